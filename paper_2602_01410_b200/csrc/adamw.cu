// One AdamW step over many tensors at once, states in 32 or 8 bits.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Binary32 states: 28 bytes per element (p, bf16 g, m, v, bf16 copy; read and written once), bound by HBM; four 1B blocks 795-834 us, 90-95 % of
// the copy rate.  8-bit states: 16 bytes; to nearest still HBM (a 7B block 541 us, 92 %), stochastic 71 instructions per element, bound by issue slots
// (62 % busy) and the power cap (644 us, 715 in a long run).  Hence arithmetic on pairs and a warp's loads all ahead of its arithmetic.  Fetching
// the next chunk into shared memory meanwhile (cp.async) costs more instructions and registers than it hides (stochastic 605 -> 703 us when it was
// measured; since then products and sums rounded one by one cost 6 %, the root of an infinite v and NaN through the rounding 3 %).  Loads and stores
// without cache hints: streaming stores cost 4 % (846 / 809 us on four 1B blocks).
// The tensors' table travels in the kernel's parameters, so that a call needs no device memory of its own and a captured graph holds it;
// a chunk of 2048 elements is the unit of work, the resident grid walks over the chunks of all tensors, and a chunk's tensor is found by
// bisection in the table.  A warp holds 128 consecutive elements at a time, four per lane: that is a block of the 8-bit states, whose
// maximum is then one warp-wide integer reduction (magnitudes order like their bits).
#include <cuda_bf16.h>
#include <float.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "quant_device.cuh"

namespace snip {

int gemm_sm_count();

namespace {

constexpr int kThreads = 128;
constexpr int kBlock = 128;      // elements that share a scale
constexpr int kChunk = 2048;     // elements a CTA takes at a time
// Tensors in a launch's table: parameters of up to 8 KB cost the launch nothing, 32 KB (all that a launch takes) 2 us (65 tensors: 8.2 -> 6.1 us a call).
constexpr int kFewTensors = 112;
constexpr int kMostTensors = 448;

struct Entry {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    uint16_t *param_bf16;
    int64_t n;
    float weight_decay;
    uint32_t first_chunk;
};
struct Hyper {
    float step_size, inv_sqrt_bc2, lr;   // lr / (1 - b1^t), (1 - b2^t)^-1/2
};
struct Common {
    double lr, beta1, beta2;
    Hyper h;                             // without device values
    const int64_t *step_device;
    const float *lr_device, *grad_scale;
    uint32_t k0, k1;                     // the generator's key
    int64_t step_host;
    uint32_t step;
    uint32_t chunks;
    int32_t count, first_tensor;
    float b1, omb1, b2, omb2, eps;
};
template <int CAP>
struct Table {
    Common c;
    Entry e[CAP];
};
static_assert(sizeof(Entry) == 72 && sizeof(Table<kMostTensors>) <= 32764, "a launch's parameters hold 32764 bytes");

__host__ __device__ inline Hyper hyper(double lr, double beta1, double beta2, int64_t step)
{
    const double bc1 = -expm1((double)step * log(beta1)), bc2 = -expm1((double)step * log(beta2));
    return {(float)(lr / bc1), (float)(1.0 / sqrt(bc2)), (float)lr};
}

// Stochastic rounding of a pair of values to E4M3, by one 32-bit word of the generator (its low half for the first): with a = |t|, lo <= a < hi
// the neighbouring grid points and u the 16-bit uniform, hi iff (a - lo)/(hi - lo) > (u + 1/2)/2^16.  On the bits, as for E2M1: from 2^-6 up a
// grid point has 20 zero bits at its end, and their value f exceeds 16 u + 8 iff f + 16 (65535 - u) + 7 carries out of them; below, the same
// holds for a + 2^-6, rounded upwards.  t comes from a block scaled by its own maximum: it passes 448 by a few last places at most, which
// leave the largest addend 9 units short of a carry.  SIGNED = false: t >= 0.  NaN is 0x7FFFFFFF, which the addition carries round to a zero;
// 0 s + v makes it NaN again.
template <bool SIGNED>
__device__ __forceinline__ float2 sr_e4m3x2(const float2 t, uint32_t w)
{
    const float2 a = SIGNED ? make_float2(fabsf(t.x), fabsf(t.y)) : t;
    float2 off;   // 1 below 2^-6, else 0: 2^120 - 2^126 a, clamped to [0, 1], on the FMA pipe
    asm("fma.rn.sat.f32 %0, %1, 0fFE800000, 0f7B800000;" : "=f"(off.x) : "f"(a.x));
    asm("fma.rn.sat.f32 %0, %1, 0fFE800000, 0f7B800000;" : "=f"(off.y) : "f"(a.y));
    const float2 s = __ffma2_ru(off, make_float2(0.015625f, 0.015625f), a);
    const uint32_t r0 = ((~w << 4) & 0xFFFF0u) | 7u, r1 = ((~w >> 12) & 0xFFFF0u) | 7u;
    const float2 q = make_float2(__uint_as_float((__float_as_uint(s.x) + r0) & 0xFFF00000u), __uint_as_float((__float_as_uint(s.y) + r1) & 0xFFF00000u));
    const float2 v = __ffma2_rn(s, make_float2(0.0f, 0.0f), __ffma2_rn(off, make_float2(-0.015625f, -0.015625f), q));
    return SIGNED ? make_float2(copysignf(v.x, t.x), copysignf(v.y, t.y)) : v;
}
// ... to bf16 bits, packed: the low 16 bits f exceed u + 1/2 iff f + 65535 - u carries, which is what the conversion's random bits do (equal to the
// integer addition on 2^31 pairs, subnormal and the largest ones among them).  It keeps a NaN, which the addition would carry round to -0.
__device__ __forceinline__ uint32_t sr_bf16x2(const float2 t, uint32_t w)
{
    uint32_t r;
    asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(r) : "f"(t.y), "f"(t.x), "r"(~w));
    return r;
}
__device__ __forceinline__ uint32_t rn_bf16x2(const float2 t)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(t.y), "f"(t.x));
    return r;
}

__device__ __forceinline__ float rcp_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// At most FLT_MAX; NaN stays NaN.
__device__ __forceinline__ float at_most_flt_max(float x)
{
    float r;
    asm("min.NaN.f32 %0, %1, 0f7F7FFFFF;" : "=f"(r) : "f"(x));
    return r;
}
// Square roots to half a last place: v times its approximate reciprocal root, and a Newton step.  (Below 2^-126, where the reciprocal root is
// held at 2^63, too small; 0 for 0.  Of an infinite v, which the square of a finite gradient can make: that of FLT_MAX, so that an 8-bit
// state stays finite.)
__device__ __forceinline__ float2 sqrt2(float2 v)
{
    v = make_float2(at_most_flt_max(v.x), at_most_flt_max(v.y));
    float2 y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(fmaxf(v.x, FLT_MIN)));
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(fmaxf(v.y, FLT_MIN)));
    const float2 s = __fmul2_rn(v, y), h = __fmul2_rn(y, make_float2(-0.5f, -0.5f));
    const float2 d = __ffma2_rn(s, s, make_float2(-v.x, -v.y));
    return __ffma2_rn(d, h, s);
}

__device__ __forceinline__ float2 unpack2(uint32_t b) { return make_float2(bf16lo(b), bf16hi(b)); }

// What a kernel ahead may have written is read past L1 (this kernel may have started before that one ended).
// Four consecutive elements of a lane, of which the tensor has `left` (the others read as zeros).
__device__ __forceinline__ void load4(const void *p, uint32_t i, int left, uint2 &v)
{
    const uint16_t *q = static_cast<const uint16_t *>(p) + i;
    if (left >= 4) {
        v = __ldcg(reinterpret_cast<const uint2 *>(q));
    } else {
        v = make_uint2(0u, 0u);
        if (left > 0) v.x = __ldcg(q);
        if (left > 1) v.x |= (uint32_t)__ldcg(q + 1) << 16;
        if (left > 2) v.y = __ldcg(q + 2);
    }
}
__device__ __forceinline__ void load4(const void *p, uint32_t i, int left, float4 &v)
{
    const float *q = static_cast<const float *>(p) + i;
    if (left >= 4) {
        v = __ldcg(reinterpret_cast<const float4 *>(q));
    } else {
        v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (left > 0) v.x = __ldcg(q);
        if (left > 1) v.y = __ldcg(q + 1);
        if (left > 2) v.z = __ldcg(q + 2);
    }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, uint32_t i, int left)
{
    if (left >= 4) return __ldcg(reinterpret_cast<const uint32_t *>(p + i));
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j < left) v |= (uint32_t)__ldcg(p + i + j) << (8 * j);
    return v;
}
__device__ __forceinline__ void to_floats(const uint2 &v, float2 (&f)[2]) { f[0] = unpack2(v.x); f[1] = unpack2(v.y); }
__device__ __forceinline__ void to_floats(const float4 &v, float2 (&f)[2]) { f[0] = make_float2(v.x, v.y); f[1] = make_float2(v.z, v.w); }
template <bool BF16>
using Vec = std::conditional_t<BF16, uint2, float4>;
template <bool FULL>
__device__ __forceinline__ void store4(float *p, uint32_t i, int left, const float2 (&f)[2])
{
    if (FULL) {
        *reinterpret_cast<float4 *>(p + i) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    } else {
        if (left > 0) p[i] = f[0].x;
        if (left > 1) p[i + 1] = f[0].y;
        if (left > 2) p[i + 2] = f[1].x;
        if (left > 3) p[i + 3] = f[1].y;
    }
}
template <bool FULL>
__device__ __forceinline__ void store4(uint16_t *p, uint32_t i, int left, uint32_t b0, uint32_t b1)
{
    if (FULL) {
        *reinterpret_cast<uint2 *>(p + i) = make_uint2(b0, b1);
    } else {
        if (left > 0) p[i] = (uint16_t)b0;
        if (left > 1) p[i + 1] = (uint16_t)(b0 >> 16);
        if (left > 2) p[i + 2] = (uint16_t)b1;
        if (left > 3) p[i + 3] = (uint16_t)(b1 >> 16);
    }
}
template <bool FULL>
__device__ __forceinline__ void store_codes(uint8_t *p, uint32_t i, int left, uint32_t v)
{
    if (FULL) {
        *reinterpret_cast<uint32_t *>(p + i) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[i + j] = (uint8_t)(v >> (8 * j));
    }
}

// The numbers of a step, the same for every element of a tensor.
struct Step {
    Hyper h;
    float b1, omb1, b2, omb2, eps, gs, keep;
    uint32_t k0, k1, tensor, count;   // of the generator: key, counter words 2 and 3 (without the kind)
};

// A chunk of a tensor: pointers to its first element.
struct Chunk {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    uint16_t *param_bf16;
    uint64_t quad;    // number of its first four elements in the tensor
    int32_t left;     // elements of the tensor from here on, if fewer than a chunk
};

__device__ __forceinline__ float2 splat(float x) { return make_float2(x, x); }

// The generator's words for the four elements at i.  A chunk's groups of four share the upper word of their number.
__device__ __forceinline__ void generator(const Step &s, const Chunk &c, uint32_t i, uint32_t kind, uint32_t (&w)[4])
{
    philox4x32_10((uint32_t)c.quad + (i >> 2), (uint32_t)(c.quad >> 32), s.tensor, s.count + kind, s.k0, s.k1, w);
}

// New moments (m, v; and r = sqrt(v)) and weights of four elements, from the old moments.  Each product and sum of the moments is rounded by
// itself: 8-bit codes sit next to rounding borders, and what is fed back should follow from a definition that can be repeated bit for bit.
// (The sums are scalar because a packed product and a packed sum are joined into an FMA, their .rn notwithstanding.)
__device__ __forceinline__ void update4(const Step &s, float2 (&p)[2], const float2 (&g)[2], float2 (&m)[2], float2 (&v)[2], float2 (&r)[2])
{
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float2 gg = __fmul2_rn(g[j], splat(s.gs));
        const float2 om = __fmul2_rn(m[j], splat(s.b1)), nm = __fmul2_rn(gg, splat(s.omb1));
        const float2 ov = __fmul2_rn(v[j], splat(s.b2)), nv = __fmul2_rn(__fmul2_rn(gg, gg), splat(s.omb2));
        m[j] = make_float2(__fadd_rn(om.x, nm.x), __fadd_rn(om.y, nm.y));
        v[j] = make_float2(__fadd_rn(ov.x, nv.x), __fadd_rn(ov.y, nv.y));
        r[j] = sqrt2(v[j]);
        // the root that the weight sees is infinite where v is: for any other v the addend is less than 2^-62 of the root and leaves it as it is
        const float2 root = __ffma2_rn(v[j], splat(FLT_MIN), r[j]);
        const float2 d = __ffma2_rn(root, splat(s.h.inv_sqrt_bc2), splat(s.eps));
        const float2 u = __fmul2_rn(__fmul2_rn(m[j], splat(-s.h.step_size)), make_float2(rcp_fast(d.x), rcp_fast(d.y)));
        p[j] = __ffma2_rn(p[j], splat(s.keep), u);
    }
}

// Code values over their scale S, correctly rounded (Markstein's division: a product with the rounded reciprocal, corrected by its exact
// remainder).
__device__ __forceinline__ float2 over_scale(const float2 code, float inv, float neg_scale)
{
    const float2 q = __fmul2_rn(code, splat(inv));
    return __ffma2_rn(__ffma2_rn(q, splat(neg_scale), code), splat(inv), q);
}
// Scale of a block: 448 times the reciprocal of its maximum, both rounded; 1 for an empty block, at most FLT_MAX.
__device__ __forceinline__ float state_scale(float most) { return most == 0.0f ? 1.0f : fminf(448.0f * __frcp_rn(most), FLT_MAX); }

template <bool FULL, bool P_BF16, bool SR>
__device__ __forceinline__ void store_param(const Step &s, const Chunk &c, uint32_t i, int left, const float2 (&p)[2])
{
    if constexpr (P_BF16) {
        uint32_t b0, b1;
        if constexpr (SR) {
            uint32_t w[4];
            generator(s, c, i, 1, w);
            b0 = sr_bf16x2(p[0], w[0]);
            b1 = sr_bf16x2(p[1], w[1]);
        } else {
            b0 = rn_bf16x2(p[0]);
            b1 = rn_bf16x2(p[1]);
        }
        store4<FULL>(static_cast<uint16_t *>(c.param), i, left, b0, b1);
    } else {
        store4<FULL>(static_cast<float *>(c.param), i, left, p);
        if (c.param_bf16) store4<FULL>(c.param_bf16, i, left, rn_bf16x2(p[0]), rn_bf16x2(p[1]));
    }
}

constexpr int kWarps = kThreads / 32;

// A warp's share of a chunk, binary32 states.
template <bool FULL, bool P_BF16, bool G_BF16, bool SR>
__device__ __forceinline__ void run_chunk32(const Step &s, const Chunk &c, int warp, int lane)
{
#pragma unroll 1
    for (int part = 0; part < kChunk / (kBlock * kWarps); ++part) {
        const uint32_t i = (uint32_t)((part * kWarps + warp) * kBlock + 4 * lane);
        const int left = FULL ? 4 : c.left - (int)i;
        Vec<P_BF16> pv;
        Vec<G_BF16> gv;
        float4 mv, vv;
        load4(c.param, i, left, pv);
        load4(c.grad, i, left, gv);
        load4(c.m, i, left, mv);
        load4(c.v, i, left, vv);
        float2 p[2], g[2], m[2], v[2], r[2];
        to_floats(pv, p);
        to_floats(gv, g);
        to_floats(mv, m);
        to_floats(vv, v);
        update4(s, p, g, m, v, r);
        store4<FULL>(static_cast<float *>(c.m), i, left, m);
        store4<FULL>(static_cast<float *>(c.v), i, left, v);
        store_param<FULL, P_BF16, SR>(s, c, i, left, p);
    }
}

// ... 8-bit states.  What is done once per block and state (reading a scale and dividing by it, making the new one) is done by one lane each:
// lanes 0 .. U-1 for the first moments of the warp's U blocks, lanes U .. 2 U - 1 for the second, and handed round by shuffles.
template <bool FULL, bool P_BF16, bool G_BF16, bool SR>
__device__ __forceinline__ void run_chunk8(const Step &s, const Chunk &c, int warp, int lane)
{
    constexpr int U = kChunk / (kBlock * kWarps);
    constexpr uint32_t kAll = 0xFFFFFFFFu;
    const uint32_t b0 = (uint32_t)(warp * U), i0 = b0 * kBlock + 4 * lane;
    if (!FULL && (int)(b0 * kBlock) >= c.left) return;     // the whole warp
    Vec<P_BF16> pv[U];
    Vec<G_BF16> gv[U];
    uint32_t mc[U], vc[U];
    const bool second = (lane & U) != 0;
    float *scales = second ? c.v_scale : c.m_scale;
    const uint32_t block = b0 + (lane & (U - 1));
    const bool owner = lane < 2 * U && (FULL || (int)(block * kBlock) < c.left);
    const float scale = owner ? __ldcg(scales + block) : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = i0 + u * kBlock;
        const int left = FULL ? 4 : c.left - (int)i;
        load4(c.param, i, left, pv[u]);
        load4(c.grad, i, left, gv[u]);
        mc[u] = load_codes(static_cast<const uint8_t *>(c.m), i, left);
        vc[u] = load_codes(static_cast<const uint8_t *>(c.v), i, left);
    }
    const float inv = scale == 0.0f ? 0.0f : __frcp_rn(scale);
    float2 m[U][2], r[U][2];
    float most = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = i0 + u * kBlock;
        const float im = __shfl_sync(kAll, inv, u), iv = __shfl_sync(kAll, inv, U + u), nm = -__shfl_sync(kAll, scale, u), nv = -__shfl_sync(kAll, scale, U + u);
        float2 p[2], g[2], v[2];
        to_floats(pv[u], p);
        to_floats(gv[u], g);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            m[u][j] = over_scale(dec_e4m3x2(mc[u] >> (16 * j)), im, nm);
            const float2 root = over_scale(dec_e4m3x2(vc[u] >> (16 * j)), iv, nv);
            v[j] = __fmul2_rn(root, root);
        }
        update4(s, p, g, m[u], v, r[u]);
        store_param<FULL, P_BF16, SR>(s, c, i, FULL ? 4 : c.left - (int)i, p);
        // magnitudes order like their bits
        const uint32_t am = __reduce_max_sync(kAll, __float_as_uint(fmaxf(fmaxf(fabsf(m[u][0].x), fabsf(m[u][0].y)), fmaxf(fabsf(m[u][1].x), fabsf(m[u][1].y)))));
        const uint32_t ar = __reduce_max_sync(kAll, __float_as_uint(fmaxf(fmaxf(r[u][0].x, r[u][0].y), fmaxf(r[u][1].x, r[u][1].y))));
        if ((lane & (U - 1)) == u) most = __uint_as_float(second ? ar : am);
    }
    const float fresh = state_scale(most);
    if (owner) scales[block] = fresh;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = i0 + u * kBlock;
        const int left = FULL ? 4 : c.left - (int)i;
        const float sm = __shfl_sync(kAll, fresh, u), sv = __shfl_sync(kAll, fresh, U + u);
        float2 tm[2], tv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            tm[j] = __fmul2_rn(m[u][j], splat(sm));
            tv[j] = __fmul2_rn(r[u][j], splat(sv));
        }
        if constexpr (SR) {
            uint32_t w[4];
            generator(s, c, i, 0, w);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                tm[j] = sr_e4m3x2<true>(tm[j], w[j]);
                tv[j] = sr_e4m3x2<false>(tv[j], w[2 + j]);
            }
        }
        uint32_t codes = cvt_e4m3x2(tv[0].x, tv[0].y) | cvt_e4m3x2(tv[1].x, tv[1].y) << 16;
        if ((codes - 0x01010101u) & 0x80808080u) {   // perhaps a code 0 (a code has 7 bits): what is positive gets the smallest one instead
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float rj = j & 1 ? r[u][j >> 1].y : r[u][j >> 1].x;
                if (((codes >> (8 * j)) & 0xFFu) == 0u && rj > 0.0f) codes |= 1u << (8 * j);
            }
        }
        store_codes<FULL>(static_cast<uint8_t *>(c.m), i, left, cvt_e4m3x2(tm[0].x, tm[0].y) | cvt_e4m3x2(tm[1].x, tm[1].y) << 16);
        store_codes<FULL>(static_cast<uint8_t *>(c.v), i, left, codes);
    }
}

// The tensor that a chunk belongs to, and the chunk in it.
template <int CAP, bool P_BF16, bool G_BF16, bool BITS8>
__device__ __forceinline__ int locate(const Table<CAP> &a, uint32_t chunk, Chunk &k)
{
    int lo = 0, hi = a.c.count;       // last entry whose first chunk is not behind this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.e[mid].first_chunk <= chunk) lo = mid;
        else hi = mid;
    }
    const Entry &e = a.e[lo];
    const int64_t base = (int64_t)(chunk - e.first_chunk) * kChunk, left = e.n - base;
    k.param = static_cast<uint8_t *>(e.param) + base * (P_BF16 ? 2 : 4);
    k.grad = static_cast<const uint8_t *>(e.grad) + base * (G_BF16 ? 2 : 4);
    k.m = static_cast<uint8_t *>(e.m) + base * (BITS8 ? 1 : 4);
    k.v = static_cast<uint8_t *>(e.v) + base * (BITS8 ? 1 : 4);
    k.m_scale = e.m_scale + base / kBlock;
    k.v_scale = e.v_scale + base / kBlock;
    k.param_bf16 = e.param_bf16 ? e.param_bf16 + base : nullptr;
    k.quad = (uint64_t)base >> 2;
    k.left = left < kChunk ? (int32_t)left : kChunk;
    return lo;
}

// CTAs per SM that the registers of the forms with 8-bit states are cut for.  A 7B block (202 M elements) in us, at four / five / six / seven / eight,
// bf16 gradients: to nearest 559 / 543 / 567 / 579 / 598 with binary32 weights, 443 / 424 / 398 / 393 / 382 with bf16 ones; stochastic 679 / 656 / 646 /
// 645 / 645 and 734 / 745 / 767 / 799 / 816 (two generator calls per four elements: the more registers, the fewer spill).
constexpr int resident_ctas(bool p16, bool bits8, bool sr)
{
    return !bits8 ? 6 : p16 ? (sr ? 4 : 8) : (sr ? 7 : 5);
}
// Most CTAs per SM that are launched, 0 for all that fit.  With binary32 states the registers leave room for eight to ten; four blocks of the 1B model
// in us, at six / at all: binary32 weights 793 / 820 (one call at a time 796 / 855; calls that follow each other on three states 833 / 832), bf16
// ones 637 / 624, and stochastic 656 / 610.
constexpr int launched_ctas(bool p16, bool bits8) { return !bits8 && !p16 ? 6 : 0; }

template <int CAP, bool P_BF16, bool G_BF16, bool BITS8, bool SR>
__global__ void __launch_bounds__(kThreads, resident_ctas(P_BF16, BITS8, SR)) adamw_kernel(const __grid_constant__ Table<CAP> a)
{
    __shared__ Hyper shared_hyper;
    chain_start(CHAIN_FIRST);   // may be set up while the kernel before it on the stream ends
    const Common &c = a.c;
    Step s;
    s.h = c.h;
    uint32_t step = c.step;
    if (c.step_device || c.lr_device) {
        int64_t t = c.step_device ? __ldcg(reinterpret_cast<const long long *>(c.step_device)) : c.step_host;
        t = t < 1 ? 1 : t;
        if (threadIdx.x == 0) shared_hyper = hyper(c.lr_device ? (double)__ldcg(c.lr_device) : c.lr, c.beta1, c.beta2, t);
        __syncthreads();
        s.h = shared_hyper;
        step = (uint32_t)t;
    }
    s.b1 = c.b1; s.omb1 = c.omb1; s.b2 = c.b2; s.omb2 = c.omb2; s.eps = c.eps;
    s.gs = c.grad_scale ? __ldcg(c.grad_scale) : 1.0f;
    s.k0 = c.k0; s.k1 = c.k1;
    s.count = 2u * step;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (uint32_t chunk = blockIdx.x; chunk < c.chunks; chunk += gridDim.x) {
        Chunk k;
        const int entry = locate<CAP, P_BF16, G_BF16, BITS8>(a, chunk, k);
        s.keep = (float)(1.0 - (double)s.h.lr * (double)a.e[entry].weight_decay);
        s.tensor = (uint32_t)(c.first_tensor + entry);
        const bool full = k.left == kChunk;
        if constexpr (BITS8) {
            if (full) run_chunk8<true, P_BF16, G_BF16, SR>(s, k, warp, lane);
            else run_chunk8<false, P_BF16, G_BF16, SR>(s, k, warp, lane);
        } else {
            if (full) run_chunk32<true, P_BF16, G_BF16, SR>(s, k, warp, lane);
            else run_chunk32<false, P_BF16, G_BF16, SR>(s, k, warp, lane);
        }
    }
}

// CTAs of a kernel that an SM holds (asked once: the same on every device of this family).
template <auto Kernel>
int resident()
{
    static const int n = [] {
        int k = 0;
        return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, Kernel, kThreads, 0) == cudaSuccess && k > 0 ? k : 1;
    }();
    return n;
}

template <int CAP, bool P_BF16, bool G_BF16, bool BITS8, bool SR>
int launch(const Table<CAP> &t, cudaStream_t st)
{
    constexpr auto kernel = adamw_kernel<CAP, P_BF16, G_BF16, BITS8, SR>;
    constexpr int most = launched_ctas(P_BF16, BITS8);
    const int fit = resident<kernel>();
    const int64_t cap = (int64_t)(most && most < fit ? most : fit) * gemm_sm_count();
    return launch_chained(kernel, (int)(t.c.chunks < cap ? t.c.chunks : cap), kThreads, 0, st, 1, t);
}

template <int CAP>
int launch_for(const Table<CAP> &t, bool p16, bool g16, bool bits8, bool sr, cudaStream_t st)
{
    const int variant = (p16 ? 8 : 0) | (g16 ? 4 : 0) | (bits8 ? 2 : 0) | (sr && (p16 || bits8) ? 1 : 0);
    switch (variant) {
        case 0: return launch<CAP, false, false, false, false>(t, st);
        case 2: return launch<CAP, false, false, true, false>(t, st);
        case 3: return launch<CAP, false, false, true, true>(t, st);
        case 4: return launch<CAP, false, true, false, false>(t, st);
        case 6: return launch<CAP, false, true, true, false>(t, st);
        case 7: return launch<CAP, false, true, true, true>(t, st);
        case 8: return launch<CAP, true, false, false, false>(t, st);
        case 9: return launch<CAP, true, false, false, true>(t, st);
        case 10: return launch<CAP, true, false, true, false>(t, st);
        case 11: return launch<CAP, true, false, true, true>(t, st);
        case 12: return launch<CAP, true, true, false, false>(t, st);
        case 13: return launch<CAP, true, true, false, true>(t, st);
        case 14: return launch<CAP, true, true, true, false>(t, st);
        case 15: return launch<CAP, true, true, true, true>(t, st);
        default: return SNIP_ERR_UNSUPPORTED;   // not reached: stochastic rounding of nothing is dropped above
    }
}

template <int CAP>
int step_some(const snip_adamw_tensor_t *ts, int64_t first, int64_t count, const Common &common, const snip_adamw_t &a, cudaStream_t st)
{
    Table<CAP> t;
    t.c = common;
    t.c.count = (int32_t)count;
    t.c.first_tensor = (int32_t)first;
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; ++i) {
        const snip_adamw_tensor_t &s = ts[first + i];
        t.e[i] = {s.param, s.grad, s.m, s.v, s.m_scale, s.v_scale, static_cast<uint16_t *>(s.param_bf16), s.n, s.weight_decay, (uint32_t)chunks};
        chunks += ceil_div(s.n, kChunk);
    }
    if (chunks == 0) return SNIP_OK;
    t.c.chunks = (uint32_t)chunks;
    return launch_for<CAP>(t, a.param_dtype == SNIP_OUT_BF16, a.grad_dtype == SNIP_OUT_BF16, a.state_bits == 8, a.rounding == SNIP_ROUND_STOCHASTIC, st);
}

}  // namespace
}  // namespace snip

extern "C" int snip_adamw_state_sizes(int64_t n, int state_bits, size_t *state_bytes, size_t *scale_bytes)
{
    using namespace snip;
    if (!state_bytes || !scale_bytes || (state_bits != 8 && state_bits != 32)) return SNIP_ERR_ARG;
    if (n < 0) return SNIP_ERR_SHAPE;
    *state_bytes = (size_t)n * (state_bits / 8);
    *scale_bytes = state_bits == 8 ? sizeof(float) * (size_t)ceil_div(n, kBlock) : 0;
    return SNIP_OK;
}

extern "C" int snip_adamw_step(const snip_adamw_tensor_t *ts, int64_t count, const snip_adamw_t *a, void *stream)
{
    using namespace snip;
    if (!a || count < 0 || (count > 0 && !ts)) return SNIP_ERR_ARG;
    if ((a->param_dtype != SNIP_OUT_BF16 && a->param_dtype != SNIP_OUT_FP32) || (a->grad_dtype != SNIP_OUT_BF16 && a->grad_dtype != SNIP_OUT_FP32)) return SNIP_ERR_ARG;
    if (a->state_bits != 8 && a->state_bits != 32) return SNIP_ERR_ARG;
    if (a->rounding != SNIP_ROUND_NEAREST_EVEN && a->rounding != SNIP_ROUND_STOCHASTIC) return SNIP_ERR_ARG;
    if (!(fabs(a->lr) <= FLT_MAX) || !(a->beta1 >= 0.0 && a->beta1 < 1.0) || !(a->beta2 >= 0.0 && a->beta2 < 1.0)) return SNIP_ERR_ARG;
    if (!((float)a->eps >= FLT_MIN && a->eps <= FLT_MAX) || (!a->step_device && a->step < 1)) return SNIP_ERR_ARG;
    if (count > INT32_MAX) return SNIP_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(a->step_device) & 7u) || (reinterpret_cast<uintptr_t>(a->lr_device) & 3u) || (reinterpret_cast<uintptr_t>(a->grad_scale) & 3u)) return SNIP_ERR_ALIGN;
    for (int64_t i = 0; i < count; ++i) {
        const snip_adamw_tensor_t &t = ts[i];
        if (t.n < 0 || t.n > (int64_t)1 << 40) return SNIP_ERR_SHAPE;
        if (!(fabsf(t.weight_decay) <= FLT_MAX)) return SNIP_ERR_ARG;
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v) return SNIP_ERR_ARG;
        if (a->state_bits == 8 ? !t.m_scale || !t.v_scale : t.m_scale || t.v_scale) return SNIP_ERR_ARG;
        if (t.param_bf16 && a->param_dtype != SNIP_OUT_FP32) return SNIP_ERR_ARG;
        if (!aligned16(t.param) || !aligned16(t.grad) || !aligned16(t.m) || !aligned16(t.v) || !aligned16(t.param_bf16)) return SNIP_ERR_ALIGN;
        if ((reinterpret_cast<uintptr_t>(t.m_scale) & 3u) || (reinterpret_cast<uintptr_t>(t.v_scale) & 3u)) return SNIP_ERR_ALIGN;
    }
    // chunks are counted in 32 bits: a launch's tensors together
    for (int64_t i = 0; i < count;) {
        int64_t chunks = 0;
        for (const int64_t end = i + kMostTensors < count ? i + kMostTensors : count; i < end; ++i) chunks += ceil_div(ts[i].n, kChunk);
        if (chunks > INT32_MAX) return SNIP_ERR_SHAPE;
    }
    if (count == 0) return SNIP_OK;
    int rc = require_sm100();
    if (rc) return rc;
    Common c = {};
    c.lr = a->lr; c.beta1 = a->beta1; c.beta2 = a->beta2;
    if (!a->step_device) c.h = hyper(a->lr, a->beta1, a->beta2, a->step);
    c.step_device = a->step_device; c.lr_device = a->lr_device; c.grad_scale = a->grad_scale;
    c.k0 = (uint32_t)a->seed; c.k1 = (uint32_t)(a->seed >> 32);
    c.step_host = a->step;
    c.step = (uint32_t)a->step;
    c.b1 = (float)a->beta1; c.omb1 = (float)(1.0 - a->beta1);
    c.b2 = (float)a->beta2; c.omb2 = (float)(1.0 - a->beta2);
    c.eps = (float)a->eps;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    for (int64_t i = 0; i < count; i += kMostTensors) {
        const int64_t some = count - i < kMostTensors ? count - i : kMostTensors;
        rc = some <= kFewTensors ? step_some<kFewTensors>(ts, i, some, c, *a, st) : step_some<kMostTensors>(ts, i, some, c, *a, st);
        if (rc) return rc;
    }
    return SNIP_OK;
}
