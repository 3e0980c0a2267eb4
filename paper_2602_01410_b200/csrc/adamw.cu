// One AdamW step over many tensors at once, states in 32 or 8 bits.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by HBM: 28 bytes per element with binary32 states (p, g, m, v, bf16 copy; read and written once), 16 with 8-bit ones.
// The tensors' table travels in the kernel's parameters, so that a call needs no device memory of its own and a captured graph holds it;
// a chunk of 4096 elements is the unit of work, the resident grid walks over the chunks of all tensors, and a chunk's tensor is found by
// bisection in the table.  A warp holds 128 consecutive elements at a time, four per lane: that is a block of the 8-bit states, whose
// maximum is then one warp-wide integer reduction (magnitudes order like their bits).
#include <cuda_bf16.h>
#include <float.h>
#include <math.h>

#include "common.cuh"
#include "quant_device.cuh"

namespace snip {

int gemm_sm_count();

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 128;      // elements that share a scale
constexpr int kChunk = 4096;     // elements a CTA takes at a time
constexpr int kMostTensors = 448;
constexpr int kFewTensors = 16;

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
    uint64_t seed;
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

// Stochastically rounded E4M3 value of t for the 16-bit uniform u: with a = min(|t|, 448), lo <= a < hi the neighbouring grid points, hi iff
// (a - lo)/(hi - lo) > (u + 1/2)/2^16.  On the bits, as for E2M1: from 2^-6 up a grid point has 20 zero bits at its end, and their
// value f exceeds 16 u + 8 iff f + 16 (65535 - u) + 7 carries out of them; below, the same holds for a + 2^-6, rounded upwards.
__device__ __forceinline__ float sr_e4m3_value(float t, uint32_t u)
{
    const float a = fminf(fabsf(t), 448.0f);
    const float off = a < 0.015625f ? 0.015625f : 0.0f;
    const uint32_t q = (__float_as_uint(__fadd_ru(a, off)) + ((65535u - u) * 16u + 7u)) & 0xFFF00000u;
    return copysignf(__uint_as_float(q) - off, t);
}
// ... and of a bf16 value, as binary32: the low 16 bits f exceed u + 1/2 iff f + 65535 - u carries.
__device__ __forceinline__ uint32_t sr_bf16_bits(float t, uint32_t u) { return (__float_as_uint(t) + (65535u - u)) >> 16; }

__device__ __forceinline__ uint32_t warp_max(float a0, float a1, float a2, float a3)
{
    return __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(fmaxf(fmaxf(a0, a1), fmaxf(a2, a3))));
}

__device__ __forceinline__ float sqrt_fast(float v)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Four consecutive elements of a lane; `left`: how many of them the tensor has.
template <bool BF16>
__device__ __forceinline__ void load4(const void *p, int64_t i, int left, float (&f)[4])
{
    if constexpr (BF16) {
        const uint16_t *q = static_cast<const uint16_t *>(p) + i;
        if (left >= 4) {
            const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(q));
            f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = j < left ? __uint_as_float((uint32_t)q[j] << 16) : 0.0f;
        }
    } else {
        const float *q = static_cast<const float *>(p) + i;
        if (left >= 4) {
            const float4 v = __ldcs(reinterpret_cast<const float4 *>(q));
            f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = j < left ? q[j] : 0.0f;
        }
    }
}
__device__ __forceinline__ void store4(float *p, int64_t i, int left, const float (&f)[4])
{
    if (left >= 4) {
        __stcs(reinterpret_cast<float4 *>(p + i), make_float4(f[0], f[1], f[2], f[3]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[i + j] = f[j];
    }
}
__device__ __forceinline__ void store4(uint16_t *p, int64_t i, int left, const uint32_t (&b)[4])
{
    if (left >= 4) {
        *reinterpret_cast<uint2 *>(p + i) = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[i + j] = (uint16_t)b[j];
    }
}
__device__ __forceinline__ uint32_t load_codes(const void *p, int64_t i, int left)
{
    const uint8_t *q = static_cast<const uint8_t *>(p) + i;
    if (left >= 4) return __ldcs(reinterpret_cast<const uint32_t *>(q));
    uint32_t v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) v |= (uint32_t)q[j] << (8 * j);
    return v;
}
__device__ __forceinline__ void store_codes(void *p, int64_t i, int left, uint32_t v)
{
    uint8_t *q = static_cast<uint8_t *>(p) + i;
    if (left >= 4) {
        __stcs(reinterpret_cast<uint32_t *>(q), v);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) q[j] = (uint8_t)(v >> (8 * j));
    }
}
__device__ __forceinline__ uint32_t bf16_bits(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }

// What a lane holds of one block.
template <bool BITS8>
struct Four {
    float p[4], g[4];
    float m[BITS8 ? 1 : 4], v[BITS8 ? 1 : 4];
    uint32_t mc, vc;
    float ms, vs;
    int left;
};

template <int CAP, bool P_BF16, bool G_BF16, bool BITS8, bool SR>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<CAP> a)
{
    __shared__ Hyper shared_hyper;
    const Common &c = a.c;
    Hyper h = c.h;
    uint32_t step = c.step;
    if (c.step_device || c.lr_device) {
        const int64_t t = c.step_device ? *c.step_device : (int64_t)c.step;
        if (threadIdx.x == 0) shared_hyper = hyper(c.lr_device ? (double)*c.lr_device : c.lr, c.beta1, c.beta2, t);
        __syncthreads();
        h = shared_hyper;
        step = (uint32_t)t;
    }
    const float gs = c.grad_scale ? *c.grad_scale : 1.0f;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int U = BITS8 ? 4 : 2;    // blocks in flight per warp
    constexpr int kWarps = kThreads / 32;
    for (uint32_t chunk = blockIdx.x; chunk < c.chunks; chunk += gridDim.x) {
        int lo = 0, hi = c.count;       // last entry whose first chunk is not behind this one
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.e[mid].first_chunk <= chunk) lo = mid;
            else hi = mid;
        }
        const Entry &e = a.e[lo];
        const int64_t base = (int64_t)(chunk - e.first_chunk) * kChunk;
        const float keep = (float)(1.0 - (double)h.lr * (double)e.weight_decay);
#pragma unroll 1
        for (int part = 0; part < kChunk / (kBlock * kWarps * U); ++part) {
            Four<BITS8> x[U];
            const int64_t b0 = base + (int64_t)(part * U * kWarps + warp) * kBlock;   // U blocks, kWarps apart
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t b = b0 + u * kWarps * kBlock, i = b + 4 * lane;
                const int64_t rest = e.n - i;
                x[u].left = rest >= 4 ? 4 : rest > 0 ? (int)rest : 0;
                load4<P_BF16>(e.param, i, x[u].left, x[u].p);
                load4<G_BF16>(e.grad, i, x[u].left, x[u].g);
                if constexpr (BITS8) {
                    x[u].mc = load_codes(e.m, i, x[u].left);
                    x[u].vc = load_codes(e.v, i, x[u].left);
                    x[u].ms = x[u].vs = 0.0f;
                    if (b < e.n) { x[u].ms = e.m_scale[b / kBlock]; x[u].vs = e.v_scale[b / kBlock]; }
                } else {
                    load4<false>(e.m, i, x[u].left, x[u].m);
                    load4<false>(e.v, i, x[u].left, x[u].v);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t b = b0 + u * kWarps * kBlock, i = b + 4 * lane;
                if (b >= e.n) break;    // the whole warp
                const int left = x[u].left;
                float m[4], v[4], r[4], p[4];
                if constexpr (BITS8) {
                    const float im = x[u].ms == 0.0f ? 0.0f : __frcp_rn(x[u].ms), iv = x[u].vs == 0.0f ? 0.0f : __frcp_rn(x[u].vs);
                    const float2 m0 = dec_e4m3x2(x[u].mc), m1 = dec_e4m3x2(x[u].mc >> 16), v0 = dec_e4m3x2(x[u].vc), v1 = dec_e4m3x2(x[u].vc >> 16);
                    m[0] = m0.x * im; m[1] = m0.y * im; m[2] = m1.x * im; m[3] = m1.y * im;
                    v[0] = v0.x * iv; v[1] = v0.y * iv; v[2] = v1.x * iv; v[3] = v1.y * iv;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= v[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) { m[j] = x[u].m[j]; v[j] = x[u].v[j]; }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float g = x[u].g[j] * gs;
                    m[j] = fmaf(c.b1, m[j], c.omb1 * g);
                    v[j] = fmaf(c.b2, v[j], c.omb2 * g * g);
                    r[j] = sqrt_fast(v[j]);
                    p[j] = fmaf(x[u].p[j], keep, -h.step_size * __fdividef(m[j], fmaf(r[j], h.inv_sqrt_bc2, c.eps)));
                }
                const uint64_t q = (uint64_t)i >> 2;
                const uint32_t tensor = (uint32_t)(c.first_tensor + lo);
                if constexpr (BITS8) {
                    const float am = __uint_as_float(warp_max(fabsf(m[0]), fabsf(m[1]), fabsf(m[2]), fabsf(m[3])));
                    const float ar = __uint_as_float(warp_max(r[0], r[1], r[2], r[3]));
                    const float sm = tile_scale<SNIP_FMT_FP8_E4M3>(am, 0), sv = tile_scale<SNIP_FMT_FP8_E4M3>(ar, 0);
                    float tm[4], tv[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) { tm[j] = m[j] * sm; tv[j] = r[j] * sv; }
                    if constexpr (SR) {
                        uint32_t w[4];
                        philox4x32_10((uint32_t)q, (uint32_t)(q >> 32), tensor, 2u * step, (uint32_t)c.seed, (uint32_t)(c.seed >> 32), w);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            tm[j] = sr_e4m3_value(tm[j], (w[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
                            tv[j] = sr_e4m3_value(tv[j], (w[2 + (j >> 1)] >> (16 * (j & 1))) & 0xFFFFu);
                        }
                    }
                    // a positive second moment stays positive: at least the smallest code
#pragma unroll
                    for (int j = 0; j < 4; ++j) tv[j] = r[j] > 0.0f ? fmaxf(tv[j], 0.001953125f) : tv[j];
                    store_codes(e.m, i, left, cvt_e4m3x2(tm[0], tm[1]) | cvt_e4m3x2(tm[2], tm[3]) << 16);
                    store_codes(e.v, i, left, cvt_e4m3x2(tv[0], tv[1]) | cvt_e4m3x2(tv[2], tv[3]) << 16);
                    if (lane == 0) { e.m_scale[b / kBlock] = sm; e.v_scale[b / kBlock] = sv; }
                } else {
                    store4(static_cast<float *>(e.m), i, left, m);
                    store4(static_cast<float *>(e.v), i, left, v);
                }
                if constexpr (P_BF16) {
                    uint32_t bits[4];
                    if constexpr (SR) {
                        uint32_t w[4];
                        philox4x32_10((uint32_t)q, (uint32_t)(q >> 32), tensor, 2u * step + 1u, (uint32_t)c.seed, (uint32_t)(c.seed >> 32), w);
#pragma unroll
                        for (int j = 0; j < 4; ++j) bits[j] = sr_bf16_bits(p[j], (w[j >> 1] >> (16 * (j & 1))) & 0xFFFFu);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) bits[j] = bf16_bits(p[j]);
                    }
                    store4(static_cast<uint16_t *>(e.param), i, left, bits);
                } else {
                    store4(static_cast<float *>(e.param), i, left, p);
                    if (e.param_bf16) {
                        uint32_t bits[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) bits[j] = bf16_bits(p[j]);
                        store4(e.param_bf16, i, left, bits);
                    }
                }
            }
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
void launch(const Table<CAP> &t, cudaStream_t st)
{
    constexpr auto kernel = adamw_kernel<CAP, P_BF16, G_BF16, BITS8, SR>;
    const int64_t cap = (int64_t)resident<kernel>() * gemm_sm_count();
    kernel<<<(unsigned)(t.c.chunks < cap ? t.c.chunks : cap), kThreads, 0, st>>>(t);
}

template <int CAP>
void launch_for(const Table<CAP> &t, bool p16, bool g16, bool bits8, bool sr, cudaStream_t st)
{
    const int variant = (p16 ? 8 : 0) | (g16 ? 4 : 0) | (bits8 ? 2 : 0) | (sr && (p16 || bits8) ? 1 : 0);
    switch (variant) {
        case 0: launch<CAP, false, false, false, false>(t, st); break;
        case 2: launch<CAP, false, false, true, false>(t, st); break;
        case 3: launch<CAP, false, false, true, true>(t, st); break;
        case 4: launch<CAP, false, true, false, false>(t, st); break;
        case 6: launch<CAP, false, true, true, false>(t, st); break;
        case 7: launch<CAP, false, true, true, true>(t, st); break;
        case 8: launch<CAP, true, false, false, false>(t, st); break;
        case 9: launch<CAP, true, false, false, true>(t, st); break;
        case 10: launch<CAP, true, false, true, false>(t, st); break;
        case 11: launch<CAP, true, false, true, true>(t, st); break;
        case 12: launch<CAP, true, true, false, false>(t, st); break;
        case 13: launch<CAP, true, true, false, true>(t, st); break;
        case 14: launch<CAP, true, true, true, false>(t, st); break;
        case 15: launch<CAP, true, true, true, true>(t, st); break;
        default: break;   // stochastic rounding of nothing: sr is dropped above
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
    launch_for<CAP>(t, a.param_dtype == SNIP_OUT_BF16, a.grad_dtype == SNIP_OUT_BF16, a.state_bits == 8, a.rounding == SNIP_ROUND_STOCHASTIC, st);
    SNIP_CUDA_TRY(cudaGetLastError());
    return SNIP_OK;
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
    if (!((float)a->eps > 0.0f && a->eps <= FLT_MAX) || (!a->step_device && a->step < 1)) return SNIP_ERR_ARG;
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
    c.seed = a->seed;
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
