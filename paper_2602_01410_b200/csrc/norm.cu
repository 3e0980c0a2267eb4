// RMS norm with the residual's addition, its quantized outputs, and its backward pass.
//   forward:  h = bf16(x + residual), rstd = (mean h^2 + eps)^-1/2, y = (h rstd) gain, in binary32; codes of y on 1x128 tiles, and
//             on 128x1 tiles stored transposed, by the quantizers' scale rule
//   backward: g = dy gain, c = mean(g h rstd), dx = rstd (g - h rstd c) + dresidual, dgain = sum over rows of dy h rstd
//
// All of it is bound by HBM: a few operations per element against 6 to 10 bytes.
//
// rmsnorm_kernel / rmsnorm_bwd_kernel: a group of warps owns a row at a time and a thread the same columns of each of its rows, so that
// the gain (and the gain's gradient) stays in registers; the grid is resident and walks over the rows.  The row is read once: it stays in
// registers between the reduction and the outputs, and the next row is on its way during both.
#include <cuda_bf16.h>
#include <float.h>

#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "quant_device.cuh"

namespace snip {

int gemm_sm_count();

namespace {

constexpr int64_t kMaxCols = 32768;
template <int N>
using Int = std::integral_constant<int, N>;

struct NormArgs {
    const uint16_t *x, *residual;
    const void *gain;
    uint16_t *h, *y;
    float *rstd;
    uint8_t *codes;
    float *scales;
    int32_t ld_x, ld_residual, ld_h, ld_y;   // 32 bits (checked on the host): index products are 32 x 32 -> 64-bit multiplies
    int32_t rows, cols;
    int gain_f32, wpr;
    float eps, inv_cols;
};

struct NormBwdArgs {
    const uint16_t *dy, *h, *dresidual;
    const void *gain;
    const float *rstd;
    uint16_t *dx;
    float *partials;   // [groups of the grid][cols], or null
    int32_t ld_dy, ld_h, ld_dresidual, ld_dx;
    int32_t rows, cols;
    int gain_f32, wpr;
    float inv_cols;
};

// Eight neighbouring elements as four pairs.
struct Eight {
    float2 p[4];
};
__device__ __forceinline__ float2 splat(float x) { return make_float2(x, x); }
__device__ __forceinline__ Eight unpack8(const uint4 &v)
{
    return {{make_float2(bf16lo(v.x), bf16hi(v.x)), make_float2(bf16lo(v.y), bf16hi(v.y)), make_float2(bf16lo(v.z), bf16hi(v.z)), make_float2(bf16lo(v.w), bf16hi(v.w))}};
}
__device__ __forceinline__ uint32_t pack2(const float2 f)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(f.y), "f"(f.x));
    return r;
}
__device__ __forceinline__ uint4 pack8(const Eight &e) { return make_uint4(pack2(e.p[0]), pack2(e.p[1]), pack2(e.p[2]), pack2(e.p[3])); }
__device__ __forceinline__ Eight zeros8() { return {{splat(0.0f), splat(0.0f), splat(0.0f), splat(0.0f)}}; }

// (h rstd) gain, each product rounded: what every form of the forward pass quantizes
__device__ __forceinline__ Eight scaled8(const Eight &h, float rstd, const Eight &gain)
{
    Eight y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y.p[i] = __fmul2_rn(__fmul2_rn(h.p[i], splat(rstd)), gain.p[i]);
    return y;
}
__device__ __forceinline__ float most8(const Eight &y)
{
    float m = fmaxf(fabsf(y.p[0].x), fabsf(y.p[0].y));
#pragma unroll
    for (int i = 1; i < 4; ++i) m = fmaxf(fmaxf(m, fabsf(y.p[i].x)), fabsf(y.p[i].y));
    return m;
}

// Codes of eight neighbouring elements under one scale.
template <int FMT>
__device__ __forceinline__ void store_codes8(uint8_t *to, const Eight &y, float s)
{
    float2 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __fmul2_rn(y.p[i], splat(s));
    if constexpr (FMT == SNIP_FMT_FP8_E4M3) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(__byte_perm(cvt_e4m3x2(t[0].x, t[0].y), cvt_e4m3x2(t[1].x, t[1].y), 0x5410),
                                                            __byte_perm(cvt_e4m3x2(t[2].x, t[2].y), cvt_e4m3x2(t[3].x, t[3].y), 0x5410));
    } else {
        *reinterpret_cast<uint32_t *>(to) = cvt_e2m1x2(t[0].x, t[0].y) | cvt_e2m1x2(t[1].x, t[1].y) << 8 | cvt_e2m1x2(t[2].x, t[2].y) << 16 |
                                                        cvt_e2m1x2(t[3].x, t[3].y) << 24;
    }
}

__device__ __forceinline__ Eight load_gain8(const void *gain, int f32, int col)
{
    if (!f32) return unpack8(__ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(gain) + col)));
    const float4 a = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(gain) + col));
    const float4 b = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(gain) + col) + 1);
    return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}

// 16 bytes into this thread's own slot of shared memory (read back by itself: nothing to wait for but its own copies).
__device__ __forceinline__ void copy_async(uint4 *slot, const uint16_t *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot)), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where a thread is: `wpr` warps per row, groups of rows side by side in the CTA (warps behind the last group have no row).  Vector k of thread t of
// a group starts at column col0 + k apart, so that 16 neighbouring threads hold a 128-long tile.
struct Place {
    int warp, lane, group, groups, col0, apart;   // warp: of the CTA
    __device__ __forceinline__ explicit Place(int wpr)
    {
        warp = (int)threadIdx.x >> 5;
        lane = (int)threadIdx.x & 31;
        groups = (int)(blockDim.x >> 5) / wpr;
        group = warp / wpr;
        col0 = 8 * (32 * (warp - group * wpr) + lane);
        apart = 256 * wpr;
    }
};

// Sum over the warps of a row group, in a fixed order; the same value in every thread.  `slots`: 32 floats, zero at first (groups of up to eight
// warps have eight each), free again when all threads have come past the next call's barrier: callers alternate between two sets.
__device__ __forceinline__ float group_sum(float v, float *slots, const Place &at, int wpr)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    if (wpr == 1) return v;
    const int first = wpr <= 8 ? 8 * at.group : 0;
    if (at.lane == 0) slots[wpr <= 8 ? first + at.warp - at.group * wpr : at.warp] = v;
    __syncthreads();
    if (wpr <= 8) {
        const float4 p = *reinterpret_cast<const float4 *>(slots + first), q = *reinterpret_cast<const float4 *>(slots + first + 4);
        return ((p.x + p.y) + (p.z + p.w)) + ((q.x + q.y) + (q.z + q.w));
    }
    v = slots[at.lane];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    return v;
}

// Rows on their way: a thread's slots for STAGES rows of N arrays of V vectors (read back by the thread itself).  A vector beyond the last column
// is never fetched: its slots are zeroed once.
template <int V, int N, int STAGES>
struct Ring {
    uint4 *mine;
    __device__ __forceinline__ uint4 *slot(int stage, int array, int k) const { return mine + ((stage * N + array) * V + k) * (int)blockDim.x; }
    __device__ __forceinline__ Ring(uint8_t *raw, const bool (&in)[V]) : mine(reinterpret_cast<uint4 *>(raw) + threadIdx.x)
    {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (!in[k])
                for (int i = 0; i < STAGES * N; ++i) *slot(0, i, k) = make_uint4(0u, 0u, 0u, 0u);
    }
};

// Scales of the tiles that a thread's V vectors belong to: 16 neighbouring threads hold a tile each.  While the maxima are combined a thread
// comes to look after one of the vectors only (own_vector), so that there is one division for all of them; the scales are handed round at
// the end.  Returns the own one.
template <int V>
__device__ __forceinline__ int own_vector(int lane) { return (lane & 15) / (16 / V); }
template <int FMT, int V>
__device__ __forceinline__ float tile_scales(float (&most)[V], float (&s)[V], int lane)
{
    if constexpr (V == 4) {
        const bool upper = (lane & 8) != 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float give = upper ? most[i] : most[i + 2], keep = upper ? most[i + 2] : most[i];
            most[i] = fmaxf(keep, __shfl_xor_sync(0xFFFFFFFFu, give, 8));
        }
    }
    if constexpr (V >= 2) {
        constexpr int kOff = V == 4 ? 4 : 8;
        const bool upper = (lane & kOff) != 0;
        const float give = upper ? most[0] : most[1], keep = upper ? most[1] : most[0];
        most[0] = fmaxf(keep, __shfl_xor_sync(0xFFFFFFFFu, give, kOff));
    }
#pragma unroll
    for (int off = 8 / V; off > 0; off >>= 1) most[0] = fmaxf(most[0], __shfl_xor_sync(0xFFFFFFFFu, most[0], off));
    const float own = tile_scale<FMT>(most[0], 0);
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = V == 1 ? own : __shfl_sync(0xFFFFFFFFu, own, (lane & 16) | k * (16 / V));
    return own;
}

// FMT: format of the row-tile codes, BF16 for none.  THREADS is the CTA's size (so that every slot is at a constant place of the ring, whose turns
// are written out): warps that no row is dealt to look on.
template <int V, int THREADS, int STAGES, bool RES, int FMT>
__global__ void __launch_bounds__(THREADS) rmsnorm_kernel(const NormArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    __shared__ __align__(16) float slots[2][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the kernel of the transposed copy, which waits for this one
    const Place at(a.wpr);
    constexpr int N = RES ? 2 : 1, kPerByte = FMT == SNIP_FMT_FP4_E2M1 ? 2 : 1;
    uint4 *const mine = reinterpret_cast<uint4 *>(raw) + threadIdx.x;
    auto slot = [&](int stage, int array, int k) { return mine + ((stage * N + array) * V + k) * THREADS; };
    const int step = (int)gridDim.x * at.groups, first = (int)blockIdx.x * at.groups, row0 = at.group < at.groups ? first + at.group : a.rows;
    bool in[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        in[k] = at.group < at.groups && at.col0 + k * at.apart < a.cols;
        if (!in[k])   // never fetched
#pragma unroll
            for (int i = 0; i < STAGES * N; ++i) *slot(0, i, k) = make_uint4(0u, 0u, 0u, 0u);
    }
    if (threadIdx.x < 64) slots[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
    __syncthreads();
    // of the widest rows neither the gain nor the row in binary32 stays in registers
    constexpr bool kWide = V > 2 && THREADS > 512;
    auto gain_of = [&](int k) { return in[k] ? load_gain8(a.gain, a.gain_f32, at.col0 + k * at.apart) : zeros8(); };
    // addresses move from row to row; those of rows behind the last are not used
    const uint16_t *px = a.x + (int64_t)row0 * a.ld_x + at.col0, *pr = RES ? a.residual + (int64_t)row0 * a.ld_residual + at.col0 : nullptr;
    const int64_t dx = (int64_t)step * a.ld_x, dr = RES ? (int64_t)step * a.ld_residual : 0;
    int64_t ahead = row0;
    auto fetch = [&](int stage) {
        if (ahead < a.rows) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (in[k]) {
                    copy_async(slot(stage, 0, k), px + k * at.apart);
                    if (RES) copy_async(slot(stage, 1, k), pr + k * at.apart);
                }
        }
        copies_commit();
        ahead += step;
        px += dx;
        if (RES) pr += dr;
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(i);
    Eight gain[kWide ? 1 : V];
    if constexpr (!kWide) {
#pragma unroll
        for (int k = 0; k < V; ++k) gain[k] = gain_of(k);
    }
    const int own = own_vector<V>(at.lane), own_col = at.col0 - 8 * (at.lane & 15) + own * at.apart;
    float *ps = FMT != SNIP_FMT_BF16 && own_col < a.cols && (at.lane & (16 / V - 1)) == 0 ? a.scales + (int64_t)(own_col >> 7) * a.rows + row0 : nullptr;
    uint8_t *pc = FMT == SNIP_FMT_BF16 ? nullptr : a.codes + ((int64_t)row0 * a.cols + at.col0) / kPerByte;
    const int64_t dc = (int64_t)step * a.cols / kPerByte;
    uint16_t *ph = RES ? a.h + (int64_t)row0 * a.ld_h + at.col0 : nullptr;
    const int64_t dh = RES ? (int64_t)step * a.ld_h : 0;
    int64_t row = row0;
    int parity = 0;
    auto turn = [&](auto which) {
        constexpr int kStage = decltype(which)::value;
        fetch(kStage == 0 ? STAGES - 1 : kStage - 1);
        copies_wait<STAGES - 1>();
        const bool live = row < a.rows;
        Eight h[kWide ? 1 : V];
        uint4 packed[V];
        float2 sum = splat(0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            packed[k] = *slot(kStage, 0, k);
            Eight e = unpack8(packed[k]);
            if (RES) {
                const Eight q = unpack8(*slot(kStage, 1, k));
#pragma unroll
                for (int i = 0; i < 4; ++i) e.p[i] = __fadd2_rn(e.p[i], q.p[i]);
                packed[k] = pack8(e);
                if (live && in[k]) *reinterpret_cast<uint4 *>(ph + k * at.apart) = packed[k];
                e = unpack8(packed[k]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = __ffma2_rn(e.p[i], e.p[i], sum);
            if constexpr (!kWide) h[k] = e;
        }
        const float total = group_sum(sum.x + sum.y, slots[parity], at, a.wpr);
        const float rstd = rsqrtf(fmaf(total, a.inv_cols, a.eps));
        if (at.col0 == 0 && a.rstd && live) a.rstd[row] = rstd;
        if (FMT != SNIP_FMT_BF16 || a.y) {
            Eight y[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if constexpr (kWide) y[k] = scaled8(unpack8(packed[k]), rstd, gain_of(k));
                else y[k] = scaled8(h[k], rstd, gain[k]);
            }
            if (a.y && live) {
                uint16_t *py = a.y + row * a.ld_y + at.col0;
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (in[k]) *reinterpret_cast<uint4 *>(py + k * at.apart) = pack8(y[k]);
            }
            if constexpr (FMT != SNIP_FMT_BF16) {
                float most[V], s[V];
#pragma unroll
                for (int k = 0; k < V; ++k) most[k] = most8(y[k]);
                const float one = tile_scales<FMT, V>(most, s, at.lane);
                if (live) {
                    if (ps) *ps = one;
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if (in[k]) store_codes8<FMT>(pc + k * at.apart / kPerByte, y[k], s[k]);
                }
                if (ps) ps += step;
                pc += dc;
            }
        }
        row += step;
        if (RES) ph += dh;
        parity ^= 1;
    };
    // all groups of a CTA take the same number of turns: nothing is written for rows behind the last
    for (int64_t base = first; base < a.rows;) {
        turn(Int<0>{});
        if constexpr (STAGES > 1) {
            if ((base += step) >= a.rows) break;
            turn(Int<1>{});
        }
        if constexpr (STAGES > 2) {
            if ((base += step) >= a.rows) break;
            turn(Int<2>{});
        }
        base += step;
    }
    copies_wait<0>();
}

// Both quantized copies of y from h and rstd: 128x128 tiles, a thread owns 8x8 elements of one (dimensions are multiples of 64: all of
// them or none).  Rows' maxima are combined over the 16 threads of a row group, columns' over the 16 row groups; the transposed codes
// leave through shared memory.
struct NormDualArgs {
    const uint16_t *h;
    const void *gain;
    const float *rstd;
    uint8_t *codes, *codes_t;
    float *scales, *scales_t;
    int32_t rows, cols, tiles_c, tiles, ld;
    int gain_f32;
};
constexpr int kTile = 128;
constexpr int kDualThreads = 256;
constexpr int kDualCtas = 3;

struct DualShared {
    uint4 slot[8][kDualThreads];                 // the thread's own eight vectors of eight elements
    __align__(16) uint8_t stage[kTile * kTile];  // transposed codes
    float col_max[8][kTile];
    float col_scale[kTile];
    float row_scale[kTile];
};

// FMT: format of the row-tile codes (BF16: none), FMT_T: of the transposed ones.
template <int FMT, int FMT_T>
__global__ void __launch_bounds__(kDualThreads, kDualCtas) rmsnorm_dual_kernel(const NormDualArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    DualShared &m = *reinterpret_cast<DualShared *>(raw);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31, warp = tid >> 5;
    // row and column of the tile, moved on without a division
    const int step_r = (int)gridDim.x / a.tiles_c, step_c = (int)gridDim.x % a.tiles_c;
    auto advance = [&](int &r, int &c) {
        r += step_r;
        c += step_c;
        if (c >= a.tiles_c) { c -= a.tiles_c; ++r; }
    };
    auto fetch = [&](int tile, int r, int c) {
        if (tile < a.tiles && r * kTile + 8 * ty < a.rows && c * kTile + 8 * tx < a.cols) {
            const uint16_t *p = a.h + (int64_t)(r * kTile + 8 * ty) * a.ld + c * kTile + 8 * tx;
#pragma unroll
            for (int i = 0; i < 8; ++i) copy_async(&m.slot[i][tid], p + (int64_t)i * a.ld);
        }
        copies_commit();
    };
    asm volatile("griddepcontrol.wait;" ::: "memory");   // for the kernel that leaves h and rstd
    int tr = (int)blockIdx.x / a.tiles_c, tc = (int)blockIdx.x % a.tiles_c;
    fetch((int)blockIdx.x, tr, tc);
    for (int tile = (int)blockIdx.x; tile < a.tiles; tile += (int)gridDim.x) {
        int next_r = tr, next_c = tc;
        advance(next_r, next_c);
        const int row0 = tr * kTile + 8 * ty, col0 = tc * kTile + 8 * tx;
        const bool ok = row0 < a.rows && col0 < a.cols;
        Eight gain = zeros8();
        float rstd[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rstd[i] = 0.0f;
        if (ok) {
            gain = load_gain8(a.gain, a.gain_f32, col0);
            const float4 p = __ldcg(reinterpret_cast<const float4 *>(a.rstd + row0)), q = __ldcg(reinterpret_cast<const float4 *>(a.rstd + row0) + 1);
            rstd[0] = p.x; rstd[1] = p.y; rstd[2] = p.z; rstd[3] = p.w; rstd[4] = q.x; rstd[5] = q.y; rstd[6] = q.z; rstd[7] = q.w;
        }
        copies_wait<0>();
        float rmax[8], cmax[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rmax[i] = cmax[i] = 0.0f;
        if (ok) {   // (the slots of what a ragged tile lacks hold anything)
#pragma unroll
        for (int p = 0; p < 8; p += 2) {
            const Eight y0 = scaled8(unpack8(m.slot[p][tid]), rstd[p], gain), y1 = scaled8(unpack8(m.slot[p + 1][tid]), rstd[p + 1], gain);
            rmax[p] = most8(y0);
            rmax[p + 1] = most8(y1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                cmax[2 * i] = fmaxf(fmaxf(cmax[2 * i], fabsf(y0.p[i].x)), fabsf(y1.p[i].x));
                cmax[2 * i + 1] = fmaxf(fmaxf(cmax[2 * i + 1], fabsf(y0.p[i].y)), fabsf(y1.p[i].y));
            }
        }
        }
        if constexpr (FMT != SNIP_FMT_BF16) {
            // rows: each step halves the number of rows a lane still looks after; lanes 2 q and 2 q + 1 of a half-warp end with row q's maximum
#pragma unroll
            for (int w = 4, off = 8; w > 0; w >>= 1, off >>= 1) {
                const bool upper = (lane & off) != 0;
#pragma unroll
                for (int i = 0; i < w; ++i) {
                    const float give = upper ? rmax[i] : rmax[i + w], keep = upper ? rmax[i + w] : rmax[i];
                    rmax[i] = fmaxf(keep, __shfl_xor_sync(0xFFFFFFFFu, give, off));
                }
            }
            rmax[0] = fmaxf(rmax[0], __shfl_xor_sync(0xFFFFFFFFu, rmax[0], 1));
            if ((lane & 1) == 0) {
                const float s = tile_scale<FMT>(rmax[0], 0);
                const int r = 8 * ty + ((lane >> 1) & 7), row = tr * kTile + r;
                m.row_scale[r] = s;
                if (row < a.rows) a.scales[(int64_t)tc * a.rows + row] = s;
            }
        }
        // columns
#pragma unroll
        for (int i = 0; i < 8; ++i) cmax[i] = fmaxf(cmax[i], __shfl_xor_sync(0xFFFFFFFFu, cmax[i], 16));
        if (lane < 16) {
            *reinterpret_cast<float4 *>(&m.col_max[warp][8 * tx]) = make_float4(cmax[0], cmax[1], cmax[2], cmax[3]);
            *reinterpret_cast<float4 *>(&m.col_max[warp][8 * tx + 4]) = make_float4(cmax[4], cmax[5], cmax[6], cmax[7]);
        }
        __syncthreads();   // also: the previous tile's codes have left the stage
        if (tid < kTile) {
            float v = m.col_max[0][tid];
#pragma unroll
            for (int w = 1; w < 8; ++w) v = fmaxf(v, m.col_max[w][tid]);
            const float s = tile_scale<FMT_T>(v, 0);
            m.col_scale[tid] = s;
            const int col = tc * kTile + tid;
            if (col < a.cols) a.scales_t[(int64_t)tr * a.cols + col] = s;
        }
        __syncthreads();
        Eight cs;
        {
            const float4 p = *reinterpret_cast<const float4 *>(&m.col_scale[8 * tx]), q = *reinterpret_cast<const float4 *>(&m.col_scale[8 * tx + 4]);
            cs = {{make_float2(p.x, p.y), make_float2(p.z, p.w), make_float2(q.x, q.y), make_float2(q.z, q.w)}};
        }
        const int line = FMT == SNIP_FMT_FP4_E2M1 ? a.cols >> 1 : a.cols;
        uint8_t *pc = FMT == SNIP_FMT_BF16 ? nullptr : a.codes + (int64_t)row0 * line + (FMT == SNIP_FMT_FP4_E2M1 ? col0 >> 1 : col0);
        uint32_t ct[8][2];   // column i: codes of its eight rows (FP4: the first word)
#pragma unroll
        for (int p = 0; p < 8; p += 4) {
            uint32_t part[2][8];
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                Eight y[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const int r = p + e + f;
                    y[f] = scaled8(unpack8(m.slot[r][tid]), rstd[r], gain);
                    if constexpr (FMT != SNIP_FMT_BF16)
                        if (ok) store_codes8<FMT>(pc + (int64_t)r * line, y[f], m.row_scale[8 * ty + r]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 t0 = __fmul2_rn(y[0].p[i], cs.p[i]), t1 = __fmul2_rn(y[1].p[i], cs.p[i]);
                    if constexpr (FMT_T == SNIP_FMT_FP8_E4M3) {
                        part[e >> 1][2 * i] = cvt_e4m3x2(t0.x, t1.x);
                        part[e >> 1][2 * i + 1] = cvt_e4m3x2(t0.y, t1.y);
                    } else {
                        part[e >> 1][2 * i] = cvt_e2m1x2(t0.x, t1.x);
                        part[e >> 1][2 * i + 1] = cvt_e2m1x2(t0.y, t1.y);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (FMT_T == SNIP_FMT_FP8_E4M3) ct[i][p >> 2] = __byte_perm(part[0][i], part[1][i], 0x5410);
                else ct[i][p >> 2] = __byte_perm(part[0][i], part[1][i], 0x0040);   // two bytes
            }
        }
        fetch(tile + (int)gridDim.x, next_r, next_c);   // the slot has been read
        // transposed codes: line = column of the tile, 128 (64) bytes each; 16-byte pieces swizzled by the line so that neither side conflicts
        constexpr bool kFp8T = FMT_T == SNIP_FMT_FP8_E4M3;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int to = 8 * tx + i;
            if constexpr (kFp8T) *reinterpret_cast<uint2 *>(&m.stage[to * 128 + ((ty >> 1) ^ (tx & 7)) * 16 + (ty & 1) * 8]) = make_uint2(ct[i][0], ct[i][1]);
            else *reinterpret_cast<uint32_t *>(&m.stage[to * 64 + ((ty >> 2) ^ (tx & 3)) * 16 + (ty & 3) * 4]) = __byte_perm(ct[i][0], ct[i][1], 0x5410);
        }
        __syncthreads();
        constexpr int kPieces = kFp8T ? 8 : 4, kRows = kFp8T ? 16 : 32;   // 16-byte pieces of a line, rows in one
#pragma unroll
        for (int j = 0; j < kTile * kPieces / kDualThreads; ++j) {
            const int from = (j * kDualThreads + tid) / kPieces, piece = tid % kPieces;
            const int row = tr * kTile + piece * kRows, col = tc * kTile + from;
            if (col >= a.cols || row >= a.rows) continue;
            const int64_t elem = (int64_t)col * a.rows + row;
            *reinterpret_cast<uint4 *>(a.codes_t + (kFp8T ? elem : elem / 2)) =
                *reinterpret_cast<const uint4 *>(&m.stage[from * (16 * kPieces) + (piece ^ ((from >> 3) & (kPieces - 1))) * 16]);
        }
        tr = next_r;
        tc = next_c;
    }
    copies_wait<0>();
}

template <int V, int THREADS, int STAGES, bool RES>
__global__ void __launch_bounds__(THREADS) rmsnorm_bwd_kernel(const NormBwdArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    __shared__ __align__(16) float slots[2][32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the reduction of the gain's gradient, which waits for this kernel
    const Place at(a.wpr);
    bool in[V];
#pragma unroll
    for (int k = 0; k < V; ++k) in[k] = at.col0 + k * at.apart < a.cols;
    const Ring<V, RES ? 3 : 2, STAGES> ring(raw, in);
    if (threadIdx.x < 64) slots[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
    __syncthreads();
    const int step = (int)gridDim.x * at.groups, first = (int)blockIdx.x * at.groups, row0 = first + at.group;
    const uint16_t *py = a.dy + (int64_t)row0 * a.ld_dy + at.col0, *ph = a.h + (int64_t)row0 * a.ld_h + at.col0;
    const uint16_t *pd = RES ? a.dresidual + (int64_t)row0 * a.ld_dresidual + at.col0 : nullptr;
    const int64_t sy = (int64_t)step * a.ld_dy, sh = (int64_t)step * a.ld_h, sd = RES ? (int64_t)step * a.ld_dresidual : 0;
    int64_t ahead = row0;
    auto fetch = [&](int stage) {
        if (ahead < a.rows) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (in[k]) {
                    copy_async(ring.slot(stage, 0, k), py + k * at.apart);
                    copy_async(ring.slot(stage, 1, k), ph + k * at.apart);
                    if (RES) copy_async(ring.slot(stage, 2, k), pd + k * at.apart);
                }
        }
        copies_commit();
        ahead += step;
        py += sy;
        ph += sh;
        if (RES) pd += sd;
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(i);
    // of the widest rows neither the gain nor the products stay in registers
    constexpr bool kWide = V > 2;
    auto gain_of = [&](int k) { return in[k] ? load_gain8(a.gain, a.gain_f32, at.col0 + k * at.apart) : zeros8(); };
    Eight gain[kWide ? 1 : V], dgain[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if constexpr (!kWide) gain[k] = gain_of(k);
        dgain[k] = zeros8();
    }
    int64_t row = row0;
    float rstd = row < a.rows ? __ldg(a.rstd + row) : 0.0f;
    uint16_t *px = a.dx + (int64_t)row0 * a.ld_dx + at.col0;
    const int64_t sx = (int64_t)step * a.ld_dx;
    int parity = 0, stage = 0;
    for (int64_t base = first; base < a.rows; base += step, parity ^= 1) {
        fetch(stage == 0 ? STAGES - 1 : stage - 1);
        copies_wait<STAGES - 1>();
        const bool live = row < a.rows;
        Eight g[kWide ? 1 : V], u[kWide ? 1 : V];   // dy gain, h rstd
        float2 dot = splat(0.0f);
        const float r = rstd;
        if (live) {   // (a group behind the last row: nothing has been fetched, nothing may be added)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                Eight &gk = g[kWide ? 0 : k], &uk = u[kWide ? 0 : k];
                gk = unpack8(*ring.slot(stage, 0, k));
                uk = unpack8(*ring.slot(stage, 1, k));
                const Eight w = kWide ? gain_of(k) : gain[kWide ? 0 : k];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uk.p[i] = __fmul2_rn(uk.p[i], splat(r));
                    dgain[k].p[i] = __ffma2_rn(gk.p[i], uk.p[i], dgain[k].p[i]);
                    gk.p[i] = __fmul2_rn(gk.p[i], w.p[i]);
                    dot = __ffma2_rn(gk.p[i], uk.p[i], dot);
                }
            }
        }
        row += step;
        if (row < a.rows) rstd = __ldg(a.rstd + row);
        const float c = group_sum(dot.x + dot.y, slots[parity], at, a.wpr) * -a.inv_cols;
        if (live) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (!in[k]) continue;
                Eight q;
                if (RES) q = unpack8(*ring.slot(stage, 2, k));
                Eight &gk = g[kWide ? 0 : k], &uk = u[kWide ? 0 : k];
                if constexpr (kWide) {
                    gk = unpack8(*ring.slot(stage, 0, k));
                    uk = unpack8(*ring.slot(stage, 1, k));
                    const Eight w = gain_of(k);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uk.p[i] = __fmul2_rn(uk.p[i], splat(r));
                        gk.p[i] = __fmul2_rn(gk.p[i], w.p[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 e = __ffma2_rn(uk.p[i], splat(c), gk.p[i]);
                    q.p[i] = RES ? __ffma2_rn(splat(r), e, q.p[i]) : __fmul2_rn(splat(r), e);
                }
                *reinterpret_cast<uint4 *>(px + k * at.apart) = pack8(q);
            }
        }
        px += sx;
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    copies_wait<0>();
    if (a.partials) {
        float *p = a.partials + (int64_t)row0 * a.cols + at.col0;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (!in[k]) continue;
            float4 *q = reinterpret_cast<float4 *>(p + k * at.apart);
            q[0] = make_float4(dgain[k].p[0].x, dgain[k].p[0].y, dgain[k].p[1].x, dgain[k].p[1].y);
            q[1] = make_float4(dgain[k].p[2].x, dgain[k].p[2].y, dgain[k].p[3].x, dgain[k].p[3].y);
        }
    }
}

// dgain[c] (+)= sum of the partials of column c, in a fixed order: 32 threads of a column take every 32nd partial each and are added in order.
__global__ void __launch_bounds__(1024) dgain_reduce_kernel(const float *partials, int n, int cols, float *dgain, int accumulate)
{
    __shared__ float part[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = blockIdx.x * 32 + threadIdx.x;
    float v = 0.0f;
    if (c < cols)
        for (int i = threadIdx.y; i < n; i += 32) v += partials[(int64_t)i * cols + c];
    part[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && c < cols) {
        v = part[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 32; ++i) v += part[i][threadIdx.x];
        dgain[c] = accumulate ? dgain[c] + v : v;
    }
}

// How rows of `cols` elements are dealt to threads: vectors per thread, warps per row, rows side by side, stages of the ring.
struct Shape {
    int v, wpr, groups, stages, smem, threads, form;
};
// Forward: CTAs of fixed sizes, as F(form, V, threads, stages).
#define SNIP_NORM_FWD_FORMS(F) F(0, 1, 256, 3) F(1, 1, 512, 3) F(2, 1, 1024, 3) F(3, 2, 256, 3) F(4, 2, 512, 3) F(5, 4, 512, 2) F(6, 4, 1024, 1) F(7, 4, 256, 2)
// More vectors per thread spread what a row costs over more elements; fewer leave more threads to fetch.  16384 x 4096 with two / four vectors in us:
// residual added 65.3 / 63.4, and y written 91.8 / 89.4, and FP8 codes 83.0 / 83.1 (8192 x 8192: 79.7 / 83.1); no residual: rstd alone 21.5 / 23.8,
// y 47.5 / 43.7, codes 41.6 / 37.9.  2048 columns: 21.3 / 22.2.
Shape fwd_shape(int64_t cols, bool residual, bool y, bool codes, bool few)
{
    Shape s;
    const bool four = cols > 2048 && (residual ? !codes : codes || y);
    s.v = cols > 8192 ? 4 : few ? 1 : four ? 4 : 2;
    s.wpr = (int)ceil_div(cols, 256 * s.v);
    s.threads = s.wpr <= 8 ? 256 : s.wpr <= 16 ? 512 : 1024;
    s.groups = s.threads / 32 / s.wpr;
    s.form = s.v == 1 ? (s.threads == 256 ? 0 : s.threads == 512 ? 1 : 2) : s.v == 2 ? (s.threads == 256 ? 3 : 4) : s.threads == 512 ? 5 : s.threads == 1024 ? 6 : 7;
    s.stages = s.form < 5 ? 3 : s.form == 6 ? 1 : 2;
    s.smem = s.stages * (residual ? 2 : 1) * s.v * s.threads * 16;   // at most 128 KB
    return s;
}
// Backward: as F(form, V, most threads, stages).
#define SNIP_NORM_BWD_FORMS(F) F(0, 1, 1024, 3) F(1, 2, 512, 3) F(2, 2, 512, 2) F(3, 4, 512, 2) F(4, 4, 1024, 1)
Shape bwd_shape(int64_t cols, int arrays, bool few)
{
    Shape s;
    s.v = cols > 8192 ? 4 : few ? 1 : 2;
    s.wpr = (int)ceil_div(cols, 256 * s.v);
    s.groups = s.wpr >= 8 ? 1 : 8 / s.wpr;
    s.threads = 32 * s.wpr * s.groups;
    const int row_bytes = arrays * s.v * s.threads * 16;
    s.form = s.v == 4 ? (s.threads > 512 ? 4 : 3) : s.v == 1 ? 0 : row_bytes <= 32 * 1024 ? 1 : 2;
    s.stages = s.form == 4 ? 1 : s.form < 2 ? 3 : 2;
    s.smem = s.stages * row_bytes;   // at most 192 KB
    return s;
}
constexpr int64_t kFewRows = 296;

// CTAs of a kernel that an SM holds, with its dynamic shared memory allowed for (asked once: the same on every device of this family; the
// allowance is per device).
template <auto Kernel>
int resident(int threads, int smem, int most_smem)
{
    static std::atomic<uint64_t> allowed{0};   // a bit per device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) || dev > 63) {
        if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem) != cudaSuccess) return 0;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    // by threads: the shared memory goes with them
    static std::atomic<int> known[33];
    int n = known[threads / 32].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, threads, smem) != cudaSuccess || n < 1) return 0;
        known[threads / 32].store(n, std::memory_order_relaxed);
    }
    return n;
}

bool bad_ld(int64_t ld, int64_t cols) { return ld < cols || (ld % 8) != 0 || ld > INT32_MAX; }
bool bad_dims(int64_t rows, int64_t cols) { return rows < 0 || rows > INT32_MAX - 128 || cols <= 0 || (cols % 8) != 0 || cols > kMaxCols; }


constexpr int kMostSmem = 200 * 1024;

// CTAs of the backward pass (each group of rows leaves one partial of dgain).  kBwdCtas bounds the workspace.
constexpr int64_t kBwdCtas = 8 * 148;
int64_t bwd_ctas(int64_t rows, int groups, int per_sm)
{
    const int64_t want = ceil_div(rows, groups), fit = (int64_t)per_sm * gemm_sm_count(), cap = fit < kBwdCtas ? fit : kBwdCtas;
    return want < cap ? want : cap;
}

// A kernel that may be set up while the one before it on the stream ends; it waits for that one's results itself.
template <typename Kernel, typename... Args>
cudaError_t launch_behind(Kernel kernel, dim3 grid, dim3 block, int smem, cudaStream_t st, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace
}  // namespace snip

extern "C" int snip_rmsnorm_fwd(const snip_rmsnorm_t *t, void *stream)
{
    using namespace snip;
    if (!t || (t->gain_dtype != SNIP_OUT_BF16 && t->gain_dtype != SNIP_OUT_FP32)) return SNIP_ERR_ARG;
    if (!(t->eps > 0.0f) || !(t->eps <= FLT_MAX)) return SNIP_ERR_ARG;
    if (bad_dims(t->rows, t->cols)) return SNIP_ERR_SHAPE;
    if (t->rows == 0) return SNIP_OK;   // matrices without rows have no addresses to check
    if (!t->x || !t->gain) return SNIP_ERR_ARG;
    if (!t->y && !t->codes && !t->codes_t && !t->h && !t->rstd) return SNIP_ERR_ARG;
    if ((t->residual != nullptr) != (t->h != nullptr)) return SNIP_ERR_ARG;
    if ((t->codes != nullptr) != (t->scales != nullptr) || (t->codes_t != nullptr) != (t->scales_t != nullptr)) return SNIP_ERR_ARG;
    if (t->codes && t->fmt != SNIP_FMT_FP8_E4M3 && t->fmt != SNIP_FMT_FP4_E2M1) return SNIP_ERR_ARG;
    if (t->codes_t && ((t->fmt_t != SNIP_FMT_FP8_E4M3 && t->fmt_t != SNIP_FMT_FP4_E2M1) || !t->rstd)) return SNIP_ERR_ARG;
    if (t->codes_t && ((t->rows % 64) != 0 || (t->cols % 64) != 0)) return SNIP_ERR_SHAPE;
    if (t->codes_t && ceil_div(t->rows, kTile) * ceil_div(t->cols, kTile) > INT32_MAX / 2) return SNIP_ERR_SHAPE;   // tiles are counted in 32 bits
    if (bad_ld(t->ld_x, t->cols) || (t->residual && (bad_ld(t->ld_residual, t->cols) || bad_ld(t->ld_h, t->cols))) || (t->y && bad_ld(t->ld_y, t->cols))) return SNIP_ERR_SHAPE;
    const void *all[] = {t->x, t->residual, t->gain, t->h, t->y, t->rstd, t->codes, t->scales, t->codes_t, t->scales_t};
    for (const void *p : all)
        if (!aligned16(p)) return SNIP_ERR_ALIGN;
    int rc = require_sm100();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool dual = t->codes_t != nullptr;
    NormArgs a = {};
    a.x = static_cast<const uint16_t *>(t->x);
    a.residual = static_cast<const uint16_t *>(t->residual);
    a.gain = t->gain;
    a.h = static_cast<uint16_t *>(t->h);
    a.y = static_cast<uint16_t *>(t->y);
    a.rstd = t->rstd;
    a.codes = dual ? nullptr : static_cast<uint8_t *>(t->codes);
    a.scales = t->scales;
    a.ld_x = (int32_t)t->ld_x; a.ld_residual = (int32_t)t->ld_residual; a.ld_h = (int32_t)t->ld_h; a.ld_y = (int32_t)t->ld_y;
    a.rows = (int32_t)t->rows;
    a.cols = (int32_t)t->cols;
    a.gain_f32 = t->gain_dtype == SNIP_OUT_FP32;
    a.eps = t->eps;
    a.inv_cols = (float)(1.0 / (double)t->cols);
    const Shape s = fwd_shape(t->cols, t->residual != nullptr, t->y != nullptr, a.codes != nullptr, t->rows <= kFewRows);
    a.wpr = s.wpr;
    int n = 0;   // 0: a CUDA call failed
    auto launch = [&](auto v, auto threads, auto stages, auto res, auto fmt) {
        constexpr auto kernel = rmsnorm_kernel<v(), threads(), stages(), res(), fmt()>;
        n = resident<kernel>(s.threads, s.smem, kMostSmem);
        const int64_t want = ceil_div(t->rows, s.groups), cap = (int64_t)n * gemm_sm_count();
        if (n) kernel<<<(unsigned)(want < cap ? want : cap), s.threads, s.smem, st>>>(a);
    };
    auto with_fmt = [&](auto v, auto threads, auto stages, auto res) {
        if (!a.codes) launch(v, threads, stages, res, Int<SNIP_FMT_BF16>{});
        else if (t->fmt == SNIP_FMT_FP8_E4M3) launch(v, threads, stages, res, Int<SNIP_FMT_FP8_E4M3>{});
        else launch(v, threads, stages, res, Int<SNIP_FMT_FP4_E2M1>{});
    };
#define SNIP_LAUNCH(FORM, V, THREADS, STAGES)                                                   \
    if (s.form == FORM) {                                                                       \
        if (t->residual) with_fmt(Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::true_type{});   \
        else with_fmt(Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::false_type{});              \
    }
    SNIP_NORM_FWD_FORMS(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(cudaGetLastError());
    if (!n) return SNIP_ERR_CUDA;
    if (!dual) return SNIP_OK;
    NormDualArgs d = {};
    d.h = static_cast<const uint16_t *>(t->residual ? t->h : t->x);
    d.gain = t->gain;
    d.rstd = t->rstd;
    d.codes = static_cast<uint8_t *>(t->codes);
    d.scales = t->scales;
    d.codes_t = static_cast<uint8_t *>(t->codes_t);
    d.scales_t = t->scales_t;
    d.ld = (int32_t)(t->residual ? t->ld_h : t->ld_x);
    d.rows = a.rows; d.cols = a.cols;
    d.tiles_c = (int32_t)ceil_div(t->cols, kTile);
    d.tiles = (int32_t)(d.tiles_c * ceil_div(t->rows, kTile));
    d.gain_f32 = a.gain_f32;
    cudaError_t e = cudaSuccess;
    auto launch_dual = [&](auto fmt, auto fmt_t) {
        constexpr auto kernel = rmsnorm_dual_kernel<fmt(), fmt_t()>;
        constexpr int smem = (int)sizeof(DualShared);
        n = resident<kernel>(kDualThreads, smem, smem);
        const int64_t cap = (int64_t)n * gemm_sm_count();
        if (n) e = launch_behind(kernel, dim3((unsigned)(d.tiles < cap ? d.tiles : cap)), dim3(kDualThreads), smem, st, d);
    };
    auto with_fmt_t = [&](auto fmt) {
        if (t->fmt_t == SNIP_FMT_FP8_E4M3) launch_dual(fmt, Int<SNIP_FMT_FP8_E4M3>{});
        else launch_dual(fmt, Int<SNIP_FMT_FP4_E2M1>{});
    };
    if (!d.codes) with_fmt_t(Int<SNIP_FMT_BF16>{});
    else if (t->fmt == SNIP_FMT_FP8_E4M3) with_fmt_t(Int<SNIP_FMT_FP8_E4M3>{});
    else with_fmt_t(Int<SNIP_FMT_FP4_E2M1>{});
    SNIP_CUDA_TRY(e);
    return n ? SNIP_OK : SNIP_ERR_CUDA;
}

extern "C" int snip_rmsnorm_bwd_workspace(int64_t rows, int64_t cols, size_t *ws_bytes)
{
    using namespace snip;
    if (!ws_bytes) return SNIP_ERR_ARG;
    if (bad_dims(rows, cols)) return SNIP_ERR_SHAPE;
    // one partial per group of rows in flight, of the largest grid
    const Shape s = bwd_shape(cols, 3, rows <= kFewRows);
    int64_t groups = kBwdCtas * s.groups;
    if (rows < groups) groups = align_up((size_t)rows, (size_t)s.groups);
    *ws_bytes = align_up(sizeof(float) * (size_t)groups * (size_t)cols, 256);
    return SNIP_OK;
}

extern "C" int snip_rmsnorm_bwd(const snip_rmsnorm_bwd_t *t, void *ws, size_t ws_bytes, void *stream)
{
    using namespace snip;
    if (!t || (t->gain_dtype != SNIP_OUT_BF16 && t->gain_dtype != SNIP_OUT_FP32)) return SNIP_ERR_ARG;
    if (bad_dims(t->rows, t->cols)) return SNIP_ERR_SHAPE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (t->rows == 0) {   // matrices without rows have no addresses to check
        if (!t->dgain || t->accumulate) return SNIP_OK;
        if (!aligned16(t->dgain)) return SNIP_ERR_ALIGN;
        int rc = require_sm100();
        if (rc) return rc;
        SNIP_CUDA_TRY(cudaMemsetAsync(t->dgain, 0, sizeof(float) * (size_t)t->cols, st));
        return SNIP_OK;
    }
    if (!t->dy || !t->h || !t->gain || !t->rstd || !t->dx) return SNIP_ERR_ARG;
    if (bad_ld(t->ld_dy, t->cols) || bad_ld(t->ld_h, t->cols) || bad_ld(t->ld_dx, t->cols) || (t->dresidual && bad_ld(t->ld_dresidual, t->cols))) return SNIP_ERR_SHAPE;
    const void *all[] = {t->dy, t->h, t->gain, t->rstd, t->dresidual, t->dx, t->dgain, t->dgain ? ws : nullptr};
    for (const void *p : all)
        if (!aligned16(p)) return SNIP_ERR_ALIGN;
    if (t->dgain) {
        size_t need = 0;
        int rc = snip_rmsnorm_bwd_workspace(t->rows, t->cols, &need);
        if (rc) return rc;
        if (!ws || ws_bytes < need) return SNIP_ERR_WORKSPACE;
    }
    int rc = require_sm100();
    if (rc) return rc;
    NormBwdArgs a = {};
    a.dy = static_cast<const uint16_t *>(t->dy);
    a.h = static_cast<const uint16_t *>(t->h);
    a.dresidual = static_cast<const uint16_t *>(t->dresidual);
    a.gain = t->gain;
    a.rstd = t->rstd;
    a.dx = static_cast<uint16_t *>(t->dx);
    a.partials = t->dgain ? static_cast<float *>(ws) : nullptr;
    a.ld_dy = (int32_t)t->ld_dy; a.ld_h = (int32_t)t->ld_h; a.ld_dresidual = (int32_t)t->ld_dresidual; a.ld_dx = (int32_t)t->ld_dx;
    a.rows = (int32_t)t->rows;
    a.cols = (int32_t)t->cols;
    a.gain_f32 = t->gain_dtype == SNIP_OUT_FP32;
    a.inv_cols = (float)(1.0 / (double)t->cols);
    const Shape s = bwd_shape(t->cols, t->dresidual ? 3 : 2, t->rows <= kFewRows);
    a.wpr = s.wpr;
    int64_t ctas = 0;   // 0: a CUDA call failed
    auto launch = [&](auto v, auto threads, auto stages, auto res) {
        constexpr auto kernel = rmsnorm_bwd_kernel<v(), threads(), stages(), res()>;
        ctas = bwd_ctas(t->rows, s.groups, resident<kernel>(s.threads, s.smem, kMostSmem));
        if (ctas) kernel<<<(unsigned)ctas, s.threads, s.smem, st>>>(a);
    };
#define SNIP_LAUNCH(FORM, V, THREADS, STAGES)                                                   \
    if (s.form == FORM) {                                                                       \
        if (t->dresidual) launch(Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::true_type{});    \
        else launch(Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::false_type{});                \
    }
    SNIP_NORM_BWD_FORMS(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(cudaGetLastError());
    if (!ctas) return SNIP_ERR_CUDA;
    if (t->dgain) {
        SNIP_CUDA_TRY(launch_behind(dgain_reduce_kernel, dim3((unsigned)ceil_div(t->cols, 32)), dim3(32, 32), 0, st, static_cast<const float *>(a.partials),
                                    (int)(ctas * s.groups), (int)a.cols, t->dgain, (int)t->accumulate));
    }
    return SNIP_OK;
}
