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

struct NormArgs {
    const uint16_t *x, *residual;
    const void *gain;
    uint16_t *h, *y;
    float *rstd;
    uint8_t *codes;
    float *scales;
    int64_t ld_x, ld_residual, ld_h, ld_y;
    int32_t rows, cols;
    int gain_f32;
    float eps, inv_cols;
};

struct NormBwdArgs {
    const uint16_t *dy, *h, *dresidual;
    const void *gain;
    const float *rstd;
    uint16_t *dx;
    float *partials;   // [groups of the grid][cols], or null
    int64_t ld_dy, ld_h, ld_dresidual, ld_dx;
    int32_t rows, cols;
    int gain_f32;
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
__device__ __forceinline__ void store_codes8(uint8_t *codes, int64_t at, const Eight &y, float s)
{
    float2 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __fmul2_rn(y.p[i], splat(s));
    if constexpr (FMT == SNIP_FMT_FP8_E4M3) {
        *reinterpret_cast<uint2 *>(codes + at) = make_uint2(__byte_perm(cvt_e4m3x2(t[0].x, t[0].y), cvt_e4m3x2(t[1].x, t[1].y), 0x5410),
                                                            __byte_perm(cvt_e4m3x2(t[2].x, t[2].y), cvt_e4m3x2(t[3].x, t[3].y), 0x5410));
    } else {
        *reinterpret_cast<uint32_t *>(codes + at / 2) = cvt_e2m1x2(t[0].x, t[0].y) | cvt_e2m1x2(t[1].x, t[1].y) << 8 | cvt_e2m1x2(t[2].x, t[2].y) << 16 |
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

// 16 bytes into this thread's own slot of shared memory (read back by itself: nothing to wait for but its own copies), or zeros.
__device__ __forceinline__ void copy_async(uint4 *slot, const uint16_t *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(slot)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sum over the WPR warps of a row group, in a fixed order; the same value in every thread.  `slots` (one float per warp of the CTA) is free again
// when all threads have come past the next call's barrier: callers alternate between two sets.
template <int WPR>
__device__ __forceinline__ float group_sum(float v, float *slots)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    if constexpr (WPR > 1) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) slots[warp] = v;
        __syncthreads();
        v = lane < WPR ? slots[warp / WPR * WPR + lane] : 0.0f;
#pragma unroll
        for (int off = WPR / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
        v = __shfl_sync(0xFFFFFFFFu, v, 0);
    }
    return v;
}

__host__ __device__ constexpr int cta_threads(int wpr) { return wpr < 8 ? 256 : 32 * wpr; }
__host__ __device__ constexpr int groups_per_cta(int wpr) { return cta_threads(wpr) / (32 * wpr); }

// Rows on their way: a thread's slots for kStages rows of N arrays of V vectors.
template <int WPR, int V, int N>
struct Ring {
    static constexpr int kRowBytes = N * V * cta_threads(WPR) * 16;
    static constexpr int kStages = kRowBytes > 100 * 1024 ? 1 : kRowBytes > 24 * 1024 ? 2 : kRowBytes > 12 * 1024 ? 3 : 4;
    static constexpr int kBytes = kStages * kRowBytes;
    static_assert(kBytes <= 224 * 1024, "an SM has 227 KB");
    uint4 *base;
    __device__ __forceinline__ uint4 *slot(int stage, int array, int k) const { return base + ((stage * N + array) * V + k) * cta_threads(WPR) + threadIdx.x; }
};

// WPR warps per row, V vectors of eight elements per thread: vector k of thread t of the group starts at column 8 (t + k 32 WPR), so
// that 16 neighbouring threads hold a 128-long tile.  FMT: format of the row-tile codes, BF16 for none.
template <int WPR, int V, bool RES, int FMT>
__global__ void __launch_bounds__(cta_threads(WPR)) rmsnorm_kernel(const NormArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ float slots[2][32];
    using R = Ring<WPR, V, RES ? 2 : 1>;
    const R ring = {reinterpret_cast<uint4 *>(raw)};
    constexpr int kGroups = groups_per_cta(WPR);
    const int t = threadIdx.x % (32 * WPR), group = threadIdx.x / (32 * WPR);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    auto fetch = [&](int stage, int64_t row) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            const bool there = col < a.cols && row < a.rows;
            copy_async(ring.slot(stage, 0, k), a.x + (there ? row * a.ld_x + col : 0), there);
            if (RES) copy_async(ring.slot(stage, 1, k), a.residual + (there ? row * a.ld_residual + col : 0), there);
        }
        copies_commit();
    };
    int64_t row = (int64_t)blockIdx.x * kGroups + group;
#pragma unroll
    for (int i = 0; i < R::kStages - 1; ++i) fetch(i, row + i * step);
    // of the widest rows neither the gain nor the row in binary32 stays in registers
    constexpr bool kWide = V > 2;
    Eight gain[kWide ? 1 : V];
    if constexpr (!kWide) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            gain[k] = col < a.cols ? load_gain8(a.gain, a.gain_f32, col) : zeros8();
        }
    }
    int parity = 0, stage = 0;
    // all groups of a CTA take the same number of turns: rows behind the last are zeros that nothing is written for
    for (int64_t base = (int64_t)blockIdx.x * kGroups; base < a.rows; base += step, row += step, parity ^= 1) {
        fetch(stage == 0 ? R::kStages - 1 : stage - 1, row + (R::kStages - 1) * step);
        copies_wait<R::kStages - 1>();
        Eight h[kWide ? 1 : V];
        uint4 packed[V];
        float2 sum = splat(0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            packed[k] = *ring.slot(stage, 0, k);
            Eight e = unpack8(packed[k]);
            if (RES) {
                const Eight q = unpack8(*ring.slot(stage, 1, k));
#pragma unroll
                for (int i = 0; i < 4; ++i) e.p[i] = __fadd2_rn(e.p[i], q.p[i]);
                packed[k] = pack8(e);
                if (col < a.cols && row < a.rows) *reinterpret_cast<uint4 *>(a.h + row * a.ld_h + col) = packed[k];
                e = unpack8(packed[k]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = __ffma2_rn(e.p[i], e.p[i], sum);
            if constexpr (!kWide) h[k] = e;
        }
        stage = stage == R::kStages - 1 ? 0 : stage + 1;
        const float total = group_sum<WPR>(sum.x + sum.y, slots[parity]);
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(total, a.inv_cols, a.eps)));
        if (t == 0 && a.rstd && row < a.rows) a.rstd[row] = rstd;
        if (FMT == SNIP_FMT_BF16 && !a.y) continue;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            const bool ok = col < a.cols && row < a.rows;
            Eight y;
            if constexpr (kWide) y = scaled8(unpack8(packed[k]), rstd, col < a.cols ? load_gain8(a.gain, a.gain_f32, col) : zeros8());
            else y = scaled8(h[k], rstd, gain[k]);
            if (a.y && ok) *reinterpret_cast<uint4 *>(a.y + row * a.ld_y + col) = pack8(y);
            if constexpr (FMT != SNIP_FMT_BF16) {
                float most = most8(y);
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, off));
                const float s = tile_scale<FMT>(most, 0);
                if (ok) {
                    if ((t & 15) == 0) a.scales[(int64_t)(col >> 7) * a.rows + row] = s;
                    store_codes8<FMT>(a.codes, row * a.cols + col, y, s);
                }
            }
        }
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
    int64_t ld;
    int32_t rows, cols, tiles_c;
    int64_t tiles;
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
    auto fetch = [&](int64_t tile) {
        const int64_t row = tile / a.tiles_c * kTile + 8 * ty, col = tile % a.tiles_c * kTile + 8 * tx;
        const bool ok = tile < a.tiles && row < a.rows && col < a.cols;
        const uint16_t *p = a.h + (ok ? row * a.ld + col : 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) copy_async(&m.slot[i][tid], p + (ok ? i * a.ld : 0), ok);
        copies_commit();
    };
    fetch(blockIdx.x);
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int tr = (int)(tile / a.tiles_c), tc = (int)(tile % a.tiles_c);
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
        for (int i = 0; i < 8; ++i) cmax[i] = 0.0f;
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
                        if (ok) store_codes8<FMT>(a.codes, (int64_t)(row0 + r) * a.cols + col0, y[f], m.row_scale[8 * ty + r]);
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
        fetch(tile + gridDim.x);   // the slot has been read
        // transposed codes: line = column of the tile, 128 (64) bytes each; 16-byte pieces swizzled by the line so that neither side conflicts
        constexpr bool kFp8T = FMT_T == SNIP_FMT_FP8_E4M3;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int line = 8 * tx + i;
            if constexpr (kFp8T) *reinterpret_cast<uint2 *>(&m.stage[line * 128 + ((ty >> 1) ^ (tx & 7)) * 16 + (ty & 1) * 8]) = make_uint2(ct[i][0], ct[i][1]);
            else *reinterpret_cast<uint32_t *>(&m.stage[line * 64 + ((ty >> 2) ^ (tx & 3)) * 16 + (ty & 3) * 4]) = __byte_perm(ct[i][0], ct[i][1], 0x5410);
        }
        __syncthreads();
        constexpr int kPieces = kFp8T ? 8 : 4, kRows = kFp8T ? 16 : 32;   // 16-byte pieces of a line, rows in one
#pragma unroll
        for (int j = 0; j < kTile * kPieces / kDualThreads; ++j) {
            const int line = (j * kDualThreads + tid) / kPieces, piece = tid % kPieces;
            const int row = tr * kTile + piece * kRows, col = tc * kTile + line;
            if (col >= a.cols || row >= a.rows) continue;
            const int64_t elem = (int64_t)col * a.rows + row;
            *reinterpret_cast<uint4 *>(a.codes_t + (kFp8T ? elem : elem / 2)) =
                *reinterpret_cast<const uint4 *>(&m.stage[line * (16 * kPieces) + (piece ^ ((line >> 3) & (kPieces - 1))) * 16]);
        }
    }
    copies_wait<0>();
}

template <int WPR, int V, bool RES>
__global__ void __launch_bounds__(cta_threads(WPR)) rmsnorm_bwd_kernel(const NormBwdArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ float slots[2][32];
    using R = Ring<WPR, V, RES ? 3 : 2>;
    const R ring = {reinterpret_cast<uint4 *>(raw)};
    constexpr int kGroups = groups_per_cta(WPR);
    const int t = threadIdx.x % (32 * WPR), group = threadIdx.x / (32 * WPR);
    const int64_t step = (int64_t)gridDim.x * kGroups, first = (int64_t)blockIdx.x * kGroups;
    auto fetch = [&](int stage, int64_t row) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            const bool there = col < a.cols && row < a.rows;
            copy_async(ring.slot(stage, 0, k), a.dy + (there ? row * a.ld_dy + col : 0), there);
            copy_async(ring.slot(stage, 1, k), a.h + (there ? row * a.ld_h + col : 0), there);
            if (RES) copy_async(ring.slot(stage, 2, k), a.dresidual + (there ? row * a.ld_dresidual + col : 0), there);
        }
        copies_commit();
    };
    int64_t row = first + group;
#pragma unroll
    for (int i = 0; i < R::kStages - 1; ++i) fetch(i, row + i * step);
    // of the widest rows neither the gain nor the products stay in registers
    constexpr bool kWide = V > 2;
    auto gain_of = [&](int k) {
        const int col = 8 * (t + k * 32 * WPR);
        return col < a.cols ? load_gain8(a.gain, a.gain_f32, col) : zeros8();
    };
    Eight gain[kWide ? 1 : V], dgain[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if constexpr (!kWide) gain[k] = gain_of(k);
        dgain[k] = zeros8();
    }
    float rstd = row < a.rows ? __ldg(a.rstd + row) : 0.0f;
    int parity = 0, stage = 0;
    for (int64_t base = first; base < a.rows; base += step, row += step, parity ^= 1) {
        fetch(stage == 0 ? R::kStages - 1 : stage - 1, row + (R::kStages - 1) * step);
        copies_wait<R::kStages - 1>();
        Eight g[kWide ? 1 : V], u[kWide ? 1 : V];   // dy gain, h rstd
        float2 dot = splat(0.0f);
        const float r = rstd;
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
        if (row + step < a.rows) rstd = __ldg(a.rstd + row + step);
        const float c = group_sum<WPR>(dot.x + dot.y, slots[parity]) * -a.inv_cols;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            if (col >= a.cols || row >= a.rows) continue;
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
            *reinterpret_cast<uint4 *>(a.dx + row * a.ld_dx + col) = pack8(q);
        }
        stage = stage == R::kStages - 1 ? 0 : stage + 1;
    }
    copies_wait<0>();
    if (a.partials) {
        float *p = a.partials + (first + group) * a.cols;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            if (col >= a.cols) continue;
            float4 *q = reinterpret_cast<float4 *>(p + col);
            q[0] = make_float4(dgain[k].p[0].x, dgain[k].p[0].y, dgain[k].p[1].x, dgain[k].p[1].y);
            q[1] = make_float4(dgain[k].p[2].x, dgain[k].p[2].y, dgain[k].p[3].x, dgain[k].p[3].y);
        }
    }
}

// dgain[c] (+)= sum of the partials of column c, in a fixed order: 32 threads of a column take every 32nd partial each and are added in order.
__global__ void __launch_bounds__(1024) dgain_reduce_kernel(const float *partials, int n, int cols, float *dgain, int accumulate)
{
    __shared__ float part[32][33];
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

// Warps per row and vectors per thread for a row of `cols` elements.
struct Shape {
    int wpr, v;
};
Shape shape_for(int64_t cols)
{
    const int64_t vecs = ceil_div(cols, 8 * 32);   // vectors per lane of one warp
    for (int wpr : {1, 4, 8, 16, 32})
        for (int v : {1, 2})
            if (vecs <= (int64_t)wpr * v) return {wpr, v};
    return {32, 4};
}

// CTAs of a kernel that an SM holds, with its dynamic shared memory allowed for (asked once: the same on every device of this family; the
// allowance is per device).
template <auto Kernel>
int resident(int threads, int smem)
{
    static std::atomic<uint64_t> allowed{0};   // a bit per device
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) || dev > 63) {
        if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    static std::atomic<int> known{0};
    int n = known.load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, threads, smem) != cudaSuccess || n < 1) return 0;
        known.store(n, std::memory_order_relaxed);
    }
    return n;
}

// F(WPR, V) of every shape
#define SNIP_NORM_SHAPES(F) F(1, 1) F(1, 2) F(4, 1) F(4, 2) F(8, 1) F(8, 2) F(16, 1) F(16, 2) F(32, 1) F(32, 2) F(32, 4)

bool bad_ld(int64_t ld, int64_t cols) { return ld < cols || (ld % 8) != 0; }
bool bad_dims(int64_t rows, int64_t cols) { return rows < 0 || rows > INT32_MAX - 128 || cols <= 0 || (cols % 8) != 0 || cols > kMaxCols; }

template <int N>
using Int = std::integral_constant<int, N>;

// CTAs of the backward pass (each group of rows leaves one partial of dgain).  kBwdCtas bounds the workspace.
constexpr int64_t kBwdCtas = 8 * 148;
int64_t bwd_ctas(int64_t rows, int wpr, int per_sm)
{
    const int64_t want = ceil_div(rows, groups_per_cta(wpr)), fit = (int64_t)per_sm * gemm_sm_count(), cap = fit < kBwdCtas ? fit : kBwdCtas;
    return want < cap ? want : cap;
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
    a.ld_x = t->ld_x; a.ld_residual = t->ld_residual; a.ld_h = t->ld_h; a.ld_y = t->ld_y;
    a.rows = (int32_t)t->rows;
    a.cols = (int32_t)t->cols;
    a.gain_f32 = t->gain_dtype == SNIP_OUT_FP32;
    a.eps = t->eps;
    a.inv_cols = (float)(1.0 / (double)t->cols);
    const Shape s = shape_for(t->cols);
    int n = 0;   // 0: a CUDA call failed
    auto launch = [&](auto wpr, auto v, auto res, auto fmt) {
        constexpr auto kernel = rmsnorm_kernel<wpr(), v(), res(), fmt()>;
        constexpr int smem = Ring<wpr(), v(), res() ? 2 : 1>::kBytes;
        n = resident<kernel>(cta_threads(wpr()), smem);
        const int64_t want = ceil_div(t->rows, groups_per_cta(wpr())), cap = (int64_t)n * gemm_sm_count();
        if (n) kernel<<<(unsigned)(want < cap ? want : cap), cta_threads(wpr()), smem, st>>>(a);
    };
    auto with_fmt = [&](auto wpr, auto v, auto res) {
        if (!a.codes) launch(wpr, v, res, Int<SNIP_FMT_BF16>{});
        else if (t->fmt == SNIP_FMT_FP8_E4M3) launch(wpr, v, res, Int<SNIP_FMT_FP8_E4M3>{});
        else launch(wpr, v, res, Int<SNIP_FMT_FP4_E2M1>{});
    };
#define SNIP_LAUNCH(W, V)                                                                       \
    if (s.wpr == W && s.v == V) {                                                               \
        if (t->residual) with_fmt(Int<W>{}, Int<V>{}, std::true_type{});                        \
        else with_fmt(Int<W>{}, Int<V>{}, std::false_type{});                                   \
    }
    SNIP_NORM_SHAPES(SNIP_LAUNCH)
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
    d.ld = t->residual ? t->ld_h : t->ld_x;
    d.rows = a.rows; d.cols = a.cols;
    d.tiles_c = (int32_t)ceil_div(t->cols, kTile);
    d.tiles = d.tiles_c * ceil_div(t->rows, kTile);
    d.gain_f32 = a.gain_f32;
    auto launch_dual = [&](auto fmt, auto fmt_t) {
        constexpr auto kernel = rmsnorm_dual_kernel<fmt(), fmt_t()>;
        n = resident<kernel>(kDualThreads, (int)sizeof(DualShared));
        const int64_t cap = (int64_t)n * gemm_sm_count();
        if (n) kernel<<<(unsigned)(d.tiles < cap ? d.tiles : cap), kDualThreads, sizeof(DualShared), st>>>(d);
    };
    auto with_fmt_t = [&](auto fmt) {
        if (t->fmt_t == SNIP_FMT_FP8_E4M3) launch_dual(fmt, Int<SNIP_FMT_FP8_E4M3>{});
        else launch_dual(fmt, Int<SNIP_FMT_FP4_E2M1>{});
    };
    if (!d.codes) with_fmt_t(Int<SNIP_FMT_BF16>{});
    else if (t->fmt == SNIP_FMT_FP8_E4M3) with_fmt_t(Int<SNIP_FMT_FP8_E4M3>{});
    else with_fmt_t(Int<SNIP_FMT_FP4_E2M1>{});
    SNIP_CUDA_TRY(cudaGetLastError());
    return n ? SNIP_OK : SNIP_ERR_CUDA;
}

extern "C" int snip_rmsnorm_bwd_workspace(int64_t rows, int64_t cols, size_t *ws_bytes)
{
    using namespace snip;
    if (!ws_bytes) return SNIP_ERR_ARG;
    if (bad_dims(rows, cols)) return SNIP_ERR_SHAPE;
    // one partial per group of rows in flight, of the largest grid
    const Shape s = shape_for(cols);
    int64_t groups = kBwdCtas * groups_per_cta(s.wpr);
    if (rows < groups) groups = align_up((size_t)rows, groups_per_cta(s.wpr));
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
    a.ld_dy = t->ld_dy; a.ld_h = t->ld_h; a.ld_dresidual = t->ld_dresidual; a.ld_dx = t->ld_dx;
    a.rows = (int32_t)t->rows;
    a.cols = (int32_t)t->cols;
    a.gain_f32 = t->gain_dtype == SNIP_OUT_FP32;
    a.inv_cols = (float)(1.0 / (double)t->cols);
    const Shape s = shape_for(t->cols);
    int64_t ctas = 0;
    auto launch = [&](auto wpr, auto v, auto res) {
        constexpr auto kernel = rmsnorm_bwd_kernel<wpr(), v(), res()>;
        constexpr int smem = Ring<wpr(), v(), res() ? 3 : 2>::kBytes;
        ctas = bwd_ctas(t->rows, wpr(), resident<kernel>(cta_threads(wpr()), smem));
        if (ctas) kernel<<<(unsigned)ctas, cta_threads(wpr()), smem, st>>>(a);
    };
#define SNIP_LAUNCH(W, V)                                                                       \
    if (s.wpr == W && s.v == V) {                                                               \
        if (t->dresidual) launch(Int<W>{}, Int<V>{}, std::true_type{});                         \
        else launch(Int<W>{}, Int<V>{}, std::false_type{});                                     \
    }
    SNIP_NORM_SHAPES(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(cudaGetLastError());
    if (!ctas) return SNIP_ERR_CUDA;
    if (t->dgain) {
        dgain_reduce_kernel<<<(unsigned)ceil_div(t->cols, 32), dim3(32, 32), 0, st>>>(a.partials, (int)(ctas * groups_per_cta(s.wpr)), a.cols, t->dgain, t->accumulate);
        SNIP_CUDA_TRY(cudaGetLastError());
    }
    return SNIP_OK;
}
