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
    int gain_f32, fmt;
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

// 16 bytes that this kernel reads once (they may be overwritten in place afterwards: not the read-only path)
__device__ __forceinline__ uint4 load_once(const uint16_t *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
    f[4] = bf16lo(v.z); f[5] = bf16hi(v.z); f[6] = bf16lo(v.w); f[7] = bf16hi(v.w);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

__device__ __forceinline__ void load_gain8(const void *gain, int f32, int col, float (&g)[8])
{
    if (f32) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(gain) + col));
        const float4 b = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(gain) + col) + 1);
        g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    } else {
        unpack8(__ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(gain) + col)), g);
    }
}

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

// WPR warps per row, V vectors of eight elements per thread: vector k of thread t of the group starts at column 8 (t + k 32 WPR), so
// that 16 neighbouring threads hold a 128-long tile.
template <int WPR, int V, bool RES>
__global__ void __launch_bounds__(cta_threads(WPR)) rmsnorm_kernel(const NormArgs a)
{
    __shared__ float slots[2][32];
    constexpr int kGroups = groups_per_cta(WPR);
    const int t = threadIdx.x % (32 * WPR);
    const int64_t step = (int64_t)gridDim.x * kGroups;
    float gain[V][8];
    bool in[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int col = 8 * (t + k * 32 * WPR);
        in[k] = col < a.cols;
#pragma unroll
        for (int i = 0; i < 8; ++i) gain[k][i] = 0.0f;
        if (in[k]) load_gain8(a.gain, a.gain_f32, col, gain[k]);
    }
    uint4 x[V], r[V];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            x[k] = make_uint4(0, 0, 0, 0);
            if (RES) r[k] = make_uint4(0, 0, 0, 0);
            if (in[k] && row < a.rows) {
                const int col = 8 * (t + k * 32 * WPR);
                x[k] = load_once(a.x + row * a.ld_x + col);
                if (RES) r[k] = load_once(a.residual + row * a.ld_residual + col);
            }
        }
    };
    // all groups of a CTA take the same number of turns: rows behind the last are zeros that nothing is written for
    const int64_t first = (int64_t)blockIdx.x * kGroups;
    const int group = threadIdx.x / (32 * WPR);
    fetch(first + group);
    int parity = 0;
    for (int64_t base = first; base < a.rows; base += step, parity ^= 1) {
        const int64_t row = base + group;
        float h[V][8];
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unpack8(x[k], h[k]);
            if (RES) {
                float q[8];
                unpack8(r[k], q);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[k][i] += q[i];
                const uint4 packed = pack8(h[k]);
                if (in[k] && row < a.rows) *reinterpret_cast<uint4 *>(a.h + row * a.ld_h + 8 * (t + k * 32 * WPR)) = packed;
                unpack8(packed, h[k]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(h[k][i], h[k][i], sum);
        }
        fetch(row + step);
        sum = group_sum<WPR>(sum, slots[parity]);
        const float rstd = __frcp_rn(__fsqrt_rn(fmaf(sum, a.inv_cols, a.eps)));
        if (t == 0 && a.rstd && row < a.rows) a.rstd[row] = rstd;
        if (!a.y && !a.codes) continue;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int col = 8 * (t + k * 32 * WPR);
            const bool ok = in[k] && row < a.rows;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] = __fmul_rn(__fmul_rn(h[k][i], rstd), gain[k][i]);
            if (a.y && ok) *reinterpret_cast<uint4 *>(a.y + row * a.ld_y + col) = pack8(h[k]);
            if (a.codes) {
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(h[k][i]));
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, off));
                const bool fp8 = a.fmt == SNIP_FMT_FP8_E4M3;
                const float s = fp8 ? tile_scale<SNIP_FMT_FP8_E4M3>(most, 0) : tile_scale<SNIP_FMT_FP4_E2M1>(most, 0);
                if (ok) {
                    if ((t & 15) == 0) a.scales[(int64_t)(col >> 7) * a.rows + row] = s;
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[k][i] *= s;
                    const int64_t at = row * a.cols + col;
                    if (fp8) {
                        *reinterpret_cast<uint2 *>(a.codes + at) = make_uint2(cvt_e4m3x2(h[k][0], h[k][1]) | cvt_e4m3x2(h[k][2], h[k][3]) << 16,
                                                                              cvt_e4m3x2(h[k][4], h[k][5]) | cvt_e4m3x2(h[k][6], h[k][7]) << 16);
                    } else {
                        *reinterpret_cast<uint32_t *>(a.codes + at / 2) = cvt_e2m1x2(h[k][0], h[k][1]) | cvt_e2m1x2(h[k][2], h[k][3]) << 8 |
                                                                          cvt_e2m1x2(h[k][4], h[k][5]) << 16 | cvt_e2m1x2(h[k][6], h[k][7]) << 24;
                    }
                }
            }
        }
    }
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
    int gain_f32, fmt, fmt_t;
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

__global__ void __launch_bounds__(kDualThreads, kDualCtas) rmsnorm_dual_kernel(const NormDualArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    DualShared &m = *reinterpret_cast<DualShared *>(raw);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, lane = tid & 31, warp = tid >> 5;
    auto fetch = [&](int64_t tile) {
        const int64_t row = tile / a.tiles_c * kTile + 8 * ty, col = tile % a.tiles_c * kTile + 8 * tx;
        const bool ok = tile < a.tiles && row < a.rows && col < a.cols;
        const uint16_t *p = a.h + (ok ? row * a.ld + col : 0);
        const int bytes = ok ? 16 : 0;   // 0: the slot is filled with zeros, nothing is read
#pragma unroll
        for (int i = 0; i < 8; ++i)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(&m.slot[i][tid])), "l"(p + (ok ? i * a.ld : 0)), "r"(bytes) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch(blockIdx.x);
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int row0 = (int)(tile / a.tiles_c) * kTile + 8 * ty, col0 = (int)(tile % a.tiles_c) * kTile + 8 * tx;
        const bool ok = row0 < a.rows && col0 < a.cols;
        float gain[8], rstd[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) gain[i] = rstd[i] = 0.0f;
        if (ok) {
            load_gain8(a.gain, a.gain_f32, col0, gain);
            const float4 p = __ldcg(reinterpret_cast<const float4 *>(a.rstd + row0)), q = __ldcg(reinterpret_cast<const float4 *>(a.rstd + row0) + 1);
            rstd[0] = p.x; rstd[1] = p.y; rstd[2] = p.z; rstd[3] = p.w; rstd[4] = q.x; rstd[5] = q.y; rstd[6] = q.z; rstd[7] = q.w;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        float rmax[8], cmax[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) cmax[i] = 0.0f;
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            float f[8];
            unpack8(m.slot[p][tid], f);
            rmax[p] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = fabsf(__fmul_rn(__fmul_rn(f[i], rstd[p]), gain[i]));
                rmax[p] = fmaxf(rmax[p], v);
                cmax[i] = fmaxf(cmax[i], v);
            }
        }
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
        if (a.codes && (lane & 1) == 0) {
            const float s = a.fmt == SNIP_FMT_FP8_E4M3 ? tile_scale<SNIP_FMT_FP8_E4M3>(rmax[0], 0) : tile_scale<SNIP_FMT_FP4_E2M1>(rmax[0], 0);
            const int q = (lane >> 1) & 7, r = 8 * ty + q;
            m.row_scale[r] = s;
            const int64_t row = tile / a.tiles_c * kTile + r;
            if (row < a.rows) a.scales[tile % a.tiles_c * a.rows + row] = s;
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
            const float s = a.fmt_t == SNIP_FMT_FP8_E4M3 ? tile_scale<SNIP_FMT_FP8_E4M3>(v, 0) : tile_scale<SNIP_FMT_FP4_E2M1>(v, 0);
            m.col_scale[tid] = s;
            const int64_t col = tile % a.tiles_c * kTile + tid;
            if (col < a.cols) a.scales_t[tile / a.tiles_c * a.cols + col] = s;
        }
        __syncthreads();
        float cs[8];
        {
            const float4 p = *reinterpret_cast<const float4 *>(&m.col_scale[8 * tx]), q = *reinterpret_cast<const float4 *>(&m.col_scale[8 * tx + 4]);
            cs[0] = p.x; cs[1] = p.y; cs[2] = p.z; cs[3] = p.w; cs[4] = q.x; cs[5] = q.y; cs[6] = q.z; cs[7] = q.w;
        }
        const bool fp8 = a.fmt == SNIP_FMT_FP8_E4M3, fp8_t = a.fmt_t == SNIP_FMT_FP8_E4M3;
        uint32_t ct[8][2];   // column i: codes of its eight rows (FP4: the first word)
#pragma unroll
        for (int i = 0; i < 8; ++i) ct[i][0] = ct[i][1] = 0u;
#pragma unroll
        for (int p = 0; p < 8; p += 2) {
            float y[2][8];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                unpack8(m.slot[p + e][tid], y[e]);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[e][i] = __fmul_rn(__fmul_rn(y[e][i], rstd[p + e]), gain[i]);
                if (a.codes && ok) {
                    const float s = m.row_scale[8 * ty + p + e];
                    float z[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = y[e][i] * s;
                    const int64_t at = (int64_t)(row0 + p + e) * a.cols + col0;
                    if (fp8) *reinterpret_cast<uint2 *>(a.codes + at) = make_uint2(cvt_e4m3x2(z[0], z[1]) | cvt_e4m3x2(z[2], z[3]) << 16, cvt_e4m3x2(z[4], z[5]) | cvt_e4m3x2(z[6], z[7]) << 16);
                    else *reinterpret_cast<uint32_t *>(a.codes + at / 2) = cvt_e2m1x2(z[0], z[1]) | cvt_e2m1x2(z[2], z[3]) << 8 | cvt_e2m1x2(z[4], z[5]) << 16 | cvt_e2m1x2(z[6], z[7]) << 24;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (fp8_t) ct[i][p >> 2] |= cvt_e4m3x2(y[0][i] * cs[i], y[1][i] * cs[i]) << (8 * (p & 3));
                else ct[i][0] |= cvt_e2m1x2(y[0][i] * cs[i], y[1][i] * cs[i]) << (4 * p);
            }
        }
        fetch(tile + gridDim.x);   // the slot has been read
        // transposed codes: line = column of the tile, 128 (64) bytes each; 16-byte pieces swizzled by the line so that neither side conflicts
        if (fp8_t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int line = 8 * tx + i, piece = (ty >> 1) ^ (tx & 7);
                *reinterpret_cast<uint2 *>(&m.stage[line * 128 + piece * 16 + (ty & 1) * 8]) = make_uint2(ct[i][0], ct[i][1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int line = 8 * tx + i, piece = (ty >> 2) ^ (tx & 3);
                *reinterpret_cast<uint32_t *>(&m.stage[line * 64 + piece * 16 + (ty & 3) * 4]) = ct[i][0];
            }
        }
        __syncthreads();
        const int64_t r0 = tile / a.tiles_c * kTile, c0 = tile % a.tiles_c * kTile;
        const int per_line = fp8_t ? 8 : 4, rows_per_piece = fp8_t ? 16 : 32;
        for (int j = tid; j < kTile * per_line; j += kDualThreads) {
            const int line = j / per_line, piece = j % per_line;
            const int64_t row = r0 + piece * rows_per_piece;
            if (c0 + line >= a.cols || row >= a.rows) continue;
            const int at = fp8_t ? line * 128 + ((piece ^ ((line >> 3) & 7)) * 16) : line * 64 + ((piece ^ ((line >> 3) & 3)) * 16);
            const int64_t elem = (c0 + line) * a.rows + row;
            *reinterpret_cast<uint4 *>(a.codes_t + (fp8_t ? elem : elem / 2)) = *reinterpret_cast<const uint4 *>(&m.stage[at]);
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int WPR, int V, bool RES>
__global__ void __launch_bounds__(cta_threads(WPR)) rmsnorm_bwd_kernel(const NormBwdArgs a)
{
    __shared__ float slots[2][32];
    constexpr int kGroups = groups_per_cta(WPR);
    const int t = threadIdx.x % (32 * WPR), group = threadIdx.x / (32 * WPR);
    const int64_t step = (int64_t)gridDim.x * kGroups, first = (int64_t)blockIdx.x * kGroups;
    float gain[V][8], dgain[V][8];
    bool in[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int col = 8 * (t + k * 32 * WPR);
        in[k] = col < a.cols;
#pragma unroll
        for (int i = 0; i < 8; ++i) gain[k][i] = dgain[k][i] = 0.0f;
        if (in[k]) load_gain8(a.gain, a.gain_f32, col, gain[k]);
    }
    uint4 dy[V], h[V], d[V];
    float rstd = 0.0f;
    auto fetch = [&](int64_t row) {
        const bool any = row < a.rows;
        if (any) rstd = __ldg(a.rstd + row);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            dy[k] = h[k] = make_uint4(0, 0, 0, 0);
            if (RES) d[k] = make_uint4(0, 0, 0, 0);
            if (in[k] && any) {
                const int col = 8 * (t + k * 32 * WPR);
                dy[k] = load_once(a.dy + row * a.ld_dy + col);
                h[k] = load_once(a.h + row * a.ld_h + col);
                if (RES) d[k] = load_once(a.dresidual + row * a.ld_dresidual + col);
            }
        }
    };
    fetch(first + group);
    int parity = 0;
    for (int64_t base = first; base < a.rows; base += step, parity ^= 1) {
        const int64_t row = base + group;
        float g[V][8], u[V][8];   // dy gain, h rstd
        uint4 res[V];
        float dot = 0.0f;
        const float r = rstd;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            unpack8(dy[k], g[k]);
            unpack8(h[k], u[k]);
            if (RES) res[k] = d[k];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[k][i] *= r;
                dgain[k][i] = fmaf(g[k][i], u[k][i], dgain[k][i]);
                g[k][i] *= gain[k][i];
                dot = fmaf(g[k][i], u[k][i], dot);
            }
        }
        fetch(row + step);
        const float c = group_sum<WPR>(dot, slots[parity]) * a.inv_cols;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (!in[k] || row >= a.rows) continue;
            float q[8];
            if (RES) unpack8(res[k], q);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = fmaf(-u[k][i], c, g[k][i]);
                q[i] = RES ? fmaf(r, e, q[i]) : r * e;
            }
            *reinterpret_cast<uint4 *>(a.dx + row * a.ld_dx + 8 * (t + k * 32 * WPR)) = pack8(q);
        }
    }
    if (a.partials) {
        float *p = a.partials + (int64_t)(first + group) * a.cols;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (in[k]) {
                float4 *q = reinterpret_cast<float4 *>(p + 8 * (t + k * 32 * WPR));
                q[0] = make_float4(dgain[k][0], dgain[k][1], dgain[k][2], dgain[k][3]);
                q[1] = make_float4(dgain[k][4], dgain[k][5], dgain[k][6], dgain[k][7]);
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

// CTAs of a kernel that an SM holds (asked once: the same on every device of this family).
template <auto Kernel>
int resident(int threads)
{
    static const int n = [threads] {
        int k = 0;
        return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, Kernel, threads, 0) == cudaSuccess && k > 0 ? k : 1;
    }();
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
    a.fmt = t->fmt;
    a.eps = t->eps;
    a.inv_cols = (float)(1.0 / (double)t->cols);
    const Shape s = shape_for(t->cols);
    auto launch = [&](auto wpr, auto v, auto res) {
        constexpr auto kernel = rmsnorm_kernel<wpr(), v(), res()>;
        const int64_t want = ceil_div(t->rows, groups_per_cta(wpr())), cap = (int64_t)resident<kernel>(cta_threads(wpr())) * gemm_sm_count();
        kernel<<<(unsigned)(want < cap ? want : cap), cta_threads(wpr()), 0, st>>>(a);
    };
#define SNIP_LAUNCH(W, V)                                                                       \
    if (s.wpr == W && s.v == V) {                                                               \
        if (t->residual) launch(Int<W>{}, Int<V>{}, std::true_type{});                          \
        else launch(Int<W>{}, Int<V>{}, std::false_type{});                                     \
    }
    SNIP_NORM_SHAPES(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(cudaGetLastError());
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
    d.gain_f32 = a.gain_f32; d.fmt = t->fmt; d.fmt_t = t->fmt_t;
    const int64_t cap = (int64_t)kDualCtas * gemm_sm_count();
    SNIP_CUDA_TRY(cudaFuncSetAttribute(rmsnorm_dual_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(DualShared)));
    rmsnorm_dual_kernel<<<(unsigned)(d.tiles < cap ? d.tiles : cap), kDualThreads, sizeof(DualShared), st>>>(d);
    SNIP_CUDA_TRY(cudaGetLastError());
    return SNIP_OK;
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
        ctas = bwd_ctas(t->rows, wpr(), resident<kernel>(cta_threads(wpr())));
        kernel<<<(unsigned)ctas, cta_threads(wpr()), 0, st>>>(a);
    };
#define SNIP_LAUNCH(W, V)                                                                       \
    if (s.wpr == W && s.v == V) {                                                               \
        if (t->dresidual) launch(Int<W>{}, Int<V>{}, std::true_type{});                         \
        else launch(Int<W>{}, Int<V>{}, std::false_type{});                                     \
    }
    SNIP_NORM_SHAPES(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(cudaGetLastError());
    if (t->dgain) {
        dgain_reduce_kernel<<<(unsigned)ceil_div(t->cols, 32), dim3(32, 32), 0, st>>>(a.partials, (int)(ctas * groups_per_cta(s.wpr)), a.cols, t->dgain, t->accumulate);
        SNIP_CUDA_TRY(cudaGetLastError());
    }
    return SNIP_OK;
}
