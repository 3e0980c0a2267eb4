// RMS norm with the residual's addition, its quantized outputs, and its backward pass.
//   forward:  h = bf16(x + residual), rstd = (mean h^2 + eps)^-1/2, y = (h rstd) gain, in binary32; codes of y on 1x128 tiles, and
//             on 128x1 tiles stored transposed, by the quantizers' scale rule
//   backward: g = dy gain, c = mean(g h rstd), dx = rstd (g - h rstd c) + dresidual, dgain = sum over rows of dy h rstd
//
// Bound by HBM where a residual is read: a few operations per element against 6 to 10 bytes; without one (3 bytes with codes) issue slots come
// next to it: 83 % of the copy rate.  16384 x 4096, bf16 gain, in us (TB/s, of 6.55 for a copy): residual
// added and FP8 row codes 80-83 (5.7), the transposed codes too 110 (4.9; 6.1 with h's second reading), both in FP4 97 (4.9; 6.2), backward with a residual
// gradient 82 (6.5), without 66 (6.1).
//
// rmsnorm_kernel / rmsnorm_bwd_kernel: a group of warps owns a row at a time and a thread the same columns of each of its rows, so that
// the gain's gradient (and, but for the widest rows, the gain) stays in registers; the grid is resident and walks over the rows.  The row is read
// once: it stays in registers between the reduction and the outputs, and the next rows are on their way during both: a ring of three stages fetches
// two rows ahead, one of two one, one of a single stage (forward and backward beyond 16384 columns) none.  The forms with four vectors per thread of
// the backward pass and the 1024-thread one of the forward pass, beyond 8192 and 16384 columns, load the gain again for each row; that backward
// pass also takes the row from shared memory a second time, and that forward pass keeps it in bf16.
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
    float *partials;   // [CTAs][cols], or null
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

// (Plain loads, not the read-only path: this kernel may have started before the one that writes the gain had ended.)
__device__ __forceinline__ Eight load_gain8(const void *gain, int f32, int col)
{
    if (!f32) return unpack8(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(gain) + col));
    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(gain) + col);
    const float4 a = p[0], b = p[1];
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
    chain_start(CHAIN_FIRST);
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

// The transposed copy, from h and rstd: codes on 128x1 tiles.  A CTA walks over 128x128 tiles; a warp takes 16 columns of 128 rows, a thread 8x8
// elements of them (dimensions are multiples of 64: a thread has all of them or none), whose y stay in registers between the maximum and the
// codes.  A column's 128 elements belong to 16 threads of the one warp, so that its maximum needs no barrier, and the eight codes that a thread
// has of a column go straight to their place, 16 threads filling a 128-byte line.  A tile comes through shared memory, fetched in whole rows of
// 256 bytes while the tile before it is worked on (fetched by the threads that use it, 32 bytes of a row at a time, 51 us instead of 38 on
// 16384 x 4096), its 16-byte pieces swizzled by the row group so that the 16 row groups of a warp read different banks; one barrier per tile.
struct NormColsArgs {
    const uint16_t *h;
    const void *gain;
    const float *rstd;
    uint8_t *codes_t;
    float *scales_t;
    int32_t rows, cols, tiles_c, tiles, ld;
    int gain_f32;
};
constexpr int kTile = 128;
constexpr int kColsThreads = 256;
constexpr int kColsCtas = 2;
struct ColsShared {
    uint4 h[2][kTile * 16];
    __align__(16) float rstd[2][kTile];
    uint4 gain[2][32];
};

template <int FMT>
__global__ void __launch_bounds__(kColsThreads, kColsCtas) rmsnorm_cols_kernel(const NormColsArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    ColsShared &m = *reinterpret_cast<ColsShared *>(raw);
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5, tx = lane & 1, ty = lane >> 1;
    const int off_r = 8 * ty, off_c = 16 * warp + 8 * tx;   // of the thread's elements in a tile
    const int piece = tid & 15, line = tid >> 4;            // what it fetches: 16 bytes of rows line, line + 16, ...
    // row and column of the tile, moved on without a division
    const int step_r = (int)gridDim.x / a.tiles_c, step_c = (int)gridDim.x % a.tiles_c;
    const int last_r = a.tiles / a.tiles_c - 1;   // from the last tile row back: what of h is still in the L2 cache is read from there
    auto fetch = [&](int buf, int tile, int r, int c) {
        r = last_r - r;
        if (tile < a.tiles) {
            const int row = r * kTile + line, col = c * kTile + 8 * piece;
            const uint16_t *p = a.h + (int64_t)row * a.ld + col;
#pragma unroll
            for (int i = 0; i < 8; ++i, p += 16 * (int64_t)a.ld)
                if (row + 16 * i < a.rows && col < a.cols) copy_async(&m.h[buf][(line + 16 * i) * 16 + (piece ^ ((line >> 3) + 2 * i))], p);
            if (tid < 32) {
                if (r * kTile + 4 * tid < a.rows) copy_async(reinterpret_cast<uint4 *>(&m.rstd[buf][4 * tid]), reinterpret_cast<const uint16_t *>(a.rstd + r * kTile + 4 * tid));
            } else if (tid < 64) {
                const int g = tid - 32, first = c * kTile + (a.gain_f32 ? 4 : 8) * g;
                if (first < a.cols && (a.gain_f32 || g < 16))
                    copy_async(&m.gain[buf][g], a.gain_f32 ? reinterpret_cast<const uint16_t *>(static_cast<const float *>(a.gain) + first) : static_cast<const uint16_t *>(a.gain) + first);
            }
        }
        copies_commit();
    };
    chain_start(CHAIN_FIRST);   // h and rstd come from the kernel before this one
    int done = (int)blockIdx.x / a.tiles_c, tc = (int)blockIdx.x % a.tiles_c, buf = 0;
    fetch(0, (int)blockIdx.x, done, tc);
    for (int tile = (int)blockIdx.x; tile < a.tiles; tile += (int)gridDim.x, buf ^= 1) {
        const int tr = last_r - done;
        int next_r = done + step_r, next_c = tc + step_c;
        if (next_c >= a.tiles_c) { next_c -= a.tiles_c; ++next_r; }
        const int row = tr * kTile + off_r, col = tc * kTile + off_c;
        const bool ok = row < a.rows && col < a.cols;
        copies_wait<0>();
        __syncthreads();   // everybody's copies are here, and the other buffer has been read
        fetch(buf ^ 1, tile + (int)gridDim.x, next_r, next_c);
        Eight y[8];
        if (ok) {
            Eight gain;
            if (a.gain_f32) {
                const float4 g0 = *reinterpret_cast<const float4 *>(&m.gain[buf][off_c >> 2]), g1 = *reinterpret_cast<const float4 *>(&m.gain[buf][(off_c >> 2) + 1]);
                gain = Eight{{make_float2(g0.x, g0.y), make_float2(g0.z, g0.w), make_float2(g1.x, g1.y), make_float2(g1.z, g1.w)}};
            } else {
                gain = unpack8(m.gain[buf][off_c >> 3]);
            }
            const float4 r0 = *reinterpret_cast<const float4 *>(&m.rstd[buf][off_r]), r1 = *reinterpret_cast<const float4 *>(&m.rstd[buf][off_r + 4]);
            const float rstd[8] = {r0.x, r0.y, r0.z, r0.w, r1.x, r1.y, r1.z, r1.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = scaled8(unpack8(m.h[buf][(off_r + i) * 16 + ((off_c >> 3) ^ ty)]), rstd[i], gain);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = zeros8();
        }
        float most[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            most[2 * i] = fabsf(y[0].p[i].x);
            most[2 * i + 1] = fabsf(y[0].p[i].y);
#pragma unroll
            for (int r = 1; r < 7; r += 2) {
                most[2 * i] = fmaxf(fmaxf(most[2 * i], fabsf(y[r].p[i].x)), fabsf(y[r + 1].p[i].x));
                most[2 * i + 1] = fmaxf(fmaxf(most[2 * i + 1], fabsf(y[r].p[i].y)), fabsf(y[r + 1].p[i].y));
            }
            most[2 * i] = fmaxf(most[2 * i], fabsf(y[7].p[i].x));
            most[2 * i + 1] = fmaxf(most[2 * i + 1], fabsf(y[7].p[i].y));
        }
        // each step halves the number of columns a lane still looks after: lanes 4 q + tx and 4 q + 2 + tx end with column q's maximum
#pragma unroll
        for (int w = 4, off = 16; w > 0; w >>= 1, off >>= 1) {
            const bool upper = (lane & off) != 0;
#pragma unroll
            for (int i = 0; i < w; ++i) {
                const float give = upper ? most[i] : most[i + w], keep = upper ? most[i + w] : most[i];
                most[i] = fmaxf(keep, __shfl_xor_sync(0xFFFFFFFFu, give, off));
            }
        }
        most[0] = fmaxf(most[0], __shfl_xor_sync(0xFFFFFFFFu, most[0], 2));
        const float own = tile_scale<FMT>(most[0], 0);
        if ((lane & 2) == 0 && col < a.cols) a.scales_t[(int64_t)tr * a.cols + col + (lane >> 2)] = own;
        Eight s;
#pragma unroll
        for (int i = 0; i < 4; ++i) s.p[i] = make_float2(__shfl_sync(0xFFFFFFFFu, own, 8 * i + tx), __shfl_sync(0xFFFFFFFFu, own, 8 * i + 4 + tx));
        if (ok) {
            constexpr int kPerByte = FMT == SNIP_FMT_FP4_E2M1 ? 2 : 1;
            uint8_t *to = a.codes_t + ((int64_t)col * a.rows + row) / kPerByte;
            const int64_t line = a.rows / kPerByte;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int r = 0; r < 8; ++r) y[r].p[i] = __fmul2_rn(y[r].p[i], s.p[i]);
#pragma unroll
                for (int e = 0; e < 2; ++e, to += line) {
                    uint32_t c[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float lo = e ? y[2 * q].p[i].y : y[2 * q].p[i].x, hi = e ? y[2 * q + 1].p[i].y : y[2 * q + 1].p[i].x;
                        c[q] = FMT == SNIP_FMT_FP8_E4M3 ? cvt_e4m3x2(lo, hi) : cvt_e2m1x2(lo, hi);
                    }
                    if constexpr (FMT == SNIP_FMT_FP8_E4M3) *reinterpret_cast<uint2 *>(to) = make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
                    else *reinterpret_cast<uint32_t *>(to) = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
                }
            }
        }
        done = next_r;
        tc = next_c;
    }
    copies_wait<0>();
}

template <int V, int THREADS, int STAGES, bool RES>
__global__ void __launch_bounds__(THREADS) rmsnorm_bwd_kernel(const NormBwdArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    __shared__ __align__(16) float slots[2][32];
    const Place at(a.wpr);
    bool in[V];
#pragma unroll
    for (int k = 0; k < V; ++k) in[k] = at.col0 + k * at.apart < a.cols;
    const Ring<V, RES ? 3 : 2, STAGES> ring(raw, in);
    if (threadIdx.x < 64) slots[threadIdx.x >> 5][threadIdx.x & 31] = 0.0f;
    __syncthreads();
    chain_start(CHAIN_FIRST);
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
    float rstd = row < a.rows ? a.rstd[row] : 0.0f;
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
        if (row < a.rows) rstd = a.rstd[row];
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
    if (!a.partials) return;
    if (at.groups > 1) {   // the groups' sums are added in order by the first one's threads, through the ring (whose copies have all arrived)
        __syncthreads();
        float4 *const mine = reinterpret_cast<float4 *>(raw) + threadIdx.x;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            mine[2 * k * blockDim.x] = make_float4(dgain[k].p[0].x, dgain[k].p[0].y, dgain[k].p[1].x, dgain[k].p[1].y);
            mine[(2 * k + 1) * blockDim.x] = make_float4(dgain[k].p[2].x, dgain[k].p[2].y, dgain[k].p[3].x, dgain[k].p[3].y);
        }
        __syncthreads();
        if (at.group > 0) return;
        for (int g = 1; g < at.groups; ++g) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float4 p = mine[2 * k * blockDim.x + 32 * a.wpr * g], q = mine[(2 * k + 1) * blockDim.x + 32 * a.wpr * g];
                dgain[k].p[0] = __fadd2_rn(dgain[k].p[0], make_float2(p.x, p.y));
                dgain[k].p[1] = __fadd2_rn(dgain[k].p[1], make_float2(p.z, p.w));
                dgain[k].p[2] = __fadd2_rn(dgain[k].p[2], make_float2(q.x, q.y));
                dgain[k].p[3] = __fadd2_rn(dgain[k].p[3], make_float2(q.z, q.w));
            }
        }
    }
    float *p = a.partials + (int64_t)blockIdx.x * a.cols + at.col0;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (!in[k]) continue;
        float4 *q = reinterpret_cast<float4 *>(p + k * at.apart);
        q[0] = make_float4(dgain[k].p[0].x, dgain[k].p[0].y, dgain[k].p[1].x, dgain[k].p[1].y);
        q[1] = make_float4(dgain[k].p[2].x, dgain[k].p[2].y, dgain[k].p[3].x, dgain[k].p[3].y);
    }
}

// dgain[c] (+)= sum of the partials of column c, in a fixed order: 32 threads of a column take every 32nd partial each and are added in order.
__global__ void __launch_bounds__(1024) dgain_reduce_kernel(const float *partials, int n, int cols, float *dgain, int accumulate)
{
    __shared__ float part[32][33];
    chain_start(CHAIN_FIRST);
    const int c = blockIdx.x * 32 + threadIdx.x;
    float v = 0.0f;
    if (c < cols)
        for (int i = threadIdx.y; i < n; i += 32) v += __ldcg(partials + (int64_t)i * cols + c);
    part[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && c < cols) {
        v = part[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 32; ++i) v += part[i][threadIdx.x];
        dgain[c] = accumulate ? __ldcg(dgain + c) + v : v;
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
constexpr Shape fwd_shape(int64_t cols, bool residual, bool y, bool codes, bool few)
{
    Shape s = {};
    const bool four = cols > 2048 && (residual ? !codes : codes || y);
    s.v = cols > 8192 ? 4 : few ? 1 : four ? 4 : 2;
    s.wpr = (int)((cols + 256 * s.v - 1) / (256 * s.v));
    s.threads = s.wpr <= 8 ? 256 : s.wpr <= 16 ? 512 : 1024;
    s.groups = s.threads / 32 / s.wpr;
    s.form = s.v == 1 ? (s.threads == 256 ? 0 : s.threads == 512 ? 1 : 2) : s.v == 2 ? (s.threads == 256 ? 3 : 4) : s.threads == 512 ? 5 : s.threads == 1024 ? 6 : 7;
    s.stages = s.form < 5 ? 3 : s.form == 6 ? 1 : 2;
    s.smem = s.stages * (residual ? 2 : 1) * s.v * s.threads * 16;   // at most 128 KB
    return s;
}
// Backward: as F(form, V, most threads, stages).
#define SNIP_NORM_BWD_FORMS(F) F(0, 1, 1024, 3) F(1, 2, 512, 3) F(2, 2, 512, 2) F(3, 4, 512, 2) F(4, 4, 1024, 1)
constexpr Shape bwd_shape(int64_t cols, int arrays, bool few)
{
    Shape s = {};
    s.v = cols > 8192 ? 4 : few ? 1 : 2;
    s.wpr = (int)((cols + 256 * s.v - 1) / (256 * s.v));
    s.groups = s.wpr >= 8 ? 1 : 8 / s.wpr;
    s.threads = 32 * s.wpr * s.groups;
    const int row_bytes = arrays * s.v * s.threads * 16;
    s.form = s.v == 4 ? (s.threads > 512 ? 4 : 3) : s.v == 1 ? 0 : row_bytes <= 32 * 1024 ? 1 : 2;
    s.stages = s.form == 4 ? 1 : s.form < 2 ? 3 : 2;
    s.smem = s.stages * row_bytes;   // at most 192 KB
    return s;
}
// Up to two rows per SM of this chip (148): one vector per thread, so that more threads fetch a row.  Us with it / without, residual and FP8 codes, at
// 512, 4096 and 8192 columns: 1 row 1.54 / 1.81, 1.91 / 2.12, 2.77 / 2.54; 148 rows 1.79 / 2.11, 2.22 / 2.43, 3.12 / 2.94; 296 rows 1.89 / 2.13,
// 3.13 / 2.81, 5.68 / 5.48; 1184 rows 2.19 / 2.24, 8.99 / 7.64, 15.9 / 12.8.  Backward: 1 row 3.03 / 3.34, 3.84 / 3.87, 5.17 / 4.88; 296 rows
// 3.87 / 4.06, 7.43 / 7.85, 10.1 / 9.0.  Beyond 4096 columns it loses up to 10 % and keeps what the forms with more vectors do not: whichever outputs
// are asked for, one form makes them, and rstd has the same bits.
constexpr int64_t kFewRows = 296;
// Whether a call reaches a form with a residual (gradient) and, forward, with row codes: only such kernels are built.  Every width of a vector group
// is looked at, the rules change nowhere else.
constexpr bool fwd_reaches(int form, bool residual, bool codes)
{
    for (int64_t cols = 256; cols <= kMaxCols; cols += 256)
        for (int i = 0; i < 4; ++i)
            if (fwd_shape(cols, residual, (i & 1) != 0, codes, (i & 2) != 0).form == form) return true;
    return false;
}
constexpr bool bwd_reaches(int form, bool residual)
{
    for (int64_t cols = 256; cols <= kMaxCols; cols += 256)
        for (int few = 0; few < 2; ++few)
            if (bwd_shape(cols, residual ? 3 : 2, few != 0).form == form) return true;
    return false;
}

// CTAs of a kernel that an SM holds, with its dynamic shared memory allowed for (asked once: the same on every device of this family; the
// allowance is per device).
template <auto Kernel>
int resident(int threads, int smem, int most_smem)
{
    static std::atomic<uint64_t> allowed{0};   // a bit per device
    int dev = 0;
    auto failed = [](const char *what) {
        set_last_error(what, cudaGetLastError());
        return 0;
    };
    if (cudaGetDevice(&dev) != cudaSuccess) return failed("cudaGetDevice");
    const uint64_t bit = 1ull << (dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit) || dev > 63) {
        if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem) != cudaSuccess) return failed("cudaFuncSetAttribute");
        allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    // by threads: the shared memory goes with them
    static std::atomic<int> known[33];
    int n = known[threads / 32].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, Kernel, threads, smem) != cudaSuccess || n < 1) return failed("cudaOccupancyMaxActiveBlocksPerMultiprocessor");
        known[threads / 32].store(n, std::memory_order_relaxed);
    }
    return n;
}

bool bad_ld(int64_t ld, int64_t cols) { return ld < cols || (ld % 8) != 0 || ld > INT32_MAX; }
bool bad_dims(int64_t rows, int64_t cols) { return rows < 0 || rows > INT32_MAX - 128 || cols <= 0 || (cols % 8) != 0 || cols > kMaxCols; }

constexpr int kMostSmem = 200 * 1024;

// CTAs of the backward pass, each of which leaves one partial of dgain.  kBwdCtas bounds the workspace, which is asked for without a device: eight per
// SM of this chip, of which fewer fit (16384 x 4096: 19.4 MB, of which 296 CTAs use 4.8).
constexpr int64_t kBwdCtas = 8 * 148;
int64_t bwd_ctas(int64_t rows, int groups, int64_t fit)
{
    const int64_t want = ceil_div(rows, groups), cap = fit < kBwdCtas ? fit : kBwdCtas;
    return want < cap ? want : cap;
}

// Every kernel here may be set up while the one before it on the stream ends, and waits for that one before it touches memory (chain_start).
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
    // of the outputs only h may be an input, row for row
    if ((t->h && t->h == t->x && t->ld_h != t->ld_x) || (t->h && t->h == t->residual && t->ld_h != t->ld_residual)) return SNIP_ERR_ARG;
    const void *out[] = {t->h, t->y, t->rstd, t->codes, t->scales, t->codes_t, t->scales_t}, *in[] = {t->x, t->residual, t->gain};
    for (int i = 0; i < 7; ++i) {
        for (int j = i + 1; out[i] && j < 7; ++j)
            if (out[i] == out[j]) return SNIP_ERR_ARG;
        for (int j = 0; out[i] && j < 3; ++j)
            if (out[i] == in[j] && (i > 0 || j == 2)) return SNIP_ERR_ARG;
    }
    int rc = require_sm100();
    if (rc) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    NormArgs a = {};
    a.x = static_cast<const uint16_t *>(t->x);
    a.residual = static_cast<const uint16_t *>(t->residual);
    a.gain = t->gain;
    a.h = static_cast<uint16_t *>(t->h);
    a.y = static_cast<uint16_t *>(t->y);
    a.rstd = t->rstd;
    a.codes = static_cast<uint8_t *>(t->codes);
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
    cudaError_t e = cudaSuccess;
    auto launch = [&](auto form, auto v, auto threads, auto stages, auto res, auto fmt) {
        if constexpr (fwd_reaches(form(), res(), fmt() != SNIP_FMT_BF16)) {
            constexpr auto kernel = rmsnorm_kernel<v(), threads(), stages(), res(), fmt()>;
            n = resident<kernel>(s.threads, s.smem, kMostSmem);
            const int64_t want = ceil_div(t->rows, s.groups), cap = (int64_t)n * gemm_sm_count();
            if (n) e = launch_behind(kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(s.threads), s.smem, st, a);
        }
    };
    auto with_fmt = [&](auto form, auto v, auto threads, auto stages, auto res) {
        if (!a.codes) launch(form, v, threads, stages, res, Int<SNIP_FMT_BF16>{});
        else if (t->fmt == SNIP_FMT_FP8_E4M3) launch(form, v, threads, stages, res, Int<SNIP_FMT_FP8_E4M3>{});
        else launch(form, v, threads, stages, res, Int<SNIP_FMT_FP4_E2M1>{});
    };
#define SNIP_LAUNCH(FORM, V, THREADS, STAGES)                                                              \
    if (s.form == FORM) {                                                                                  \
        if (t->residual) with_fmt(Int<FORM>{}, Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::true_type{}); \
        else with_fmt(Int<FORM>{}, Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::false_type{});            \
    }
    SNIP_NORM_FWD_FORMS(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(e);
    if (!n) return SNIP_ERR_CUDA;
    if (!t->codes_t) return SNIP_OK;
    NormColsArgs d = {};
    d.h = static_cast<const uint16_t *>(t->residual ? t->h : t->x);
    d.gain = t->gain;
    d.rstd = t->rstd;
    d.codes_t = static_cast<uint8_t *>(t->codes_t);
    d.scales_t = t->scales_t;
    d.ld = (int32_t)(t->residual ? t->ld_h : t->ld_x);
    d.rows = a.rows;
    d.cols = a.cols;
    d.tiles_c = (int32_t)ceil_div(t->cols, kTile);
    d.tiles = (int32_t)(d.tiles_c * ceil_div(t->rows, kTile));
    d.gain_f32 = a.gain_f32;
    auto launch_cols = [&](auto fmt) {
        constexpr auto kernel = rmsnorm_cols_kernel<fmt()>;
        constexpr int smem = (int)sizeof(ColsShared);
        n = resident<kernel>(kColsThreads, smem, smem);
        const int64_t cap = (int64_t)n * gemm_sm_count();
        if (n) e = launch_behind(kernel, dim3((unsigned)(d.tiles < cap ? d.tiles : cap)), dim3(kColsThreads), smem, st, d);
    };
    if (t->fmt_t == SNIP_FMT_FP8_E4M3) launch_cols(Int<SNIP_FMT_FP8_E4M3>{});
    else launch_cols(Int<SNIP_FMT_FP4_E2M1>{});
    SNIP_CUDA_TRY(e);
    return n ? SNIP_OK : SNIP_ERR_CUDA;
}

extern "C" int snip_rmsnorm_bwd_workspace(int64_t rows, int64_t cols, size_t *ws_bytes)
{
    using namespace snip;
    if (!ws_bytes) return SNIP_ERR_ARG;
    if (bad_dims(rows, cols)) return SNIP_ERR_SHAPE;
    // one partial per CTA of the largest grid
    const int64_t ctas = bwd_ctas(rows, bwd_shape(cols, 3, rows <= kFewRows).groups, kBwdCtas);
    *ws_bytes = align_up(sizeof(float) * (size_t)ctas * (size_t)cols, 256);
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
    if ((t->dx == t->dy && t->ld_dx != t->ld_dy) || (t->dx == t->dresidual && t->ld_dx != t->ld_dresidual) || t->dx == t->h || t->dx == t->gain ||
        t->dx == t->rstd || (t->dgain && (t->dgain == t->gain || t->dgain == t->dx || t->dgain == t->rstd || t->dgain == t->dy || t->dgain == t->h ||
                                          t->dgain == t->dresidual || t->dgain == ws)))
        return SNIP_ERR_ARG;
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
    cudaError_t e = cudaSuccess;
    auto launch = [&](auto form, auto v, auto threads, auto stages, auto res) {
        if constexpr (bwd_reaches(form(), res())) {
            constexpr auto kernel = rmsnorm_bwd_kernel<v(), threads(), stages(), res()>;
            ctas = bwd_ctas(t->rows, s.groups, (int64_t)resident<kernel>(s.threads, s.smem, kMostSmem) * gemm_sm_count());
            if (ctas) e = launch_behind(kernel, dim3((unsigned)ctas), dim3(s.threads), s.smem, st, a);
        }
    };
#define SNIP_LAUNCH(FORM, V, THREADS, STAGES)                                                              \
    if (s.form == FORM) {                                                                                  \
        if (t->dresidual) launch(Int<FORM>{}, Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::true_type{});  \
        else launch(Int<FORM>{}, Int<V>{}, Int<THREADS>{}, Int<STAGES>{}, std::false_type{});              \
    }
    SNIP_NORM_BWD_FORMS(SNIP_LAUNCH)
#undef SNIP_LAUNCH
    SNIP_CUDA_TRY(e);
    if (!ctas) return SNIP_ERR_CUDA;
    if (t->dgain) {
        SNIP_CUDA_TRY(launch_behind(dgain_reduce_kernel, dim3((unsigned)ceil_div(t->cols, 32)), dim3(32, 32), 0, st, static_cast<const float *>(a.partials),
                                    (int)ctas, (int)a.cols, t->dgain, (int)t->accumulate));
    }
    return SNIP_OK;
}
