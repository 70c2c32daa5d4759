// What an eviction from a quantized cache goes by, and the eviction, for gfx950.
//
// key_weights: W_j (+)= sum over the queries i and the heads of a group of P_ij = exp(S_ij - m_i) / l_i, S as in the attention calls.  A weight needs m and l of its
// whole row, so the scores are gone through twice.  With few rows to a key head (a decode step) the first pass leaves the scores in the workspace and K is read once;
// with many (a prompt) the second computes them again, now a key to a lane: 32x32 accumulators of Q K^T hold 16 queries of one key each, whose weights a lane adds up by itself.
// All sums are in a fixed order (no atomics on floating point values): equal calls give equal results.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "intfa.h"
#include "intfa_internal.h"
#include "intfa_device.h"
#include "intfa_cache.h"
#include "intfa_cache_plan.h"

namespace {

using namespace ifa_cache;

struct WeightsCall {
    const int8_t *Q, *K;
    const float *sQ, *sK, *W;                                    // W null: zeros
    const int *lens;
    int B, Hkv, G, Nq, Nk;
    unsigned G_inverse;                                          // 2^32 / G, rounded up (G > 1)
    int parts;                                                   // of the keys, in the first pass
    int slices;                                                  // of the rows, in the second
    float2 *stats;                                               // [part][unit][rows]: maximum (log2 units) and sum of a row over that part
    float2 *rows_out;                                            // [unit][rows]: maximum + log2(sum) of a row (inf: it sees nothing) and s_Q log2(e); null with stored scores
    float *scores;                                               // [unit][rows][score_stride] in log2 units, or null
    long score_stride;
    float *sums;                                                 // [slice][unit][Nk], or null: straight to out
    float *out;
};
__device__ __forceinline__ long query_row(const WeightsCall &c, int unit, int row) {             // row (i, g) of unit (b, hk), in the order of Q
    return (static_cast<long>(unit) * c.G + row % c.G) * c.Nq + row / c.G;
}

// what the second pass takes of a row
__device__ __forceinline__ float2 row_of_second_pass(float m, float sum, float sq) {
    return float2{m == -INFINITY ? INFINITY : m + __builtin_amdgcn_logf(sum), sq * LOG2E};
}
[[maybe_unused]] __device__ __forceinline__ void write_stats(const WeightsCall &c, int units, int part, int unit, int row, float m, float sum) {
    const long rows = static_cast<long>(c.G) * c.Nq, at = unit * rows + row;
    if (c.rows_out && c.parts == 1) c.rows_out[at] = row_of_second_pass(m, sum, c.sQ[query_row(c, unit, row)]);
    else c.stats[part * units * rows + at] = float2{m, sum};
}

// ---- first pass: maximum and sum of 32 rows over a part of the keys, the wavefronts taking every fourth tile of 32 keys, each for itself -----------------
constexpr int KW_WAVES = 4, KW_ST = 2;
template <int D> struct SmemRows {
    alignas(4096) int8_t k[KW_WAVES][KW_ST][32 * D];
    alignas(128) float sk[KW_WAVES][KW_ST][32];
    float2 ml[KW_WAVES][32];
};

template <int D, bool NT>
__global__ __launch_bounds__(64 * KW_WAVES) void key_weights_rows_kernel(WeightsCall c, int units, int row_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemRows<D> sm;
    constexpr int KS = D / 32, KB = 32 * D, PER_TILE = K_PIECES<D> + 1;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int block = blockIdx.x, in8 = block % (8 * row_tiles), share = block / (8 * row_tiles) * 8 + (in8 & 7), rt = in8 >> 3;
    const int unit = share / c.parts, part = share % c.parts;
    if (unit >= units) return;
    const int rows = c.G * c.Nq, row0 = 32 * rt, last_row = imin(row0 + 31, rows - 1), row = imin(row0 + r, rows - 1);
    const int L = keys_of(c.lens, unit / c.Hkv, c.Nk);
    const int p0 = L - c.Nq + row0 / c.G, p1 = L - c.Nq + last_row / c.G, p = L - c.Nq + row / c.G;
    const int keys = imax(0, p1 + 1);                            // that any of the rows sees
    const int tiles = (keys + 31) / 32, per = (tiles + c.parts - 1) / c.parts, t0 = part * per, t1 = imin(tiles, t0 + per);
    const BufRsrc rK = make_rsrc(c.K + static_cast<long>(unit) * c.Nk * D, keys * D), rS = make_rsrc(c.sK + static_cast<long>(unit) * c.Nk, keys * 4);

    const Lane<D, true> lo(lane);
    const lds_ptr kbuf = (lds_ptr)(&sm.k[wave][0][0]), skbuf = (lds_ptr)(&sm.sk[wave][0][0]);
    auto stage = [&](int t, int slot) {
        copy_pieces<K_PIECES<D>, NT>(rK, kbuf + slot * KB, lo.gk, lo.gk, t < t1 ? 32 * t * D : NOTHING);
        if (g == 0) lds_copy4(rS, skbuf + slot * 128, 4 * r, t < t1 ? 128 * t : NOTHING);
    };
    const int first = t0 + wave;
#pragma unroll
    for (int s = 0; s < KW_ST; ++s) stage(first + s * KW_WAVES, s);
    const long qrow = query_row(c, unit, row);
    v4i qf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const v4i *>(c.Q + qrow * D + 32 * kk + 16 * g);
    const float sq2 = c.sQ[qrow] * LOG2E;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[kk]));
    v16i bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I;
    asm volatile("" : "+v"(bias));

    float m2 = -INFINITY, l = 0.0f;
    float *const scores = c.scores ? c.scores + (static_cast<long>(unit) * rows + row0 + r) * c.score_stride + 4 * g : nullptr;
    int slot = 0;
    for (int t = first; t < t1; t += KW_WAVES) {
        // (a stored score counts with the copies: no more of them than KW_ST - 1 tiles have can be behind this tile's)
        wait_vmcnt<PER_TILE *(KW_ST - 1)>();
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        v4i kop[KS];
        v4f skv[4];
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) kop[kk] = *reinterpret_cast<LDS_AS const v4i *>(lds_xor(kbuf + slot * KB, 32 * kk, lo.k0));
#pragma unroll
        for (int vq = 0; vq < 4; ++vq) skv[vq] = *reinterpret_cast<LDS_AS const v4f *>(skbuf + slot * 128 + 16 * g + 32 * vq);
        wait_lds();
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        v16i acc = bias;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kop[kk], qf[kk], acc, 0, 0, 0);
        float x[16], tmax = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = (__int_as_float(acc[v]) - ACC_BIAS_F) * skv[v >> 2][v & 3] * sq2;
        if (32 * t + 31 > p0) {                                  // (wave-uniform) a row that does not see the whole tile
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (32 * t + 8 * (v >> 2) + 4 * g + (v & 3) > p) x[v] = -INFINITY;
        }
        if (scores && row0 + r < rows) {                         // (rows of whole tiles of 32: the last one is stored past the keys)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) *reinterpret_cast<v4f *>(scores + 32 * t + 8 * vq) = v4f{x[4 * vq], x[4 * vq + 1], x[4 * vq + 2], x[4 * vq + 3]};
        }
        stage(t + KW_ST * KW_WAVES, slot);                       // behind the scores, so that the wait above counts only copies that are younger than its tile
        __builtin_amdgcn_sched_barrier(0);
        slot = slot == KW_ST - 1 ? 0 : slot + 1;
#pragma unroll
        for (int v = 0; v < 16; ++v) tmax = fmaxf(tmax, x[v]);
        tmax = pair_max(tmax);
        const float m_new = fmaxf(m2, tmax), m_at = m_new == -INFINITY ? 0.0f : m_new;
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; ++v) s += __builtin_amdgcn_exp2f(x[v] - m_at);
        l = __builtin_fmaf(l, __builtin_amdgcn_exp2f(m2 - m_at), s);
        m2 = m_new;
    }
    wait_all_memory();
    l += swap32(l);
    if (g == 0) sm.ml[wave][r] = float2{m2, l};
    __syncthreads();
    if (tid < 32 && row0 + tid < rows) {
        float m = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < KW_WAVES; ++w) m = fmaxf(m, sm.ml[w][tid].x);
#pragma unroll
        for (int w = 0; w < KW_WAVES; ++w)
            if (sm.ml[w][tid].x != -INFINITY) sum += sm.ml[w][tid].y * __builtin_amdgcn_exp2f(sm.ml[w][tid].x - m);
        write_stats(c, units, part, unit, row0 + tid, m, sum);
    }
#endif
}

// ---- the same for tiles of 128 rows, which share the keys, 64 at a time, through LDS ------------------------------------------------
// A score costs the vector unit a subtraction, s_K, half a maximum, s_Q and m, exp2 (16 cycles) and an addition, four times the 8 cycles of its products.  The maximum that
// a sum refers to moves only when a block exceeds it by 2^8, a row by itself.
template <int D> struct SmemRowTile {
    alignas(4096) int8_t k[2][TILE_KEYS * D];
    alignas(256) float sk[2][TILE_KEYS];
};
template <int D>
__global__ __launch_bounds__(256, 4) void key_weights_row_tiles_kernel(WeightsCall c, int units, int row_tiles, int head_group) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemRowTile<D> sm;
    constexpr int KS = D / 32, KB = TILE_KEYS * D, KP = KB / 4096;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit, ord;
    map_workgroup(blockIdx.x, units, row_tiles * c.parts, head_group, true, unit, ord);
    const int rt = row_tiles - 1 - ord / c.parts, part = ord % c.parts;
    const int rows = c.G * c.Nq, row0 = TILE_ROWS * rt, last_row = imin(row0 + TILE_ROWS - 1, rows - 1), row = imin(row0 + 32 * wave + r, last_row);
    const int shift = keys_of(c.lens, unit / c.Hkv, c.Nk) - c.Nq;
    const int keys = imax(0, shift + last_row / c.G + 1), p = shift + row / c.G;
    const int w0 = shift + imin(row0 + 32 * wave, last_row) / c.G, w1 = shift + imin(row0 + 32 * wave + 31, last_row) / c.G;     // of the wavefront's first and last row
    const int blocks = (keys + TILE_KEYS - 1) / TILE_KEYS, per = (blocks + c.parts - 1) / c.parts, t0 = part * per, t1 = imin(blocks, t0 + per);
    const BufRsrc rK = make_rsrc(c.K + static_cast<long>(unit) * c.Nk * D, keys * D), rS = make_rsrc(c.sK + static_cast<long>(unit) * c.Nk, keys * 4);
    const Lane<D, true> lo(lane);
    const lds_ptr kbuf = (lds_ptr)(&sm.k[0][0]), skbuf = (lds_ptr)(&sm.sk[0][0]);
    auto stage = [&](int t, int slot) {
        copy_pieces<KP>(rK, kbuf + slot * KB + wave * KP * 1024, lo.gk, lo.gk, t * KB + wave * KP * 1024);
        if (wave == 3) lds_copy4(rS, skbuf + slot * 256, 4 * lane, t * 256);
    };
    if (t0 < t1) stage(t0, 0);
    const long qrow = query_row(c, unit, row);
    v4i qf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const v4i *>(c.Q + qrow * D + 32 * kk + 16 * g);
    const float sq2 = p >= 0 ? query_scale(c.sQ[qrow], qf) : 1.0f;        // (padding: whatever its scale holds)
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[kk]));
    v16i bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I;
    asm volatile("" : "+v"(bias));
    float m2 = -INFINITY, l = 0.0f;
    wait_all_memory();
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int slot = (t - t0) & 1, j0 = TILE_KEYS * t;
        if (t + 1 < t1) stage(t + 1, slot ^ 1);
        if (w1 >= j0 && row0 + 32 * wave < rows) {               // (wave-uniform)
            float a[2][16];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                v16i acc = bias;
#pragma unroll
                for (int kk = 0; kk < KS; ++kk)
                    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<LDS_AS const v4i *>(lds_xor(kbuf + slot * KB, 32 * kk, lo.k0) + 32 * mt * D), qf[kk], acc, 0, 0, 0);
#pragma unroll
                for (int vq = 0; vq < 4; ++vq) {
                    const v4f skv = *reinterpret_cast<LDS_AS const v4f *>(skbuf + slot * 256 + 16 * g + 128 * mt + 32 * vq);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[mt][4 * vq + e] = (__int_as_float(acc[4 * vq + e]) - ACC_BIAS_F) * skv[e];
                }
            }
            if (w0 < j0 + TILE_KEYS - 1) {
                const uint64_t seen = keys_seen(p - j0, 0, 0);
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (!(static_cast<uint32_t>(seen >> (32 * mt)) >> (4 * g) & (1u << (8 * (v >> 2) + (v & 3))))) a[mt][v] = -INFINITY;
            }
            float bmax = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int v = 0; v < 16; ++v) bmax = fmaxf(bmax, a[mt][v]);
            const float top = pair_max(bmax) * sq2;
            if (top > m2 + 8.0f) {
                l *= __builtin_amdgcn_exp2f(m2 - top);           // exp2(-inf) = 0
                m2 = top;
            }
            const float m = m2 == -INFINITY ? 0.0f : m2;
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int v = 0; v < 16; ++v) s[v & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(a[mt][v], sq2, -m));
            l += (s[0] + s[1]) + (s[2] + s[3]);
        }
        wait_all_memory();
        __syncthreads();
    }
    l += swap32(l);
    if (g == 0 && row0 + 32 * wave + r < rows) write_stats(c, units, part, unit, row, m2, l);
#endif
}

// parts first, first + step, ... of a row, eight loads at a time
__device__ __forceinline__ float2 join_parts(const float2 *stats, long stride, int parts, int first, int step) {
    float m = -INFINITY, sum = 0.0f;
    for (int i0 = first; i0 < parts; i0 += 8 * step) {
        float2 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            x[k] = float2{-INFINITY, 0.0f};
            if (i0 + k * step < parts) x[k] = stats[(i0 + k * step) * stride];
        }
        float m_new = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) m_new = fmaxf(m_new, x[k].x);
        if (m_new == -INFINITY) continue;
        sum *= __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k].y * __builtin_amdgcn_exp2f(x[k].x - m);
    }
    return float2{m, sum};
}
__global__ __launch_bounds__(256) void key_weights_join_kernel(WeightsCall c, long rows) {
    const long at = blockIdx.x * 256L + threadIdx.x;
    if (at >= rows) return;
    const float2 x = join_parts(c.stats + at, rows, c.parts, 0, 1);
    const int per = c.G * c.Nq;
    c.rows_out[at] = row_of_second_pass(x.x, x.y, c.sQ[query_row(c, static_cast<int>(at / per), static_cast<int>(at % per))]);
}

// ---- second pass, from stored scores: four keys to a thread ------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void key_weights_stored_kernel(WeightsCall c, int units, int blocks, bool whole) {
    __shared__ float2 st[STORED_ROWS];
    const int unit = blockIdx.x / blocks, j = (blockIdx.x % blocks * 256 + threadIdx.x) * 4, rows = c.G * c.Nq;
    const int L = c.lens ? imax(0, imin(c.lens[unit / c.Hkv], c.Nk)) : c.Nk;
    static_assert(STORED_ROWS * 16 == 256, "16 lanes to a row");
    const int row = threadIdx.x >> 4, lane = threadIdx.x & 15;
    float2 x = row < rows ? join_parts(c.stats + static_cast<long>(unit) * rows + row, static_cast<long>(units) * rows, c.parts, lane, 16) : float2{-INFINITY, 0.0f};
#pragma unroll
    for (int s = 8; s; s >>= 1) {
        const float2 y = {__shfl_xor(x.x, s), __shfl_xor(x.y, s)};
        const float m = fmaxf(x.x, y.x), at = m == -INFINITY ? 0.0f : m;
        x = float2{m, x.y * __builtin_amdgcn_exp2f(x.x - at) + y.y * __builtin_amdgcn_exp2f(y.x - at)};
    }
    // maximum and 1 / sum; a row that sees nothing: 0 and 0, so that its weights are 0
    if (lane == 0) st[row] = x.x == -INFINITY ? float2{0.0f, 0.0f} : float2{x.x, 1.0f / x.y};
    __syncthreads();
    if (j >= c.Nk) return;
    v4f w = {0.0f, 0.0f, 0.0f, 0.0f};
    if (j < L) {
        const float *x = c.scores + static_cast<long>(unit) * rows * c.score_stride + j;
        for (int r0 = 0; r0 < rows; r0 += 4) {
            // Tiles of 32 keys are stored up to the last that a row sees, and its scores are -inf behind what it sees.
            v4f y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = *reinterpret_cast<const v4f *>(x + imin(r0 + k, rows - 1) * c.score_stride);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 s = st[imin(r0 + k, rows - 1)];
                const float f = r0 + k < rows ? s.y : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(y[k][e] - s.x), f, w[e]);
            }
        }
    }
    const long at = static_cast<long>(unit) * c.Nk + j;
    if (whole) {                                                 // rows of W of whole 16 bytes
        v4f old = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c.W) old = *reinterpret_cast<const v4f *>(c.W + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) old[e] = (j + e < L ? w[e] : 0.0f) + old[e];
        *reinterpret_cast<v4f *>(c.out + at) = old;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (j + e < c.Nk) c.out[at + e] = (j + e < L ? w[e] : 0.0f) + (c.W ? c.W[at + e] : 0.0f);
}

// ---- second pass, scores computed again: 256 keys to a workgroup, a key to a lane ---------------------------------------------------------------
// The rows go by in tiles of 64 through LDS, shared by the four wavefronts of 64 keys (two operands of K in registers, so that what is read of the rows counts
// twice); a slice of them per workgroup.  They are packed like everywhere, row (i, g) with g fastest: a row is a copy from a place of its own, and a few queries of many heads fill a tile.  The vector unit's part of a score: s_Q s_K, the subtraction of the start value, their product less the row's maximum + log2(sum), exp2 and the
// addition.  (Maximum and log2 in one number: it rounds by 2^-24 of itself, as scores do, and the rows' errors do not add up.)
template <int D> struct SmemKeys {
    alignas(4096) int8_t q[2][KW_ROWS * D];
    alignas(256) float2 row[2][KW_ROWS];
};
template <int D>
__global__ __launch_bounds__(256, 3) void key_weights_keys_kernel(WeightsCall c, int units, int key_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemKeys<D> sm;
    constexpr int KS = D / 32, QB = KW_ROWS * D, PIECES = QB / 4096;             // copies of a wavefront to a tile
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the workgroups of a unit on one XCD as far as units go round; the first keys, which most rows see, first
    const int per_unit = key_tiles * c.slices, x = blockIdx.x & 7, s = blockIdx.x >> 3;
    const int unit = s / per_unit * 8 + x, kt = s % per_unit / c.slices, slice = s % c.slices;
    if (unit >= units) return;
    const int L = keys_of(c.lens, unit / c.Hkv, c.Nk), shift = L - c.Nq;
    const int j0 = KW_KEYS * kt, jw = j0 + 64 * wave;
    const int rows = c.G * c.Nq;
    auto first_row = [&](int j) { return imin(imax(0, j - shift), c.Nq) * c.G; };               // the first row that sees key j
    const int r0 = first_row(j0), total = j0 < L ? (rows - r0 + KW_ROWS - 1) / KW_ROWS : 0;
    const int per = (total + c.slices - 1) / c.slices, t0 = slice * per, t1 = imin(total, t0 + per);
    float sum[2] = {0.0f, 0.0f};
    if (t0 < t1) {
        const long kb = static_cast<long>(unit) * c.Nk;
        v4i kop[2][KS];                                          // (keys at or beyond L: zeros, left out at the end)
        float sk[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = jw + 32 * h + r;
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                v4i y = {0, 0, 0, 0};
                if (j < L) y = *reinterpret_cast<const v4i *>(c.K + (kb + j) * D + 32 * kk + 16 * g);
                kop[h][kk] = y;
            }
            sk[h] = j < L ? c.sK[kb + j] : 0.0f;
        }
        const int lane_first[2] = {first_row(jw + r), first_row(jw + 32 + r)}, wave_first = first_row(jw), wave_last = first_row(jw + 63);
        const Lane<D, true> lo(lane);
        const lds_ptr qbuf = (lds_ptr)(&sm.q[0][0]), rbuf = (lds_ptr)(&sm.row[0][0]);
        const BufRsrc rQ = make_rsrc(c.Q + static_cast<long>(unit) * rows * D, rows * D), rM = make_rsrc(c.rows_out + static_cast<long>(unit) * rows, rows * 8);
        auto stage = [&](int t, int slot) {                      // (rows past the last come as zeros)
            const int tile = r0 + t * KW_ROWS;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int in = (wave * PIECES + i) * (1024 / D) + lane / (D / 16), row = tile + in;
                // row = q G + g; the product with 2^32 / G, rounded up, is right or one too large
                int q = c.G == 1 ? row : static_cast<int>(__umulhi(static_cast<unsigned>(row), c.G_inverse)), g_of = row - q * c.G;
                if (g_of < 0) --q, g_of += c.G;
                const unsigned from = row < rows ? static_cast<unsigned>(g_of * c.Nq + q) * D + (lo.gk & (D - 1)) : static_cast<unsigned>(NOTHING);
                lds_copy16(rQ, qbuf + slot * QB + (wave * PIECES + i) * 1024, from, 0);
            }
            if (wave < 2) lds_copy4(rM, rbuf + slot * 512 + 256 * wave, 4 * lane, tile * 8 + 256 * wave);
        };
        v16i bias;
#pragma unroll
        for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I;
        asm volatile("" : "+v"(bias));
        stage(t0, 0);
        wait_all_memory();
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int slot = (t - t0) & 1;
            if (t + 1 < t1) stage(t + 1, slot ^ 1);
#pragma unroll
            for (int q = 0; q < KW_ROWS / 32; ++q) {
                const int tile = r0 + t * KW_ROWS + 32 * q;      // the first of these rows
                if (tile >= rows || tile + 31 < wave_first) continue;            // (wave-uniform) none sees any of the wavefront's keys
                v4i qop[KS];
                v4f row[4][2];
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) qop[kk] = *reinterpret_cast<LDS_AS const v4i *>(lds_xor(qbuf + slot * QB, 32 * kk, lo.k0) + 32 * q * D);
#pragma unroll
                for (int vq = 0; vq < 4; ++vq)
#pragma unroll
                    for (int e = 0; e < 2; ++e) row[vq][e] = *reinterpret_cast<LDS_AS const v4f *>(rbuf + slot * 512 + 256 * q + 64 * vq + 32 * g + 16 * e);
                const bool masked = tile < wave_last || tile + 32 > rows;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v16i acc = bias;
#pragma unroll
                    for (int kk = 0; kk < KS; ++kk) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(qop[kk], kop[h][kk], acc, 0, 0, 0);
                    float y[16];
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const v4f &x4 = row[v >> 2][(v & 3) >> 1];
                        y[v] = __builtin_fmaf(__int_as_float(acc[v]) - ACC_BIAS_F, sk[h] * x4[2 * (v & 1) + 1], -x4[2 * (v & 1)]);
                    }
                    if (masked) {
                        // from the first row that sees the lane's key to the last there is
                        const uint32_t seen = static_cast<uint32_t>(below(rows - tile) & ~below(lane_first[h] - tile)) >> (4 * g);
#pragma unroll
                        for (int v = 0; v < 16; ++v)
                            if (!(seen & (1u << (8 * (v >> 2) + (v & 3))))) y[v] = -INFINITY;
                    }
#pragma unroll
                    for (int v = 0; v < 16; ++v) sum[h] += __builtin_amdgcn_exp2f(y[v]);
                }
            }
            wait_all_memory();
            __syncthreads();
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = jw + 32 * h + r;
        float w = sum[h] + swap32(sum[h]);
        if (g == 0 && j < c.Nk) {
            const long at = static_cast<long>(unit) * c.Nk + j;
            if (j >= L) w = 0.0f;
            if (c.sums) c.sums[static_cast<long>(slice) * units * c.Nk + at] = w;
            else c.out[at] = w + (c.W ? c.W[at] : 0.0f);
        }
    }
#endif
}
__global__ __launch_bounds__(256) void key_weights_add_kernel(WeightsCall c, long n) {
    const long at = blockIdx.x * 256L + threadIdx.x;
    if (at >= n) return;
    float s = 0.0f;
    for (int i = 0; i < c.slices; ++i) s += c.sums[i * n + at];
    c.out[at] = s + (c.W ? c.W[at] : 0.0f);
}

// ---- host --------------------------------------------------------------------------------------------------------
template <int D> int launch(WeightsCall c, const WeightsPlan &plan, hipStream_t st) {
    const int units = c.B * c.Hkv, unit_rows = c.G * c.Nq;
    const long rows = static_cast<long>(units) * unit_rows;
    if (plan.few) {
        const int row_tiles = (unit_rows + 31) / 32;
        const long grid = (static_cast<long>(units) * c.parts + 7) / 8 * 8 * row_tiles;
        if (plan.once) hipLaunchKernelGGL((key_weights_rows_kernel<D, true>), dim3(static_cast<unsigned>(grid)), dim3(64 * KW_WAVES), 0, st, c, units, row_tiles);
        else hipLaunchKernelGGL((key_weights_rows_kernel<D, false>), dim3(static_cast<unsigned>(grid)), dim3(64 * KW_WAVES), 0, st, c, units, row_tiles);
    } else {
        const int row_tiles = (unit_rows + TILE_ROWS - 1) / TILE_ROWS;
        hipLaunchKernelGGL((key_weights_row_tiles_kernel<D>), dim3(static_cast<unsigned>(static_cast<long>(units) * row_tiles * c.parts)), dim3(256), 0, st, c, units, row_tiles, head_group_for(true, 0, 0));
    }
    if (plan.stored) {
        const int blocks = (c.Nk + 1023) / 1024;
        const bool whole = c.Nk % 4 == 0 && ifa_aligned16(c.W) && ifa_aligned16(c.out);
        hipLaunchKernelGGL(key_weights_stored_kernel, dim3(static_cast<unsigned>(units) * blocks), dim3(256), 0, st, c, units, blocks, whole);
    } else {
        if (c.parts > 1) hipLaunchKernelGGL(key_weights_join_kernel, dim3(static_cast<unsigned>((rows + 255) / 256)), dim3(256), 0, st, c, rows);
        const int key_tiles = (c.Nk + KW_KEYS - 1) / KW_KEYS;
        hipLaunchKernelGGL((key_weights_keys_kernel<D>), dim3(static_cast<unsigned>(key_tiles) * ((units + 7) / 8 * 8) * c.slices), dim3(256), 0, st, c, units, key_tiles);
        if (c.sums) {
            const long n = static_cast<long>(units) * c.Nk;
            hipLaunchKernelGGL(key_weights_add_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, st, c, n);
        }
    }
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}

int refuse_sizes(int B, int H, int Hkv, int Nq, int Nk, int d) {
    if (B <= 0 || H <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0 || d <= 0 || H % Hkv) return IFA_ERR_SHAPE;
    const long heads = static_cast<long>(B) * H, N = Nq > Nk ? Nq : Nk;
    if (heads > (1L << 40) / N / d) return IFA_ERR_SHAPE;
    if (d != 64 && d != 128) return IFA_ERR_UNSUPPORTED;
    if (static_cast<long>(Nk) * d * 2 > 0x7ff00000L || heads * Nq > 1L << 26 || heads > 1L << 23) return IFA_ERR_UNSUPPORTED;
    if (static_cast<long>(H / Hkv) * Nq * d > 0x7ff00000L || static_cast<long>(B) * Hkv * Nk > 1L << 30) return IFA_ERR_UNSUPPORTED;      // (a launch has less than 2^32 threads: two to a key)
    return IFA_OK;
}

// ---- eviction -----------------------------------------------------------------------------------------------------
// One workgroup to a key head finds the weight of the last key that stays (radix selection, 11 bits at a time) and writes the list of those that do, in order; a second launch moves the
// rows.  What bounds the pair is memory: 16 sequences x 8 heads, 4096 of 16384 keys of d = 128 with fp16 V, 421 MB moved.
struct EvictCall {
    const int8_t *K, *V;
    const float *sK, *W;
    const int *lens;
    int B, Hkv, Nk, d, v_row, keep, recent, sinks;               // v_row: bytes of a row of V
    int8_t *K_out, *V_out;
    float *sK_out, *W_out;
    int *index, *lens_out;
};
constexpr int SEL_WAVES = SEL_THREADS / 64, BINS = 2048;

// Larger weight, larger number; -0 is 0, a NaN is below everything.  Between 1 and 0xff800000 (+inf): 0 is left for places without a key, the largest number for keys that stay anyway.
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    return w != w ? 1u : u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t NO_KEY = 0, STAYS = 0xffffffffu;

// The keys go by in rounds of 4096: wavefront w has 256 of them in a row, its lanes 64 at a time.  ROUNDS: of buffers of at most so many rounds the weights are read once and stay in
// registers; 0: longer ones are read again each time (from the caches: 4 bytes a key).  What bounds it is the vector unit: 16 keys a lane, each looked at four times (sinks and
// recent keys as the largest numbers rather than as conditions of their own: 15.8 us for 128 heads of 16384 keys, 18.5 before).
template <int ROUNDS>
__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(EvictCall c) {
    __shared__ uint32_t bins[BINS];
    __shared__ uint32_t wave_total[SEL_WAVES];
    __shared__ uint32_t found[2];                                // digit, how many keys are wanted among those that have it
    __shared__ int2 counts[2][SEL_WAVES];
    const int unit = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = c.lens ? imax(0, imin(c.lens[unit / c.Hkv], c.Nk)) : c.Nk;
    int *const index = c.index + static_cast<long>(unit) * c.keep;
    if (unit % c.Hkv == 0 && tid == 0) c.lens_out[unit / c.Hkv] = imin(n, c.keep);
    if (n <= c.keep) {
        for (int s = tid; s < c.keep; s += SEL_THREADS) index[s] = s < n ? s : -1;
        return;
    }
    const float *const W = c.W + static_cast<long>(unit) * c.Nk;
    const int first = c.sinks, last = n - c.recent;              // the keys that are chosen from: [first, last)
    const int mine = wave * 256 + lane;                          // (of a round: and 64, 128, 192 further on)
    auto number = [&](int j, float w) { return j >= n ? NO_KEY : j < first || j >= last ? STAYS : order_of(w); };
    uint32_t kept[ROUNDS > 0 ? ROUNDS : 1][4];
    if constexpr (ROUNDS > 0) {
        float w[ROUNDS][4];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = i * SEL_ROUND + mine + 64 * e;
                w[i][e] = j < n ? W[j] : 0.0f;
            }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) kept[i][e] = number(i * SEL_ROUND + mine + 64 * e, w[i][e]);
    }
    // f(place of a round, the number there) for every place of every round; all of them, so that wavefronts stay together.  after(round)
    auto rounds = [&](auto f, auto after) {
        auto one = [&](int i, int slot) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = i * SEL_ROUND + mine + 64 * e;
                f(e, ROUNDS > 0 ? kept[slot][e] : number(j, j < n ? W[j] : 0.0f));
            }
            after(i);
        };
        if constexpr (ROUNDS > 0) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i)
                if (i * SEL_ROUND < n) one(i, i);
        } else
            for (int i = 0; i * SEL_ROUND < n; ++i) one(i, 0);
    };
    // The want-th largest weight, 11 + 11 + 10 bits from the top.  Keys that stay anyway and places without one are left out of the first count (the later ones leave them out by
    // their bits): so many equal numbers would queue at one bin.
    uint32_t want = c.keep - c.sinks - c.recent, prefix = 0;
    auto digit = [&](auto above, auto shift_) {                  // among the numbers whose bits from `above` on are `prefix`
        constexpr int ABOVE = decltype(above)::value, SHIFT = decltype(shift_)::value, WIDTH = ABOVE - SHIFT;
        for (int i = tid; i < BINS; i += SEL_THREADS) bins[i] = 0;
        __syncthreads();
        rounds([&](int, uint32_t u) {
            if (ABOVE == 32 ? u + 1 > 1 : u >> (ABOVE & 31) == prefix) atomicAdd(&bins[u >> SHIFT & ((1u << WIDTH) - 1)], 1u);
        }, [](int) {});
        __syncthreads();
        // from the top bin down: thread t has bins 2047 - 2 t and the one below
        const int b0 = BINS - 1 - 2 * tid;
        const uint32_t c0 = bins[b0], c1 = bins[b0 - 1];
        uint32_t run = c0 + c1;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t y = __shfl_up(run, s);
            if (lane >= s) run += y;
        }
        if (lane == 63) wave_total[wave] = run;
        __syncthreads();
        uint32_t before = run - c0 - c1;
#pragma unroll
        for (int w = 0; w < SEL_WAVES; ++w) before += w < wave ? wave_total[w] : 0;
        if (before < want && want <= before + c0) found[0] = b0, found[1] = want - before;
        else if (before + c0 < want && want <= before + c0 + c1) found[0] = b0 - 1, found[1] = want - before - c0;
        __syncthreads();
        prefix = prefix << WIDTH | found[0];
        want = found[1];
    };
    if (want) {
        digit(std::integral_constant<int, 32>{}, std::integral_constant<int, 21>{});
        digit(std::integral_constant<int, 21>{}, std::integral_constant<int, 10>{});
        digit(std::integral_constant<int, 10>{}, std::integral_constant<int, 0>{});
    } else prefix = STAYS - 1;                                   // none by its weight
    // `prefix` is the number of the last key that stays, `want` how many of those equal to it do: the first ones
    int base = 0, equal_base = 0, n_more = 0, n_equal = 0;
    bool more[4], equal[4];
    auto in_front = [](uint64_t ballot) { return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(ballot >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(ballot), 0))); };
    rounds([&](int e, uint32_t u) {
        more[e] = u > prefix, equal[e] = u == prefix;
        n_more += __popcll(__ballot(more[e])), n_equal += __popcll(__ballot(equal[e]));
    }, [&](int i) {
        int2 *const all = counts[i & 1];
        if (lane == 0) all[wave] = int2{n_more, n_equal};
        __syncthreads();
        int my_more = base, my_equal = equal_base;               // kept (without the equal ones) and equal ones in front of this wavefront's keys
#pragma unroll
        for (int w = 0; w < SEL_WAVES; ++w) {
            const int2 x = all[w];
            if (w < wave) my_more += x.x, my_equal += x.y;
            base += x.x, equal_base += x.y;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t bm = __ballot(more[e]), be = __ballot(equal[e]);
            const int rank = my_equal + in_front(be);
            if (more[e] || (equal[e] && rank < static_cast<int>(want)))
                index[my_more + in_front(bm) + imin(rank, static_cast<int>(want))] = i * SEL_ROUND + mine + 64 * e;
            my_more += __popcll(bm), my_equal += __popcll(be);
        }
        n_more = n_equal = 0;
    });
}

// d / 16 lanes to a key, each with 16 bytes of K and of V (fp16: twice) of four keys at a time; the scales and weights go with the first two lanes
constexpr int MOVE_AT_ONCE = 4;
template <int VB>
__global__ __launch_bounds__(256) void evict_move_kernel(EvictCall c, int lanes, int blocks) {
    const int unit = blockIdx.x / blocks, per_block = 256 / lanes, in = threadIdx.x / lanes, part = threadIdx.x % lanes;
    if (in >= per_block) return;
    const long from = static_cast<long>(unit) * c.Nk, to = static_cast<long>(unit) * c.keep;
    const int s0 = blockIdx.x % blocks * per_block * MOVE_AT_ONCE + in;
    int j[MOVE_AT_ONCE];
    v4i k[MOVE_AT_ONCE], v[MOVE_AT_ONCE][VB];
    float x[MOVE_AT_ONCE];
#pragma unroll
    for (int i = 0; i < MOVE_AT_ONCE; ++i) {
        const int s = s0 + i * per_block;
        j[i] = s < c.keep ? c.index[to + s] : -1;
    }
    const float *const small = part == 0 ? c.sK : c.W;
#pragma unroll
    for (int i = 0; i < MOVE_AT_ONCE; ++i) {
        k[i] = v4i{0, 0, 0, 0};
        x[i] = 0.0f;
#pragma unroll
        for (int e = 0; e < VB; ++e) v[i][e] = v4i{0, 0, 0, 0};
        if (j[i] >= 0) {
            k[i] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(c.K + (from + j[i]) * c.d + 16 * part));
#pragma unroll
            for (int e = 0; e < VB; ++e) v[i][e] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(c.V + (from + j[i]) * c.v_row + 16 * (part + e * lanes)));
            if (part < 2) x[i] = small[from + j[i]];
        }
    }
    float *const small_out = part == 0 ? c.sK_out : c.W_out;
#pragma unroll
    for (int i = 0; i < MOVE_AT_ONCE; ++i) {
        const int s = s0 + i * per_block;
        if (s >= c.keep) continue;
        __builtin_nontemporal_store(k[i], reinterpret_cast<v4i *>(c.K_out + (to + s) * c.d + 16 * part));
#pragma unroll
        for (int e = 0; e < VB; ++e) __builtin_nontemporal_store(v[i][e], reinterpret_cast<v4i *>(c.V_out + (to + s) * c.v_row + 16 * (part + e * lanes)));
        if (part < 2) small_out[to + s] = x[i];
        if (lanes == 1) c.W_out[to + s] = j[i] < 0 ? 0.0f : c.W[from + j[i]];
    }
}

bool overlap(const void *a, long na, const void *b, long nb) {
    const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
    return x < y + nb && y < x + na;
}

}  // namespace

extern "C" long ifa_key_weights_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d) {
    if (refuse_sizes(B, H, Hkv, Nq, Nk, d)) return -1;
    return weights_plan(B, Hkv, H / Hkv, Nq, Nk, d).bytes();
}

extern "C" int key_weights(const signed char *Q_i8, const signed char *K_i8, const float *s_Q, const float *s_K, const int *lens, const float *W,
                           int B, int H, int Hkv, int Nq, int Nk, int d, float *W_out, void *workspace, long workspace_bytes, void *hip_stream) {
    if (const int rc = refuse_sizes(B, H, Hkv, Nq, Nk, d)) return rc;
    if (!Q_i8 || !K_i8 || !s_Q || !s_K || !W_out || !workspace) return IFA_ERR_NULL;
    if (!ifa_aligned16(Q_i8) || !ifa_aligned16(K_i8) || (reinterpret_cast<uintptr_t>(workspace) & 255)) return IFA_ERR_UNSUPPORTED;
    for (const void *p : {static_cast<const void *>(s_Q), static_cast<const void *>(s_K), static_cast<const void *>(lens), static_cast<const void *>(W), static_cast<const void *>(W_out)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return IFA_ERR_UNSUPPORTED;
    const long n = static_cast<long>(B) * Hkv * Nk * 4;
    if (W && W != W_out && overlap(W, n, W_out, n)) return IFA_ERR_UNSUPPORTED;      // (in place or apart, not shifted)
    const WeightsPlan plan = weights_plan(B, Hkv, H / Hkv, Nq, Nk, d);
    if (workspace_bytes < plan.bytes()) return IFA_ERR_WORKSPACE;
    WeightsCall c = {};
    c.Q = Q_i8, c.K = K_i8, c.sQ = s_Q, c.sK = s_K, c.W = W, c.lens = lens, c.out = W_out;
    c.B = B, c.Hkv = Hkv, c.G = H / Hkv, c.Nq = Nq, c.Nk = Nk, c.G_inverse = static_cast<unsigned>(((1ull << 32) + c.G - 1) / c.G), c.parts = plan.parts, c.slices = plan.slices;
    char *const ws = static_cast<char *>(workspace);
    c.stats = reinterpret_cast<float2 *>(ws);
    c.rows_out = plan.stored ? nullptr : reinterpret_cast<float2 *>(ws + plan.stats);
    c.scores = plan.stored ? reinterpret_cast<float *>(ws + plan.stats) : nullptr;
    c.score_stride = plan.stride;
    c.sums = plan.sums ? reinterpret_cast<float *>(ws + plan.stats + plan.rows) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return d == 128 ? launch<128>(c, plan, st) : launch<64>(c, plan, st);
}

extern "C" int evict_keys(const signed char *K_i8, const float *s_K, const void *V, int v_bytes, const float *W, const int *lens,
                          int B, int Hkv, int Nk, int d, int keep, int recent, int sinks,
                          signed char *K_out, float *s_K_out, void *V_out, float *W_out, int *index, int *lens_out, void *hip_stream) {
    if (!K_i8 || !s_K || !V || !W || !K_out || !s_K_out || !V_out || !W_out || !index || !lens_out) return IFA_ERR_NULL;
    if (B <= 0 || Hkv <= 0 || Nk <= 0 || d <= 0 || keep <= 0 || recent < 0 || sinks < 0) return IFA_ERR_SHAPE;
    const long units = static_cast<long>(B) * Hkv;
    if (keep > Nk || static_cast<long>(recent) + sinks > keep || units > (1L << 40) / Nk / d) return IFA_ERR_SHAPE;
    if (v_bytes != 1 && v_bytes != 2) return IFA_ERR_DTYPE;
    if ((d & 15) || d > 1024 || Nk > 0x7fffffff - 8192 || units >= 1L << 22 || units * keep > (1L << 35) / d) return IFA_ERR_UNSUPPORTED;      // (a launch has less than 2^32 threads: 1024 to a head)
    for (const void *p : {static_cast<const void *>(K_i8), V, static_cast<const void *>(K_out), static_cast<const void *>(V_out)})
        if (!ifa_aligned16(p)) return IFA_ERR_UNSUPPORTED;
    for (const void *p : {static_cast<const void *>(s_K), static_cast<const void *>(W), static_cast<const void *>(lens), static_cast<const void *>(s_K_out),
                          static_cast<const void *>(W_out), static_cast<const void *>(index), static_cast<const void *>(lens_out)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return IFA_ERR_UNSUPPORTED;
    // rows move while others are still read: nothing is evicted in place
    const long in = units * Nk, out = units * keep;
    const struct { const void *p; long n; } read[] = {{K_i8, in * d}, {s_K, in * 4}, {V, in * d * v_bytes}, {W, in * 4}, {lens, lens ? 4L * B : 0}},
        written[] = {{K_out, out * d}, {s_K_out, out * 4}, {V_out, out * d * v_bytes}, {W_out, out * 4}, {index, out * 4}, {lens_out, 4L * B}};
    for (const auto &w : written) {
        for (const auto &r : read)
            if (overlap(w.p, w.n, r.p, r.n)) return IFA_ERR_UNSUPPORTED;
        for (const auto &o : written)
            if (&o != &w && overlap(w.p, w.n, o.p, o.n)) return IFA_ERR_UNSUPPORTED;
    }
    EvictCall c = {K_i8, static_cast<const int8_t *>(V), s_K, W, lens, B, Hkv, Nk, d, d * v_bytes, keep, recent, sinks,
                   K_out, static_cast<int8_t *>(V_out), s_K_out, W_out, index, lens_out};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto select = [&](auto rounds) { hipLaunchKernelGGL((evict_select_kernel<decltype(rounds)::value>), dim3(static_cast<unsigned>(units)), dim3(SEL_THREADS), 0, st, c); };
    switch (evict_rounds(Nk)) {
    case 1: select(std::integral_constant<int, 1>{}); break;
    case 4: select(std::integral_constant<int, 4>{}); break;
    case 8: select(std::integral_constant<int, 8>{}); break;
    default: select(std::integral_constant<int, 0>{});
    }
    const int lanes = d / 16, per_block = 256 / lanes * MOVE_AT_ONCE, blocks = (keep + per_block - 1) / per_block;
    auto move = [&](auto vb) { hipLaunchKernelGGL((evict_move_kernel<decltype(vb)::value>), dim3(static_cast<unsigned>(units) * blocks), dim3(256), 0, st, c, lanes, blocks); };
    if (v_bytes == 1) move(std::integral_constant<int, 1>{});
    else move(std::integral_constant<int, 2>{});
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}
