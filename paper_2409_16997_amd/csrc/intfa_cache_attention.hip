// Attention over a quantized cache for gfx950: with a sliding window and sinks, and over keys that a batch shares.
//
//     S = s_Q s_K (Q K^T)        v_mfma_i32_32x32x32_i8, exact in int32, fp32 scales
//     P~ = fp16(exp(S - m))      m 15 (in tiles of 128 rows 7 to 15) log2 units below the running maximum; l = the sum of the rounded weights in fp32
//     O = P~ V / l               v_mfma_f32_32x32x16_f16, fp32 accumulation; INT8 V enters as fp16 (exactly) and its scale meets O
//
// The weights are fp16 like those of the half-INT8 variant, for INT8 V too: rounded relative to themselves (2^-11) rather than on the grid of a running maximum, they hardly
// depend on where a sequence is cut, so its keys may be shared out over workgroups and the parts joined with e^{m_part - m}.  What ends that is the lower end of fp16: below 2^-14 a weight is
// rounded by 2^-25, whatever it is.  With the largest weight near the upper end rather than at 1 those 2^-25 are 2^-40 of it (tiles: 2^-32 at worst), so that a long rest of small weights
// counts: with 1 as the largest weight what 16384 keys give 18 nats below the first was 25 % off (tiles, 9000 keys: 100 %), like this .01 % (.9 %), in the same time.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <hip/hip_bf16.h>
#include <stdint.h>
#include <type_traits>

#include "intfa.h"
#include "intfa_internal.h"
#include "intfa_device.h"
#include "intfa_cache.h"
#include "intfa_cache_plan.h"

namespace {

using namespace ifa_cache;

// Four outputs of a row, to fp32, fp16 or bf16
__device__ __forceinline__ void store4(void *O, int o_dtype, long at, float a, float b, float c, float d) {
    if (o_dtype == IFA_F32) *reinterpret_cast<float4 *>(static_cast<float *>(O) + at) = float4{a, b, c, d};
    else if (o_dtype == IFA_F16) *reinterpret_cast<uint2 *>(static_cast<__half *>(O) + at) = Pack4<__half>::pack(a, b, c, d);
    else *reinterpret_cast<uint2 *>(static_cast<__hip_bfloat16 *>(O) + at) = Pack4<__hip_bfloat16>::pack(a, b, c, d);
}

// Row `row` of unit `unit` in Q and O (in rows)
__device__ __forceinline__ long row_of(const Call &c, bool all, int unit, int row) {
    const int per = c.Nq * c.G, b = all ? row / per : unit / c.Hkv, hk = all ? unit : unit % c.Hkv;
    const int in = all ? row % per : row, i = in / c.G, g = in % c.G;
    return (static_cast<long>(b * c.Hkv + hk) * c.G + g) * c.Nq + i;
}

// INT8 V: o is in units of one scale.  Own V whose scale is 0, or vanishes beside the shared one's so that the ratio of the two could leave the range of fp32 (|o| < 2^46), is
// taken as the zeros it is then: its keys have their weights, its values are not read and o stays in the shared keys' units.
[[maybe_unused]] __device__ __forceinline__ bool counts_as_zero(float own, float shared) { return fabsf(own) <= fabsf(shared) * 0x1p-64f; }

// ---- 32 rows against many keys: every wavefront for itself -------------------------------------------------------
// The four wavefronts of a workgroup hold the same 32 rows and take every fourth tile of 32 keys each, with an online softmax of their own; they meet
// once, at the end.  So the loop has no barrier: a wavefront copies its tile into LDS, ST tiles ahead, takes the operands of a tile to registers and
// asks for the one that goes into its place before it computes.  What bounds it is memory: 32 sequences x 8 heads on 4096 keys of d = 128 in 66.5 us, 6.1 TB/s.
constexpr int FEW_WAVES = 4;
[[maybe_unused]] constexpr float FEW_BELOW = 15.0f;              // the largest weight is 2^15
template <int D, bool VI8, int ST> struct SmemFew {
    static constexpr int KB = 32 * D, VB = 32 * V_ROW<D, VI8>;
    union {
        struct {
            alignas(4096) int8_t k[FEW_WAVES][ST][KB];
            alignas(4096) int8_t v[FEW_WAVES][ST][VB];
            alignas(128) float sk[FEW_WAVES][ST][32];
        };
        float o[FEW_WAVES][32][64];                              // when the loop is over: 64 columns at a time
    };
    float2 ml[FEW_WAVES][32];
};

// ALL: unit = key head, rows of the whole batch, the shared keys alone.  Otherwise unit = (sequence, key head), shared keys (if any) and its own.
#if defined(__HIP_DEVICE_COMPILE__)
template <int D, bool VI8, bool ALL, int ST, bool NT>
__device__ __forceinline__ void few_rows_of_a_unit(SmemFew<D, VI8, ST> &sm, const Call &c, int block, int units, int row_tiles) {
    constexpr int KS = D / 32, DT = D / 32, KB = 32 * D, VB = 32 * V_ROW<D, VI8>;
    constexpr int PER_TILE = K_PIECES<D> + V_PIECES<D, VI8> + 1;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the row tiles of one share of the keys run 8 apart: on one XCD
    const int in8 = block % (8 * row_tiles), share = block / (8 * row_tiles) * 8 + (in8 & 7), rt = in8 >> 3;
    const int unit = share / c.splits, split = share % c.splits;
    if (unit >= units) return;
    const int b = ALL ? 0 : unit / c.Hkv, hk = ALL ? unit : unit % c.Hkv;
    const int row0 = 32 * rt, last_row = imin(row0 + 31, c.rows - 1), row = imin(row0 + r, c.rows - 1);
    const bool shared = ALL || c.Kp != nullptr;
    const int L = ALL ? 0 : keys_of(c.lens, b, c.Nk);
    // positions of the first and the last row, and of this lane's
    const int p0 = ALL ? -1 : L - c.Nq + row0 / c.G, p1 = ALL ? -1 : L - c.Nq + last_row / c.G, p = ALL ? -1 : L - c.Nq + row / c.G;
    const Runs runs(shared, c.Np, c.window, c.sinks, p0, p1);
    const int tilesA = (runs.lenA + 31) / 32, tiles = tilesA + (runs.lenB + 31) / 32;
    const int per = (tiles + c.splits - 1) / c.splits, t0 = split * per, t1 = imin(tiles, t0 + per);

    const long kA = shared ? static_cast<long>(hk) * c.Np : static_cast<long>(unit) * c.Nk, kB = static_cast<long>(unit) * c.Nk + runs.lo;
    const int8_t *vA = static_cast<const int8_t *>(shared ? c.Vp : c.V), *vB = static_cast<const int8_t *>(c.V);
    const BufRsrc rKA = make_rsrc((shared ? c.Kp : c.K) + kA * D, runs.lenA * D), rVA = make_rsrc(vA + kA * V_ROW<D, VI8>, runs.lenA * V_ROW<D, VI8>),
                  rSA = make_rsrc((shared ? c.sKp : c.sK) + kA, runs.lenA * 4);
    const BufRsrc rKB = ALL ? rKA : make_rsrc(c.K + kB * D, runs.lenB * D), rVB = ALL ? rVA : make_rsrc(vB + kB * V_ROW<D, VI8>, runs.lenB * V_ROW<D, VI8>),
                  rSB = ALL ? rSA : make_rsrc(c.sK + kB, runs.lenB * 4);
    const float unitA = VI8 ? (shared ? c.sVp[hk] : c.sV[unit]) : 1.0f, unitB = VI8 && !ALL ? c.sV[unit] : unitA;
    const bool zeros = VI8 && !ALL && counts_as_zero(unitB, unitA);

    const Lane<D, VI8> lo(lane);
    const lds_ptr kbuf = (lds_ptr)(&sm.k[wave][0][0]), vbuf = (lds_ptr)(&sm.v[wave][0][0]), skbuf = (lds_ptr)(&sm.sk[wave][0][0]);
    auto stage = [&](int t, int slot) {                          // (a tile past the last costs as many copies, of nothing)
        const bool inA = t < tilesA;
        const int j0 = 32 * (inA ? t : t - tilesA);
        const bool real = t < t1;
        copy_pieces<K_PIECES<D>, NT>(pick(inA, rKA, rKB), kbuf + slot * KB, lo.gk, lo.gk, real ? j0 * D : NOTHING);
        copy_pieces<V_PIECES<D, VI8>, NT>(pick(inA, rVA, rVB), vbuf + slot * VB, lo.gv[0], lo.gv[1], real && (inA || !zeros) ? j0 * V_ROW<D, VI8> : NOTHING);
        if (g == 0) lds_copy4(pick(inA, rSA, rSB), skbuf + slot * 128, 4 * r, real ? j0 * 4 : NOTHING);
    };
    const int first = t0 + wave;
#pragma unroll
    for (int s = 0; s < ST; ++s) stage(first + s * FEW_WAVES, s);

    const long qrow = row_of(c, ALL, unit, row);
    v4i qf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const v4i *>(c.Q + qrow * D + 32 * kk + 16 * g);
    const float sq2 = shared || p >= 0 ? query_scale(c.sQ[qrow], qf) : 1.0f;       // (padding: whatever its scale holds, 0 and NaN too, its row is zeros)
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(qf[kk]));    // landed before the loop
    v16i bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I;
    asm volatile("" : "+v"(bias));

    float m2 = -INFINITY, l = 0.0f, unit_of_o = first < tilesA ? unitA : unitB;      // m2: what the weights refer to, FEW_BELOW under the maximum
    v16f o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] = 0.0f;
    const h2 ones = {(_Float16)1.0f, (_Float16)1.0f};

    int slot = 0;
    for (int t = first; t < t1; t += FEW_WAVES) {
        wait_vmcnt<PER_TILE *(ST - 1)>();                        // this tile has landed
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        v4i kop[KS];
        v4f skv[4];
        h8 vop[DT][2];
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) kop[kk] = *reinterpret_cast<LDS_AS const v4i *>(lds_xor(kbuf + slot * KB, 32 * kk, lo.k0));
#pragma unroll
        for (int vq = 0; vq < 4; ++vq) skv[vq] = *reinterpret_cast<LDS_AS const v4f *>(skbuf + slot * 128 + 16 * g + 32 * vq);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int s = 0; s < 2; ++s) vop[dt][s] = v_operand<D, VI8>(vbuf + slot * VB, lo.v0, dt, 16 * s);
        wait_lds();
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        stage(t + ST * FEW_WAVES, slot);                         // into the place this tile has left
        __builtin_amdgcn_sched_barrier(0);
        slot = slot == ST - 1 ? 0 : slot + 1;

        v16i acc = bias;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kop[kk], qf[kk], acc, 0, 0, 0);
        const bool inA = t < tilesA;
        const int j0 = 32 * (inA ? t : t - tilesA);
        float a[16], tmax = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) a[v] = (__int_as_float(acc[v]) - ACC_BIAS_F) * skv[v >> 2][v & 3];
        // whether all 32 rows see all 32 keys (wave-uniform)
        const bool clear = inA ? j0 + 32 <= runs.lenA && (shared || p0 >= 0)
                               : p0 >= 0 && j0 + 31 <= p0 - runs.lo && (j0 > p1 - runs.lo - c.window || j0 + 31 < c.sinks - runs.lo);
        if (!clear) {
            const int hi = inA ? (shared || p >= 0 ? runs.lenA - 1 : -1) - j0 : p - runs.lo - j0;
            const int from = inA ? 0 : p - runs.lo - c.window + 1 - j0, sink = inA ? 0 : c.sinks - runs.lo - j0;
            const uint32_t seen = static_cast<uint32_t>(keys_seen(hi, from, sink)) >> (4 * g);
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (!(seen & (1u << (8 * (v >> 2) + (v & 3))))) a[v] = -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) tmax = fmaxf(tmax, a[v]);
        tmax = pair_max(tmax);
        const float m_new = fmaxf(m2, __builtin_fmaf(tmax, sq2, -FEW_BELOW));
        const float m_at = m_new == -INFINITY ? 0.0f : m_new;    // a row that has seen nothing yet: weights of 0, no NaN
        float alpha = __builtin_amdgcn_exp2f(m2 - m_at);         // exp2(-inf) = 0
        m2 = m_new;
        h2 ph[8];
        float psum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ph[e] = h2{(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(a[2 * e], sq2, -m_at)),
                       (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(a[2 * e + 1], sq2, -m_at))};
            psum = __builtin_amdgcn_fdot2(ph[e], ones, psum, false);
        }
        l = __builtin_fmaf(l, alpha, psum);
        if (VI8 && !inA && !zeros && unit_of_o != unitB) {       // from the shared keys' scale of V to the own ones', once
            alpha *= unit_of_o / unitB;
            unit_of_o = unitB;
        }
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const h8 pb = {ph[4 * s][0], ph[4 * s][1], ph[4 * s + 1][0], ph[4 * s + 1][1], ph[4 * s + 2][0], ph[4 * s + 2][1], ph[4 * s + 3][0], ph[4 * s + 3][1]};
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vop[dt][s], pb, o[dt], 0, 0, 0);
        }
    }
    wait_all_memory();                                           // requests past the last tile
    __syncthreads();                                             // every wavefront is done with its buffers: o may lie there

    // ---- the four meet
    l += swap32(l);
    if (g == 0) sm.ml[wave][r] = float2{m2, l};
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) m_all = fmaxf(m_all, sm.ml[w][r].x);
    const float f = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - m_all) * unit_of_o;
    const int valid = last_row - row0 + 1;
    for (int half = 0; half < D / 64; ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            if (dt >> 1 == half) {
#pragma unroll
                for (int vq = 0; vq < 4; ++vq) {
                    // 16-byte chunks, the row's bits mixed into the chunk so that a column of rows spreads over the banks
                    const int chunk = (8 * (dt & 1) + 2 * vq + g) ^ (r & 7);
                    *reinterpret_cast<v4f *>(&sm.o[wave][r][4 * chunk]) = v4f{o[dt][4 * vq] * f, o[dt][4 * vq + 1] * f, o[dt][4 * vq + 2] * f, o[dt][4 * vq + 3] * f};
                }
            }
        __syncthreads();
        for (int at = tid; at < valid * 16; at += 64 * FEW_WAVES) {
            const int rr = at / 16, cc = at % 16;
            float m = -INFINITY, ls = 0.0f;
            v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) m = fmaxf(m, sm.ml[w][rr].x);
#pragma unroll
            for (int w = 0; w < FEW_WAVES; ++w) {
                const float2 x = sm.ml[w][rr];
                ls += x.x == -INFINITY ? 0.0f : x.y * __builtin_amdgcn_exp2f(x.x - m);
                s += *reinterpret_cast<const v4f *>(&sm.o[w][rr][4 * (cc ^ (rr & 7))]);
            }
            if (c.part_o) {
                const long pr = (static_cast<long>(unit) * c.splits + split) * c.rows + row0 + rr;
                *reinterpret_cast<v4f *>(c.part_o + pr * D + 64 * half + 4 * cc) = s;
                if (cc == 0 && half == 0) c.part_ml[pr] = float2{m, ls};
            } else {
                const float q = ls > 0.0f ? 1.0f / ls : 0.0f;    // a row that sees nothing: zeros
                store4(c.O, c.o_dtype, row_of(c, ALL, unit, row0 + rr) * D + 64 * half + 4 * cc, s[0] * q, s[1] * q, s[2] * q, s[3] * q);
            }
        }
    }
}
#endif
template <int D, bool VI8, int ST, bool NT>
__global__ __launch_bounds__(64 * FEW_WAVES) void cache_attention_few_kernel(Call c, int units, int row_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemFew<D, VI8, ST> sm;
    few_rows_of_a_unit<D, VI8, false, ST, NT>(sm, c, blockIdx.x, units, row_tiles);
#endif
}

// ---- many rows: tiles of 128 ----------------------------------------------------------------------------------------
// Four wavefronts of 32 rows share the keys, 64 at a time, through LDS (double-buffered).  What bounds it is the vector unit: 32 keys of 32 rows are 12 matrix
// instructions (384 cycles at d = 128), and of the vector instructions on each of their scores (subtract the start value, s_K, the maximum, s_Q and m, exp2, the conversion
// in pairs, the sum in pairs) exp2 alone takes 16 cycles: 1116 vector cycles of the 2004 that 64 keys take a wavefront, 768 of the matrix unit (the chip runs it at 1.8 - 2.0 GHz).
// So the number that the weights refer to, 2^7 under the maximum when it was taken, only moves when a block exceeds that maximum by 2^8 (a row by itself: what a row gives does not depend on
// its neighbours), which fp16 weights of up to 2^15 hold, and only then are o and l rescaled: 64 multiplications a block that are hardly ever made.
template <int D, bool VI8> struct SmemTile {
    alignas(4096) int8_t k[2][TILE_KEYS * D];
    alignas(4096) int8_t v[2][TILE_KEYS * V_ROW<D, VI8>];
    alignas(256) float sk[2][TILE_KEYS];
};

#if defined(__HIP_DEVICE_COMPILE__)
template <int D> struct RowState {
    float m2, l;                                                 // m2: what the weights refer to, log2 units
    v16f o[D / 32];
};
constexpr float SLACK = 8.0f, TILE_BELOW = 7.0f;                 // (below a maximum that may be exceeded: weights of up to 2^15)

// 64 keys in LDS against the wavefront's rows.  `clear`: all of them count for every row, otherwise those of `seen`.  (One body for both, with a branch around
// the mask alone: two bodies and o would be moved from one's registers to the other's at every block.)
template <int D, bool VI8>
__device__ __forceinline__ void tile_block(lds_ptr ks, lds_ptr vs, lds_ptr sk, const Lane<D, VI8> &lo, const v4i (&qf)[D / 32], float sq2, bool clear, uint64_t seen, int g,
                                           const v16i &bias, RowState<D> &st) {
    constexpr int KS = D / 32, DT = D / 32;
    v16i acc[2];
    float a[2][16];
    v4i kop[KS];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) kop[kk] = *reinterpret_cast<LDS_AS const v4i *>(lds_xor(ks, 32 * kk, lo.k0) + 32 * mt * D);
        acc[mt] = bias;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) acc[mt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(kop[kk], qf[kk], acc[mt], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int vq = 0; vq < 4; ++vq) {
            const v4f skv = *reinterpret_cast<LDS_AS const v4f *>(sk + 16 * g + 128 * mt + 32 * vq);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[mt][4 * vq + e] = (__int_as_float(acc[mt][4 * vq + e]) - ACC_BIAS_F) * skv[e];
        }
    if (!clear) {
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
    __builtin_amdgcn_sched_barrier(0);
    const float top = __builtin_fmaf(pair_max(bmax), sq2, -TILE_BELOW);
    const bool moves = top > st.m2 + SLACK;                      // (st.m2 = -inf: whenever a key counts)
    if (__any(moves)) {
        const float m_new = moves ? top : st.m2;
        const float alpha = moves ? __builtin_amdgcn_exp2f(st.m2 - m_new) : 1.0f;
        st.m2 = m_new;
        st.l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) st.o[dt][v] *= alpha;
    }
    const float m = st.m2 == -INFINITY ? 0.0f : st.m2; // a row that has seen nothing yet: weights of 0, no NaN
    const h2 ones = {(_Float16)1.0f, (_Float16)1.0f};
    h2 ph[2][8];
    float sum = 0.0f;                                            // of the block: small weights do not meet l one by one
    auto weights = [&](int mt, int e) {
        ph[mt][e] = h2{(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(a[mt][2 * e], sq2, -m)), (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(a[mt][2 * e + 1], sq2, -m))};
        sum = __builtin_amdgcn_fdot2(ph[mt][e], ones, sum, false);
    };
    // the weights of the second 32 keys between the products of the first
    h8 vop[DT][2];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int s = 0; s < 2; ++s) vop[dt][s] = v_operand<D, VI8>(vs, lo.v0, dt, 16 * s);
#pragma unroll
    for (int e = 0; e < 8; ++e) weights(0, e);
    __builtin_amdgcn_s_setprio(3);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const h8 pb = {ph[mt][4 * s][0], ph[mt][4 * s][1], ph[mt][4 * s + 1][0], ph[mt][4 * s + 1][1], ph[mt][4 * s + 2][0], ph[mt][4 * s + 2][1], ph[mt][4 * s + 3][0], ph[mt][4 * s + 3][1]};
                st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vop[dt][s], pb, st.o[dt], 0, 0, 0);
                if (mt == 0) vop[dt][s] = v_operand<D, VI8>(vs, lo.v0, dt, 32 + 16 * s);
            }
            if (mt == 0) {
#pragma unroll
                for (int q = 0; q < 8 / DT; ++q) weights(1, dt * (8 / DT) + q);
            }
        }
    st.l += sum;
    __builtin_amdgcn_s_setprio(0);
}

// A wavefront's 32 x D outputs through 64 D bytes of LDS of its own, so that whole (fp32: half) rows are stored.  at(row): where row `row` goes, null for nowhere.
template <int D, typename OutT, typename Val, typename At>
__device__ __forceinline__ void store_rows(lds_ptr stage, int lane, Val val, At at) {
    constexpr int PASSES = sizeof(OutT) / 2, DTP = (D / 32) / PASSES, CH = D * 2 / 16, ROWS = 64 / CH;
    const int r = lane & 31, g = lane >> 5, cc = lane % CH, rr = lane / CH;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
#pragma unroll
        for (int dl = 0; dl < DTP; ++dl)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) {
                const int dt = pass * DTP + dl;
                if constexpr (sizeof(OutT) == 2)
                    *reinterpret_cast<LDS_AS uint2 *>(stage + r * (2 * D) + (((4 * dl + vq) ^ (r & (CH - 1))) * 16) + 8 * g) =
                        Pack4<OutT>::pack(val(dt, 4 * vq), val(dt, 4 * vq + 1), val(dt, 4 * vq + 2), val(dt, 4 * vq + 3));
                else
                    *reinterpret_cast<LDS_AS v4f *>(stage + r * (2 * D) + (((8 * dl + 2 * vq + g) ^ (r & (CH - 1))) * 16)) =
                        v4f{val(dt, 4 * vq), val(dt, 4 * vq + 1), val(dt, 4 * vq + 2), val(dt, 4 * vq + 3)};
            }
#pragma unroll
        for (int rd = 0; rd < 32 / ROWS; ++rd) {
            const int row = rd * ROWS + rr;
            const v4i x = *reinterpret_cast<LDS_AS const v4i *>(stage + row * (2 * D) + ((cc ^ (row & (CH - 1))) * 16));
            char *const to = at(row);
            if (to) __builtin_nontemporal_store(x, reinterpret_cast<v4i *>(to + pass * (2 * D) + 16 * cc));
        }
    }
}
#endif

// What a tile walks: the own keys through a window; the shared keys, for rows of the whole batch; or the shared keys and then the own ones of its sequence.
enum Walk { OWN, SHARED, SHARED_AND_OWN };
#if defined(__HIP_DEVICE_COMPILE__)
template <int D, bool VI8, Walk WALK>
__device__ __forceinline__ void tile_of_a_unit(SmemTile<D, VI8> &sm, const Call &c, int block, int units, int row_tiles, int head_group) {
    constexpr int DT = D / 32, KB = TILE_KEYS * D, VB = TILE_KEYS * V_ROW<D, VI8>, KP = KB / 4096, VP = VB / 4096;
    constexpr bool ALL = WALK == SHARED, FRONT = WALK == SHARED_AND_OWN;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit, ord;                                               // the row tiles and parts of a unit on one XCD, the last rows, which may see more, first
    map_workgroup(block, units, row_tiles * c.splits, head_group, !ALL, unit, ord);
    const int rt = row_tiles - 1 - ord / c.splits, split = ord % c.splits;
    const int L = ALL ? c.Np : keys_of(c.lens, unit / c.Hkv, c.Nk), window = ALL ? c.Np : c.window;
    const int row0 = TILE_ROWS * rt, last_row = imin(row0 + TILE_ROWS - 1, c.rows - 1), row = imin(row0 + 32 * wave + r, last_row);
    // the position of a row; every row sees all of the shared keys
    auto position = [&](int i) { return ALL ? L - 1 : L - c.Nq + i / c.G; };
    const int pos0 = position(row0), pos1 = position(last_row);
    // The two runs one after the other, cut into blocks of 64 with no seam: key v of them is key v for v < lenA, else key v + gap.  All of it lies in front of key pos1 + 1.
    const Runs runs(false, 0, window, ALL ? 0 : c.sinks, pos0, pos1);
    const int lenA = runs.lenA, gap = runs.lo - lenA, keys = lenA + runs.lenB;
    const int front = FRONT ? (c.Np + TILE_KEYS - 1) / TILE_KEYS : 0;            // blocks of shared keys in front
    const int blocks = front + (keys + TILE_KEYS - 1) / TILE_KEYS, per = (blocks + c.splits - 1) / c.splits, t0 = split * per, t1 = imin(blocks, t0 + per);
    // a row at p sees key v iff v <= p - gap and (v > p - gap - window or v < sink); one at p < 0 none
    const int p = position(row), hi = p < 0 ? -1 : p - gap, sink = imax(lenA, (ALL ? 0 : c.sinks) - gap);
    const int w0 = position(imin(row0 + 32 * wave, last_row)), w1 = position(imin(row0 + 32 * wave + 31, last_row));      // of the wavefront's first and last row
    const int hi0 = w0 < 0 ? -1 : w0 - gap, hi1 = w1 < 0 ? -1 : w1 - gap;

    const int8_t *const K = ALL ? c.Kp : c.K, *const V = static_cast<const int8_t *>(ALL ? c.Vp : c.V);
    const float *const sK = ALL ? c.sKp : c.sK;
    const long first_key = static_cast<long>(unit) * (ALL ? c.Np : c.Nk);
    const int seen_end = imax(0, pos1 + 1);
    const BufRsrc rK = make_rsrc(K + first_key * D, seen_end * D), rV = make_rsrc(V + first_key * V_ROW<D, VI8>, seen_end * V_ROW<D, VI8>), rS = make_rsrc(sK + first_key, seen_end * 4);
    const long front_key = FRONT ? static_cast<long>(unit % c.Hkv) * c.Np : 0;
    const BufRsrc fK = FRONT ? make_rsrc(c.Kp + front_key * D, c.Np * D) : rK,
                  fV = FRONT ? make_rsrc(static_cast<const int8_t *>(c.Vp) + front_key * V_ROW<D, VI8>, c.Np * V_ROW<D, VI8>) : rV, fS = FRONT ? make_rsrc(c.sKp + front_key, c.Np * 4) : rS;
    const float unit_own = VI8 ? (ALL ? c.sVp : c.sV)[unit] : 1.0f, unit_front = VI8 && FRONT ? c.sVp[unit % c.Hkv] : unit_own;
    const bool zeros = VI8 && FRONT && counts_as_zero(unit_own, unit_front);
    const Lane<D, VI8> lo(lane);
    const lds_ptr kbuf = (lds_ptr)(&sm.k[0][0]), vbuf = (lds_ptr)(&sm.v[0][0]), skbuf = (lds_ptr)(&sm.sk[0][0]);
    auto stage = [&](int t, int slot) {                          // a quarter of the block to each wavefront
        const lds_ptr kl = kbuf + slot * KB + wave * KP * 1024, vl = vbuf + slot * VB + wave * VP * 1024, sl = skbuf + slot * 256;
        if (FRONT && t < front) {
            const int f0 = TILE_KEYS * t;
            copy_pieces<KP>(fK, kl, lo.gk, lo.gk, f0 * D + wave * KP * 1024);
            copy_pieces<VP>(fV, vl, lo.gv[0], lo.gv[1], f0 * V_ROW<D, VI8> + wave * VP * 1024);
            if (wave == 3) lds_copy4(fS, sl, 4 * lane, f0 * 4);
            return;
        }
        int v0 = TILE_KEYS * (t - front);
        if (v0 < lenA && v0 + TILE_KEYS > lenA) {                // the block with the seam: row by row
            constexpr int K_ROWS = 1024 / D, V_ROWS = 1024 / V_ROW<D, VI8>;
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const int at = v0 + (wave * KP + i) * K_ROWS + lane / (D / 16);
                lds_copy16(rK, kl + 1024 * i, lo.gk + (at < lenA ? 0 : gap * D), v0 * D + (wave * KP + i) * 1024);
            }
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                const int at = v0 + (wave * VP + i) * V_ROWS + lane / (V_ROW<D, VI8> / 16);
                lds_copy16(rV, vl + 1024 * i, lo.gv[i & 1] + 1024 * (i & 1) + (at < lenA ? 0 : gap * V_ROW<D, VI8>), v0 * V_ROW<D, VI8> + (wave * VP + (i & ~1)) * 1024);
            }
            if (wave == 3) lds_copy4(rS, sl, 4 * (lane + (v0 + lane < lenA ? 0 : gap)), v0 * 4);
            return;
        }
        if (v0 >= lenA) v0 += gap;
        copy_pieces<KP>(rK, kl, lo.gk, lo.gk, v0 * D + wave * KP * 1024);
        copy_pieces<VP>(rV, vl, lo.gv[0], lo.gv[1], zeros ? NOTHING : v0 * V_ROW<D, VI8> + wave * VP * 1024);
        if (wave == 3) lds_copy4(rS, sl, 4 * lane, v0 * 4);
    };
    if (t0 < t1) stage(t0, 0);

    const long qrow = row_of(c, ALL, unit, row);
    v4i qf[D / 32];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) qf[kk] = *reinterpret_cast<const v4i *>(c.Q + qrow * D + 32 * kk + 16 * g);
    const float sq2 = FRONT || p >= 0 ? query_scale(c.sQ[qrow], qf) : 1.0f;       // (padding: whatever its scale holds, 0 and NaN too, its row is zeros)
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) asm volatile("" : "+v"(qf[kk]));
    v16i bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I;
    asm volatile("" : "+v"(bias));
    RowState<D> st;
    st.m2 = -INFINITY, st.l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) st.o[dt][v] = 0.0f;
    float unit_of_o = t0 < front ? unit_front : unit_own;

    const bool alive = row0 + 32 * wave < c.rows;                // (wave-uniform) a wavefront without rows copies only
    wait_all_memory();
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int slot = (t - t0) & 1, v0 = TILE_KEYS * (t - front);
        if (t + 1 < t1) stage(t + 1, slot ^ 1);
        if (VI8 && FRONT && t == front && t > t0 && !zeros) {    // from the shared keys' scale of V to the own ones', once
            const float f = unit_of_o / unit_own;
            unit_of_o = unit_own;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) st.o[dt][v] *= f;
        }
        const bool in_front = FRONT && t < front;
        // (wave-uniform) whether some of the rows see some of the keys, and whether all see all
        const bool any = alive && (in_front || (hi1 >= v0 && (hi0 - window < v0 + TILE_KEYS - 1 || v0 < sink)));
        const bool clear = in_front ? TILE_KEYS * (t + 1) <= c.Np : hi0 >= v0 + TILE_KEYS - 1 && (hi1 - window < v0 || v0 + TILE_KEYS <= sink);
        const uint64_t seen = clear ? 0 : in_front ? below(c.Np - TILE_KEYS * t) : keys_seen(hi - v0, hi - window + 1 - v0, sink - v0);
        if (any) tile_block<D, VI8>(kbuf + slot * KB, vbuf + slot * VB, skbuf + slot * 256, lo, qf, sq2, clear, seen, g, bias, st);
        wait_all_memory();                                       // my part of the next block has landed
        __syncthreads();                                         // everyone's has, and this one's place is free
    }

    const float l = st.l + swap32(st.l);
    const lds_ptr stage_out = (lds_ptr)(&sm) + wave * (64 * D);
    const int first = row0 + 32 * wave;
    if (c.part_o) {
        const long pr = (static_cast<long>(unit) * c.splits + split) * c.rows;
        const int n = c.rows;
        float *const po = c.part_o + pr * D;
        const float u = st.m2 == -INFINITY ? 0.0f : unit_of_o;   // (a part without keys of its row: zeros, whatever the scale that it did not use is)
        store_rows<D, float>(stage_out, lane, [&](int dt, int v) { return st.o[dt][v] * u; },
                             [&](int k) { return first + k < n ? reinterpret_cast<char *>(po + static_cast<long>(first + k) * D) : nullptr; });
        if (g == 0 && first + r < n) c.part_ml[pr + first + r] = float2{st.m2, l};
        return;
    }
    const float f = l > 0.0f ? unit_of_o / l : 0.0f;             // a row that sees nothing: zeros
    auto store = [&](auto type) {
        using OutT = decltype(type);
        store_rows<D, OutT>(stage_out, lane, [&](int dt, int v) { return st.o[dt][v] * f; },
                            [&](int k) { return first + k < c.rows ? reinterpret_cast<char *>(static_cast<OutT *>(c.O) + row_of(c, ALL, unit, first + k) * D) : nullptr; });
    };
    if (c.o_dtype == IFA_F32) store(float{});
    else if (c.o_dtype == IFA_F16) store(__half{});
    else store(__hip_bfloat16{});
}
#endif
template <int D, bool VI8, Walk WALK>
__global__ __launch_bounds__(256, 2) void cache_attention_tile_kernel(Call c, int units, int row_tiles, int head_group) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemTile<D, VI8> sm;
    tile_of_a_unit<D, VI8, WALK>(sm, c, blockIdx.x, units, row_tiles, head_group);
#endif
}

// ---- shared keys and own keys in one launch --------------------------------------------------------------------------
// The first `blocks` workgroups take the shared keys for the whole batch (TILE: in tiles of 128 rows, otherwise 32), the others every sequence's own: the former are bound by their
// arithmetic, the latter by memory, and neither waits for the end of the other.
template <int D, bool VI8, bool TILE>
__global__ __launch_bounds__(256, 2) void cache_attention_both_kernel(Call shared, Call own, int blocks, int shared_tiles, int own_units, int own_tiles, int head_group) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ union {
        SmemTile<D, VI8> tile;
        SmemFew<D, VI8, 1> few;
    } sm;
    if (static_cast<int>(blockIdx.x) >= blocks) few_rows_of_a_unit<D, VI8, false, 1, false>(sm.few, own, blockIdx.x - blocks, own_units, own_tiles);
    else if constexpr (TILE) tile_of_a_unit<D, VI8, SHARED>(sm.tile, shared, blockIdx.x, shared.Hkv, shared_tiles, head_group);
    else few_rows_of_a_unit<D, VI8, true, 1, false>(sm.few, shared, blockIdx.x, shared.Hkv, shared_tiles);
#endif
}

// ---- the parts of a row joined -----------------------------------------------------------------------------------
// `shared` > 0: that many parts of the shared keys first (unit hk, row (b, i, g)), then `own` of the sequence's own.  P groups of D / 4 threads take every P-th part of a
// row, each with a maximum of its own, and meet in LDS: what there is to wait for is a few loads in a row, not one for each part (33 parts of 2048 rows: 26 us one after the other, 9 like this).
struct Parts {
    const float *o_shared, *o_own;
    const float2 *ml_shared, *ml_own;
    int shared, own;
};
template <int D, int P>
__global__ __launch_bounds__(256) void cache_attention_join_kernel(Call c, Parts parts, long all_rows) {
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * P);
    __shared__ v4f so[P > 1 ? P : 1][ROWS][TPR];
    __shared__ float2 sml[P > 1 ? P : 1][ROWS];
    const int cc = threadIdx.x % TPR, pg = threadIdx.x / TPR % P, in_block = threadIdx.x / (TPR * P);
    const long idx = static_cast<long>(blockIdx.x) * ROWS + in_block;
    const bool valid = idx < all_rows;
    const int per = c.Nq * c.G, unit = static_cast<int>(idx / per), in = static_cast<int>(idx % per), n = valid ? parts.shared + parts.own : 0;
    const long s_step = static_cast<long>(c.B) * per, s0 = static_cast<long>(unit % c.Hkv) * parts.shared * s_step + static_cast<long>(unit / c.Hkv) * per + in;
    const long o0 = (static_cast<long>(unit) * parts.own - parts.shared) * per + in;
    float m = -INFINITY, l = 0.0f;
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int AT_ONCE = 4;
    for (int i0 = pg; i0 < n; i0 += AT_ONCE * P) {
        float2 x[AT_ONCE];
        v4f y[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = i0 + k * P;
            x[k] = float2{-INFINITY, 0.0f};
            y[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if (i < n) {
                const bool shared = i < parts.shared;
                const long at = shared ? s0 + i * s_step : o0 + static_cast<long>(i) * per;
                x[k] = (shared ? parts.ml_shared : parts.ml_own)[at];
                y[k] = *reinterpret_cast<const v4f *>((shared ? parts.o_shared : parts.o_own) + at * D + 4 * cc);
            }
        }
        float m_new = m;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) m_new = fmaxf(m_new, x[k].x);
        if (m_new == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(m - m_new);       // exp2(-inf) = 0
        l *= f, s *= f, m = m_new;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const float w = __builtin_amdgcn_exp2f(x[k].x - m);
            l += x[k].y * w;
            s += y[k] * w;
        }
    }
    if constexpr (P > 1) {
        so[pg][in_block][cc] = s;
        if (cc == 0) sml[pg][in_block] = float2{m, l};
        __syncthreads();
        if (pg) return;
        float m_all = m;
#pragma unroll
        for (int k = 1; k < P; ++k) m_all = fmaxf(m_all, sml[k][in_block].x);
        if (m_all != -INFINITY) {
            const float f = __builtin_amdgcn_exp2f(m - m_all);
            l *= f, s *= f;
#pragma unroll
            for (int k = 1; k < P; ++k) {
                const float w = __builtin_amdgcn_exp2f(sml[k][in_block].x - m_all);
                l += sml[k][in_block].y * w;
                s += so[k][in_block][cc] * w;
            }
        }
    }
    if (!valid) return;
    const float q = l > 0.0f ? 1.0f / l : 0.0f;
    store4(c.O, c.o_dtype, row_of(c, false, unit, in) * D + 4 * cc, s[0] * q, s[1] * q, s[2] * q, s[3] * q);
}

// ---- host --------------------------------------------------------------------------------------------------------
template <int D, bool VI8>
int launch(Call c, const AttentionPlan &plan, void *workspace, hipStream_t st) {
    const int units = c.B * c.Hkv;
    float *const o = static_cast<float *>(workspace);
    float2 *const ml = reinterpret_cast<float2 *>(o + (plan.rows_shared + plan.rows_own) * D);
    auto tiles = [&](auto walk, const Call &k, int n_units) {
        const int n = static_cast<int>(row_tiles(false, k.rows));
        hipLaunchKernelGGL((cache_attention_tile_kernel<D, VI8, decltype(walk)::value>), dim3(static_cast<unsigned>(static_cast<long>(n_units) * n * k.splits)), dim3(256), 0, st, k, n_units, n,
                           head_group_for(true, 0, 0));
    };
    Call shared = c;                                             // the shared keys for the rows of the whole batch, if they are taken so
    if (plan.shared > 0) {
        shared.rows = c.rows * c.B;
        shared.splits = plan.shared;
        shared.part_o = o, shared.part_ml = ml;
        c.Kp = nullptr, c.Np = 0;                                // the own keys alone
    }
    c.splits = plan.own;
    if (plan.join()) c.part_o = o + plan.rows_shared * D, c.part_ml = ml + plan.rows_shared;
    const int own_tiles = static_cast<int>(row_tiles(true, c.rows));
    const long own_grid = few_grid(units, c.splits, c.rows);
    auto few = [&](auto ahead, auto once) {
        hipLaunchKernelGGL((cache_attention_few_kernel<D, VI8, decltype(ahead)::value, decltype(once)::value>), dim3(static_cast<unsigned>(own_grid)), dim3(64 * FEW_WAVES), 0, st, c, units, own_tiles);
    };
    auto both = [&](auto tile) {
        constexpr bool TILE = decltype(tile)::value;
        const int n = static_cast<int>(row_tiles(!TILE, shared.rows));
        const long blocks = TILE ? static_cast<long>(c.Hkv) * n * shared.splits : few_grid(c.Hkv, shared.splits, shared.rows);
        hipLaunchKernelGGL((cache_attention_both_kernel<D, VI8, TILE>), dim3(static_cast<unsigned>(blocks + own_grid)), dim3(256), 0, st, shared, c, static_cast<int>(blocks), n, units, own_tiles,
                           head_group_for(true, 0, 0));
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 2> two{};
    switch (plan.way) {
    case WAY_FEW:
        if (plan.ahead == 1) plan.once ? few(one, std::true_type{}) : few(one, std::false_type{});
        else plan.once ? few(two, std::true_type{}) : few(two, std::false_type{});
        break;
    case WAY_BOTH_FEW: both(std::false_type{}); break;
    case WAY_BOTH_TILE: both(std::true_type{}); break;
    case WAY_TILE_APART: tiles(std::integral_constant<Walk, SHARED>{}, shared, c.Hkv); [[fallthrough]];
    case WAY_TILE: tiles(std::integral_constant<Walk, OWN>{}, c, units); break;
    case WAY_TILE_FRONT: tiles(std::integral_constant<Walk, SHARED_AND_OWN>{}, c, units); break;
    }
    if (plan.join()) {
        const Parts parts = {o, c.part_o, ml, c.part_ml, plan.shared, plan.own};
        const long all_rows = static_cast<long>(units) * c.rows;
        auto join = [&](auto p) {
            constexpr int P = decltype(p)::value, ROWS = 1024 / D / P;
            hipLaunchKernelGGL((cache_attention_join_kernel<D, P>), dim3(static_cast<unsigned>((all_rows + ROWS - 1) / ROWS)), dim3(256), 0, st, c, parts, all_rows);
        };
        if (plan.shared + plan.own > 8) join(std::integral_constant<int, 8>{});
        else join(std::integral_constant<int, 1>{});
    }
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}

// The argument rules that both entry points share
int refuse(const Call &c, int d, const void *workspace, long workspace_bytes, const AttentionPlan &plan) {
    const bool prefix = c.Np > 0;
    if (!c.Q || !c.K || !c.V || !c.sQ || !c.sK || !c.O || (prefix && (!c.Kp || !c.Vp || !c.sKp || !c.sVp != !c.sV))) return IFA_ERR_NULL;
    if (c.o_dtype < IFA_F32 || c.o_dtype > IFA_BF16) return IFA_ERR_DTYPE;
    for (const void *p : {static_cast<const void *>(c.Q), static_cast<const void *>(c.K), c.V, static_cast<const void *>(c.O), static_cast<const void *>(c.Kp), c.Vp})
        if (!ifa_aligned16(p)) return IFA_ERR_UNSUPPORTED;
    for (const void *p : {static_cast<const void *>(c.sQ), static_cast<const void *>(c.sK), static_cast<const void *>(c.sV), static_cast<const void *>(c.sKp), static_cast<const void *>(c.sVp), static_cast<const void *>(c.lens)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return IFA_ERR_UNSUPPORTED;
    if (plan.bytes(d)) {
        if (!workspace) return IFA_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 255) return IFA_ERR_UNSUPPORTED;
        if (workspace_bytes < plan.bytes(d)) return IFA_ERR_WORKSPACE;
    }
    return IFA_OK;
}

// Sizes alone: what a call or a workspace query takes
int refuse_sizes(int B, int H, int Hkv, int Nq, int Np, int Nk, int d) {
    if (B <= 0 || H <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0 || Np < 0 || d <= 0 || H % Hkv) return IFA_ERR_SHAPE;
    const long heads = static_cast<long>(B) * H, N = Nq > Nk ? Nq : Nk;
    if (heads > (1L << 40) / N / d) return IFA_ERR_SHAPE;
    if (d != 64 && d != 128) return IFA_ERR_UNSUPPORTED;
    if (static_cast<long>(Nk) * d * 2 > 0x7ff00000L || static_cast<long>(Np) * d * 2 > 0x7ff00000L) return IFA_ERR_UNSUPPORTED;
    if (heads * Nq > 1L << 26 || heads > 1L << 23) return IFA_ERR_UNSUPPORTED;      // a launch has less than 2^32 threads: 256 to 32 rows or to a unit, d / 4 to a joined row
    return IFA_OK;
}

int entry(const Call &c, int d, void *workspace, long workspace_bytes, void *hip_stream) {
    const bool i8 = c.sV != nullptr;
    const AttentionPlan plan = attention_plan(c.B, c.Hkv, c.G, c.Nq, c.Np, c.Nk, c.window, c.sinks, i8 ? 2 * d : 3 * d);
    if (const int rc = refuse(c, d, workspace, workspace_bytes, plan)) return rc;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (d == 128) return i8 ? launch<128, true>(c, plan, workspace, st) : launch<128, false>(c, plan, workspace, st);
    return i8 ? launch<64, true>(c, plan, workspace, st) : launch<64, false>(c, plan, workspace, st);
}

}  // namespace

extern "C" long ifa_window_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d, int window, int sinks) {
    if (refuse_sizes(B, H, Hkv, Nq, 0, Nk, d) || window <= 0 || sinks < 0) return -1;
    return attention_plan(B, Hkv, H / Hkv, Nq, 0, Nk, imin(window, Nk), imin(sinks, Nk), d).bytes(d);
}

extern "C" int int_flash_attn_fwd_window(const signed char *Q_i8, const signed char *K_i8, const void *V, const float *s_Q, const float *s_K,
                                         const float *s_V, const int *lens, int B, int H, int Hkv, int Nq, int Nk, int d, int window, int sinks,
                                         void *O, int o_dtype, void *workspace, long workspace_bytes, void *hip_stream) {
    if (window <= 0 || sinks < 0) return IFA_ERR_SHAPE;
    if (const int rc = refuse_sizes(B, H, Hkv, Nq, 0, Nk, d)) return rc;
    Call c = {};
    c.Q = Q_i8, c.K = K_i8, c.V = V, c.sQ = s_Q, c.sK = s_K, c.sV = s_V, c.lens = lens;
    c.B = B, c.Hkv = Hkv, c.G = H / Hkv, c.Nq = Nq, c.Nk = Nk, c.window = imin(window, Nk), c.sinks = imin(sinks, Nk);
    c.rows = c.G * Nq, c.O = O, c.o_dtype = o_dtype;
    return entry(c, d, workspace, workspace_bytes, hip_stream);
}

extern "C" long ifa_prefix_workspace_bytes(int B, int H, int Hkv, int Nq, int Np, int Nk, int d) {
    if (refuse_sizes(B, H, Hkv, Nq, Np, Nk, d) || Np <= 0) return -1;
    return attention_plan(B, Hkv, H / Hkv, Nq, Np, Nk, Nk, 0, d).bytes(d);
}

extern "C" int int_flash_attn_fwd_prefix(const signed char *Q_i8, const signed char *Kp_i8, const void *Vp, const signed char *K_i8, const void *V,
                                         const float *s_Q, const float *s_Kp, const float *s_K, const float *s_Vp, const float *s_V, const int *lens,
                                         int B, int H, int Hkv, int Nq, int Np, int Nk, int d, void *O, int o_dtype,
                                         void *workspace, long workspace_bytes, void *hip_stream) {
    if (Np <= 0) return IFA_ERR_SHAPE;
    if (const int rc = refuse_sizes(B, H, Hkv, Nq, Np, Nk, d)) return rc;
    Call c = {};
    c.Q = Q_i8, c.K = K_i8, c.V = V, c.sQ = s_Q, c.sK = s_K, c.sV = s_V, c.Kp = Kp_i8, c.Vp = Vp, c.sKp = s_Kp, c.sVp = s_Vp, c.lens = lens;
    c.B = B, c.Hkv = Hkv, c.G = H / Hkv, c.Nq = Nq, c.Np = Np, c.Nk = Nk, c.window = Nk, c.sinks = 0;
    c.rows = c.G * Nq, c.O = O, c.o_dtype = o_dtype;
    return entry(c, d, workspace, workspace_bytes, hip_stream);
}
