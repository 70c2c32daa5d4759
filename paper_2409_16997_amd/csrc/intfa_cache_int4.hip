// Attention over a cache held in 4 bits for gfx950: K and V as codes u - 8, u = 0 .. 15, with one fp32 scale a token and head, window and sinks as for the cache in 8 bits.
//
//     S = s_Q s_K (sum q u - 8 sum q)       v_mfma_i32_16x16x64_i8 (32x32x32 in tiles), exact in int32: the accumulator starts at -8 sum q
//     w~ = fp16(exp(S - M) |s_V|)           M per row: 15 log2 units below the largest exp(S) |s_V| (tiles: 7 to 15 below a bound of it), so that w~ <= 2^15; l = sum of exp(S - M) in fp32
//     O = sum w~ (u - 8) / l                v_mfma_f32_16x16x32_f16 (32x32x16 in tiles), fp32 accumulation
//
// The scale of a token joins its weight, where applied to V it would cost a multiplication a code.  Then the weights' range is that of p s_V, and what fp16 cuts off is small beside the largest summand.
// For few rows M is that summand itself, 2^15 exactly: the key that draws most of a row is not rounded at all.  (With a bound in its place single rows were off by up to 2^-11, a decode step of 32 rows by
// 1.6 times what the rounding of its output leaves.)  Scales below 2^-80 count as 2^-80 for M and l, so that exp(S - M) <= 2^95 and the sum of 2^24 of them is a number; the largest are below 2^20, so that
// a weight of 2^-100 of the largest product, or what an M that moves by 100 leaves of l, is still 26 powers of 2 above the smallest normal number.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <hip/hip_bf16.h>
#include <stdint.h>
#include <type_traits>
#include <utility>

#include "intfa.h"
#include "intfa_internal.h"
#include "intfa_device.h"
#include "intfa_cache.h"
#include "intfa_cache_plan.h"
#include "intfa_cache_rows.h"
#include "intfa_divisor.h"

namespace {

using namespace ifa_cache;
using ifa::Divisor;

constexpr int KEYS4 = 64;                  // keys of a tile
template <int D> constexpr int ROW4 = D / 2;                 // bytes of a row of codes,
template <int D> constexpr int TILE4 = KEYS4 * D / 2;        // and of a tile's K or V
[[maybe_unused]] constexpr float LEAST_SCALE = 0x1p-80f;
[[maybe_unused]] constexpr float FEW4_BELOW = 15.0f, TILE4_BELOW = 7.0f, SLACK4 = 8.0f;     // the largest weight is 2^15; in tiles 2^7, and 2^15 until M moves
[[maybe_unused]] constexpr int ALIKE4 = 4;                   // tiles, log2: scales of a block that are no further apart take M to the smallest of them where keys are hidden

// Sequences of different lengths, which the host does not know: a sequence of t tiles has ceil(t / C) parts, at least one, with C so that there are about `places` parts of all units, which is what the chip
// holds at once; workgroup w counts its way to its part.  (In as many parts each, the longest sequence decides: 8 x 4 heads, 40 rows on 0 .. 16391 keys 31.1 us, like this 25.8; 16 x 8 heads, one of 16384 keys and 15 of 100 26.3 and 13.6.)  A unit in one part goes straight
// to O; parts_of[unit] = (its first part, their number).
struct Sharing {
    int places;                            // 0: c.splits parts of every unit
    int2 *parts_of;
};

// What indexes are divided by.  (A quotient by a number that comes as an argument takes 30 instructions, one after the other, and the start and end of a workgroup had a dozen: a decode step on 700 keys 6.0 -> 5.8 us,
// 12 heads of 1777 queries under a window 19.4 -> 19.0.)
struct Divisors {
    Divisor G, Hkv, splits, row_tiles8;
};

// Row `row` of a unit in Q and O (in rows): heads of a unit, and units, follow each other there
__device__ __forceinline__ long row_of(const Call &c, const Divisors &by, int unit, int row) {
    const int i = by.G.of(row), g = row - i * c.G;
    return static_cast<long>(unit) * c.rows + static_cast<long>(g) * c.Nq + i;
}

#if defined(__HIP_DEVICE_COMPILE__)
// Sums over the lanes up to each: inside rows of 16, then row by row
__device__ __forceinline__ int sums_up_to(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(sums_up_to(x), 63); }
struct Part { int unit, split, splits, first; };                 // `first`: of the unit's
// False: there is no part w
__device__ __forceinline__ bool part_of(const Call &c, const Sharing &sh, const Divisors &by, int units, int w, int lane, Part &p) {
    if (!sh.places) {
        p.splits = c.splits, p.unit = by.splits.of(w), p.first = p.unit * c.splits, p.split = w - p.first;
        return p.unit < units;
    }
    const int span = imin(c.Nk, c.window + c.Nq + c.sinks);      // (window, sinks <= Nk < 2^25, Nq <= 2^26) the keys that some query sees, nearly
    auto load = [&](int b) { return b < c.B ? (imin(imax(c.lens[b], 0), span) + KEYS4 - 1) / KEYS4 : 0; };
    const int of_first_64 = load(lane);
    auto tiles_of = [&](int b0) { return b0 == 0 ? of_first_64 : load(b0 + lane); };
    auto parts_of = [&](int t, int C) { return imax(1, (t + C - 1) / C); };
    int all = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64) all += wave_sum(tiles_of(b0));
    // C: whole rounds of the wavefronts; half a part a unit is lost to rounding up, and where it is more C grows
    const int wanted = imax(1, sh.places - units / 2);
    int C = imax(1, static_cast<int>((static_cast<unsigned>(all) * static_cast<unsigned>(c.Hkv) / wanted + 3) / 4)) * 4;      // (less than 2^31 tiles: B Hkv Nk d <= 2^40)
    for (int tries = 0; tries < 4; ++tries) {
        int n = 0;
        for (int b0 = 0; b0 < c.B; b0 += 64) n += wave_sum(b0 + lane < c.B ? parts_of(tiles_of(b0), C) : 0);
        if (n * c.Hkv <= sh.places) break;
        C += 4;
    }
    int base = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64) {
        const int n = b0 + lane < c.B ? parts_of(tiles_of(b0), C) : 0;
        const int end = base + sums_up_to(n * c.Hkv);
        const uint64_t past = __ballot(end > w);
        if (past) {
            const int at = __ffsll(static_cast<long long>(past)) - 1;
            p.splits = __builtin_amdgcn_readlane(n, at);
            const int begin = __builtin_amdgcn_readlane(end, at) - p.splits * c.Hkv, head = (w - begin) / p.splits;
            p.unit = (b0 + at) * c.Hkv + head, p.split = (w - begin) % p.splits, p.first = begin + head * p.splits;
            return true;
        }
        base = __builtin_amdgcn_readlane(end, 63);
    }
    return false;
}

// 16-byte chunks of a row are exchanged by the row so that what is read at once spreads over the banks.  K is read a row to a lane; V transposed, rows 4 q .. 4 q + 3
// and those 16 further at once.
template <int D> __device__ __forceinline__ int k4_slot(int row) { return D == 128 ? (row >> 1) & 3 : (row >> 2) & 1; }
template <int D> __device__ __forceinline__ int v4_slot(int row) { return D == 128 ? (((row >> 1) ^ (row >> 2)) & 1) | (row >> 3 & 2) : row >> 4 & 1; }

constexpr uint32_t LOW4 = 0x0f0f0f0fu;

// 8 keys of a column of bytes (dwords of keys 0 - 3 and 4 - 7) as fp16 operands of the low and of the high channel; keys in the order 0, 2, 1, 3, 4, 6, 5, 7.  u in bits 0 - 3 of a half with the
// exponent of 1024 above it is 1024 + u, u in bits 4 - 7 with that of 64 is 64 + u; what is taken off leaves u - 8 exactly.  (u alone, as a subnormal number, would save the subtraction, but the matrix
// unit aligns such operands by their exponent: sums of them were off by 2^-14 and, in bits 4 - 7, 2^-18.)
// (v_and_or_b32 takes one scalar operand: the masks live in two registers.)
struct NibbleMasks {
    uint32_t low = 0x000f000fu, high = 0x00f000f0u;
    __device__ __forceinline__ NibbleMasks() { asm volatile("" : "+v"(low), "+v"(high)); }
};
__device__ __forceinline__ h2 low_codes(uint32_t w, const NibbleMasks &m) { return __builtin_bit_cast(h2, (w & m.low) | 0x64006400u) - h2{(_Float16)1032.0f, (_Float16)1032.0f}; }
__device__ __forceinline__ h2 high_codes(uint32_t w, const NibbleMasks &m) { return __builtin_bit_cast(h2, (w & m.high) | 0x54005400u) - h2{(_Float16)72.0f, (_Float16)72.0f}; }
__device__ __forceinline__ void values_of(const v2i &w, const NibbleMasks &m, h8 &low, h8 &high) {
    const uint32_t a = static_cast<uint32_t>(w[0]), b = static_cast<uint32_t>(w[1]), a8 = a >> 8, b8 = b >> 8;
    const h2 l0 = low_codes(a, m), l1 = low_codes(a8, m), l2 = low_codes(b, m), l3 = low_codes(b8, m), u0 = high_codes(a, m), u1 = high_codes(a8, m), u2 = high_codes(b, m), u3 = high_codes(b8, m);
    low = h8{l0[0], l0[1], l1[0], l1[1], l2[0], l2[1], l3[0], l3[1]};
    high = h8{u0[0], u0[1], u1[0], u1[1], u2[0], u2[1], u3[0], u3[1]};
}
__device__ __forceinline__ int high_nibbles(int w) { return static_cast<int>(static_cast<uint32_t>(w) >> 4 & LOW4); }
__device__ __forceinline__ int low_nibbles(int w) { return w & static_cast<int>(LOW4); }

__device__ __forceinline__ float swap16_max(float x) {           // with the lane 16 apart
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float quarters_sum(float x) {         // of the four lanes 16 apart
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// the largest of 64 lanes, in all of them
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xf, 0xf, true)));
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xf, 0xf, true)));
    return pair_max(swap16_max(x));
}
// Lane 16 r + N of x in every lane 16 r .. 16 r + 15: an operand modifier of the instruction that takes it.  Scales of keys reach the lanes that hold their scores so, a register for 16 keys; read from LDS, four
// at a time, they took 128 of the 294 cycles that LDS is busy for 32 rows and 64 keys in tiles (2 x 32 heads, prompts of 4096 284 -> 272 us).
template <int N> __device__ __forceinline__ float of_row(float x) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x150 + N, 0xf, 0xf, true)); }
template <typename F, int... I> __device__ __forceinline__ void unrolled(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
#endif

// ---- up to 16 RT rows against many keys: every wavefront for itself ----------------------------------------------------
// As in the kernel for 8 bits, the four wavefronts of a workgroup hold the same rows, take every fourth tile of keys, without a barrier in the loop, and meet once at the end.  A matrix
// instruction has 16 query columns, so that a decode step's few rows leave fewer of them idle, and all of a lane's softmax work is for keys of its 16 bytes of K.
template <int D, int RT, int W, int ST> struct SmemFew4 {
    union {
        struct {
            alignas(4096) int8_t k[W][ST][TILE4<D>];
            alignas(4096) int8_t v[W][ST][TILE4<D>];
            alignas(256) float sk[W][ST][KEYS4], sv[W][ST][KEYS4];
            alignas(256) float log_sv[W][KEYS4], inv_sv[W][KEYS4], rest[W][KEYS4];     // of the tile at hand
        };
        float o[W][16 * RT][D];                                  // when the loop is over
    };
    float2 ml[W][16 * RT];
};

#if defined(__HIP_DEVICE_COMPILE__)
template <int D, int RT, int W, int ST, bool NT>
__device__ __forceinline__ void few4_rows_of_a_unit(SmemFew4<D, RT, W, ST> &sm, const Call &c, const Divisors &by, const Part &part, int share, int row0) {
    constexpr int ROW = ROW4<D>, TB = TILE4<D>, PIECES = TB / 1024, KS = D / 64, CT = D / 32;
    constexpr int PER_TILE = 2 * PIECES + 2;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int unit = part.unit, last_row = imin(row0 + 16 * RT - 1, c.rows - 1);
    const int L = keys_of(c.lens, by.Hkv.of(unit), c.Nk);
    auto position = [&](int row) { return L - c.Nq + static_cast<int>(by.G.of(row)); };
    const int p0 = position(row0), p1 = position(last_row);
    const Runs runs(false, 0, c.window, c.sinks, p0, p1);
    const int tilesA = (runs.lenA + KEYS4 - 1) / KEYS4, tiles = tilesA + (runs.lenB + KEYS4 - 1) / KEYS4;
    const int per = (tiles + part.splits - 1) / part.splits, t0 = part.split * per, t1 = imin(tiles, t0 + per);

    const long kA = static_cast<long>(unit) * c.Nk, kB = kA + runs.lo;
    const int8_t *const V = static_cast<const int8_t *>(c.V);
    const BufRsrc rKA = make_rsrc(c.K + kA * ROW, runs.lenA * ROW), rVA = make_rsrc(V + kA * ROW, runs.lenA * ROW), rSKA = make_rsrc(c.sK + kA, runs.lenA * 4), rSVA = make_rsrc(c.sV + kA, runs.lenA * 4);
    const BufRsrc rKB = make_rsrc(c.K + kB * ROW, runs.lenB * ROW), rVB = make_rsrc(V + kB * ROW, runs.lenB * ROW), rSKB = make_rsrc(c.sK + kB, runs.lenB * 4), rSVB = make_rsrc(c.sV + kB, runs.lenB * 4);

    constexpr int CH = ROW / 16;
    const int crow = lane / CH, cslot = lane % CH;               // of a copied piece; an odd one is 16 (d = 64: 32) rows further
    const unsigned gk = crow * ROW + 16 * (cslot ^ k4_slot<D>(crow));
    const unsigned gv0 = crow * ROW + 16 * (cslot ^ v4_slot<D>(crow)), gv1 = crow * ROW + 16 * (cslot ^ v4_slot<D>(crow + 1024 / ROW));
    const lds_ptr kbuf = (lds_ptr)(&sm.k[wave][0][0]), vbuf = (lds_ptr)(&sm.v[wave][0][0]), skbuf = (lds_ptr)(&sm.sk[wave][0][0]), svbuf = (lds_ptr)(&sm.sv[wave][0][0]);
    const lds_ptr logbuf = (lds_ptr)(&sm.log_sv[wave][0]), invbuf = (lds_ptr)(&sm.inv_sv[wave][0]), restbuf = (lds_ptr)(&sm.rest[wave][0]);
    auto stage = [&](int t, int slot) {
        const bool inA = t < tilesA;
        const int j0 = KEYS4 * (inA ? t : t - tilesA);
        copy_pieces<PIECES, NT>(pick(inA, rKA, rKB), kbuf + slot * TB, gk, gk, j0 * ROW);
        copy_pieces<PIECES, NT>(pick(inA, rVA, rVB), vbuf + slot * TB, gv0, gv1, j0 * ROW);
        lds_copy4(pick(inA, rSKA, rSKB), skbuf + slot * 256, 4 * lane, j0 * 4);
        lds_copy4(pick(inA, rSVA, rSVB), svbuf + slot * 256, 4 * lane, j0 * 4);
    };
    const int first = t0 + wave;
#pragma unroll
    for (int s = 0; s < ST; ++s)
        if (first + s * W < t1) stage(first + s * W, s);

    // where this lane reads K (key r of 16; the 16 bytes, at d = 64 8 bytes, of quarter q) and V (row i / 2 of the 8 that are transposed, half i & 1 of 16 columns)
    const unsigned k0 = D == 128 ? r * ROW + 16 * (q ^ k4_slot<D>(r)) : r * ROW + 16 * ((q >> 1) ^ k4_slot<D>(r)) + 8 * (q & 1);
    const int vkey = 4 * q + (r >> 1 & 3) + 16 * (r >> 3);
    const unsigned v0 = vkey * ROW + 16 * v4_slot<D>(vkey) + 8 * (r & 1);

    v4i qf[RT][KS], bias[RT];
    float sq2[RT];
    int p[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int row = imin(row0 + 16 * rt + r, c.rows - 1);
        p[rt] = position(row);
        const long qrow = row_of(c, by, unit, row);
        const int8_t *const at = c.Q + qrow * D;
        if constexpr (D == 128) {
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[rt][s] = *reinterpret_cast<const v4i *>(at + 64 * s + 16 * q);
        } else {                                                 // channels in the order in which 8 bytes of K hold them: 8 low ones, then the 8 that are 32 further
            const v2i a = *reinterpret_cast<const v2i *>(at + 8 * q), b = *reinterpret_cast<const v2i *>(at + 32 + 8 * q);
            qf[rt][0] = v4i{a[0], a[1], b[0], b[1]};
        }
        sq2[rt] = c.sQ[qrow];
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        sq2[rt] = query_scale(p[rt] >= 0 ? sq2[rt] : 1.0f, qf[rt]);      // (padding: whatever its scale holds, its row is zeros)
        v4i sum = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(v4i{0x01010101, 0x01010101, 0x01010101, 0x01010101}, qf[rt][s], sum, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[rt][i] = ACC_BIAS_I - 8 * sum[i];
    }

    float m2[RT], l[RT];                                         // m2: M
    v4f o[RT][2][CT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m2[rt] = -INFINITY, l[rt] = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[rt][h][ct] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const NibbleMasks masks;
    int slot = 0;
    for (int t = first; t < t1; t += W) {
        if (ST > 1 && t + W < t1) wait_vmcnt<PER_TILE *(ST - 1)>();      // this tile has landed
        else wait_vmcnt<0>();
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        v4i kw[4];                                               // 16 keys each: the bytes of this lane (d = 64: two dwords)
        v2i vw[2][CT];                                           // 32 keys each
        v4f skv[4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            const lds_ptr at = lds_xor(kbuf + slot * TB + 16 * kb * ROW, 0, k0);
            if constexpr (D == 128) kw[kb] = *reinterpret_cast<LDS_AS const v4i *>(at);
            else {
                const v2i x = *reinterpret_cast<LDS_AS const v2i *>(at);
                kw[kb] = v4i{x[0], x[1], 0, 0};
            }
        }
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) skv[kb] = *reinterpret_cast<LDS_AS const v4f *>(skbuf + slot * 256 + 16 * q + 64 * kb);
        const float sv_here = *reinterpret_cast<LDS_AS const float *>(svbuf + slot * 256 + 4 * lane);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) vw[h][ct] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<LDS_AS v2i *>(lds_xor(vbuf + slot * TB + 32 * h * ROW, 16 * ct, v0)));
        wait_lds();
        __builtin_amdgcn_sched_barrier(0);
        memory_fence_of_the_compiler();
        if (t + ST * W < t1) stage(t + ST * W, slot);            // into the place this tile has left
        __builtin_amdgcn_sched_barrier(0);
        slot = slot == ST - 1 ? 0 : slot + 1;

        // log2 |s_V| and 1 / |s_V|, at least 2^-80, a key to a lane, handed round to the lanes that have the key's scores.  What s_V is beside that, its sign, 0 or 2^80 s_V, is a factor of the weight, later
        const float sv_size = fmaxf(fabsf(sv_here), LEAST_SCALE);
        *reinterpret_cast<LDS_AS float *>(logbuf + 4 * lane) = __builtin_amdgcn_logf(sv_size);
        *reinterpret_cast<LDS_AS float *>(invbuf + 4 * lane) = __builtin_amdgcn_rcpf(sv_size);
        const bool odd = __any(!(sv_here >= LEAST_SCALE));
        if (odd) *reinterpret_cast<LDS_AS float *>(restbuf + 4 * lane) = fminf(fmaxf(sv_here * (1.0f / LEAST_SCALE), -1.0f), 1.0f);
        v4i kop[4][KS];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            if constexpr (D == 128) {
                kop[kb][0] = v4i{low_nibbles(kw[kb][0]), low_nibbles(kw[kb][1]), low_nibbles(kw[kb][2]), low_nibbles(kw[kb][3])};
                kop[kb][KS - 1] = v4i{high_nibbles(kw[kb][0]), high_nibbles(kw[kb][1]), high_nibbles(kw[kb][2]), high_nibbles(kw[kb][3])};
            } else kop[kb][0] = v4i{low_nibbles(kw[kb][0]), low_nibbles(kw[kb][1]), high_nibbles(kw[kb][0]), high_nibbles(kw[kb][1])};
        }
        const bool inA = t < tilesA;
        const int j0 = KEYS4 * (inA ? t : t - tilesA);
        // whether all rows see all 64 keys (wave-uniform)
        const bool clear = p0 >= 0 && (inA ? j0 + KEYS4 <= runs.lenA : j0 + KEYS4 - 1 <= p0 - runs.lo && (j0 > p1 - runs.lo - c.window || j0 + KEYS4 - 1 < c.sinks - runs.lo));
        h8 pb[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float a[16], tmax = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                v4i acc = bias[rt];
#pragma unroll
                for (int s = 0; s < KS; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(kop[kb][s], qf[rt][s], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[4 * kb + i] = (__int_as_float(acc[i]) - ACC_BIAS_F) * skv[kb][i];
            }
            if (!clear) {
                const int hi = (inA ? (p[rt] >= 0 ? runs.lenA - 1 : -1) : p[rt] - runs.lo) - j0;
                const int from = inA ? 0 : p[rt] - runs.lo - c.window + 1 - j0, sink = inA ? 0 : c.sinks - runs.lo - j0;
                const uint64_t seen = keys_seen(hi, from, sink) >> (4 * q);
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(static_cast<uint32_t>(seen >> (32 * (kb >> 1))) & (1u << (16 * (kb & 1) + i)))) a[4 * kb + i] = -INFINITY;
            }
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {                     // log2 (p s_V), but for M
                const v4f ls = *reinterpret_cast<LDS_AS const v4f *>(logbuf + 16 * q + 64 * kb);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[4 * kb + i] = __builtin_fmaf(a[4 * kb + i], sq2[rt], ls[i]);
                    tmax = fmaxf(tmax, a[4 * kb + i]);
                }
            }
            const float m_new = fmaxf(m2[rt], pair_max(swap16_max(tmax)) - FEW4_BELOW);
            const float m_at = m_new == -INFINITY ? 0.0f : m_new;    // a row that has seen nothing yet: weights of 0, no NaN
            const float alpha = __builtin_amdgcn_exp2f(m2[rt] - m_at);   // exp2(-inf) = 0
            m2[rt] = m_new;
            float psum = 0.0f;
            h2 w[8];                                             // keys 0, 2 and 1, 3 of each four: the order of values_of
            auto weights = [&](auto odd_) {
#pragma unroll
                for (int kb = 0; kb < 4; ++kb) {
                    const v4f is = *reinterpret_cast<LDS_AS const v4f *>(invbuf + 16 * q + 64 * kb);
                    v4f x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[i] = __builtin_amdgcn_exp2f(a[4 * kb + i] - m_at);
                        psum = __builtin_fmaf(x[i], is[i], psum);
                    }
                    if constexpr (decltype(odd_)::value) x *= *reinterpret_cast<LDS_AS const v4f *>(restbuf + 16 * q + 64 * kb);      // (before the weight is rounded: once)
#pragma unroll
                    for (int i = 0; i < 2; ++i) w[2 * kb + i] = h2{(_Float16)x[i], (_Float16)x[i + 2]};
                }
            };
            if (odd) weights(std::true_type{});
            else weights(std::false_type{});
            l[rt] = __builtin_fmaf(l[rt], alpha, psum);
            if (__any(alpha != 1.0f)) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) o[rt][h][ct] *= alpha;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) pb[rt][h] = h8{w[4 * h][0], w[4 * h][1], w[4 * h + 1][0], w[4 * h + 1][1], w[4 * h + 2][0], w[4 * h + 2][1], w[4 * h + 3][0], w[4 * h + 3][1]};
            __builtin_amdgcn_sched_barrier(0);                   // (two row tiles between each other take 26 more registers than there are)
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                h8 low, high;
                values_of(vw[h][ct], masks, low, high);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[rt][0][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(low, pb[rt][h], o[rt][0][ct], 0, 0, 0);
                    o[rt][1][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(high, pb[rt][h], o[rt][1][ct], 0, 0, 0);
                }
            }
    }
    __syncthreads();                                             // every wavefront is done with its buffers: o may lie there

    // ---- they meet: M, l and o of each as they are, then whoever has four columns of a row weighs them.  (All rows at once: 16 by 16, 8 x 4 heads with 40 rows on up to 16391 keys 27.3 -> 26.7 us.)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const float sum = quarters_sum(l[rt]);
        if (q == 0) sm.ml[wave][16 * rt + r] = float2{m2[rt], sum};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)                      // 16-byte chunks, the row's bits mixed into the chunk so that a column of rows spreads over the banks
                *reinterpret_cast<v4f *>(&sm.o[wave][16 * rt + r][4 * ((D / 8 * h + 4 * ct + q) ^ r)]) = o[rt][h][ct];
    }
    __syncthreads();
    const int valid = last_row - row0 + 1;
    // Threads of a row, how many times four columns each has, rows at once.  What is the row's alone is done N times less often than by threads with four columns each, which however share out the few rows of a
    // decode step evenly (us, 32 key heads, 40 and 4 rows on 256 keys: N = 4 6.9 and 5.3, N = 1 7.6 and 5.2).
    constexpr int TPR = RT == 1 ? D / 4 : 2 * W, N = D / 4 / TPR, ROWS = 64 * W / TPR;
#pragma unroll
    for (int first_row = 0; first_row < 16 * RT; first_row += ROWS) {
        const int rr = first_row + tid / TPR, to = row0 + rr, col = 4 * (tid % TPR);
        if (rr >= valid) break;
        float2 x[W];
        float m = -INFINITY, ls = 0.0f, f[W];
#pragma unroll
        for (int k = 0; k < W; ++k) x[k] = sm.ml[k][rr], m = fmaxf(m, x[k].x);
        const float m_at = m == -INFINITY ? 0.0f : m;            // (a row that has seen nothing: factors of 0)
#pragma unroll
        for (int k = 0; k < W; ++k) f[k] = __builtin_amdgcn_exp2f(x[k].x - m_at), ls = __builtin_fmaf(x[k].y, f[k], ls);
        v4f s[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            s[n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < W; ++k) s[n] += *reinterpret_cast<const v4f *>(&sm.o[k][rr][(col + 4 * TPR * n) ^ (4 * (rr & 15))]) * f[k];
        }
        if (part.splits > 1) {
            const long pr = static_cast<long>(share) * c.rows + to;
#pragma unroll
            for (int n = 0; n < N; ++n) *reinterpret_cast<v4f *>(c.part_o + pr * D + col + 4 * TPR * n) = s[n];
            if (col == 0) c.part_ml[pr] = float2{m, ls};
        } else {
            const float i = ls > 0.0f ? 1.0f / ls : 0.0f;        // a row that sees nothing: zeros
            const long at = row_of(c, by, unit, to) * D + col;
            auto store = [&](auto type) {
#pragma unroll
                for (int n = 0; n < N; ++n) store4(c.O, decltype(type)::value, at + 4 * TPR * n, s[n][0] * i, s[n][1] * i, s[n][2] * i, s[n][3] * i);
            };
            if (c.o_dtype == IFA_F32) store(std::integral_constant<int, IFA_F32>{});
            else if (c.o_dtype == IFA_F16) store(std::integral_constant<int, IFA_F16>{});
            else store(std::integral_constant<int, IFA_BF16>{});
        }
    }
}
#endif
template <int D, int RT, int W, int ST, bool NT>
__global__ __launch_bounds__(64 * W, 2) void int4_few_kernel(Call c, Sharing sh, Divisors by, int units, int row_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemFew4<D, RT, W, ST> sm;
    // the row tiles of one share of the keys run 8 apart: on one XCD
    const int block = blockIdx.x, eight = by.row_tiles8.of(block), in8 = block - eight * 8 * row_tiles, share = 8 * eight + (in8 & 7), row0 = 16 * RT * (in8 >> 3);
    Part part;
    if (!part_of(c, sh, by, units, share, threadIdx.x & 63, part)) return;
    if (sh.places && row0 == 0 && part.split == 0 && threadIdx.x == 0) sh.parts_of[part.unit] = int2{part.first, part.splits};
    few4_rows_of_a_unit<D, RT, W, ST, NT>(sm, c, by, part, share, row0);
#endif
}

// ---- as many parts of a row as its unit has, joined --------------------------------------------------------------------
// D / 4 threads a row, JOIN4_GROUPS of them taking every such part, with AT_ONCE loads in flight each; then they meet in LDS.
constexpr int JOIN4_GROUPS = 8;
template <int D>
__global__ __launch_bounds__(JOIN4_GROUPS * D / 4) void int4_join_kernel(Call c, Sharing sh, Divisors by) {
    constexpr int TPR = D / 4, P = JOIN4_GROUPS, AT_ONCE = 4;
    __shared__ v4f so[P][TPR];
    __shared__ float2 sml[P];
    const int unit = blockIdx.y, row = blockIdx.x, cc = threadIdx.x % TPR, pg = threadIdx.x / TPR;
    const int2 of = sh.parts_of[unit];
    const int n = of.y;
    if (n <= 1) return;                                          // (it is in O already)
    float m = -INFINITY, l = 0.0f;
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = pg; i0 < n; i0 += AT_ONCE * P) {
        float2 x[AT_ONCE];
        v4f y[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = i0 + k * P;
            x[k] = float2{-INFINITY, 0.0f};
            y[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            if (i < n) {
                const long at = static_cast<long>(of.x + i) * c.rows + row;
                x[k] = c.part_ml[at];
                y[k] = *reinterpret_cast<const v4f *>(c.part_o + at * D + 4 * cc);
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
    so[pg][cc] = s;
    if (cc == 0) sml[pg] = float2{m, l};
    __syncthreads();
    if (pg) return;
    float m_all = m;
#pragma unroll
    for (int k = 1; k < P; ++k) m_all = fmaxf(m_all, sml[k].x);
    if (m_all != -INFINITY) {
        const float f = __builtin_amdgcn_exp2f(m - m_all);
        l *= f, s *= f;
#pragma unroll
        for (int k = 1; k < P; ++k) {
            const float w = __builtin_amdgcn_exp2f(sml[k].x - m_all);
            l += sml[k].y * w;
            s += so[k][cc] * w;
        }
    }
    const float q = l > 0.0f ? 1.0f / l : 0.0f;
    store4(c.O, c.o_dtype, row_of(c, by, unit, row) * D + 4 * cc, s[0] * q, s[1] * q, s[2] * q, s[3] * q);
}

// ---- many rows: tiles of 128 ------------------------------------------------------------------------------------------
// Four wavefronts of 32 rows share the keys, 64 at a time, through LDS (double-buffered).  What bounds it is the vector unit, so a block is unpacked once for the four: each thread takes
// 16 bytes of a row of K and of V from memory a block ahead, and writes them to LDS as the matrix operands are: K in bytes, V in fp16, which the transposing reads then serve as in the kernel for 8 bits.
template <int D> struct SmemTile4 {
    alignas(4096) int8_t k[2][KEYS4 * D];
    alignas(4096) int8_t v[2][KEYS4 * 2 * D];
    alignas(256) float sk[2][KEYS4], sv[2][KEYS4];
    float2 sv_size[2];                     // log2 of the largest |s_V|; that |s_V| 2^-ALIKE4
};

#if defined(__HIP_DEVICE_COMPILE__)
template <int D> struct RowState4 {
    float m2, l;                                                 // m2: M
    v16f o[D / 32];                                              // channels 1 and 2 of four are exchanged, as V's columns are
    __device__ __forceinline__ float channel(int dt, int v) const { return o[dt][(v & ~3) | (v & 1) << 1 | (v >> 1 & 1)]; }
};

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
// 16 bytes of a row of codes to where they belong: `low` and, for the high nibbles, `high`
__device__ __forceinline__ void unpack_k(const u4 &w, lds_ptr low, lds_ptr high) {
    *reinterpret_cast<LDS_AS u4 *>(low) = w & LOW4;
    *reinterpret_cast<LDS_AS u4 *>(high) = w >> 4 & LOW4;
}
__device__ __forceinline__ void unpack_v(const u4 &w, const NibbleMasks &m, lds_ptr low, lds_ptr high) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        u4 lo, hi;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t a = w[i + e], b = w[i + e] >> 8;      // channels 0, 2 and 1, 3 of four: columns lie in LDS in this order
            lo[2 * e] = __builtin_bit_cast(uint32_t, low_codes(a, m)), lo[2 * e + 1] = __builtin_bit_cast(uint32_t, low_codes(b, m));
            hi[2 * e] = __builtin_bit_cast(uint32_t, high_codes(a, m)), hi[2 * e + 1] = __builtin_bit_cast(uint32_t, high_codes(b, m));
        }
        *reinterpret_cast<LDS_AS u4 *>(low + 8 * i) = lo;
        *reinterpret_cast<LDS_AS u4 *>(high + 8 * i) = hi;
    }
}

// 64 keys in LDS against the wavefront's rows.  `clear`: all of them count for every row, otherwise those of `seen`, none behind key `last`.
template <int D>
__device__ __forceinline__ void tile4_block(lds_ptr ks, lds_ptr vs, lds_ptr sk, lds_ptr sv, float2 size, int last, int lane, const Lane<D, false> &lo, const v4i (&qf)[D / 32], float sq2, bool clear, uint64_t seen,
                                            const v16i &bias, RowState4<D> &st) {
    constexpr int KS = D / 32, DT = D / 32;
    const int g = lane >> 5;
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
    const unsigned mine = 4 * (8 * (lane >> 2 & 3) + 4 * g + (lane & 3));        // lane 16 x + v: the key whose scores lie in element v of acc[0]
    float skv[2], svv[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
        skv[mt] = *reinterpret_cast<LDS_AS const float *>(sk + mine + 128 * mt);
        svv[mt] = *reinterpret_cast<LDS_AS const float *>(sv + mine + 128 * mt);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
        unrolled([&](auto v_) { constexpr int v = decltype(v_)::value; a[mt][v] = (__int_as_float(acc[mt][v]) - ACC_BIAS_F) * of_row<v>(skv[mt]); }, std::make_integer_sequence<int, 16>{});
    // log2 of bounds of the largest |s_V| that the row sees, from above and from below: M moves when it has to by the one, and to where the other puts it.  A hidden key's scale in M would take the
    // weights that count under fp16's range.  Scales of a block within 2^ALIKE4 bound each other; otherwise each row finds its own largest.  (M by all 64 keys, seen or not: 3 x 12 heads of 64, up to 1777 queries, window 333, 19.0 us, like
    // this 19.9, with the row's own in every block that is not clear 21.4.)
    float high = size.x, low = size.x;
    if (!clear) {
        const float one = fabsf(*reinterpret_cast<LDS_AS const float *>(sv + 4 * lane));
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (!(static_cast<uint32_t>(seen >> (32 * mt)) >> (4 * g) & (1u << (8 * (v >> 2) + (v & 3))))) a[mt][v] = -INFINITY;
        if (!__any(lane <= last && one < size.y)) low = high - ALIKE4;
        else {
            int most = 0;                                        // (as integers, which numbers that are not negative compare like)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                const float abs_sv = fabsf(svv[mt]);
                unrolled([&](auto v_) {                          // a hidden key's -inf is a negative integer, other scores + 2^100 are above any scale
                    constexpr int v = decltype(v_)::value;
                    most = imax(most, imin(__float_as_int(of_row<v>(abs_sv)), __float_as_int(a[mt][v] + 0x1p100f)));
                }, std::make_integer_sequence<int, 16>{});
            }
            high = low = __builtin_amdgcn_logf(fmaxf(pair_max(__int_as_float(most)), LEAST_SCALE));
        }
    }
    float bmax = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int v = 0; v < 16; ++v) bmax = fmaxf(bmax, a[mt][v]);
    __builtin_amdgcn_sched_barrier(0);
    const float top = __builtin_fmaf(pair_max(bmax), sq2, high - TILE4_BELOW);
    const bool moves = top > st.m2 + SLACK4;                     // (st.m2 = -inf: whenever a key counts)
    if (__any(moves)) {
        const float m_new = moves ? top - (high - low) : st.m2;
        const float alpha = moves ? __builtin_amdgcn_exp2f(st.m2 - m_new) : 1.0f;
        st.m2 = m_new;
        st.l *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) st.o[dt][v] *= alpha;
    }
    const float m = st.m2 == -INFINITY ? 0.0f : st.m2;           // a row that has seen nothing yet: weights of 0, no NaN
    h2 ph[2][8];
    float sum = 0.0f;                                            // of the block: small weights do not meet l one by one
    auto weights = [&](int mt, auto vq_) {                      // of 4 keys
        constexpr int vq = decltype(vq_)::value;
        float x[4];
        unrolled([&](auto i) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(a[mt][4 * vq + i], sq2, -m));
            sum += e;
            x[i] = e * of_row<4 * vq + decltype(i)::value>(svv[mt]);
        }, std::make_integer_sequence<int, 4>{});
        ph[mt][2 * vq] = h2{(_Float16)x[0], (_Float16)x[1]};
        ph[mt][2 * vq + 1] = h2{(_Float16)x[2], (_Float16)x[3]};
    };
    // the weights of the second 32 keys between the products of the first
    h8 vop[DT][2];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int s = 0; s < 2; ++s) vop[dt][s] = v_operand<D, false>(vs, lo.v0, dt, 16 * s);
    unrolled([&](auto vq) { weights(0, vq); }, std::make_integer_sequence<int, 4>{});
    __builtin_amdgcn_s_setprio(3);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
        unrolled([&](auto dt) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const h8 pb = {ph[mt][4 * s][0], ph[mt][4 * s][1], ph[mt][4 * s + 1][0], ph[mt][4 * s + 1][1], ph[mt][4 * s + 2][0], ph[mt][4 * s + 2][1], ph[mt][4 * s + 3][0], ph[mt][4 * s + 3][1]};
                st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vop[dt][s], pb, st.o[dt], 0, 0, 0);
                if (mt == 0) vop[dt][s] = v_operand<D, false>(vs, lo.v0, dt, 32 + 16 * s);
            }
            if (mt == 0) unrolled([&](auto q) { weights(1, std::integral_constant<int, decltype(dt)::value * (4 / DT) + decltype(q)::value>{}); }, std::make_integer_sequence<int, 4 / DT>{});
        }, std::make_integer_sequence<int, DT>{});
    st.l += sum;
    __builtin_amdgcn_s_setprio(0);
}

template <int D>
__device__ __forceinline__ void tile4_of_a_unit(SmemTile4<D> &sm, const Call &c, const Divisors &by, int block, int units, int row_tiles, int head_group) {
    constexpr int ROW = ROW4<D>, KB = KEYS4 * D, VB = KEYS4 * 2 * D, DT = D / 32, CH = ROW / 16;
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int unit, ord;                                               // the row tiles and parts of a unit on one XCD, the last rows, which may see more, first
    map_workgroup(block, units, row_tiles * c.splits, head_group, true, unit, ord);
    const int tile = by.splits.of(ord), rt = row_tiles - 1 - tile, split = ord - tile * c.splits;
    const int L = keys_of(c.lens, by.Hkv.of(unit), c.Nk), window = c.window;
    const int row0 = TILE_ROWS * rt, last_row = imin(row0 + TILE_ROWS - 1, c.rows - 1), row = imin(row0 + 32 * wave + r, last_row);
    auto position = [&](int i) { return L - c.Nq + static_cast<int>(by.G.of(i)); };
    const int pos0 = position(row0), pos1 = position(last_row);
    // The two runs one after the other, cut into blocks of 64 with no seam: key v of them is key v for v < lenA, else key v + gap.  All of it lies in front of key pos1 + 1.
    const Runs runs(false, 0, window, c.sinks, pos0, pos1);
    const int lenA = runs.lenA, gap = runs.lo - lenA, keys = lenA + runs.lenB;
    const int blocks = (keys + KEYS4 - 1) / KEYS4, per = (blocks + c.splits - 1) / c.splits, t0 = split * per, t1 = imin(blocks, t0 + per);
    // a row at p sees key v iff v <= p - gap and (v > p - gap - window or v < sink); one at p < 0 none
    const int p = position(row), hi = p < 0 ? -1 : p - gap, sink = imax(lenA, c.sinks - gap);
    const int w0 = position(imin(row0 + 32 * wave, last_row)), w1 = position(imin(row0 + 32 * wave + 31, last_row));      // of the wavefront's first and last row
    const int hi0 = w0 < 0 ? -1 : w0 - gap, hi1 = w1 < 0 ? -1 : w1 - gap;

    // Of a block this thread takes 16 bytes of K and of V (d = 64: the first half of the threads of K, the second of V), and a scale of K (first wavefront) or of V (second)
    const long first_key = static_cast<long>(unit) * c.Nk;
    const int seen_end = imax(0, pos1 + 1);
    const auto rsrc = [&](const void *at, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, bytes, 0x00020000); };
    const auto rK = rsrc(c.K + first_key * ROW, seen_end * ROW), rV = rsrc(static_cast<const int8_t *>(c.V) + first_key * ROW, seen_end * ROW), rSK = rsrc(c.sK + first_key, seen_end * 4),
               rSV = rsrc(c.sV + first_key, seen_end * 4);
    const int piece = D == 128 ? tid : tid & 127, prow = piece / CH, pc = piece % CH;
    u4 kraw = {}, vraw = {};                                     // (d = 64: `kraw` of either)
    float sraw = 0.0f;
    auto fetch = [&](int t) {
        const int at = KEYS4 * t;
        auto key = [&](int in) { return at + in + (at + in >= lenA ? gap : 0); };       // (row by row: a block may hold the seam)
        const int from = key(prow) * ROW + 16 * pc;
        kraw = __builtin_amdgcn_raw_buffer_load_b128(D == 128 || wave < 2 ? rK : rV, from, 0, 0);
        if constexpr (D == 128) vraw = __builtin_amdgcn_raw_buffer_load_b128(rV, from, 0, 0);
        if (wave < 2) sraw = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(wave == 0 ? rSK : rSV, key(lane) * 4, 0, 0));
    };
    const lds_ptr kbuf = (lds_ptr)(&sm.k[0][0]), vbuf = (lds_ptr)(&sm.v[0][0]), skbuf = (lds_ptr)(&sm.sk[0][0]), svbuf = (lds_ptr)(&sm.sv[0][0]);
    const NibbleMasks masks;
    const unsigned kat = prow * D, kx = k_slot<D>(prow), vat = prow * 2 * D + 32 * (pc & 1), vx = v_slot<D, false>(prow);
    auto unpack = [&](int slot) {
        const lds_ptr k = kbuf + slot * KB + kat, v = vbuf + slot * VB + vat;
        if (D == 128 || wave < 2) unpack_k(kraw, k + 16 * (pc ^ kx), k + 16 * ((pc + D / 32) ^ kx));
        if (D == 128 || wave >= 2) unpack_v(D == 128 ? vraw : kraw, masks, v + 64 * ((pc >> 1) ^ vx), v + 64 * (((pc >> 1) + D / 64) ^ vx));
        if (wave < 2) *reinterpret_cast<LDS_AS float *>((wave == 0 ? skbuf : svbuf) + slot * 256 + 4 * lane) = sraw;
        if (wave == 1) {
            const float most = wave_max(fabsf(sraw)), high = __builtin_amdgcn_logf(fmaxf(most, LEAST_SCALE));
            if (lane == 0) sm.sv_size[slot] = float2{high, most * (1.0f / (1 << ALIKE4))};
        }
    };
    if (t0 < t1) fetch(t0);

    const long qrow = row_of(c, by, unit, row);
    v4i qf[DT];
#pragma unroll
    for (int kk = 0; kk < DT; ++kk) qf[kk] = *reinterpret_cast<const v4i *>(c.Q + qrow * D + 32 * kk + 16 * g);
    const float sq = c.sQ[qrow], sq2 = query_scale(p >= 0 ? sq : 1.0f, qf);        // (padding: whatever its scale holds, its row is zeros)
    v16i bias;
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = 0;
#pragma unroll
    for (int kk = 0; kk < DT; ++kk) bias = __builtin_amdgcn_mfma_i32_32x32x32_i8(v4i{0x01010101, 0x01010101, 0x01010101, 0x01010101}, qf[kk], bias, 0, 0, 0);
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = ACC_BIAS_I - 8 * bias[v];
    asm volatile("" : "+v"(bias));
    const Lane<D, false> lo(lane);
    RowState4<D> st;
    st.m2 = -INFINITY, st.l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) st.o[dt][v] = 0.0f;

    const bool alive = row0 + 32 * wave < c.rows;                // (wave-uniform) a wavefront without rows unpacks only
    if (t0 < t1) unpack(0);
    if (t0 + 1 < t1) fetch(t0 + 1);
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int slot = (t - t0) & 1, v0 = KEYS4 * t;
        if (t + 1 < t1) unpack(slot ^ 1);                        // (whose readers have passed the last barrier)
        if (t + 2 < t1) fetch(t + 2);
        // (wave-uniform) whether some of the rows see some of the keys, and whether all see all
        const bool any = alive && hi1 >= v0 && (hi0 - window < v0 + KEYS4 - 1 || v0 < sink);
        const bool clear = hi0 >= v0 + KEYS4 - 1 && (hi1 - window < v0 || v0 + KEYS4 <= sink);
        const uint64_t seen = clear ? 0 : keys_seen(hi - v0, hi - window + 1 - v0, sink - v0);
        if (any) tile4_block<D>(kbuf + slot * KB, vbuf + slot * VB, skbuf + slot * 256, svbuf + slot * 256, sm.sv_size[slot], hi1 - v0, lane, lo, qf, sq2, clear, seen, bias, st);
        __syncthreads();
    }

    const float l = st.l + swap32(st.l);
    const lds_ptr stage_out = (lds_ptr)(&sm) + wave * (64 * D);
    const int first = row0 + 32 * wave;
    if (c.part_o) {
        const long pr = (static_cast<long>(unit) * c.splits + split) * c.rows;
        float *const po = c.part_o + pr * D;
        store_rows<D, float>(stage_out, lane, [&](int dt, int v) { return st.channel(dt, v); },
                             [&](int k) { return first + k < c.rows ? reinterpret_cast<char *>(po + static_cast<long>(first + k) * D) : nullptr; });
        if (g == 0 && first + r < c.rows) c.part_ml[pr + first + r] = float2{st.m2, l};
        return;
    }
    const float f = l > 0.0f ? 1.0f / l : 0.0f;                  // a row that sees nothing: zeros
    auto store = [&](auto type) {
        using OutT = decltype(type);
        store_rows<D, OutT>(stage_out, lane, [&](int dt, int v) { return st.channel(dt, v) * f; },
                            [&](int k) { return first + k < c.rows ? reinterpret_cast<char *>(static_cast<OutT *>(c.O) + row_of(c, by, unit, first + k) * D) : nullptr; });
    };
    if (c.o_dtype == IFA_F32) store(float{});
    else if (c.o_dtype == IFA_F16) store(__half{});
    else store(__hip_bfloat16{});
}
#endif
// (d = 64: three wavefronts fit a SIMD, which took 32 heads, prompts of 4096 from 114 us to 102, with the scales as lane modifiers 96; at d = 128 there are 52 registers too few for it, 279 -> 700)
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void int4_tile_kernel(Call c, Divisors by, int units, int row_tiles, int head_group) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ SmemTile4<D> sm;
    tile4_of_a_unit<D>(sm, c, by, blockIdx.x, units, row_tiles, head_group);
#endif
}

// ---- host --------------------------------------------------------------------------------------------------------------
template <int D>
int launch(Call c, const Int4Plan &plan, void *workspace, hipStream_t st) {
    const int units = c.B * c.Hkv, row_tiles = static_cast<int>(plan.row_tiles);
    c.splits = static_cast<int>(plan.parts / units);
    Sharing sh = {plan.places, nullptr};
    const Divisors by = {Divisor(c.G), Divisor(c.Hkv), Divisor(c.splits), Divisor(8 * row_tiles)};
    if (plan.parts > units) {
        c.part_o = static_cast<float *>(workspace);
        c.part_ml = reinterpret_cast<float2 *>(c.part_o + plan.parts * c.rows * D);
        sh.parts_of = reinterpret_cast<int2 *>(c.part_ml + plan.parts * c.rows);
    }
    auto few = [&](auto rt, auto waves, auto once) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((int4_few_kernel<D, decltype(rt)::value, W, W == 8 ? 2 : 1, decltype(once)::value>), dim3(static_cast<unsigned>((plan.parts + 7) / 8 * 8 * row_tiles)), dim3(64 * W), 0, st, c, sh, by, units, row_tiles);
    };
    auto few_waves = [&](auto rt) {
        constexpr std::integral_constant<int, 4> four{};
        if (plan.waves == 8) few(rt, std::integral_constant<int, 8>{}, std::false_type{});
        else if (plan.once) few(rt, four, std::true_type{});
        else few(rt, four, std::false_type{});
    };
    if (plan.tile) hipLaunchKernelGGL((int4_tile_kernel<D>), dim3(static_cast<unsigned>(plan.parts * row_tiles)), dim3(256), 0, st, c, by, units, row_tiles, head_group_for(true, 0, 0));
    else if (plan.rows_at_once == 16) few_waves(std::integral_constant<int, 1>{});
    else few_waves(std::integral_constant<int, 2>{});
    const long all_rows = static_cast<long>(units) * c.rows;
    if (plan.places) hipLaunchKernelGGL((int4_join_kernel<D>), dim3(static_cast<unsigned>(c.rows), static_cast<unsigned>(units)), dim3(JOIN4_GROUPS * D / 4), 0, st, c, sh, by);
    else if (c.splits > 1) {
        const Parts parts = {nullptr, c.part_o, nullptr, c.part_ml, 0, c.splits};
        auto join = [&](auto p) {
            constexpr int P = decltype(p)::value, ROWS = 1024 / D / P;
            hipLaunchKernelGGL((cache_attention_join_kernel<D, P>), dim3(static_cast<unsigned>((all_rows + ROWS - 1) / ROWS)), dim3(256), 0, st, c, parts, all_rows);
        };
        if (c.splits > 8) join(std::integral_constant<int, 8>{});
        else join(std::integral_constant<int, 1>{});
    }
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}

// Sizes alone: what a call or a workspace query takes
int refuse_sizes(int B, int H, int Hkv, int Nq, int Nk, int d, int window, int sinks) {
    if (B <= 0 || H <= 0 || Hkv <= 0 || Nq <= 0 || Nk <= 0 || d <= 0 || H % Hkv || window <= 0 || sinks < 0) return IFA_ERR_SHAPE;
    const long heads = static_cast<long>(B) * H, N = Nq > Nk ? Nq : Nk;
    if (heads > (1L << 40) / N / d) return IFA_ERR_SHAPE;
    if (d != 64 && d != 128) return IFA_ERR_UNSUPPORTED;
    if (static_cast<long>(Nk) * d * 2 > 0x7ff00000L) return IFA_ERR_UNSUPPORTED;
    if (heads * Nq > 1L << 26 || heads > 1L << 23) return IFA_ERR_UNSUPPORTED;      // a launch has less than 2^32 threads: 256 to 16 rows or to a unit, d / 4 to a joined row
    return IFA_OK;
}

}  // namespace

extern "C" long ifa_int4_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d, int window, int sinks) {
    if (refuse_sizes(B, H, Hkv, Nq, Nk, d, window, sinks)) return -1;
    return int4_plan(B, Hkv, H / Hkv, Nq, Nk, d, imin(window, Nk), imin(sinks, Nk), true).bytes;
}

extern "C" int int_flash_attn_fwd_int4(const signed char *Q_i8, const void *K_i4, const void *V_i4, const float *s_Q, const float *s_K, const float *s_V, const int *lens,
                                       int B, int H, int Hkv, int Nq, int Nk, int d, int window, int sinks, void *O, int o_dtype, void *workspace, long workspace_bytes, void *hip_stream) {
    if (const int rc = refuse_sizes(B, H, Hkv, Nq, Nk, d, window, sinks)) return rc;
    if (!Q_i8 || !K_i4 || !V_i4 || !s_Q || !s_K || !s_V || !O) return IFA_ERR_NULL;
    if (o_dtype < IFA_F32 || o_dtype > IFA_BF16) return IFA_ERR_DTYPE;
    for (const void *p : {static_cast<const void *>(Q_i8), K_i4, V_i4, static_cast<const void *>(O)})
        if (!ifa_aligned16(p)) return IFA_ERR_UNSUPPORTED;
    for (const void *p : {static_cast<const void *>(s_Q), static_cast<const void *>(s_K), static_cast<const void *>(s_V), static_cast<const void *>(lens)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return IFA_ERR_UNSUPPORTED;
    Call c = {};
    c.Q = Q_i8, c.K = static_cast<const int8_t *>(K_i4), c.V = V_i4, c.sQ = s_Q, c.sK = s_K, c.sV = s_V, c.lens = lens;
    c.B = B, c.Hkv = Hkv, c.G = H / Hkv, c.Nq = Nq, c.Nk = Nk, c.window = imin(window, Nk), c.sinks = imin(sinks, Nk);
    c.rows = c.G * Nq, c.O = O, c.o_dtype = o_dtype;
    const Int4Plan plan = int4_plan(B, Hkv, c.G, Nq, Nk, d, c.window, c.sinks, lens != nullptr);
    if (plan.bytes) {
        if (!workspace) return IFA_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(workspace) & 255) return IFA_ERR_UNSUPPORTED;
        if (workspace_bytes < plan.bytes) return IFA_ERR_WORKSPACE;
    }
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return d == 128 ? launch<128>(c, plan, workspace, st) : launch<64>(c, plan, workspace, st);
}
