// What the kernels that read a quantized cache share (intfa_cache_attention.hip, intfa_cache_weights.hip): the call as the kernels take it, which
// keys a group of query rows sees, and the tiles of 32 keys in LDS.
#ifndef INTFA_CACHE_H
#define INTFA_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "intfa_device.h"

namespace ifa_cache {

using namespace ifa_dev;

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));

// One call.  Q [B, H, Nq, d], own keys [B, Hkv, Nk, d], shared keys [Hkv, Np, d] in front of them (Kp null: none); H = G Hkv.
//   The rows of a UNIT are the queries that read the same keys, packed so that a group of heads fills the 32 columns of a matrix instruction
// that one decode query alone would leave empty: row (i, g) of unit (b, hk) with g fastest; for the shared keys alone (`all`) row (b, i, g) of unit hk.
struct Call {
    const int8_t *Q, *K, *Kp;
    const void *V, *Vp;
    const float *sQ, *sK, *sKp, *sV, *sVp;                       // sV, sVp null: V is fp16
    const int *lens;                                             // null: Nk everywhere
    int B, Hkv, G, Nq, Nk, Np, window, sinks;                    // window <= Nk
    int rows, splits;                                            // rows of a unit; workgroups that share the keys of a unit
    float *part_o;                                               // [unit][split][rows][d] and [unit][split][rows] (m, l): where parts go (null: straight to O)
    float2 *part_ml;
    void *O;
    int o_dtype;
};

__host__ __device__ __forceinline__ int imin(int a, int b) { return a < b ? a : b; }
__host__ __device__ __forceinline__ int imax(int a, int b) { return a > b ? a : b; }

// How many keys sequence b has: what lies at or beyond that is never looked at.
__device__ __forceinline__ int keys_of(const int *lens, int b, int Nk) {
    return __builtin_amdgcn_readfirstlane(lens ? imax(0, imin(lens[b], Nk)) : Nk);
}

// The keys that rows at positions p0 .. p1 see between them, as two runs that start where the first row begins to see (not at a multiple of the tile:
// no key that nobody sees is read, whatever its bytes are):
//   A  the shared keys, or the sinks in front of the window: every row sees all of them (without shared keys: every row with p >= 0)
//   B  keys from `lo` on: row p sees lo + k iff k <= p - lo and (k > p - lo - window or k < sinks - lo)
struct Runs {
    int lo, lenA, lenB;
    __device__ __forceinline__ Runs(bool shared, int Np, int window, int sinks, int p0, int p1) {
        if (shared) {
            lo = 0, lenA = Np, lenB = imax(0, p1 + 1);
        } else {
            lo = imax(0, imax(p0, 0) - window + 1);
            lenB = imax(0, p1 + 1 - lo);
            lenA = lenB ? imin(sinks, lo) : 0;
        }
    }
};

// 16-byte slot of K chunk c of row r: c ^ k_slot(r), so that 32 rows read at one chunk spread over the banks
template <int D> __device__ __forceinline__ int k_slot(int row) { return (D == 128) ? (row & 7) : ((row >> 1) & 3); }
// V, fp16: 64-byte chunks, read 4 keys at a time; INT8: 16-byte chunks, read 8 keys (0-3, 8-11 or 4-7, 12-15) at a time
template <int D, bool VI8> __device__ __forceinline__ int v_slot(int row) {
    if constexpr (VI8) {
        const int s = (row & 3) | ((row >> 1) & 4);
        return (D == 128) ? s : (s & 3);
    } else return (D == 128) ? (row & 3) : (row & 1);
}

template <int D, bool VI8> constexpr int V_ROW = D * (VI8 ? 1 : 2);    // bytes of a row of V
// Copies of 1 KB that a tile of 32 keys takes
template <int D> constexpr int K_PIECES = 32 * D / 1024;
template <int D, bool VI8> constexpr int V_PIECES = 32 * V_ROW<D, VI8> / 1024;

#if defined(__HIP_DEVICE_COMPILE__)

// This lane's part of a tile: where it copies from (byte offset inside the tile in memory; piece i is 1024 i further, which the slots do not see except
// INT8 V of d = 128, where odd pieces have the other `gv`), and where it reads its matrix operands.
template <int D, bool VI8> struct Lane {
    unsigned k0, v0, gk, gv[2];
    __device__ __forceinline__ explicit Lane(int lane) {
        const int r = lane & 31, g = lane >> 5;
        constexpr int CH = D / 16, VR = V_ROW<D, VI8>, CHV = VR / 16;
        { const int row = lane / CH, slot = lane % CH; gk = row * D + 16 * (slot ^ k_slot<D>(row)); }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int p = 64 * i + lane, row = p / CHV, slot = p % CHV;
            gv[i] = row * VR + 16 * (slot ^ (VI8 ? v_slot<D, VI8>(row) : v_slot<D, VI8>(row) << 2)) - 1024 * i;
        }
        k0 = r * D + ((g ^ k_slot<D>(r)) * 16);                                  // k-step kk at k0 ^ 32 kk
        const int i = lane & 15, G = lane >> 4;
        if constexpr (VI8) {
            const int kidx = i >> 1, key = 8 * (kidx >> 2) + 4 * g + (kidx & 3);
            v0 = key * D + (((G & 1) ^ v_slot<D, VI8>(key)) * 16) + 8 * (i & 1);     // d tile dt at v0 ^ 32 dt
        } else {
            const int key = 4 * g + (i >> 2);
            v0 = key * VR + (v_slot<D, VI8>(key) * 64) + 32 * (G & 1) + 8 * (i & 3); // d tile dt at v0 ^ 64 dt
        }
    }
};

// Four INT8 codes as fp16, exactly: 1024 + u has the bit pattern 0x6400 | u for 0 <= u < 1024; u = code + 128.
__device__ __forceinline__ void codes_to_half(uint32_t w, h2 &a, h2 &b) {
    w ^= 0x80808080u;
    const h2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    a = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) + off;
    b = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) + off;
}

// A operand of O^T = V^T P^T for 16 keys from `key` on (a multiple of 16) and d tile dt: 8 keys of one column of V, in the order in which the S^T accumulators
// hold the weights (4 g + 0 .. 3, then 8 further on)
template <int D, bool VI8>
__device__ __forceinline__ h8 v_operand(lds_ptr vs, unsigned v0, int dt, int key) {
    if constexpr (VI8) {
        const v2i w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<LDS_AS v2i *>(lds_xor(vs, 32 * dt, v0) + key * D));
        h2 a, b, c, d;
        codes_to_half(static_cast<uint32_t>(w[0]), a, b);
        codes_to_half(static_cast<uint32_t>(w[1]), c, d);
        return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        const lds_ptr at = lds_xor(vs, 64 * dt, v0) + key * (2 * D);
        const h4 t0 = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s4 *>(at)));
        const h4 t1 = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s4 *>(at + 8 * (2 * D))));
        return h8{t0[0], t0[1], t0[2], t0[3], t1[0], t1[1], t1[2], t1[3]};
    }
}

// Which of 64 keys count for a row, a bit each: key k iff k <= hi and (k >= from or k < sink)
__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t keys_seen(int hi, int from, int sink) { return below(hi + 1) & (~below(from) | below(sink)); }

// N pieces of 1 KB, one after the other (N a power of two up to 8); NT: bytes that are read once
template <int N, bool NT = false> __device__ __forceinline__ void copy_pieces(const BufRsrc &r, lds_ptr lds, unsigned even, unsigned odd, int soff) {
    if constexpr (N <= 4) lds_copy16_run<N, NT>(r, lds, even, odd, soff);
    else {
        copy_pieces<N / 2, NT>(r, lds, even, odd, soff);
        copy_pieces<N / 2, NT>(r, lds + N / 2 * 1024, even, odd, soff + N / 2 * 1024);
    }
}
// Offset of a request that fetches nothing: past the end of any tensor (the scalar offset takes part in the range check), so the copy writes zeros.
constexpr int NOTHING = 0x7fff0000;

__device__ __forceinline__ BufRsrc pick(bool a, const BufRsrc &x, const BufRsrc &y) {
    return {{a ? x.w[0] : y.w[0], a ? x.w[1] : y.w[1], a ? x.w[2] : y.w[2], x.w[3]}};
}
// s_Q log2(e) of a live query.  One whose scale is 0 scores 0 with every key: its codes become 0 and its scale 1, so that the -inf of masked scores, to which the scale comes last,
// is never multiplied by 0.
template <int KS> __device__ __forceinline__ float query_scale(float sq, v4i (&codes)[KS]) {
    if (sq == 0.0f) {
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) codes[kk] = v4i{0, 0, 0, 0};
        sq = 1.0f;
    }
    return sq * LOG2E;
}
// Copies into LDS are assembly that the compiler does not see write memory: nothing is read across this.
__device__ __forceinline__ void memory_fence_of_the_compiler() { asm volatile("" ::: "memory"); }

#endif  // __HIP_DEVICE_COMPILE__

}  // namespace ifa_cache

#endif  // INTFA_CACHE_H
