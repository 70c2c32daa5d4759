// Tokens into a quantized cache and back, gfx950: append_keys, read_keys.
//
//     append   the row x of token i goes to slot p = L_b - Nn + i:  q = rint(x (R / a)), s = a / R,  a = max|x|,  R = 127 or 7
//     read     x' = q s  (rotated keys: H (q s) / d)
//
// Both move every byte once and compute next to nothing: what bounds them is memory, or the launch where there are few tokens.  As in the quantizers of whole tensors a lane
// owns 8 consecutive elements of a row and d / 8 adjacent lanes a row; K and V of a token go together, so that up to 2 x AT_ONCE loads of a lane are in flight.
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <hip/hip_bf16.h>
#include <stdint.h>
#include <type_traits>

#include "intfa.h"
#include "intfa_internal.h"
#include "intfa_divisor.h"
#include "intfa_rows.h"

namespace {

using namespace ifa_rows;
using ifa::Divisor;

struct Tokens {                            // activations [B, Hkv, Nn, d], rows contiguous
    const void *X;
    long b, h, n;                          // strides, in elements
};
struct AppendCall {
    Tokens K, V;
    const int *lens;
    int8_t *Kc;
    void *Vc;
    float *sK, *sV;
    unsigned rows, Hkv, Nn;
    int Nk;
    Divisor by_tokens, by_heads;
};
struct ReadCall {
    const int8_t *Kc;
    const void *Vc;
    const float *sK, *sV;
    const int *lens;
    void *K, *V;
    unsigned rows, Hkv, count;
    int Nk;
    long first;                            // -1: the last `count` of each sequence
    Divisor by_count, by_heads;
};

constexpr int THREADS = 256;
constexpr long MOST_ROWS = 1L << 28;        // a launch has less than 2^32 threads: 8 or 16 to a row, or to two

__device__ __forceinline__ int keys_of(const int *lens, unsigned b, int Nk) {
    if (!lens) return Nk;
    const int n = lens[b];
    return n < 0 ? 0 : n > Nk ? Nk : n;
}

// ---- four bits -------------------------------------------------------------------------------------------------------
// Below 2^-118 7 / a or a / 7 would leave the normal range of fp32: such a row counts as zeros.
constexpr float LEAST4 = 0x1p-118f;
__device__ __forceinline__ float inverse4(float a) { return a >= LEAST4 ? 7.0f / a : 0.0f; }
__device__ __forceinline__ float scale4(float a) { return a >= LEAST4 ? a / 7.0f : 1.0f; }
// q + 8 of 8 elements, one a byte.  Adding 1.5 2^23 rounds the product, |x (7 / a)| < 7.5, to an integer (half to even) in the low bits of the sum.
__device__ __forceinline__ uint2 codes4(const float (&x)[8], float inv) {
    uint32_t u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(x[i] * inv + 12582920.0f);
    const uint32_t a = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), b = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu), c = __builtin_amdgcn_perm(u[5], u[4], 0x0c0c0400u),
                   d = __builtin_amdgcn_perm(u[7], u[6], 0x04000c0cu);
    return make_uint2((a | b) & 0x0f0f0f0fu, (c | d) & 0x0f0f0f0fu);      // (NaN may bring any byte, and has a neighbour)
}
// Byte j of a row: channel j low, channel j + d/2 high.  Lane `sub` has channels 8 sub .. 8 sub + 7, the lane LPR / 2 further the ones that share their bytes: they exchange
// half of what they have and write 4 bytes each.
template <int LPR> __device__ __forceinline__ void store4bit(int8_t *row, uint2 mine, int sub) {
    const bool high = sub >= LPR / 2;
    const uint32_t theirs = __float_as_uint(lane_xor<LPR / 2>(__uint_as_float(high ? mine.x : mine.y)));
    const uint32_t w = high ? theirs | (mine.y << 4) : mine.x | (theirs << 4);
    *reinterpret_cast<uint32_t *>(row + 8 * (sub & (LPR / 2 - 1)) + (high ? 4 : 0)) = w;
}

// ---- append ------------------------------------------------------------------------------------------------------------
template <typename T, int LPR, int HELD, bool HADAMARD, int AT_ONCE>
__global__ __launch_bounds__(THREADS) void append_keys_kernel(AppendCall c) {
    constexpr int ROWS = THREADS / LPR, D = 8 * LPR;
    const int sub = threadIdx.x % LPR;
    const unsigned row0 = blockIdx.x * (ROWS * AT_ONCE) + threadIdx.x / LPR;
    Raw8<T> k[AT_ONCE], v[AT_ONCE];
    long slot[AT_ONCE];
    unsigned unit[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const unsigned r = row0 + i * ROWS;
        slot[i] = -1, unit[i] = 0;
        if (r < c.rows) {
            const unsigned u = c.by_tokens.of(r), n = r - u * c.Nn, b = c.by_heads.of(u), h = u - b * c.Hkv;
            const long p = static_cast<long>(keys_of(c.lens, b, c.Nk)) - c.Nn + n;
            unit[i] = u;
            if (p >= 0) {
                slot[i] = static_cast<long>(u) * c.Nk + p;
                k[i].load(c.K.X, b * c.K.b + h * c.K.h + n * c.K.n + 8 * sub);
                v[i].load(c.V.X, b * c.V.b + h * c.V.h + n * c.V.n + 8 * sub);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        if (slot[i] < 0) continue;                               // (the lanes of a row together)
        float x[8];
        k[i].widen(x);
        if (HADAMARD) hadamard_row<LPR>(x, sub);
        float a = group_max<LPR>(absmax8(x));
        if constexpr (HELD == IFA_CACHE_I4) {
            store4bit<LPR>(c.Kc + slot[i] * (D / 2), codes4(x, inverse4(a)), sub);
            if (sub == 0) c.sK[slot[i]] = scale4(a);
        } else {
            *reinterpret_cast<uint2 *>(c.Kc + slot[i] * D + 8 * sub) = quant8(x, a == 0.0f ? 0.0f : 127.0f / a);
            if (sub == 0) c.sK[slot[i]] = a == 0.0f ? 1.0f : a / 127.0f;
        }
        v[i].widen(x);
        if constexpr (HELD == IFA_CACHE_I4) {
            a = group_max<LPR>(absmax8(x));
            store4bit<LPR>(static_cast<int8_t *>(c.Vc) + slot[i] * (D / 2), codes4(x, inverse4(a)), sub);
            if (sub == 0) c.sV[slot[i]] = scale4(a);
        } else if constexpr (HELD == IFA_CACHE_I8) {
            const float s = c.sV[unit[i]];
            *reinterpret_cast<uint2 *>(static_cast<int8_t *>(c.Vc) + slot[i] * D + 8 * sub) = quant8(x, s == 0.0f ? 0.0f : 1.0f / s);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __floats2half2_rn(x[2 * e], x[2 * e + 1]));
            *reinterpret_cast<uint4 *>(static_cast<__half *>(c.Vc) + slot[i] * D + 8 * sub) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// ---- read ---------------------------------------------------------------------------------------------------------------
// Values in fp32 are 32 bytes of a lane's 8 channels, and a store of 16 of them would leave every other 16 bytes to the next: there lane `sub` has channels 4 sub .. and d/2 + 4 sub .. instead, so that a row's lanes
// store 128 or 256 bytes without a gap (4 x 8 heads x 8000 of 128 numbers from 4 bits 105 -> 44 us, 36 x 1777 of 64 from 8 bits, rotated, 12.5 -> 7.7).
template <typename T> constexpr bool HALVES = std::is_same_v<T, float>;
template <typename T, int LPR> __device__ __forceinline__ void store_row(void *to, long row, int sub, const float (&x)[8]) {
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    if constexpr (HALVES<T>) {
        u4 *const p = reinterpret_cast<u4 *>(static_cast<float *>(to) + row * (8 * LPR)) + sub;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            __builtin_nontemporal_store(u4{__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]), __float_as_uint(x[4 * h + 2]), __float_as_uint(x[4 * h + 3])}, p + h * LPR);
    } else {
        u4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (std::is_same_v<T, __half>) w[e] = __builtin_bit_cast(uint32_t, __floats2half2_rn(x[2 * e], x[2 * e + 1]));
            else w[e] = __builtin_bit_cast(uint32_t, bf2{static_cast<__bf16>(x[2 * e]), static_cast<__bf16>(x[2 * e + 1])});
        }
        __builtin_nontemporal_store(w, reinterpret_cast<u4 *>(static_cast<T *>(to) + row * (8 * LPR)) + sub);
    }
}
// hadamard_row for channels 4 sub .. and d/2 + 4 sub ..: the same sums in the same order
template <int LPR> __device__ __forceinline__ void hadamard_halves(float (&x)[8], int sub) {
    auto inside = [&](int h) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & h) == 0) {
                const float a = x[i], b = x[i + h];
                x[i] = a + b;
                x[i + h] = a - b;
            }
    };
    inside(1), inside(2);
    hadamard_lane_stage<1, LPR>(x, sub);
    hadamard_lane_stage<2, LPR>(x, sub);
    hadamard_lane_stage<4, LPR>(x, sub);
    hadamard_lane_stage<8, LPR>(x, sub);
    inside(4);
}
// (u - 8) s of four nibbles, one a byte
__device__ __forceinline__ void values4(uint32_t w, float s, float *x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (static_cast<float>(w >> (8 * e) & 0xffu) - 8.0f) * s;
}
__device__ __forceinline__ void values8(uint32_t w, float s, float *x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = static_cast<float>(static_cast<int8_t>(w >> (8 * e))) * s;
}

template <typename T, int LPR, int HELD, bool HADAMARD, int AT_ONCE>
__global__ __launch_bounds__(THREADS) void read_keys_kernel(ReadCall c) {
    constexpr int ROWS = THREADS / LPR, D = 8 * LPR;
    constexpr bool I4 = HELD == IFA_CACHE_I4, VF16 = HELD == IFA_CACHE_I8_F16, HALF = HALVES<T>;
    const int sub = threadIdx.x % LPR;
    const unsigned row0 = blockIdx.x * (ROWS * AT_ONCE) + threadIdx.x / LPR;
    uint2 k[AT_ONCE];
    std::conditional_t<VF16, Raw8<__half>, uint2> v[AT_ONCE];
    float sk[AT_ONCE], sv[AT_ONCE];
    bool there[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const unsigned r = row0 + i * ROWS;
        there[i] = false;
        if (r >= c.rows) continue;
        const unsigned u = c.by_count.of(r), n = r - u * c.count, b = c.by_heads.of(u);
        const long L = keys_of(c.lens, b, c.Nk), p = (c.first < 0 ? L - c.count : c.first) + n;
        there[i] = p >= 0 && p < L;
        if (!there[i]) continue;
        const long slot = static_cast<long>(u) * c.Nk + p;
        const int8_t *const V = static_cast<const int8_t *>(c.Vc);
        if constexpr (HALF) {                                    // bytes of the two halves; in 4 bits both are in the same four
            auto codes = [&](const int8_t *p) {
                const uint32_t *const row = reinterpret_cast<const uint32_t *>(p + slot * (I4 ? D / 2 : D)) + sub;
                if constexpr (I4) return make_uint2(row[0], row[0] >> 4);
                else return make_uint2(row[0], row[LPR]);
            };
            k[i] = codes(c.Kc);
            sk[i] = c.sK[slot];
            if constexpr (VF16) {
                const uint2 *const row = reinterpret_cast<const uint2 *>(V + slot * (2 * D)) + sub;
                const uint2 a = row[0], b = row[LPR];
                v[i].raw = make_uint4(a.x, a.y, b.x, b.y);
            } else v[i] = codes(V);
        } else {
            const long at = I4 ? slot * (D / 2) + 8 * (sub & (LPR / 2 - 1)) : slot * D + 8 * sub;
            k[i] = *reinterpret_cast<const uint2 *>(c.Kc + at);
            sk[i] = c.sK[slot];
            if constexpr (VF16) v[i].load(c.Vc, at);
            else v[i] = *reinterpret_cast<const uint2 *>(V + at);
        }
        if constexpr (!VF16) sv[i] = c.sV[I4 ? slot : u];
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const unsigned r = row0 + i * ROWS;
        if (r >= c.rows) continue;
        float x[8] = {}, y[8] = {};
        if (there[i]) {
            if constexpr (I4) {
                const int up = !HALF && sub >= LPR / 2 ? 4 : 0;        // which nibble of the bytes
                values4(k[i].x >> up & 0x0f0f0f0fu, sk[i], x), values4(k[i].y >> up & 0x0f0f0f0fu, sk[i], x + 4);
                values4(v[i].x >> up & 0x0f0f0f0fu, sv[i], y), values4(v[i].y >> up & 0x0f0f0f0fu, sv[i], y + 4);
            } else {
                values8(k[i].x, sk[i], x), values8(k[i].y, sk[i], x + 4);
                if constexpr (VF16) v[i].widen(y);
                else values8(v[i].x, sv[i], y), values8(v[i].y, sv[i], y + 4);
            }
        }
        if constexpr (HADAMARD) {                                // H H = d I, 1 / d is exact
            if constexpr (HALF) hadamard_halves<LPR>(x, sub);
            else hadamard_row<LPR>(x, sub);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= 1.0f / D;
        }
        store_row<T, LPR>(c.K, r, sub, x);
        store_row<T, LPR>(c.V, r, sub, y);
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
// Rows of a thread: one for the first 8192 workgroups' worth, then two, which saves divisions (us with one, two, four everywhere: 5331 x 12 rows of 64 fp32 numbers, rotated, into 8 bits and back 14.4, 15.4,
// 17.8; 32768 x 8 of 128 bf16 numbers into 4 bits and back 60.9, 60.9, 63.7; 16 x 8 x 16384 read from 4 bits 241, 236, 247).
constexpr int MANY = 2;
template <typename F> void by_rows(long rows, int lpr, F f) {
    const long per = THREADS / lpr, one = (rows + per - 1) / per;
    if (one <= 8192) f(std::integral_constant<int, 1>{}, static_cast<unsigned>(one));
    else f(std::integral_constant<int, MANY>{}, static_cast<unsigned>((one + MANY - 1) / MANY));
}
template <typename F> void by_type(int dtype, F f) {
    if (dtype == IFA_F32) f(float{});
    else if (dtype == IFA_F16) f(__half{});
    else f(__hip_bfloat16{});
}
template <typename F> void by_held(int held, F f) {
    if (held == IFA_CACHE_I8_F16) f(std::integral_constant<int, IFA_CACHE_I8_F16>{});
    else if (held == IFA_CACHE_I8) f(std::integral_constant<int, IFA_CACHE_I8>{});
    else f(std::integral_constant<int, IFA_CACHE_I4>{});
}
template <typename F> void by_flag(bool x, F f) {
    if (x) f(std::true_type{});
    else f(std::false_type{});
}

bool overlap(const void *a, long na, const void *b, long nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && x < y + static_cast<uintptr_t>(nb) && y < x + static_cast<uintptr_t>(na);
}
bool odd4(const void *p) { return reinterpret_cast<uintptr_t>(p) & 3; }

// What both calls ask of a cache
int refuse_cache(const void *Kc, const float *sK, const void *Vc, const float *sV, const int *lens, int B, int Hkv, int Nk, int d, int held) {
    if (!Kc || !sK || !Vc || (held != IFA_CACHE_I8_F16 && !sV)) return IFA_ERR_NULL;
    if (B <= 0 || Hkv <= 0 || Nk <= 0 || d <= 0 || static_cast<long>(B) * Hkv > (1L << 40) / Nk / d) return IFA_ERR_SHAPE;
    if (held < IFA_CACHE_I8_F16 || held > IFA_CACHE_I4) return IFA_ERR_DTYPE;
    if ((d != 64 && d != 128) || static_cast<long>(B) * Hkv > 0x7fffffffL) return IFA_ERR_UNSUPPORTED;
    if (!ifa_aligned16(Kc) || !ifa_aligned16(Vc) || odd4(sK) || odd4(sV) || odd4(lens)) return IFA_ERR_UNSUPPORTED;
    return IFA_OK;
}
struct Span { const void *p; long n; };
// The cache's arrays: K, s_K, V, s_V
void spans_of(Span (&s)[4], const void *Kc, const float *sK, const void *Vc, const float *sV, long units, int Nk, int d, int held) {
    const long keys = units * Nk;
    s[0] = {Kc, held == IFA_CACHE_I4 ? keys * d / 2 : keys * d};
    s[1] = {sK, keys * 4};
    s[2] = {Vc, held == IFA_CACHE_I4 ? keys * d / 2 : held == IFA_CACHE_I8 ? keys * d : keys * d * 2};
    s[3] = {held == IFA_CACHE_I8_F16 ? nullptr : sV, held == IFA_CACHE_I4 ? keys * 4 : units * 4};
}

}  // namespace

extern "C" int append_keys(const void *K, const void *V, int x_dtype, long K_stride_b, long K_stride_h, long K_stride_n, long V_stride_b, long V_stride_h, long V_stride_n,
                           const int *lens, int B, int Hkv, int Nn, int Nk, int d, int held, int hadamard, void *K_c, float *s_K, void *V_c, float *s_V, void *hip_stream) {
    if (!K || !V) return IFA_ERR_NULL;
    if (const int rc = refuse_cache(K_c, s_K, V_c, s_V, lens, B, Hkv, Nk, d, held)) return rc;
    if (Nn <= 0) return IFA_ERR_SHAPE;
    if (x_dtype < IFA_F32 || x_dtype > IFA_BF16) return IFA_ERR_DTYPE;
    const int sizes[3] = {B, Hkv, Nn};
    long strides[2][3] = {{K_stride_b, K_stride_h, K_stride_n}, {V_stride_b, V_stride_h, V_stride_n}};
    const long rows = static_cast<long>(B) * Hkv * Nn, bytes = x_dtype == IFA_F32 ? 4 : 2;
    if (rows > MOST_ROWS || !ifa_aligned16(K) || !ifa_aligned16(V)) return IFA_ERR_UNSUPPORTED;
    for (auto &t : strides)
        for (int i = 0; i < 3; ++i) {
            if (sizes[i] == 1) t[i] = 0;                         // (never used)
            if (t[i] < 0 || t[i] > (1L << 42) / sizes[i]) return IFA_ERR_SHAPE;
            if (t[i] * bytes % 16) return IFA_ERR_UNSUPPORTED;   // a row starts at a multiple of 16 bytes
        }
    // tokens are read while slots are written: neither the tokens nor lens overlap the cache, nor do its arrays each other
    Span c[4];
    spans_of(c, K_c, s_K, V_c, s_V, static_cast<long>(B) * Hkv, Nk, d, held);
    auto extent = [&](const long (&t)[3]) { return ((B - 1) * t[0] + (Hkv - 1) * t[1] + (Nn - 1) * t[2] + d) * bytes; };
    const Span read[3] = {{K, extent(strides[0])}, {V, extent(strides[1])}, {lens, 4L * B}};
    for (int i = 0; i < 4; ++i) {
        for (const Span &r : read)
            if ((i < 3 || held == IFA_CACHE_I4) && overlap(c[i].p, c[i].n, r.p, r.n)) return IFA_ERR_UNSUPPORTED;
        for (int j = 0; j < i; ++j)
            if (overlap(c[i].p, c[i].n, c[j].p, c[j].n)) return IFA_ERR_UNSUPPORTED;
    }
    const AppendCall call = {{K, strides[0][0], strides[0][1], strides[0][2]}, {V, strides[1][0], strides[1][1], strides[1][2]}, lens, static_cast<int8_t *>(K_c), V_c, s_K, s_V,
                             static_cast<unsigned>(rows), static_cast<unsigned>(Hkv), static_cast<unsigned>(Nn), Nk, Divisor(Nn), Divisor(Hkv)};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    by_type(x_dtype, [&](auto x) {
        by_held(held, [&](auto h) {
            by_flag(hadamard != 0, [&](auto rotated) {
                by_flag(d == 128, [&](auto wide) {
                    constexpr int LPR = decltype(wide)::value ? 16 : 8;
                    by_rows(rows, LPR, [&](auto at_once, unsigned blocks) {
                        hipLaunchKernelGGL((append_keys_kernel<decltype(x), LPR, decltype(h)::value, decltype(rotated)::value, decltype(at_once)::value>), dim3(blocks), dim3(THREADS), 0, st, call);
                    });
                });
            });
        });
    });
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}

extern "C" int read_keys(const void *K_c, const float *s_K, const void *V_c, const float *s_V, const int *lens, int B, int Hkv, int Nk, int d, int held, int hadamard,
                         long first, int count, void *K, void *V, int x_dtype, void *hip_stream) {
    if (!K || !V) return IFA_ERR_NULL;
    if (const int rc = refuse_cache(K_c, s_K, V_c, s_V, lens, B, Hkv, Nk, d, held)) return rc;
    const long units = static_cast<long>(B) * Hkv;
    if (count <= 0 || first < -1 || first > Nk || units > (1L << 40) / count / d) return IFA_ERR_SHAPE;
    if (x_dtype < IFA_F32 || x_dtype > IFA_BF16) return IFA_ERR_DTYPE;
    const long rows = units * count, out = rows * d * (x_dtype == IFA_F32 ? 4 : 2);
    if (rows > MOST_ROWS || !ifa_aligned16(K) || !ifa_aligned16(V)) return IFA_ERR_UNSUPPORTED;
    Span c[4];
    spans_of(c, K_c, s_K, V_c, s_V, units, Nk, d, held);
    for (const void *o : {K, V}) {
        for (const Span &r : c)
            if (overlap(o, out, r.p, r.n)) return IFA_ERR_UNSUPPORTED;
        if (overlap(o, out, lens, 4L * B)) return IFA_ERR_UNSUPPORTED;
    }
    if (overlap(K, out, V, out)) return IFA_ERR_UNSUPPORTED;
    const ReadCall call = {static_cast<const int8_t *>(K_c), V_c, s_K, s_V, lens, K, V, static_cast<unsigned>(rows), static_cast<unsigned>(Hkv), static_cast<unsigned>(count), Nk, first,
                           Divisor(count), Divisor(Hkv)};
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    by_type(x_dtype, [&](auto x) {
        by_held(held, [&](auto h) {
            by_flag(hadamard != 0, [&](auto rotated) {
                by_flag(d == 128, [&](auto wide) {
                    constexpr int LPR = decltype(wide)::value ? 16 : 8;
                    by_rows(rows, LPR, [&](auto at_once, unsigned blocks) {
                        hipLaunchKernelGGL((read_keys_kernel<decltype(x), LPR, decltype(h)::value, decltype(rotated)::value, decltype(at_once)::value>), dim3(blocks), dim3(THREADS), 0, st, call);
                    });
                });
            });
        });
    });
    return hipGetLastError() == hipSuccess ? IFA_OK : IFA_ERR_HIP;
}
