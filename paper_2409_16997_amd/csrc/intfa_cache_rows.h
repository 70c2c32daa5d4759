// Where the outputs of the attention calls on a cache go: rows, whole tiles of them, and the parts of a row joined.  Shared by the kernels for 8 and for 4 bits.
#ifndef INTFA_CACHE_ROWS_H
#define INTFA_CACHE_ROWS_H

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <hip/hip_bf16.h>
#include <stdint.h>

#include "intfa.h"
#include "intfa_device.h"
#include "intfa_cache.h"

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

#if defined(__HIP_DEVICE_COMPILE__)
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

}  // namespace

#endif  // INTFA_CACHE_ROWS_H
