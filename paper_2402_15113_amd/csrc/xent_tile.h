// The ends of the logits' tiled product: what the cross entropy makes of a tile's sums in
// the registers that hold them, so that no logit is stored.
//
// A lane has columns 4 (lane / 16) .. + 3 of each block of 16, of row lane % 16: a row's
// sums go over its own values and then over the four lanes that share it.
#pragma once

#include "linear_tile.h"
#include "xent.h"

namespace tgm {

constexpr float kLog2e = 1.44269504088896340736f;
// exp(d) of a difference from a maximum: its rounding is 2^-24 of d, which is large only
// where the result is small.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

struct XentSums {
    using Args = XentArgs;
    template <class T, int NA, int MA>
    static __device__ __forceinline__ void finish(const Args &e, const LinearOut &o,
                                                  f4 (&acc)[NA][MA], int32_t n0, int32_t m0,
                                                  int32_t run, int32_t, int32_t M)
    {
        const int lane = threadIdx.x & 63, n1 = n0 + 4 * (lane >> 4);
        if (e.bias)
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int32_t n = min(n1 + 16 * a + j, o.N - 1);
                    const float bias = to_f32(((const T *)e.bias)[n]);
#pragma unroll
                    for (int b = 0; b < MA; ++b)
                        acc[a][b][j] += bias;
                }
        if (n0 + 16 * NA > o.N)   // columns that there are not
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (n1 + 16 * a + j >= o.N)
#pragma unroll
                        for (int b = 0; b < MA; ++b)
                            acc[a][b][j] = -INFINITY;
#pragma unroll
        for (int b = 0; b < MA; ++b) {
            const int32_t m = m0 + 16 * b + (lane & 15);
            float top = -INFINITY;
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    top = fmaxf(top, acc[a][b][j]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float ref = fabsf(top) == INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum += exp_of(acc[a][b][j] - ref);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (m < M) {
                if (lane < 16)
                    e.part[(int64_t)run * e.rows + m] = f2{top == -INFINITY ? top : ref, sum};
                // (a target may be any number)
                const int32_t at = (int32_t)((uint32_t)e.target[m] - (uint32_t)(e.n_first + n1));
                if (at >= 0 && at < 16 * NA && (at & 15) < 4) {
                    float z = 0.f;
#pragma unroll
                    for (int a = 0; a < NA; ++a)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            z = at == 16 * a + j ? acc[a][b][j] : z;
                    e.at_target[m] = z;
                }
            }
        }
    }
};

struct XentGrad {
    using Args = XentArgs;
    template <class T, int NA, int MA>
    static __device__ __forceinline__ void finish(const Args &e, const LinearOut &o,
                                                  f4 (&acc)[NA][MA], int32_t n0, int32_t m0,
                                                  int32_t, int32_t run, int32_t M)
    {
        const int lane = threadIdx.x & 63, n1 = n0 + 4 * (lane >> 4);
        const float scale = e.scale ? e.scale[0] : 1.f;
        float l[MA], dl[MA];
        int32_t at[MA];
#pragma unroll
        for (int b = 0; b < MA; ++b) {
            const int32_t m = min(m0 + 16 * b + (lane & 15), M - 1), t = e.target[m];
            l[b] = e.lse[m], dl[b] = e.dloss[m] * scale;
            at[b] = (int32_t)((uint32_t)t - (uint32_t)(e.n_first + n1));
            // rows that have no part in the loss
            if (t < 0 || t >= e.classes || l[b] == -INFINITY || m0 + 16 * b + (lane & 15) >= M)
                at[b] = INT32_MIN;
        }
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            const int32_t n = n1 + 16 * a;
            f4 bias{0.f, 0.f, 0.f, 0.f}, sum{0.f, 0.f, 0.f, 0.f};
            if (e.bias)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    bias[j] = to_f32(((const T *)e.bias)[min(n + j, o.N - 1)]);
#pragma unroll
            for (int b = 0; b < MA; ++b) {
                const int32_t m = m0 + 16 * b + (lane & 15);
                Pack<T, 4> out;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float d = exp_of(acc[a][b][j] + bias[j] - l[b]);
                    d = (at[b] == 16 * a + j ? d - 1.f : d) * dl[b];
                    d = at[b] == INT32_MIN ? 0.f : d;
                    sum[j] += d;
                    out.v[j] = from_f32<T>(d);
                }
                T *dz = (T *)e.dz + (int64_t)m * e.ld_dz + n;
                if (m < M) {
                    if (n + 4 <= o.N)
                        store_pack(dz, out);
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (n + j < o.N)
                                dz[j] = out.v[j];
                }
            }
            if (e.db)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s = row16_sum(sum[j]);
                    if ((lane & 15) == 0 && n + j < o.N)
                        e.db[(int64_t)run * o.N + n + j] = s;
                }
        }
    }
};

// Whether the large tiles take a product of logits.  Of many tiles it does not matter that the
// last round of them is not full, so that here a tenth more of rounds is taken for what a large
// tile saves: 8,192 rows x 65,537 x 2,048 bf16: TUNE.
template <class T> bool xent_large(int64_t M, int64_t N, int64_t K)
{
    const bool f32 = sizeof(T) == 4;
    const int64_t side = f32 ? 128 : 256, half = side / 2;
    const int64_t large = cdiv(M, side) * cdiv(N, side), small = cdiv(M, half) * cdiv(N, half);
    return large >= (f32 ? 512 : 192) && (f32 || K >= 1024) &&
           cdiv(large, 256) * 40 <= cdiv(small, 256) * 11;
}

// The sum of a tile comes in one part.
template <class T, class End, int BN, int BM, int NW, int MW, bool DIRECT>
tgm_status_t launch_xent(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    *r = XentRuns{(int32_t)cdiv(p.o.N, BN) * NW, BM, MW};
    return launch_tile<T, T, true, true, BN, BM, NW, MW, DIRECT, End>(p, 1, e);
}
template <class T, class End>
tgm_status_t xent_product(const LinearProduct &p, const XentArgs &e, XentRuns *r)
{
    const bool large = xent_large<T>(p.o.M, p.o.N, p.K);
    const bool lies = direct<T, true, true>(p);
    if constexpr (sizeof(T) == 4) {
        if (large)
            return lies ? launch_xent<T, End, 128, 128, 2, 2, true>(p, e, r)
                        : launch_xent<T, End, 128, 128, 2, 2, false>(p, e, r);
        return lies ? launch_xent<T, End, 64, 64, 1, 4, true>(p, e, r)
                    : launch_xent<T, End, 64, 64, 1, 4, false>(p, e, r);
    } else {
        if (!lies)
            return launch_xent<T, End, 128, 128, 2, 2, false>(p, e, r);
        return large ? launch_xent<T, End, 256, 256, 2, 4, true>(p, e, r)
                     : launch_xent<T, End, 128, 128, 2, 2, true>(p, e, r);
    }
}
// dx of 16-bit operands with fp32 results.
template <class T> tgm_status_t xent_dx(const LinearProduct &p)
{
    const LinearPlan l = linear_plan(p.o.M, p.o.N, p.K, TypeCode<T>::code);
    if (!direct<T, false, true>(p))
        return launch_tile<T, float, false, true, 128, 128, 2, 2, false>(p, l.parts);
    return l.large ? launch_tile<T, float, false, true, 256, 256, 2, 4, true>(p, l.parts)
                   : launch_tile<T, float, false, true, 128, 128, 2, 2, true>(p, l.parts);
}

}  // namespace tgm
