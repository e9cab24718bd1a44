// The ends of the logits' tiled product: what the cross entropy makes of a tile's sums in
// the registers that hold them, so that no logit is stored.
//
// A lane has columns 4 (lane / 16) .. + 3 of each block of 16, of row lane % 16: a row's
// sums go over its own values and then over the four lanes that share it.
#pragma once

#include <type_traits>

#include "linear_tile.h"
#include "xent.h"

namespace tgm {

constexpr float kLog2e = 1.44269504088896340736f;
// exp(z - m).  For results of 32 bits by the difference, whose rounding is 2^-24 of it, large
// only where the result is small; for 16 bits in one step, with 2^-24 of m besides.
// (From 2^100 on differences are 0 or at least 2^76: whatever factor they get, the exponential is
// that of 0, or 0, or infinite, and log2(e) m could leave fp32, as that of bf16's lowest value does.)
template <bool FULL> struct ExpFrom {
    float m, f;   // m times -f unless FULL
    __device__ __forceinline__ explicit ExpFrom(float from)
        : m(from), f(FULL || fabsf(from) < 0x1p100f ? kLog2e : 0x1p-10f)
    {
        if (!FULL)
            m *= -f;
    }
    __device__ __forceinline__ float operator()(float z) const
    {
        return __builtin_amdgcn_exp2f(FULL ? (z - m) * f : fmaf(z, f, m));
    }
};

// The sums of the loss.  Bound by the matrix cores: 8,192 rows x 65,537 x 2,048 bf16 in 1.59 ms
// (1.39 PFLOP/s), 12,000 x 9,228 x 100 fp32 in 275 us.
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
            const ExpFrom<sizeof(T) == 4> exp_of(ref);
            float sum = 0.f;
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum += exp_of(acc[a][b][j]);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (m < M) {
                if (lane < 16)
                    e.part[(int64_t)run * e.rows + m] = f2{top, sum};
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

// dz.  Bound by the matrix cores and, where K is small, by its stores: 8,192 rows x 32,768 x 2,048
// bf16 in 931 us (1.18 PFLOP/s), 1,174 with stores of 8 bytes; 12,000 x 9,228 x 100 fp32 in 360 us
// (443 MB stored).
struct XentGrad {
    using Args = XentArgs;
    template <class T, int NA, int MA>
    static __device__ __forceinline__ void finish(const Args &e, const LinearOut &o,
                                                  f4 (&acc)[NA][MA], int32_t n0, int32_t m0,
                                                  int32_t, int32_t run, int32_t M)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, n1 = n0 + 4 * g;
        const float scale = e.scale ? e.scale[0] : 1.f;
        float l[MA], dl[MA];
        int32_t at[MA];
        bool here = false;   // a row's target is among the columns
#pragma unroll
        for (int b = 0; b < MA; ++b) {
            const int32_t m = min(m0 + 16 * b + (lane & 15), M - 1), t = e.target[m];
            l[b] = e.lse[m], dl[b] = e.dloss[m] * scale;
            at[b] = (int32_t)((uint32_t)t - (uint32_t)(e.n_first + n1));
            // rows that have no part in the loss
            if (t < 0 || t >= e.classes || l[b] == -INFINITY || m0 + 16 * b + (lane & 15) >= M)
                at[b] = INT32_MIN;
            here |= at[b] >= 0 && at[b] < 16 * NA;
        }
        if (e.bias)
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float bias = to_f32(((const T *)e.bias)[min(n1 + 16 * a + j, o.N - 1)]);
#pragma unroll
                    for (int b = 0; b < MA; ++b)
                        acc[a][b][j] += bias;
                }
        // softmax, less 1 at the target where one is here (few tiles have any)
#pragma unroll
        for (int b = 0; b < MA; ++b) {
            const ExpFrom<sizeof(T) == 4> exp_of(l[b]);
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[a][b][j] = exp_of(acc[a][b][j]);
        }
        if (__any(here))
#pragma unroll
            for (int b = 0; b < MA; ++b)
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[a][b][j] -= at[b] == 16 * a + j ? 1.f : 0.f;
#pragma unroll
        for (int b = 0; b < MA; ++b)
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[a][b][j] = at[b] == INT32_MIN ? 0.f : acc[a][b][j] * dl[b];
        if (e.db)
#pragma unroll
            for (int a = 0; a < NA; ++a)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float sum = 0.f;
#pragma unroll
                    for (int b = 0; b < MA; ++b)
                        sum += acc[a][b][j];
                    sum = row16_sum(sum);
                    if ((lane & 15) == 0 && n1 + 16 * a + j < o.N)
                        e.db[(int64_t)run * o.N + n1 + 16 * a + j] = sum;
                }
        T *dz = (T *)e.dz + (int64_t)(m0 + (lane & 15)) * e.ld_dz + n0;
        const bool whole = n0 + 16 * NA <= o.N;
#pragma unroll
        for (int b = 0; b < MA; ++b, dz += 16 * e.ld_dz) {
            if (m0 + 16 * b + (lane & 15) >= M)
                continue;
            if constexpr (sizeof(T) == 2 && NA % 2 == 0) {
                // A lane has 4 columns of a block and of the next one.  Of two neighbouring
                // groups of lanes the first takes 8 of the one and the second 8 of the other:
                // stores of 16 bytes, 64 a row.
                if (whole) {
#pragma unroll
                    for (int a = 0; a < NA; a += 2) {
                        uint32_t x[2], y[2];
                        Pack<T, 4> p, q;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            p.v[j] = from_f32<T>(acc[a][b][j]),
                            q.v[j] = from_f32<T>(acc[a + 1][b][j]);
                        __builtin_memcpy(x, &p, 8);
                        __builtin_memcpy(y, &q, 8);
                        uint32_t out[4];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const auto r = __builtin_amdgcn_permlane16_swap(x[k], y[k], false,
                                                                            false);
                            out[k] = r[0], out[2 + k] = r[1];
                        }
                        __builtin_memcpy(dz + 16 * (a + (g & 1)) + 8 * (g >> 1), out, 16);
                    }
                    continue;
                }
            }
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const int32_t n = n1 + 16 * a;
                Pack<T, 4> out;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    out.v[j] = from_f32<T>(acc[a][b][j]);
                if (n + 4 <= o.N)
                    store_pack(dz + 16 * a + 4 * g, out);
                else
#pragma unroll
                    for (int j = 0; j < 3; ++j)
                        if (n + j < o.N)
                            dz[16 * a + 4 * g + j] = out.v[j];
            }
        }
    }
};

// Whether the large tiles take a product of logits.  Of many tiles it does not matter that the
// last round of them is not full, so that here a tenth more of rounds is taken for what a large
// tile saves.  us with small and large tiles, forward alone and with its gradient:
//     bf16  8,192 x 65,537 x 2,048   2,031  1,573     7,884  6,931
//           4,096 x 32,768 x 256       108     92       440    423
//           4,096 x 32,768 x 64         79     61       304    278
//           512 x 32,768 x 1,024        44     36       193    178
//     fp32  8,192 x 16,384 x 2,048   4,083  3,848    16,156 15,689
//           4,096 x 32,768 x 256       571    538     2,240  2,202
//           12,000 x 9,228 x 128       271    265     1,053  1,095
//           4,096 x 32,768 x 64        197    191       773    819
// so fp32's gradient, whose end stores 64 KB a tile, takes them for sums of 256 or more.
template <class T, class End> bool xent_large(int64_t M, int64_t N, int64_t K)
{
    const bool f32 = sizeof(T) == 4;
    const int64_t side = f32 ? 128 : 256, half = side / 2;
    const int64_t large = cdiv(M, side) * cdiv(N, side), small = cdiv(M, half) * cdiv(N, half);
    return large >= (f32 ? 512 : 192) && cdiv(large, 256) * 40 <= cdiv(small, 256) * 11 &&
           (!f32 || K >= 256 || std::is_same_v<End, XentSums>);
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
    const bool large = xent_large<T, End>(p.o.M, p.o.N, p.K);
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
    const LinearPlan l = linear_plan(p, TypeCode<T>::code);
    if (!direct<T, false, true>(p))
        return launch_tile<T, float, false, true, 128, 128, 2, 2, false>(p, l.parts);
    return l.large ? launch_tile<T, float, false, true, 256, 256, 2, 4, true>(p, l.parts)
                   : launch_tile<T, float, false, true, 128, 128, 2, 2, true>(p, l.parts);
}
// dW, of another x where the device has found that it takes one.
template <class T, int BN, int BM, int NW, int MW, bool DIRECT>
tgm_status_t launch_dw(const LinearProduct &p, int parts, const LinearEither::Args &x)
{
    return launch_tile<T, T, false, false, BN, BM, NW, MW, DIRECT, LinearEither>(p, parts, x);
}
template <class T> tgm_status_t xent_dw(const LinearProduct &p, const LinearEither::Args &x)
{
    const LinearPlan l = linear_plan(p, TypeCode<T>::code);
    const bool lies = direct<T, false, false>(p);
    if constexpr (sizeof(T) == 4) {
        if (l.large)
            return lies ? launch_dw<T, 128, 128, 2, 2, true>(p, l.parts, x)
                        : launch_dw<T, 128, 128, 2, 2, false>(p, l.parts, x);
        return lies ? launch_dw<T, 64, 64, 1, 4, true>(p, l.parts, x)
                    : launch_dw<T, 64, 64, 1, 4, false>(p, l.parts, x);
    } else {
        if (!lies)
            return launch_dw<T, 128, 128, 2, 2, false>(p, l.parts, x);
        return l.large ? launch_dw<T, 256, 256, 2, 4, true>(p, l.parts, x)
                       : launch_dw<T, 128, 128, 2, 2, true>(p, l.parts, x);
    }
}

}  // namespace tgm
