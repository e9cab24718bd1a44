// What the kernels of tgm_linear share: fragments and the matrix instructions,
// activations, the end of a product, and the description of one.
#pragma once

#include "seq.h"

namespace tgm {

typedef __bf16 b8v __attribute__((ext_vector_type(8)));
typedef _Float16 h8v __attribute__((ext_vector_type(8)));

// 16 bytes of an operand along the sum: VEC elements.
template <class T> struct Frag {
    static constexpr int VEC = 16 / sizeof(T);
    Pack<T, VEC> v;
};

// One 16 x 16 block of C over the 4 VEC k that a wavefront's fragments hold:
// lane l has those of row (P) or column (Q) l % 16, in group l / 16.  Which k a
// group's elements are is all one to the sum, as long as P and Q agree.
__device__ __forceinline__ f4 mfma(const Frag<float> &p, const Frag<float> &q, f4 c)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(p.v.v[j], q.v.v[j], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f4 mfma(const Frag<bf16> &p, const Frag<bf16> &q, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8v, p.v),
                                                   __builtin_bit_cast(b8v, q.v), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma(const Frag<f16> &p, const Frag<f16> &q, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8v, p.v),
                                                  __builtin_bit_cast(h8v, q.v), c, 0, 0, 0);
}
typedef long l2v __attribute__((ext_vector_type(2)));
// The 8-bit instructions add products in groups of 8 neighbouring ones of a
// lane: aligned to the group's largest, what lies below 2^-13 of it is cut, and
// the group's sum is added in fp32 (measured; the order and unit are the
// hardware's).  Below what a result of 16 bits keeps; a result of 32 bits has
// its operands widened to bf16 instead (mfma_wide), which is exact.
__device__ __forceinline__ f4 mfma(const Frag<e4m3> &p, const Frag<e4m3> &q, f4 c)
{
    const l2v a = __builtin_bit_cast(l2v, p.v), b = __builtin_bit_cast(l2v, q.v);
    c = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(a.x, b.x, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(a.y, b.y, c, 0, 0, 0);
}
// 8 e4m3 values as bf16: their 4 significant bits fit.
__device__ __forceinline__ b8v widen(int lo, int hi)
{
    typedef int i4v __attribute__((ext_vector_type(4)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(lo, false);
    const f2 b = __builtin_amdgcn_cvt_pk_f32_fp8(lo, true);
    const f2 c = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false);
    const f2 d = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    auto pack = [](f2 v) {   // the upper halves of two fp32 values
        return (int)__builtin_amdgcn_perm(__float_as_uint(v.y), __float_as_uint(v.x), 0x07060302);
    };
    return __builtin_bit_cast(b8v, i4v{pack(a), pack(b), pack(c), pack(d)});
}
__device__ __forceinline__ f4 mfma_wide(const Frag<e4m3> &p, const Frag<e4m3> &q, f4 c)
{
    typedef int i4v __attribute__((ext_vector_type(4)));
    const i4v a = __builtin_bit_cast(i4v, p.v), b = __builtin_bit_cast(i4v, q.v);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a.x, a.y), widen(b.x, b.y), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(a.z, a.w), widen(b.z, b.w), c, 0, 0, 0);
}

// ---------------------------------------------------------------- activations
__device__ __forceinline__ float act_of(float z, int act)
{
    switch (act) {
    case TGM_ACT_RELU: return z > 0.f || z != z ? z : 0.f;
    case TGM_ACT_SILU: return z / (1.f + __expf(-z));
    case TGM_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    default: return z;
    }
}
__device__ __forceinline__ float act_grad(float z, int act)
{
    switch (act) {
    case TGM_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case TGM_ACT_SILU: {
        const float p = 1.f / (1.f + __expf(-z));
        return p * (1.f + z * (1.f - p));
    }
    case TGM_ACT_GELU:
        return 0.5f * (1.f + erff(z * 0.70710678118654752f)) +
               z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    default: return 1.f;
    }
}

// ---------------------------------------------------------------- the end of a product
struct LinearOut {
    void *y, *z;
    const void *bias, *res;
    const float *sm, *sn;   // scales of the rows and columns of C
    int64_t ld_y, ld_z, ld_res;
    int32_t M, N, act;
    const int32_t *n_rows;  // bounds M where given
};

// Columns n .. n + 3 of row m from their sums.
template <class O> __device__ __forceinline__ void finish(const LinearOut &o, int64_t m, int32_t n, f4 c)
{
    float v[4] = {c.x, c.y, c.z, c.w};
    const int left = o.N - n;
    if (o.sm) {
        const float s = o.sm[m];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left)
                v[j] *= s * o.sn[n + j];
    }
    const O *bias = (const O *)o.bias + n, *res = (const O *)o.res + m * o.ld_res + n;
    O *z = (O *)o.z + m * o.ld_z + n, *y = (O *)o.y + m * o.ld_y + n;
    if (left >= 4) {
        Pack<O, 4> p;
        if (o.bias) {
            p = load_pack<O, 4>(bias);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] += to_f32(p.v[j]);
        }
        if (o.z) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                p.v[j] = from_f32<O>(v[j]);
            store_pack(z, p);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = act_of(v[j], o.act);
        if (o.res) {
            p = load_pack<O, 4>(res);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] += to_f32(p.v[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p.v[j] = from_f32<O>(v[j]);
        store_pack(y, p);
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < left) {
                float u = v[j] + (o.bias ? to_f32(bias[j]) : 0.f);
                if (o.z)
                    z[j] = from_f32<O>(u);
                u = act_of(u, o.act) + (o.res ? to_f32(res[j]) : 0.f);
                y[j] = from_f32<O>(u);
            }
    }
}

// C[m, n] = sum_k P(n, k) Q(m, k), C of o.M rows and o.N columns.
struct LinearProduct {
    const void *P, *Q;
    int64_t ld_p, ld_q;
    int32_t K;
    const int32_t *k_rows;   // bounds K where given
    LinearOut o;
    float *work;             // for the partial sums of linear_splits() parts
    hipStream_t s;
};

// Tiled products (csrc/linear_tile.h); which: 0 forward (P = W, Q = x, results of
// type code out), 1 dx, 2 dW.
tgm_status_t linear_tile_f32(const LinearProduct &p, int which, int out);
tgm_status_t linear_tile_bf16(const LinearProduct &p, int which, int out);
tgm_status_t linear_tile_f16(const LinearProduct &p, int which, int out);
tgm_status_t linear_tile_e4m3(const LinearProduct &p, int which, int out);

// Parts that the sum of a product of this size and type is split into.
int linear_splits(int64_t M, int64_t N, int64_t K, int code);

}  // namespace tgm
