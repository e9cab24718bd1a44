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
// FULL: for results of 32 bits, to a few units of the last place, of small values too; else
// for 16 bits, with the exponent's rounding (2^-24 times its size) besides.
//
// The normal distribution function Phi(z) = erfc(-z / sqrt 2) / 2 and e = exp(-z^2 / 2).
// For x >= 0, erfc(x) = exp(-x^2) t p(t) with t = 1 / (1 + c x); Phi of a negative z is half
// of that, so it does not cancel.  p is fitted to the scaled function exp(x^2) erfc(x) by
// least squares in relative error, reweighted towards the smallest maximum, over every x
// whose exp(-x^2) is not zero: FULL 9 coefficients, within 4.4e-8 (evaluated in fp32 8e-8
// rms and 3.5e-7 at most), else 8, within 1.3e-7 (5.1e-7).  About 22 instructions, with an
// exponential that the derivative needs as well (FULL 32).
struct Normal {
    float phi, e;
};
template <bool FULL> __device__ __forceinline__ Normal normal_of(float z)
{
    constexpr float k = -0.72134752f;   // -log2(e) / 2, and what is left of it
    constexpr float k_lo = -9.6298149e-09f;
    float p, e, t;
    if constexpr (FULL) {
        const float a = fabsf(z) > 16.f ? 16.f : fabsf(z);   // exp(-128) is zero
        t = __builtin_amdgcn_rcpf(fmaf(0.5f * 0.70710678118654752f, a, 1.f));
        p = fmaf(-0.05926307663321495f, t, 0.2855231761932373f);
        p = fmaf(p, t, -0.4891655147075653f);
        p = fmaf(p, t, 0.28031840920448303f);
        p = fmaf(p, t, -0.028178079053759575f);
        p = fmaf(p, t, 0.20334427058696747f);
        p = fmaf(p, t, 0.24293752014636993f);
        p = fmaf(p, t, 0.28239816427230835f);
        p = fmaf(p, t, 0.282085120677948f);
        // the exponent and what its roundings have left out
        const float s = a * a, v = s * k;
        const float rest = fmaf(fmaf(a, a, -s), k, fmaf(s, k_lo, fmaf(s, k, -v)));
        e = __builtin_amdgcn_exp2f(v);
        e = fmaf(e, rest * 0.69314718f, e);
    } else {
        t = __builtin_amdgcn_rcpf(fmaf(0.33f * 0.70710678118654752f, fabsf(z), 1.f));
        p = fmaf(-0.13381193578243256f, t, 0.4537965655326843f);
        p = fmaf(p, t, -0.33991068601608276f);
        p = fmaf(p, t, 0.3979606032371521f);
        p = fmaf(p, t, 0.052942752838134766f);
        p = fmaf(p, t, 0.1994291990995407f);
        p = fmaf(p, t, 0.18325647711753845f);
        p = fmaf(p, t, 0.18633709847927094f);
        e = __builtin_amdgcn_exp2f(k * z * z);
    }
    const float tail = 0.5f * p * t * e;
    return Normal{z > 0.f ? 1.f - tail : tail, e};
}
// sigmoid(z) and sigmoid(-z)
struct Sigmoid {
    float p, q;
};
template <bool FULL> __device__ __forceinline__ Sigmoid sigmoid_of(float z)
{
    if constexpr (FULL) {
        // neither loses its small values, and a step of Newton's for the reciprocal
        const float e = expf(-fabsf(z)), d = 1.f + e, r0 = __builtin_amdgcn_rcpf(d);
        const float r = fmaf(r0, fmaf(-d, r0, 1.f), r0), s = e * r;
        return z > 0.f ? Sigmoid{r, s} : Sigmoid{s, r};
    } else {
        const float p = __builtin_amdgcn_rcpf(1.f + __expf(-z));
        return Sigmoid{p, 1.f - p};
    }
}

template <bool FULL> __device__ __forceinline__ float act_of(float z, int act)
{
    switch (act) {
    case TGM_ACT_RELU: return z > 0.f || z != z ? z : 0.f;
    case TGM_ACT_SILU: return z * sigmoid_of<FULL>(z).p;
    case TGM_ACT_GELU: return z * normal_of<FULL>(z).phi;
    default: return z;
    }
}
template <bool FULL> __device__ __forceinline__ float act_grad(float z, int act)
{
    switch (act) {
    case TGM_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case TGM_ACT_SILU: {
        const Sigmoid s = sigmoid_of<FULL>(z);
        return s.p * fmaf(z, s.q, 1.f);
    }
    case TGM_ACT_GELU: {
        const Normal n = normal_of<FULL>(z);
        return fmaf(z * 0.39894228040143268f, n.e, n.phi);
    }
    default: return 1.f;
    }
}

// ---------------------------------------------------------------- the end of a product
struct LinearOut {
    void *y, *z;
    const void *bias, *res;
    const float *sm, *sn;   // scales of the rows (1 where null) and columns of C
    int64_t ld_y, ld_z, ld_res;
    int32_t M, N, act;
    const int32_t *n_rows;  // bounds M where given
};

// W neighbouring columns of C, from n on: what they share in every row, and their
// results in row m.  `left` of them exist (all of them if that is W or more).
template <class O, int W> struct Columns {
    float bias[W], scale[W];
    int left;

    __device__ __forceinline__ void load(const LinearOut &o, int32_t n)
    {
        left = o.N - n;
#pragma unroll
        for (int j = 0; j < W; ++j)
            bias[j] = 0.f, scale[j] = 1.f;
        if (left >= W) {
            if (o.bias) {
                const Pack<O, W> p = load_wide((const O *)o.bias + n);
#pragma unroll
                for (int j = 0; j < W; ++j)
                    bias[j] = to_f32(p.v[j]);
            }
            if (o.sn)
#pragma unroll
                for (int j = 0; j < W; j += 4) {
                    const Pack<float, 4> p = load_pack<float, 4>(o.sn + n + j);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        scale[j + i] = p.v[i];
                }
        } else {
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
                if (j < left) {
                    if (o.bias)
                        bias[j] = to_f32(((const O *)o.bias)[n + j]);
                    if (o.sn)
                        scale[j] = o.sn[n + j];
                }
        }
    }
    __device__ __forceinline__ Pack<O, W> residual(const LinearOut &o, int64_t m, int32_t n) const
    {
        const O *res = (const O *)o.res + m * o.ld_res + n;
        if (left >= W)
            return load_wide(res);
        Pack<O, W> p;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            if (j < left)
                p.v[j] = res[j];
        return p;
    }
    // v: the sums; sm: the row's scale
    __device__ __forceinline__ void finish(const LinearOut &o, int64_t m, int32_t n, float (&v)[W],
                                           float sm, const Pack<O, W> &res) const
    {
        Pack<O, W> p;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if (o.sn)   // one after the other: the scales' product may leave fp32
                v[j] = v[j] * sm * scale[j];
            v[j] += bias[j];
            p.v[j] = from_f32<O>(v[j]);
        }
        if (o.z)
            store((O *)o.z + m * o.ld_z + n, p);
        if (o.act != TGM_ACT_NONE)
#pragma unroll
            for (int j = 0; j < W; ++j)
                v[j] = act_of<sizeof(O) == 4>(v[j], o.act);
#pragma unroll
        for (int j = 0; j < W; ++j)
            p.v[j] = from_f32<O>(o.res ? v[j] + to_f32(res.v[j]) : v[j]);
        store((O *)o.y + m * o.ld_y + n, p);
    }

private:
    // 16 bytes a load and store at most
    static constexpr int PART = sizeof(O) * W <= 16 ? W : 16 / (int)sizeof(O);
    static __device__ __forceinline__ Pack<O, W> load_wide(const O *from)
    {
        Pack<O, W> p;
#pragma unroll
        for (int j = 0; j < W; j += PART) {
            const Pack<O, PART> q = load_pack<O, PART>(from + j);
#pragma unroll
            for (int i = 0; i < PART; ++i)
                p.v[j + i] = q.v[i];
        }
        return p;
    }
    __device__ __forceinline__ void store(O *to, const Pack<O, W> &p) const
    {
        if (left >= W) {
#pragma unroll
            for (int j = 0; j < W; j += PART) {
                Pack<O, PART> q;
#pragma unroll
                for (int i = 0; i < PART; ++i)
                    q.v[i] = p.v[j + i];
                store_pack(to + j, q);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
                if (j < left)
                    to[j] = p.v[j];
        }
    }
};

// Columns n .. n + 3 of row m from their sums.
template <class O>
__device__ __forceinline__ void finish(const LinearOut &o, int64_t m, int32_t n, f4 c)
{
    Columns<O, 4> q;
    q.load(o, n);
    Pack<O, 4> res;
    if (o.res)
        res = q.residual(o, m, n);
    float v[4] = {c.x, c.y, c.z, c.w};
    q.finish(o, m, n, v, o.sm ? o.sm[m] : 1.f, res);
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

// The tile of a product and the parts that its sum is split into, by its size and
// type.
struct LinearPlan {
    bool large;
    int parts;
};
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, int code);

}  // namespace tgm
