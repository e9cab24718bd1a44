// What the sequence operators (norm, product, scan) share: element types, wide
// loads at any alignment, checks of their arguments.
#pragma once

#include "common.h"

namespace tgm {

struct bf16 {
    uint16_t u;
};
struct f16 {
    _Float16 v;
};
struct e4m3 {
    uint8_t u;
};

// Type codes to types.
template <class T> struct TypeCode;
template <> struct TypeCode<float> { static constexpr int code = TGM_F32; };
template <> struct TypeCode<bf16> { static constexpr int code = TGM_BF16; };
template <> struct TypeCode<f16> { static constexpr int code = TGM_F16; };
template <> struct TypeCode<e4m3> { static constexpr int code = TGM_E4M3; };

inline int elem_bytes(int code) { return code == TGM_F32 ? 4 : code == TGM_E4M3 ? 1 : 2; }
inline bool wide_type(int code) { return code == TGM_F32 || code == TGM_BF16 || code == TGM_F16; }
// A row stride as given (0: dense) for rows of `width`; negative if it is refused.
inline int64_t stride_of(int64_t ld, int64_t width)
{
    return ld == 0 ? width : ld < width || ld >= (1 << 24) ? -1 : ld;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __uint_as_float((uint32_t)v.u << 16); }
__device__ __forceinline__ float to_f32(f16 v) { return (float)v.v; }

// Rounding to nearest, ties to even; NaN stays one.
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v)
{
    const __bf16 b = (__bf16)v;
    return bf16{__builtin_bit_cast(uint16_t, b)};
}
template <> __device__ __forceinline__ f16 from_f32<f16>(float v) { return f16{(_Float16)v}; }
// |v| <= 448 or NaN
template <> __device__ __forceinline__ e4m3 from_f32<e4m3>(float v)
{
    return e4m3{(uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xff)};
}

// N consecutive elements.  The global memory path takes wide accesses at any
// byte address, so no alignment beyond the element's own is asked for.
template <class T, int N> struct Pack {
    T v[N];
};
template <class T, int N> __device__ __forceinline__ Pack<T, N> load_pack(const T *p)
{
    Pack<T, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <class T, int N> __device__ __forceinline__ void store_pack(T *p, const Pack<T, N> &r)
{
    __builtin_memcpy(p, &r, sizeof(r));
}

__device__ __forceinline__ int32_t rows_in_use(int32_t rows, const int32_t *n_rows)
{
    return n_rows ? max(0, min(rows, *n_rows)) : rows;
}

// Sum and maximum over the G lanes (16, 32 or 64 consecutive ones) of a group;
// every lane of it ends with the same value.
template <int G> __device__ __forceinline__ float group_sum(float v)
{
    v = row16_sum(v);
    if (G >= 32)
        v += __shfl_xor(v, 16);
    if (G >= 64)
        v += __shfl_xor(v, 32);
    return v;
}
template <int G> __device__ __forceinline__ float group_max(float v)
{
    v = row16_max(v);
    if (G >= 32)
        v = fmaxf(v, __shfl_xor(v, 16));
    if (G >= 64)
        v = fmaxf(v, __shfl_xor(v, 32));
    return v;
}

}  // namespace tgm
