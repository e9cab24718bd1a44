// Root-mean-square norm with the residual's addition, its 8-bit output and its
// gradient (tgm_norm, tgm_norm_backward).
//
// One pass: a row's elements stay in the registers of the G lanes that hold
// it (16 to 64 lanes, or a workgroup), 16 bytes a load, between the sum of
// squares and the result, so every input is read once and every output
// written once.  Bound by memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq.h"

using namespace tgm;

namespace {

// Lane `lane` of G holds vectors lane, lane + G, ... of VEC elements.  The last
// vector of a row whose width is no multiple of VEC is moved back to end at
// the row's end: its first `skip` elements are its neighbour's too, count in
// no sum, and come out the same from both.
struct Span {
    int at, skip;   // first element; elements that belong to the vector before
    bool on;
};
template <int VEC> __device__ __forceinline__ Span span_of(int vec, int D)
{
    const int e = vec * VEC, at = min(e, D - VEC);
    return Span{at, e - at, e < D};
}

// Sum (or maximum) over the G lanes of a row; G above 64: over the workgroup,
// by LDS.  `slot` gives two exchanges in a row separate words.
template <int G, bool MAX> __device__ __forceinline__ float row_all(float v, float *lds, int slot)
{
    v = MAX ? group_max<(G > 64 ? 64 : G)>(v) : group_sum<(G > 64 ? 64 : G)>(v);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        float *p = lds + slot * W;
        if ((threadIdx.x & 63) == 0)
            p[threadIdx.x >> 6] = v;
        __syncthreads();
        v = p[0];
#pragma unroll
        for (int w = 1; w < W; ++w)
            v = MAX ? fmaxf(v, p[w]) : v + p[w];
    }
    return v;
}

// 8,192 rows of 4,096 bf16, added to a residual and out in 8 bits (235 MB): 50.8 us, 4.6 TB/s.
template <class T, class O, int VEC, int G, int NV>
__global__ __launch_bounds__((G > 256 ? G : 256)) void k_norm(
    const T *x, const T *res, const T *__restrict__ w, const int32_t *__restrict__ n_rows,
    T *total, O *y, float *scale, int32_t rows, int32_t D, float eps, int64_t ld_x,
    int64_t ld_res, int64_t ld_total, int64_t ld_y)
{
    __shared__ float lds[G > 64 ? 4 * (G / 64) : 1];
    constexpr int GROUPS = G > 256 ? 1 : 256 / G;
    const int lane = threadIdx.x % G;
    const int64_t R = rows_in_use(rows, n_rows);
    int turn = 0;   // words of two rows in a row are apart: a wavefront may be a row ahead
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G; row < R;
         row += (int64_t)gridDim.x * GROUPS, turn ^= 1) {
        Pack<T, VEC> px[NV], pr[NV], pw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
                px[i] = load_pack<T, VEC>(x + row * ld_x + s.at);
                if (res)
                    pr[i] = load_pack<T, VEC>(res + row * ld_res + s.at);
                pw[i] = load_pack<T, VEC>(w + s.at);
            }
        }
        float t[NV][VEC], sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    t[i][j] = to_f32(px[i].v[j]);
                    if (res)
                        t[i][j] += to_f32(pr[i].v[j]);
                    sum += j >= s.skip ? t[i][j] * t[i][j] : 0.f;
                }
            }
        }
        sum = row_all<G, false>(sum, lds, 2 * turn);
        const float q = 1.f / sqrtf(sum / (float)D + eps);
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
                Pack<T, VEC> pt;
                Pack<O, VEC> py;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    pt.v[j] = from_f32<T>(t[i][j]);
                    t[i][j] = t[i][j] * q * to_f32(pw[i].v[j]);
                    if constexpr (sizeof(O) == 1)
                        top = fmaxf(top, fabsf(t[i][j]));
                    else
                        py.v[j] = from_f32<O>(t[i][j]);
                }
                if (total)
                    store_pack(total + row * ld_total + s.at, pt);
                if constexpr (sizeof(O) != 1)
                    store_pack(y + row * ld_y + s.at, py);
            }
        }
        if constexpr (sizeof(O) == 1) {
            top = row_all<G, true>(top, lds, 2 * turn + 1);
            const float sc = fmaxf(top / 448.f, 0x1p-126f);
            if (lane == 0)
                scale[row] = sc;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const Span s = span_of<VEC>(lane + G * i, D);
                if (s.on) {
                    Pack<O, VEC> py;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        // a quotient that rounds past 448 stays 448; NaN stays NaN
                        const float v = t[i][j] / sc;
                        py.v[j] = from_f32<O>(v > 448.f ? 448.f : v < -448.f ? -448.f : v);
                    }
                    store_pack(y + row * ld_y + s.at, py);
                }
            }
        }
    }
}

// The gradient.  A workgroup takes every gridDim.x-th set of rows, keeps its
// lanes' part of dw in registers over all of them and leaves one partial row
// of dw in `part`; k_norm_dw adds the partial rows in order.  Bound by memory: 8,192
// bf16 rows of 8,192 (403 MB), both: 87 us, 4.6 TB/s; 12,000 fp32 rows of 100 (14 MB): 5.4
// and 2.8 us, of which a launch that does nothing would take half.
template <class T, int VEC, int G, int NV>
__global__ __launch_bounds__((G > 256 ? G : 256)) void k_norm_bwd(
    const T *t_, const T *__restrict__ w, const T *dy, const T *dtotal,
    const int32_t *__restrict__ n_rows, T *dx, float *__restrict__ part, int32_t rows, int32_t D,
    float eps, int64_t ld_t, int64_t ld_dy, int64_t ld_dt, int64_t ld_dx)
{
    __shared__ float lds[G > 64 ? 4 * (G / 64) : 256 * NV * VEC];
    constexpr int GROUPS = G > 256 ? 1 : 256 / G;
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const int64_t R = rows_in_use(rows, n_rows);
    Pack<T, VEC> pw[NV];
    float dw[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Span s = span_of<VEC>(lane + G * i, D);
        if (s.on)
            pw[i] = load_pack<T, VEC>(w + s.at);
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            dw[i][j] = 0.f;
    }
    int turn = 0;   // as in k_norm
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < R;
         row += (int64_t)gridDim.x * GROUPS, turn ^= 1) {
        Pack<T, VEC> pt[NV], py[NV], pd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
                pt[i] = load_pack<T, VEC>(t_ + row * ld_t + s.at);
                py[i] = load_pack<T, VEC>(dy + row * ld_dy + s.at);
                if (dtotal)
                    pd[i] = load_pack<T, VEC>(dtotal + row * ld_dt + s.at);
            }
        }
        float tt = 0.f, wt = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float t = to_f32(pt[i].v[j]);
                    const float g = to_f32(py[i].v[j]) * to_f32(pw[i].v[j]);
                    tt += j >= s.skip ? t * t : 0.f;
                    wt += j >= s.skip ? g * t : 0.f;
                }
            }
        }
        tt = row_all<G, false>(tt, lds, 2 * turn);
        wt = row_all<G, false>(wt, lds, 2 * turn + 1);
        const float q = 1.f / sqrtf(tt / (float)D + eps);
        const float c = q * q * (wt / (float)D);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
            if (s.on) {
                Pack<T, VEC> po;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float t = to_f32(pt[i].v[j]), g = to_f32(py[i].v[j]);
                    float v = q * (g * to_f32(pw[i].v[j]) - t * c);
                    if (dtotal)
                        v += to_f32(pd[i].v[j]);
                    dw[i][j] += g * (t * q);
                    po.v[j] = from_f32<T>(v);
                }
                store_pack(dx + row * ld_dx + s.at, po);
            }
        }
    }
    if (!part)
        return;
    float *out = part + (int64_t)blockIdx.x * D;
    if constexpr (G > 64) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Span s = span_of<VEC>(lane + G * i, D);
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (s.on && j >= s.skip)
                    out[s.at + j] = dw[i][j];
        }
    } else {
        // the workgroup's rows' lanes: group 0 + group 1 + ...
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                lds[group * (G * NV * VEC) + (G * i + lane) * VEC + j] = dw[i][j];
        __syncthreads();
        for (int e = threadIdx.x; e < D; e += 256) {
            // element e by the vector that owns it
            const int vec = e / VEC, skip = span_of<VEC>(vec, D).skip;
            float a = 0.f;
            for (int g = 0; g < GROUPS; ++g)
                a += lds[g * (G * NV * VEC) + vec * VEC + (e - vec * VEC) + skip];
            out[e] = a;
        }
    }
}

// dw = the P partial rows added up: 32 columns a workgroup, 32 threads each.
template <class T>
__global__ __launch_bounds__(1024) void k_norm_dw(const float *__restrict__ part, int32_t P,
                                                  int32_t D, T *__restrict__ dw)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + c;
    float a = 0.f;
    if (col < D)
#pragma unroll 8
        for (int p = r; p < P; p += 32)
            a += part[(int64_t)p * D + col];
    lds[r][c] = a;
    __syncthreads();
    if (r == 0 && col < D) {
        for (int k = 1; k < 32; ++k)
            a += lds[k][c];
        dw[col] = from_f32<T>(a);
    }
}

constexpr int kNormMaxD = 32768;
constexpr int kNormParts = 512;   // partial rows of dw: two workgroups a CU

struct NormArgs {
    const tgm_norm_desc *d;
    int64_t ld_x, ld_res, ld_total, ld_y;
    const void *x, *res, *w, *dy;
    const int32_t *n_rows;
    void *total, *y;
    float *scale;
    float *part;
    int32_t parts;
    hipStream_t s;
};

template <class T, class O, int VEC, int G, int NV> tgm_status_t launch_norm(const NormArgs &a)
{
    constexpr int GROUPS = G > 256 ? 1 : 256 / G;
    const int64_t grid = std::min<int64_t>(cdiv(a.d->rows, GROUPS), 1 << 20);
    TGM_LAUNCH((k_norm<T, O, VEC, G, NV>), dim3((uint32_t)grid), dim3(GROUPS * G), 0, a.s,
               (const T *)a.x, (const T *)a.res, (const T *)a.w, a.n_rows, (T *)a.total, (O *)a.y,
               a.scale, a.d->rows, a.d->D, a.d->eps, a.ld_x, a.ld_res, a.ld_total, a.ld_y);
    return TGM_OK;
}
template <class T, class O, int VEC, int G, int NV> tgm_status_t launch_norm_bwd(const NormArgs &a)
{
    constexpr int GROUPS = G > 256 ? 1 : 256 / G;
    const int32_t grid = (int32_t)std::min<int64_t>(a.parts, cdiv(a.d->rows, GROUPS));
    if (grid > 0)
        TGM_LAUNCH((k_norm_bwd<T, VEC, G, NV>), dim3(grid), dim3(GROUPS * G), 0, a.s,
                   (const T *)a.x, (const T *)a.w, (const T *)a.dy, (const T *)a.res, a.n_rows,
                   (T *)a.total, a.part, a.d->rows, a.d->D, a.d->eps, a.ld_x, a.ld_y, a.ld_res,
                   a.ld_total);
    if (a.y)
        TGM_LAUNCH((k_norm_dw<T>), dim3((uint32_t)cdiv(a.d->D, 32)), dim3(1024), 0, a.s, a.part,
                   grid, a.d->D, (T *)a.y);
    return TGM_OK;
}

// Lanes and vectors a row: the fewest lanes of 16, 32, 64 that hold it in few
// vectors each, a workgroup of 256 or 1,024 past that: rows that share a wavefront or a
// workgroup keep its lanes busy.  us of 8,192 bf16 rows, few lanes against more: 512
// wide, 64 against 256: 5.0, 8.1; 1,024: 7.1, 9.8; 8,192, 256 against 1,024: 43, 44 (4,096: 23,
// 32).  2,048 wide one vector a lane of 256 takes 12.7 where four a lane of 64 take
// 14.0 (4 rows: 2.3, 3.4), but the gradient, which keeps its part of dw in registers
// over all its rows, 28.7 and 24.2.
template <class T, class O, bool BWD, int VEC, int G, int NV>
tgm_status_t go(const NormArgs &a)
{
    if constexpr (BWD)
        return launch_norm_bwd<T, O, VEC, G, NV>(a);
    else
        return launch_norm<T, O, VEC, G, NV>(a);
}
template <class T, class O, bool BWD> tgm_status_t pick(const NormArgs &a)
{
    constexpr int VEC = 16 / sizeof(T);
    const int D = a.d->D, n = (int)cdiv(D, VEC);
    if (D < VEC)
        return go<T, O, BWD, 1, 16, 1>(a);
    if (n <= 16)
        return go<T, O, BWD, VEC, 16, 1>(a);
    if (n <= 32)
        return go<T, O, BWD, VEC, 32, 1>(a);
    if (n <= 64)
        return go<T, O, BWD, VEC, 64, 1>(a);
    if (n <= 128)
        return go<T, O, BWD, VEC, 64, 2>(a);
    if (n <= 256) {
        if constexpr (BWD)
            return go<T, O, BWD, VEC, 64, 4>(a);
        else
            return go<T, O, BWD, VEC, 256, 1>(a);
    }
    if (n <= 512)
        return go<T, O, BWD, VEC, 256, 2>(a);
    if (n <= 1024)
        return go<T, O, BWD, VEC, 256, 4>(a);
    if (n <= 2048)
        return go<T, O, BWD, VEC, 1024, 2>(a);
    if (n <= 4096)
        return go<T, O, BWD, VEC, 1024, 4>(a);
    return go<T, O, BWD, VEC, 1024, 8>(a);
}

tgm_status_t norm_args(const tgm_norm_desc *d, NormArgs *a)
{
    if (!d || d->rows < 0 || d->D < 1 || d->D > kNormMaxD || !wide_type(d->dtype) ||
        !(d->eps >= 0.f))
        return TGM_EINVAL;
    a->d = d;
    a->ld_x = stride_of(d->ld_x, d->D);
    a->ld_res = stride_of(d->ld_res, d->D);
    a->ld_total = stride_of(d->ld_total, d->D);
    a->ld_y = stride_of(d->ld_y, d->D);
    if (a->ld_x < 0 || a->ld_res < 0 || a->ld_total < 0 || a->ld_y < 0)
        return TGM_EINVAL;
    return TGM_OK;
}

int32_t norm_parts(int32_t rows) { return std::min<int32_t>(rows, kNormParts); }

}  // namespace

extern "C" tgm_status_t tgm_norm(const tgm_norm_desc *d, const void *x, const void *res,
                                 const void *w, const int32_t *n_rows, void *total, void *y,
                                 float *scale, void *stream)
{
    NormArgs a{};
    TGM_TRY_STATUS(norm_args(d, &a));
    if (d->out_dtype != d->dtype && d->out_dtype != TGM_E4M3)
        return TGM_EINVAL;
    if (!w || (d->rows && (!x || !y)) || (d->out_dtype == TGM_E4M3 ? d->rows && !scale : !!scale))
        return TGM_EINVAL;
    if (d->rows == 0)
        return TGM_OK;
    a.x = x, a.res = res, a.w = w, a.n_rows = n_rows, a.total = total, a.y = y, a.scale = scale;
    a.s = as_stream(stream);
    const bool q = d->out_dtype == TGM_E4M3;
    switch (d->dtype) {
    case TGM_F32: return q ? pick<float, e4m3, false>(a) : pick<float, float, false>(a);
    case TGM_BF16: return q ? pick<bf16, e4m3, false>(a) : pick<bf16, bf16, false>(a);
    default: return q ? pick<f16, e4m3, false>(a) : pick<f16, f16, false>(a);
    }
}

extern "C" tgm_status_t tgm_norm_work_bytes(int32_t rows, int32_t D, size_t *bytes)
{
    if (rows < 0 || D < 1 || D > kNormMaxD || !bytes)
        return TGM_EINVAL;
    *bytes = (size_t)norm_parts(rows) * D * 4;
    return TGM_OK;
}

extern "C" tgm_status_t tgm_norm_backward(const tgm_norm_desc *d, const void *t, const void *w,
                                          const void *dy, const void *dtotal,
                                          const int32_t *n_rows, void *dx, void *dw, void *work,
                                          size_t work_bytes, void *stream)
{
    NormArgs a{};
    TGM_TRY_STATUS(norm_args(d, &a));
    if (!w || (d->rows && (!t || !dy || !dx)))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_norm_work_bytes(d->rows, d->D, &need));
    if (dw && need) {
        if (!work || ((uintptr_t)work & 15))
            return TGM_EINVAL;
        if (work_bytes < need)
            return TGM_ESIZE;
    }
    a.x = t, a.w = w, a.dy = dy, a.res = dtotal, a.n_rows = n_rows, a.total = dx, a.y = dw;
    a.part = dw ? (float *)work : nullptr;
    a.parts = norm_parts(d->rows);
    a.s = as_stream(stream);
    if (d->rows == 0 && !dw)
        return TGM_OK;
    switch (d->dtype) {
    case TGM_F32: return pick<float, float, true>(a);
    case TGM_BF16: return pick<bf16, bf16, true>(a);
    default: return pick<f16, f16, true>(a);
    }
}
