// Rotary positions (tgm_rotary, tgm_rotary_frequencies).
//
// A pair (x_a, x_b) of a head's columns is turned by the angle pos omega_j: all heads of a
// row share its angles.  A workgroup forms the cosines and sines of a few rows in LDS, a
// pair a thread, and then turns the rows' heads by vectors, so that every element is read
// and written once.  Bound by memory: 65,536 rows of 20 fp16 heads of 128, half of each turned
// by event times (671 MB): 130 us, 5.1 TB/s, a copy's rate; 4 rows of 40 bf16 heads take the
// call's own 7.7 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "seq.h"

using namespace tgm;

namespace {

constexpr int kRotaryPairs = 2048;   // of the rows of a workgroup, in LDS
constexpr int kRotaryThreads = 256;

struct RotaryArgs {
    const void *x;
    void *y;
    const void *pos;
    const double *omega;
    const int32_t *n_rows;
    int64_t ld_x, ld_y;
    int32_t rows, H, d, rot, pos_type;
    float amplitude, sign;
    int32_t row_block, head_block;   // rows and heads of a workgroup
    int32_t lanes;                   // threads to a head, a power of two
    int32_t tail;                    // columns of a unit of those that are not turned
};

// cos and sin of pos omega.  The angle is formed and taken modulo a quarter turn in fp64
// (a position of 10^9 keeps 2e-7 of a radian), the rest, within pi / 4, goes by the power
// series in fp32: the first term left out is below 1.8e-9 and 1.2e-10.
__device__ __forceinline__ f2 turn_of(double pos, double omega)
{
    const double t = pos * omega;
    const double q = rint(t * 0.63661977236758134308);
    const float f = (float)fma(t, 0.63661977236758134308, -q) * 1.57079632679489661923f;
    const float s2 = f * f;
    float s = fmaf(s2, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(s, s2, 8.3333333e-3f);
    s = fmaf(s, s2, -1.6666667e-1f);
    s = fmaf(s * s2, f, f);
    float c = fmaf(s2, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(c, s2, -1.3888889e-3f);
    c = fmaf(c, s2, 4.1666667e-2f);
    c = fmaf(c, s2, -0.5f);
    c = fmaf(c, s2, 1.f);
    // which quarter; an angle that is infinite or NaN has f NaN
    const int k = (int)(q - 4. * floor(q * 0.25));
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    return f2{k == 1 || k == 2 ? -a : a, k >= 2 ? -b : b};
}

__device__ __forceinline__ double position(const RotaryArgs &a, int64_t row)
{
    if (!a.pos)
        return (double)row;
    switch (a.pos_type) {
    case TGM_POS_I32: return (double)((const int32_t *)a.pos)[row];
    case TGM_POS_I64: return (double)((const int64_t *)a.pos)[row];
    default: return ((const double *)a.pos)[row];
    }
}

template <class T, int VEC, bool HALF>
__global__ __launch_bounds__(kRotaryThreads) void k_rotary(RotaryArgs a)
{
    __shared__ f2 turn[kRotaryPairs];
    const int32_t R = rows_in_use(a.rows, a.n_rows);
    const int32_t h0 = (int32_t)blockIdx.y * a.head_block, nh = min(a.head_block, a.H - h0);
    const int pairs = a.rot / 2;
    // units of a head: pairs of vectors (HALF) or vectors of pairs, then what is not turned
    const int turned = HALF ? pairs / VEC : a.rot / VEC;
    const int units = turned + (a.tail ? (a.d - a.rot) / a.tail : 0);
    const int lane = threadIdx.x & (a.lanes - 1), slots = kRotaryThreads / a.lanes;
    const int dr = slots / nh, dh = slots - dr * nh;
    for (int64_t r0 = (int64_t)blockIdx.x * a.row_block; r0 < R;
         r0 += (int64_t)gridDim.x * a.row_block) {
        const int nr = (int)min((int64_t)a.row_block, R - r0);
        for (int i = threadIdx.x; i < nr * pairs; i += kRotaryThreads) {
            const int r = i / pairs, j = i - r * pairs;
            const f2 t = turn_of(position(a, r0 + r), a.omega[j]);
            turn[i] = f2{t.x * a.amplitude, t.y * a.amplitude * a.sign};
        }
        __syncthreads();
        for (int u = lane; u < units; u += a.lanes) {
            // (row, head) pairs, a row's heads one after the other
            const int i = threadIdx.x / a.lanes;
            for (int r = i / nh, h = i - i / nh * nh; r < nr; h += dh, r += dr) {
                if (h >= nh) {
                    h -= nh;
                    if (++r >= nr)
                        break;
                }
                const T *x = (const T *)a.x + (r0 + r) * a.ld_x + (int64_t)(h0 + h) * a.d;
                T *y = (T *)a.y + (r0 + r) * a.ld_y + (int64_t)(h0 + h) * a.d;
                if (u >= turned) {
                    const int at = a.rot + (u - turned) * a.tail;
                    if (a.tail == 1)
                        y[at] = x[at];
                    else
                        store_pack(y + at, load_pack<T, VEC>(x + at));
                } else if constexpr (HALF) {
                    const f2 *t = turn + r * pairs + u * VEC;
                    Pack<T, VEC> p = load_pack<T, VEC>(x + u * VEC);
                    Pack<T, VEC> q = load_pack<T, VEC>(x + pairs + u * VEC);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float v = to_f32(p.v[j]), w = to_f32(q.v[j]);
                        p.v[j] = from_f32<T>(v * t[j].x - w * t[j].y);
                        q.v[j] = from_f32<T>(w * t[j].x + v * t[j].y);
                    }
                    store_pack(y + u * VEC, p);
                    store_pack(y + pairs + u * VEC, q);
                } else {
                    const f2 *t = turn + r * pairs + u * (VEC / 2);
                    Pack<T, VEC> p = load_pack<T, VEC>(x + u * VEC);
#pragma unroll
                    for (int j = 0; j < VEC; j += 2) {
                        const float v = to_f32(p.v[j]), w = to_f32(p.v[j + 1]);
                        p.v[j] = from_f32<T>(v * t[j / 2].x - w * t[j / 2].y);
                        p.v[j + 1] = from_f32<T>(w * t[j / 2].x + v * t[j / 2].y);
                    }
                    store_pack(y + u * VEC, p);
                }
            }
        }
        __syncthreads();   // the next rows' angles take the same place
    }
}

template <class T, int VEC, bool HALF> tgm_status_t launch_rotary(RotaryArgs a, hipStream_t s)
{
    const int pairs = a.rot / 2, rest = a.d - a.rot;
    a.tail = rest == 0 || a.x == a.y ? 0 : rest % VEC ? 1 : VEC;
    const int units = (HALF ? pairs : a.rot) / VEC + (a.tail ? rest / a.tail : 0);
    a.lanes = 1;
    while (a.lanes < units && a.lanes < kRotaryThreads)
        a.lanes *= 2;
    a.row_block = std::max(1, kRotaryThreads / pairs);   // a pair for every thread
    const int64_t blocks = cdiv(a.rows, a.row_block);
    a.head_block = a.H;
    if (blocks < 1024)
        a.head_block = std::min(a.H, std::max(1, kRotaryThreads / a.lanes / a.row_block));
    TGM_LAUNCH((k_rotary<T, VEC, HALF>),
               dim3((uint32_t)std::min<int64_t>(blocks, 1 << 20),
                    (uint32_t)cdiv(a.H, a.head_block)),
               dim3(kRotaryThreads), 0, s, a);
    return TGM_OK;
}

// The widest vectors, 16 bytes at most, that the turned columns of a head are whole numbers
// of: vectors that overlapped could not be turned in place.
template <class T, bool HALF> tgm_status_t pick_rotary(const RotaryArgs &a, hipStream_t s)
{
    constexpr int MOST = 16 / (int)sizeof(T);
    const int part = HALF ? a.rot / 2 : a.rot;
    if constexpr (MOST == 8)
        if (part % 8 == 0)
            return launch_rotary<T, 8, HALF>(a, s);
    if (part % 4 == 0)
        return launch_rotary<T, 4, HALF>(a, s);
    if (!HALF || part % 2 == 0)
        return launch_rotary<T, 2, HALF>(a, s);
    return launch_rotary<T, HALF ? 1 : 2, HALF>(a, s);
}

}  // namespace

extern "C" tgm_status_t tgm_rotary(const tgm_rotary_desc *d, const void *x, const double *omega,
                                   const void *pos, const int32_t *n_rows, void *y, void *stream)
{
    if (!d || d->rows < 0 || d->H < 1 || d->H > 4096 || d->d < 2 || d->d > 1024 || d->rot < 2 ||
        d->rot > d->d || d->rot % 2 || !wide_type(d->dtype) || d->pos_type < TGM_POS_I32 ||
        d->pos_type > TGM_POS_F64 || d->layout < TGM_ROTARY_HALF ||
        d->layout > TGM_ROTARY_INTERLEAVED)
        return TGM_EINVAL;
    RotaryArgs a{};
    a.ld_x = stride_of(d->ld_x, (int64_t)d->H * d->d);
    a.ld_y = stride_of(d->ld_y, (int64_t)d->H * d->d);
    if (a.ld_x < 0 || a.ld_y < 0 || !omega || (d->rows && (!x || !y)))
        return TGM_EINVAL;
    if (x == y && a.ld_x != a.ld_y)
        return TGM_EINVAL;
    if (d->rows == 0)
        return TGM_OK;
    a.x = x, a.y = y, a.pos = pos, a.omega = omega, a.n_rows = n_rows;
    a.rows = d->rows, a.H = d->H, a.d = d->d, a.rot = d->rot, a.pos_type = d->pos_type;
    a.amplitude = d->amplitude, a.sign = d->inverse ? -1.f : 1.f;
    const hipStream_t s = as_stream(stream);
    const bool half = d->layout == TGM_ROTARY_HALF;
    switch (d->dtype) {
    case TGM_F32: return half ? pick_rotary<float, true>(a, s) : pick_rotary<float, false>(a, s);
    case TGM_BF16: return half ? pick_rotary<bf16, true>(a, s) : pick_rotary<bf16, false>(a, s);
    default: return half ? pick_rotary<f16, true>(a, s) : pick_rotary<f16, false>(a, s);
    }
}

extern "C" tgm_status_t tgm_rotary_frequencies(int32_t rot, int32_t scaling, double base,
                                               double factor, double original, double often,
                                               double seldom, double *omega, float *amplitude)
{
    if (rot < 2 || rot > 1024 || rot % 2 || scaling < TGM_ROTARY_PLAIN ||
        scaling > TGM_ROTARY_PARTS || !omega || !amplitude || !(base > 0) || !std::isfinite(base))
        return TGM_EINVAL;
    if (scaling != TGM_ROTARY_PLAIN && !(factor >= 1 && std::isfinite(factor)))
        return TGM_EINVAL;
    if (scaling == TGM_ROTARY_PARTS &&
        !(original > 0 && std::isfinite(original) && seldom >= 0 && often > seldom &&
          std::isfinite(often)))
        return TGM_EINVAL;
    *amplitude = scaling == TGM_ROTARY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    for (int j = 0; j < rot / 2; ++j) {
        double w = std::pow(base, -2.0 * j / rot);
        if (scaling == TGM_ROTARY_BASE && j)   // (the new base may be past fp64's range)
            w *= std::pow(factor, -2.0 * j / (rot - 2.0));
        double keep = 1;
        if (scaling == TGM_ROTARY_LINEAR)
            keep = 0;
        else if (scaling == TGM_ROTARY_PARTS)
            keep = std::min(1.0, std::max(0.0, (original * w / 6.283185307179586477 - seldom) /
                                                   (often - seldom)));
        omega[j] = keep == 1 ? w : w * keep + w / factor * (1 - keep);
    }
    return TGM_OK;
}
