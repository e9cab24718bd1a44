// Matrix product with bias, activation and residual (tgm_linear) and its
// gradient.
//
// One engine for three products, C[m, n] = sum_k P(n, k) Q(m, k):
//   forward  P = W,   Q = x      sums over K, both contiguous along them
//   dx       P = W^T, Q = dz     sums over N, P contiguous along its rows
//   dW       P = x^T, Q = dz^T   sums over the rows, both contiguous along theirs
// P is the matrix instructions' first operand, so that a lane ends with four
// neighbouring columns of one row of C and bias, residual and result move as
// vectors.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "linear.h"

using namespace tgm;

namespace {

constexpr int kMaxDim = 1 << 20;

// ---------------------------------------------------------------- few rows
// 16 bytes of an operand's row from k on; zeros from K on.
template <class T> __device__ __forceinline__ Frag<T> load_frag(const T *row, int32_t k, int32_t K)
{
    constexpr int VEC = Frag<T>::VEC;
    Frag<T> f;
    if (k + VEC <= K) {
        f.v = load_pack<T, VEC>(row + k);
        return f;
    }
    __builtin_memset(&f, 0, sizeof(f));
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (k + j < K)
            f.v.v[j] = row[k + j];
    return f;
}

// Few rows, or a small product: bound by reading W once, or by what a launch takes.  A
// workgroup takes 16 columns and 16 MB rows of C; its wavefronts share the sum, each a
// run of it, and add up through LDS, so that a short sum needs no second launch.
// Operands come straight from memory into the matrix instructions, eight loads of
// a row of W at a time.  fp16, 4 rows, 4,096 x 2,048 (W of 16.8 MB): 6.8 us, 2.5
// TB/s; fp32, 16 rows, 8,192 x 2,048: 18.3 us, 3.7 TB/s.
template <class T, class O, int MB, int W>
__global__ __launch_bounds__(64 * W) void k_linear_few(const T *__restrict__ P,
                                                       const T *__restrict__ Q, int64_t ld_p,
                                                       int64_t ld_q, int32_t K, LinearOut o,
                                                       int32_t tn)
{
    constexpr int VEC = Frag<T>::VEC, STEP = 4 * VEC, AHEAD = MB == 1 ? 8 : 4;
    __shared__ f4 lds[W][MB][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int32_t M = rows_in_use(o.M, o.n_rows);
    const int32_t n0 = (int32_t)(blockIdx.x % tn) * 16, m0 = (int32_t)(blockIdx.x / tn) * (16 * MB);
    if (m0 >= M)
        return;
    const T *p = P + (int64_t)min(n0 + r, o.N - 1) * ld_p;
    const T *x[MB];
    f4 acc[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
        x[b] = Q + (int64_t)min(m0 + 16 * b + r, M - 1) * ld_q;
        acc[b] = f4{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t steps = (K + STEP - 1) / STEP, per = (steps + W - 1) / W;
    const int32_t s1 = min(steps, (w + 1) * per);
    auto multiply = [&](const Frag<T> &f, const Frag<T> &g, int b) __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 1 && sizeof(O) == 4)
            acc[b] = mfma_wide(f, g, acc[b]);
        else
            acc[b] = mfma(f, g, acc[b]);
    };
    int32_t s = w * per;
    for (; s + AHEAD <= s1 && (s + AHEAD) * STEP <= K; s += AHEAD) {
        Frag<T> f[AHEAD], g[AHEAD][MB];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int32_t k = (s + u) * STEP + q * VEC;
            f[u].v = load_pack<T, VEC>(p + k);
#pragma unroll
            for (int b = 0; b < MB; ++b)
                g[u][b].v = load_pack<T, VEC>(x[b] + k);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int b = 0; b < MB; ++b)
                multiply(f[u], g[u][b], b);
    }
    for (; s < s1; ++s) {
        const int32_t k = s * STEP + q * VEC;
        const Frag<T> f = load_frag<T>(p, k, K);
#pragma unroll
        for (int b = 0; b < MB; ++b)
            multiply(f, load_frag<T>(x[b], k, K), b);
    }
#pragma unroll
    for (int b = 0; b < MB; ++b)
        lds[w][b][lane] = acc[b];
    __syncthreads();
    for (int b = w; b < MB; b += W) {
        f4 c = lds[0][b][lane];
#pragma unroll
        for (int u = 1; u < W; ++u)
            c += lds[u][b][lane];
        const int32_t m = m0 + 16 * b + r;
        if (m < M && n0 + 4 * q < o.N)
            finish<O>(o, m, n0 + 4 * q, c);
    }
}

// ---------------------------------------------------------------- dz and db
// The largest finite |dy| of each workgroup's rows, a wavefront a row.  Bound by memory: 8,192
// x 4,096 fp16 (67 MB): 19 us, 3.6 TB/s, of a gradient of 320.
constexpr int kTops = 512;
template <class T, int VEC>
__global__ __launch_bounds__(1024) void k_linear_top(const T *__restrict__ dy,
                                                     const int32_t *n_rows,
                                                     float *__restrict__ tops, int32_t rows,
                                                     int32_t N, int64_t ld_y)
{
    constexpr int W = 16;
    __shared__ float lds[W];
    const int32_t R = rows_in_use(rows, n_rows);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    float top = 0.f;
    for (int64_t m = (int64_t)blockIdx.x * W + w; m < R; m += W * kTops)
#pragma unroll 4
        for (int32_t e = lane * VEC; e < N; e += 64 * VEC) {
            const Pack<T, VEC> p = load_pack<T, VEC>(dy + m * ld_y + min(e, N - VEC));
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = fabsf(to_f32(p.v[j]));
                top = v < INFINITY && v > top ? v : top;
            }
        }
    top = group_max<64>(top);
    if (lane == 0)
        lds[w] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < W; ++k)
            top = fmaxf(top, lds[k]);
        tops[blockIdx.x] = top;
    }
}
// The power of two that dz is held times: |act'| <= 1.13 keeps it within 65,504.
__device__ __forceinline__ float dz_scale(const float *__restrict__ tops, float *lds)
{
    const int t = threadIdx.x;
    const float top = group_max<64>(fmaxf(tops[t], tops[t + 256]));
    static_assert(kTops == 512, "");
    if ((t & 63) == 0)
        lds[t >> 6] = top;
    __syncthreads();
    const float most = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
    __syncthreads();   // lds has other uses
    return most > 0.f ? ldexpf(1.f, ilogbf(65504.f / 1.13f / most)) : 1.f;
}

// dz = dy act'(z) (stored where `dz` is given) and, with `part`, partial column sums of it;
// SCALED: dz is stored times a power of two, whose reciprocal goes to `unscale` as the
// scale of the products' K columns.  A wavefront takes 64 vectors of VEC columns and every
// 4 gridDim.y-th row.  A last vector of fewer columns moves back to end at the edge; its
// first columns are counted by the one before.  Bound by memory: 8,192 x 4,096
// bf16, GELU (201 MB): 49 us, 4.1 TB/s.
template <class T, int VEC, bool SCALED>
__global__ __launch_bounds__(256) void k_linear_dz(const T *__restrict__ dy,
                                                   const T *__restrict__ z,
                                                   const int32_t *n_rows, T *__restrict__ dz,
                                                   float *__restrict__ part, int32_t rows,
                                                   int32_t N, int64_t ld_y, int64_t ld_z, int act,
                                                   const float *__restrict__ tops,
                                                   float *__restrict__ unscale, int32_t K)
{
    constexpr int AHEAD = 4;
    __shared__ float lds[4][64 * VEC];
    float scale = 1.f;
    if (SCALED) {
        scale = dz_scale(tops, &lds[0][0]);
        const int32_t at = (int32_t)(blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
        for (int32_t k = at; k < K; k += (int32_t)(gridDim.x * gridDim.y) * 256)
            unscale[k] = 1.f / scale;
    }
    const int32_t R = rows_in_use(rows, n_rows);
    const int c = threadIdx.x & 63, r = threadIdx.x >> 6;
    const int32_t e = (int32_t)(blockIdx.x * 64 + c) * VEC, n = min(e, N - VEC);
    float sum[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        sum[j] = 0.f;
    const int64_t by = (int64_t)gridDim.y * 4;
    if (e < N)
        for (int64_t m0 = (int64_t)blockIdx.y * 4 + r; m0 < R; m0 += AHEAD * by) {
            Pack<T, VEC> py[AHEAD], pz[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t m = min(m0 + u * by, (int64_t)R - 1);
                py[u] = load_pack<T, VEC>(dy + m * ld_y + n);
                if (act != TGM_ACT_NONE)
                    pz[u] = load_pack<T, VEC>(z + m * ld_z + n);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (m0 + u * by < R) {
                    Pack<T, VEC> po;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        float v = to_f32(py[u].v[j]);
                        if (act != TGM_ACT_NONE)
                            v *= act_grad<sizeof(T) == 4>(to_f32(pz[u].v[j]), act);
                        po.v[j] = from_f32<T>(SCALED ? v * scale : v);
                        sum[j] += v;
                    }
                    if (dz)
                        store_pack(dz + (m0 + u * by) * N + n, po);
                }
        }
    if (!part)
        return;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        lds[r][c * VEC + j] = sum[j];
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * VEC; i += 256) {
        const int32_t e0 = (int32_t)(blockIdx.x * 64 + i / VEC) * VEC;
        const int32_t at = min(e0, N - VEC) + i % VEC;
        if (e0 < N && i % VEC >= e0 - min(e0, N - VEC))
            part[(int64_t)blockIdx.y * N + at] = lds[0][i] + lds[1][i] + lds[2][i] + lds[3][i];
    }
}

// db = the P partial sums added up in order: 32 columns a workgroup, 32 threads each (128
// partial rows of 4,096: 5.5 us, most of it the launch).
template <class T>
__global__ __launch_bounds__(1024) void k_linear_db(const float *__restrict__ part, int32_t P,
                                                    int32_t N, T *__restrict__ db)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int32_t n = blockIdx.x * 32 + c;
    float a = 0.f;
    if (n < N)
#pragma unroll 8
        for (int p = r; p < P; p += 32)
            a += part[(int64_t)p * N + n];
    lds[r][c] = a;
    __syncthreads();
    if (r == 0 && n < N) {
        for (int k = 1; k < 32; ++k)
            a += lds[k][c];
        db[n] = from_f32<T>(a);
    }
}

// ---------------------------------------------------------------- host
template <class T, class O, int MB> tgm_status_t few(const LinearProduct &p)
{
    constexpr int W = 8;
    const int64_t tn = cdiv(p.o.N, 16), wg = tn * cdiv(p.o.M, 16 * MB);
    TGM_LAUNCH((k_linear_few<T, O, MB, W>), dim3((uint32_t)wg), dim3(64 * W), 0, p.s,
               (const T *)p.P, (const T *)p.Q, p.ld_p, p.ld_q, p.K, p.o, (int32_t)tn);
    return TGM_OK;
}

// Blocks of 16 rows a workgroup of k_linear_few has for a forward product, 0 where the
// tiles take it.  Its time grows with the length of a sum (each wavefront has an eighth)
// and with the workgroups past one a CU; the tiles' is 9 to 10 us until they fill
// the chip.  One block against four against tiles, us, fp16 (rows x columns x sum): 40 x 1,024 x
// 512: 3.4, 4.6, 8.1; 512 x 512 x 1,024: 10.0, 7.4, 10.3; 128 x 1,024 x 2,048: 9.4, 11.5, 10.8;
// 64 x 4,096 x 2,048: 17.2, 12.6, 11.1; 1,000 x 1,024 x 512: 18.2, 12.7, 9.8; 16 x 1,024 x
// 8,192: 16.1, 22.9, 12.1.  Up to 16 rows the tiles multiply four times as many, which shows in fp32:
// 16 x 8,192 x 8,192: 67, 102, 78 (fp16: 31, 45, 26; 8 bit: 17.6, 24.0, 17.1).
int few_blocks(int64_t M, int64_t N, int64_t K, int code)
{
    const int64_t bytes = K * elem_bytes(code);
    const int64_t one = cdiv(N, 16) * cdiv(M, 16), four = cdiv(N, 16) * cdiv(M, 64);
    if (M <= 16)
        return bytes <= 8192 || (code == TGM_F32 && one >= 256) ? 1 : 0;
    if (one <= 768)
        return bytes * std::max<int64_t>(one, 256) <= 8192 * 256 ? 1 : 0;
    return four <= 512 && bytes * std::max<int64_t>(four, 256) < 4096 * 256 ? 4 : 0;
}

template <class T, class O, bool PK, bool QK> tgm_status_t product(const LinearProduct &p)
{
    if constexpr (PK && QK) {
        const int blocks = few_blocks(p.o.M, p.o.N, p.K, TypeCode<T>::code);
        if (blocks)
            return blocks == 1 ? few<T, O, 1>(p) : few<T, O, 4>(p);
    }
    constexpr int which = PK ? 0 : QK ? 1 : 2, out = TypeCode<O>::code;
    if constexpr (sizeof(T) == 4)
        return linear_tile_f32(p, which, out);
    else if constexpr (sizeof(T) == 1)
        return linear_tile_e4m3(p, which, out);
    else if constexpr (TypeCode<T>::code == TGM_BF16)
        return linear_tile_bf16(p, which, out);
    else
        return linear_tile_f16(p, which, out);
}

// Bytes that the parts of a product need.
size_t split_bytes(int64_t M, int64_t N, int64_t K, int code)
{
    if (M <= 0 || K <= 0)
        return 0;
    const int parts = linear_plan(M, N, K, code).parts;
    return parts == 1 ? 0 : (size_t)parts * M * ((N + 3) / 4 * 4) * 4;
}

constexpr int kDbParts = 128;

// The work space of the gradient: dz, the partial sums of db, dz's scale, then the partial
// sums of a product.
size_t db_bytes(int32_t rows, int32_t N)
{
    return ((size_t)std::min<int64_t>(cdiv(rows, 4), kDbParts) * N * 4 + 15) / 16 * 16;
}
size_t dz_bytes(int32_t rows, int32_t N, int32_t dtype, int32_t act)
{
    return act == TGM_ACT_NONE ? 0 : ((size_t)rows * N * elem_bytes(dtype) + 15) / 16 * 16;
}
// fp16's range is narrower than that of dy times a derivative
bool scales_dz(int32_t dtype, int32_t act)
{
    return dtype == TGM_F16 && (act == TGM_ACT_SILU || act == TGM_ACT_GELU);
}
size_t scale_bytes(int32_t rows, int32_t K, int32_t dtype, int32_t act)
{
    return rows && scales_dz(dtype, act) ? (kTops + (size_t)round_up(K, 4)) * sizeof(float) : 0;
}

template <class T>
tgm_status_t backward(const tgm_linear_desc *d, const int64_t *ld, const void *x, const void *W,
                      const void *z, const void *dy, const int32_t *n_rows, void *dx, void *dW,
                      void *db, char *work, hipStream_t s)
{
    const size_t zb = dz_bytes(d->rows, d->N, d->dtype, d->act);
    T *dz = zb && (dx || dW) ? (T *)work : nullptr;
    float *part = (float *)(work + zb);
    const size_t sb = scale_bytes(d->rows, d->K, d->dtype, d->act);
    float *tops = dz && sb ? (float *)(work + zb + db_bytes(d->rows, d->N)) : nullptr;
    float *unscale = tops ? tops + kTops : nullptr;
    float *split = (float *)(work + zb + db_bytes(d->rows, d->N) + sb);
    const int32_t parts = (int32_t)std::min<int64_t>(cdiv(d->rows, 4), kDbParts);
    if ((dz || db) && parts) {
        auto go = [&](auto vec) -> tgm_status_t {
            constexpr int VEC = decltype(vec)::value;
            const dim3 grid((uint32_t)cdiv(d->N, 64 * VEC), parts);
            if constexpr (TypeCode<T>::code == TGM_F16)
                if (tops) {
                    TGM_LAUNCH((k_linear_top<T, VEC>), dim3(kTops), dim3(1024), 0, s,
                               (const T *)dy, n_rows, tops, d->rows, d->N, ld[4]);
                    TGM_LAUNCH((k_linear_dz<T, VEC, true>), grid, dim3(256), 0, s, (const T *)dy,
                               (const T *)z, n_rows, dz, db ? part : nullptr, d->rows, d->N,
                               ld[4], ld[3], d->act, tops, unscale, d->K);
                    return TGM_OK;
                }
            TGM_LAUNCH((k_linear_dz<T, VEC, false>), grid, dim3(256), 0, s, (const T *)dy,
                       (const T *)z, n_rows, dz, db ? part : nullptr, d->rows, d->N, ld[4], ld[3],
                       d->act, tops, unscale, d->K);
            return TGM_OK;
        };
        constexpr int VEC = 16 / (int)sizeof(T);
        TGM_TRY_STATUS(d->N < VEC ? go(std::integral_constant<int, 1>{})
                                  : go(std::integral_constant<int, VEC>{}));
    }
    if (db)
        TGM_LAUNCH((k_linear_db<T>), dim3((uint32_t)cdiv(d->N, 32)), dim3(1024), 0, s, part, parts,
                   d->N, (T *)db);
    const void *g = zb ? (const void *)dz : dy;
    const int64_t ld_g = zb ? d->N : ld[4];
    if (dx && d->rows) {
        LinearProduct p{W, g, ld[1], ld_g, d->N, nullptr, {}, split, s};
        p.o.y = dx, p.o.ld_y = ld[5], p.o.M = d->rows, p.o.N = d->K, p.o.n_rows = n_rows;
        p.o.sn = unscale;
        TGM_TRY_STATUS((product<T, T, false, true>(p)));
    }
    if (dW) {
        LinearProduct p{x, g, ld[0], ld_g, d->rows, n_rows, {}, split, s};
        p.o.y = dW, p.o.ld_y = ld[6], p.o.M = d->N, p.o.N = d->K, p.o.sn = unscale;
        TGM_TRY_STATUS((product<T, T, false, false>(p)));
    }
    return TGM_OK;
}

// ld: x, w, res, z, y, dx, dw
tgm_status_t linear_args(const tgm_linear_desc *d, int64_t *ld)
{
    if (!d || d->rows < 0 || d->N < 1 || d->N > kMaxDim || d->K < 1 || d->K > kMaxDim ||
        d->act < TGM_ACT_NONE || d->act > TGM_ACT_GELU)
        return TGM_EINVAL;
    // a launch has fewer than 2^32 threads, 256 a tile
    const int64_t side = d->dtype == TGM_F32 ? 64 : 128, most = (int64_t)1 << 24;
    const int64_t r = cdiv(d->rows, side), n = cdiv(d->N, side), k = cdiv(d->K, side);
    if (r * n >= most || r * k >= most || n * k >= most)
        return TGM_EINVAL;
    const int64_t given[7] = {d->ld_x, d->ld_w, d->ld_res, d->ld_z, d->ld_y, d->ld_dx, d->ld_dw};
    const int32_t width[7] = {d->K, d->K, d->N, d->N, d->N, d->K, d->K};
    for (int k = 0; k < 7; ++k)
        if ((ld[k] = stride_of(given[k], width[k])) < 0)
            return TGM_EINVAL;
    return TGM_OK;
}

tgm_status_t check_work(size_t need, const void *work, size_t bytes)
{
    if (!need)
        return TGM_OK;
    if (!work || ((uintptr_t)work & 15))
        return TGM_EINVAL;
    return bytes < need ? TGM_ESIZE : TGM_OK;
}

}  // namespace

// A sum is split as far as there are CUs for the parts and 8 steps of 128 bytes for
// each.  Of the two tiles the large one is taken where its busiest CU has no more
// to multiply than with the small ones, its sums are whole and (16 and 8 bits) at
// least 16 steps long: a CU holds one of it, so that nothing hides how a tile begins
// and ends.  Large against small, us, bf16: 16,384 x 4,096 x 8,192: 865, 974; 8,192 x
// 4,096 x 4,096: 231, 290; 4,096 x 4,096 x 4,096: 134, 145; 8,192 x 8,192 x 1,024: 159,
// 166; but 16,384 x 4,096 x 512: 118, 110; 2,048 x 2,048 x 2,048 (in 4 parts): 51, 32.  8 bit:
// 16,384 x 4,096 x 8,192: 427, 492; 8,192 x 8,192 x 1,024 (8 steps): 112, 107.  fp32, where the
// matrix cores take 16 times as long: 4,096 x 2,048 x 1,024: 135, 143; 12,000 x 200 x 472:
// 43, 31.
LinearPlan tgm::linear_plan(int64_t M, int64_t N, int64_t K, int code)
{
    const bool f32 = code == TGM_F32;
    const int64_t steps = cdiv(K * elem_bytes(code), 128);
    const int64_t side = f32 ? 128 : 256, half = side / 2;
    const int64_t large = cdiv(M, side) * cdiv(N, side), small = cdiv(M, half) * cdiv(N, half);
    if (cdiv(large, 256) * 4 <= cdiv(small, 256) && large >= (f32 ? 512 : 192) &&
        (f32 || steps >= 16))
        return LinearPlan{true, 1};
    // half as many large tiles as CUs or a little less, and a sum that is long in halves too.
    // us, bf16, two parts of the large tile against the small one's, rows x columns x sum:
    // 4,096 x 2,048 x 8,192: 123, 130 (x 4,096: 72, 65; x 2,048: 50, 37); 2,560 x 2,560 x 16,384: 178,
    // 204; 6,144 x 1,024 x 8,192: 98, 102; but 2,048 x 2,048 (64 tiles) x 8,192: 85, 72; weights'
    // gradients: 4,096 x 2,048 x 8,192: 124, 129 (x 4,096: 76, 70); 2,560 x 2,560 x 8,192: 108, 115;
    // 2,048 x 2,048 x 8,192: 95, 76.
    if (!f32 && large >= 96 && large <= 128 && steps >= 128)
        return LinearPlan{true, 2};
    return LinearPlan{
        false, (int)std::max<int64_t>(1, std::min<int64_t>({512 / small, steps / 8, 64}))};
}

extern "C" tgm_status_t tgm_linear_work_bytes(int32_t rows, int32_t N, int32_t K, int32_t dtype,
                                              int32_t act, int32_t backward, size_t *bytes)
{
    if (!bytes || rows < 0 || N < 1 || N > kMaxDim || K < 1 || K > kMaxDim || act < 0 ||
        act > TGM_ACT_GELU || !(wide_type(dtype) || (dtype == TGM_E4M3 && !backward)))
        return TGM_EINVAL;
    *bytes = backward ? dz_bytes(rows, N, dtype, act) + db_bytes(rows, N) +
                            scale_bytes(rows, K, dtype, act) +
                            std::max(split_bytes(rows, K, N, dtype), split_bytes(N, K, rows, dtype))
                      : few_blocks(rows, N, K, dtype) ? 0 : split_bytes(rows, N, K, dtype);
    return TGM_OK;
}

extern "C" tgm_status_t tgm_linear(const tgm_linear_desc *d, const void *x, const float *scale_x,
                                   const void *W, const float *scale_w, const void *bias,
                                   const void *res, const int32_t *n_rows, void *z, void *y,
                                   void *work, size_t work_bytes, void *stream)
{
    int64_t ld[7];
    TGM_TRY_STATUS(linear_args(d, ld));
    const bool q = d->dtype == TGM_E4M3;
    if (!(q ? wide_type(d->out_dtype) : wide_type(d->dtype) && d->out_dtype == d->dtype))
        return TGM_EINVAL;
    if (!W || (d->rows && (!x || !y)) || (q ? !scale_w || (d->rows && !scale_x)
                                            : scale_x || scale_w))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_linear_work_bytes(d->rows, d->N, d->K, d->dtype, d->act, 0, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    if (d->rows == 0)
        return TGM_OK;
    LinearProduct p{W, x, ld[1], ld[0], d->K, nullptr, {}, (float *)work, as_stream(stream)};
    p.o = LinearOut{y, z, bias, res, scale_x, scale_w, ld[4], ld[3], ld[2], d->rows, d->N, d->act,
              n_rows};
    if (q)
        switch (d->out_dtype) {
        case TGM_F32: return product<e4m3, float, true, true>(p);
        case TGM_BF16: return product<e4m3, bf16, true, true>(p);
        default: return product<e4m3, f16, true, true>(p);
        }
    switch (d->dtype) {
    case TGM_F32: return product<float, float, true, true>(p);
    case TGM_BF16: return product<bf16, bf16, true, true>(p);
    default: return product<f16, f16, true, true>(p);
    }
}

extern "C" tgm_status_t tgm_linear_backward(const tgm_linear_desc *d, const void *x, const void *W,
                                            const void *z, const void *dy, const int32_t *n_rows,
                                            void *dx, void *dW, void *db, void *work,
                                            size_t work_bytes, void *stream)
{
    int64_t ld[7];
    TGM_TRY_STATUS(linear_args(d, ld));
    if (!wide_type(d->dtype) || d->out_dtype != d->dtype)
        return TGM_EINVAL;
    if ((dx && !W) || (d->rows && (!dy || (dW && !x) || (d->act != TGM_ACT_NONE && !z))))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_linear_work_bytes(d->rows, d->N, d->K, d->dtype, d->act, 1, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    char *w = (char *)work;
    const hipStream_t s = as_stream(stream);
    switch (d->dtype) {
    case TGM_F32: return backward<float>(d, ld, x, W, z, dy, n_rows, dx, dW, db, w, s);
    case TGM_BF16: return backward<bf16>(d, ld, x, W, z, dy, n_rows, dx, dW, db, w, s);
    default: return backward<f16>(d, ld, x, W, z, dy, n_rows, dx, dW, db, w, s);
    }
}
