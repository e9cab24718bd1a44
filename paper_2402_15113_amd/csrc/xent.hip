// Softmax cross entropy of x W^T + bias over many classes, the nodes of a table (tgm_xent),
// and its gradient (tgm_xent_backward), without keeping the logits.
//
// Forward: the logits' product ends in each tile's largest value and sum of exponentials a
// row (XentSums); k_xent_loss joins them.  Backward, for a piece of the classes at a time:
// the same product ends in dz = (softmax - onehot) dloss (XentGrad), rounded to the operands'
// type for the two products that read it, dx += dz W (fp32 between the pieces) and dW = dz^T
// x.  Bound by the matrix cores: 2 rows N K operations forward, 6 back.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "xent.h"

using namespace tgm;

namespace {

constexpr int kMaxDim = 1 << 20;

// lse and loss of 16 rows a workgroup, 64 threads a row with every 64th run of columns.  Bound by
// memory and, with few rows, its latency: 514 runs of 8,192 rows (34 MB) in 11 us, 42 with a
// thread a row.
__global__ __launch_bounds__(1024) void k_xent_loss(const f2 *__restrict__ part, int32_t runs,
                                                    int32_t rows, int32_t classes,
                                                    const int32_t *__restrict__ n_rows,
                                                    const int32_t *__restrict__ target,
                                                    const float *__restrict__ at_target,
                                                    float *__restrict__ loss,
                                                    float *__restrict__ lse)
{
    constexpr int ROWS = 16, LANES = 64;
    __shared__ f2 lds[LANES][ROWS + 1];
    const int row = threadIdx.x % ROWS, lane = threadIdx.x / ROWS;
    const int32_t R = rows_in_use(rows, n_rows);
    // the sum relative to the largest so far; -infinity: nothing yet (or no more than NaN); beside
    // an infinite one the others are nothing, if they are numbers
    auto join = [](f2 a, f2 b) __attribute__((always_inline)) {
        const float t = fmaxf(a.x, b.x);
        const bool far = fabsf(t) == INFINITY;
        auto part = [&](f2 v) __attribute__((always_inline)) {
            return far ? (v.x == t ? v.y : v.y * 0.f) : v.y * expf(v.x - t);
        };
        return f2{t, part(a) + part(b)};
    };
    for (int64_t m0 = (int64_t)blockIdx.x * ROWS; m0 < R; m0 += (int64_t)gridDim.x * ROWS) {
        const int64_t m = m0 + row;
        const bool on = m < R;
        f2 all{-INFINITY, 0.f};
        if (on)
#pragma unroll 8
            for (int r = lane; r < runs; r += LANES)
                all = join(all, part[(int64_t)r * rows + m]);
        lds[lane][row] = all;
        for (int half = LANES / 2; half; half /= 2) {
            __syncthreads();
            if (lane < half)
                lds[lane][row] = join(lds[lane][row], lds[lane + half][row]);
        }
        if (lane || !on)
            continue;   // (what is read behind the last barrier is this wavefront's own)
        all = lds[0][row];
        const float l = all.x == -INFINITY ? (all.y == 0.f ? all.x : all.y) : all.x + logf(all.y);
        const int32_t t = target[m];
        if (lse)
            lse[m] = l;
        if (loss) {
            const float z = t >= 0 && t < classes ? at_target[m] : 0.f;
            // a class that is left out has probability 0, wherever the others are
            loss[m] = t < 0 || t >= classes ? 0.f : z == -INFINITY && l == l ? INFINITY : l - z;
        }
    }
}

// A row that has no part in the loss (its target is outside the classes, or every one of its
// logits is -infinity) has zeros in dz, but dW = dz^T x would have 0 x of it, NaN where x is not
// finite.  So the rows of which that is so are looked for, and where there is one, x is copied
// with zeros for all that have no part, and dW takes the copy.
__device__ __forceinline__ bool no_part(int32_t target, float lse, int32_t classes)
{
    return target < 0 || target >= classes || lse == -INFINITY;
}
constexpr int kLookRows = 16, kLookGroups = 1024;   // rows a wavefront, workgroups at most
uint32_t look_groups(int32_t rows)
{
    return (uint32_t)std::min<int64_t>(cdiv(rows, 4 * kLookRows), kLookGroups);
}
// Whether a workgroup's rows hold one.  Reads only those of x's rows that have no part, one after
// another in a wavefront, whose latency bounds it: 8,192 rows x 2,048 bf16, a tenth of them without
// a target, in 10 us; 12,000 x 100 fp32 in 5.
template <class T>
__global__ __launch_bounds__(256) void k_xent_look(const T *__restrict__ x, int64_t ld, int32_t K,
                                                   const int32_t *__restrict__ target,
                                                   const float *__restrict__ lse, int32_t classes,
                                                   int32_t rows, const int32_t *n_rows,
                                                   int32_t *__restrict__ found)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    __shared__ int32_t lds[4];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int32_t R = rows_in_use(rows, n_rows);
    bool any = false;
    for (int64_t m0 = ((int64_t)blockIdx.x * 4 + w) * kLookRows; m0 < R;
         m0 += (int64_t)gridDim.x * 4 * kLookRows) {
        const int64_t m = m0 + lane;
        uint64_t todo = __ballot(lane < kLookRows && m < R && no_part(target[m], lse[m], classes));
        for (; todo; todo &= todo - 1) {
            const T *row = x + (m0 + __builtin_ctzll(todo)) * ld;
            const int32_t whole = K / VEC * VEC;
            float sum = 0.f;   // NaN once a value is not finite
            for (int32_t k = lane * VEC; k < whole; k += 64 * VEC) {
                const Pack<T, VEC> p = load_pack<T, VEC>(row + k);
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    sum = fmaf(to_f32(p.v[j]), 0.f, sum);
            }
            if (whole + lane < K)
                sum = fmaf(to_f32(row[whole + lane]), 0.f, sum);
            any |= sum != 0.f;
        }
    }
    any = __any(any);
    if (lane == 0)
        lds[w] = any;
    __syncthreads();
    if (threadIdx.x == 0)
        found[blockIdx.x] = lds[0] | lds[1] | lds[2] | lds[3];
}
// take = whether any workgroup has found one; x's copy if so, with zeros up to `wide` columns.
// 3 to 5 us where none has; the copy is bound by memory: 100,000 x 256 bf16 (102 MB) 20 us more.
template <class T>
__global__ __launch_bounds__(256) void k_xent_keep(const T *__restrict__ x, int64_t ld, int32_t K,
                                                   const int32_t *__restrict__ target,
                                                   const float *__restrict__ lse, int32_t classes,
                                                   int32_t rows, const int32_t *n_rows,
                                                   const int32_t *__restrict__ found,
                                                   uint32_t groups, int32_t *__restrict__ take,
                                                   T *__restrict__ copy, int32_t wide)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    int32_t any = 0;
    for (uint32_t i = threadIdx.x; i < groups; i += 256)
        any |= found[i];
    any = __syncthreads_or(any);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *take = any;
    if (!any)
        return;
    const int32_t R = rows_in_use(rows, n_rows), vectors = wide / VEC;
    const int64_t n = (int64_t)R * vectors;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / vectors;
        const int32_t k = (int32_t)(i - m * vectors) * VEC;
        Pack<T, VEC> p;
        __builtin_memset(&p, 0, sizeof(p));
        if (!no_part(target[m], lse[m], classes)) {
            const T *from = x + m * ld + k;
            if (k + VEC <= K)
                p = load_pack<T, VEC>(from);
            else
#pragma unroll
                for (int j = 0; j < VEC - 1; ++j)
                    if (k + j < K)
                        p.v[j] = from[j];
        }
        store_pack(copy + m * wide + k, p);
    }
}

// The power of two that dz is held times in fp16, whose range is narrower than that of
// dloss: the largest finite |dloss| comes to between 2^14 and 2^15; and its reciprocal for the
// products' K columns.  One workgroup: 8,192 rows take it 5 us.
__global__ __launch_bounds__(1024) void k_xent_scale(const float *__restrict__ dloss,
                                                     const int32_t *__restrict__ target,
                                                     const int32_t *__restrict__ n_rows,
                                                     int32_t rows, int32_t classes, int32_t K,
                                                     float *__restrict__ scale,
                                                     float *__restrict__ unscale)
{
    __shared__ float lds[16];
    const int32_t R = rows_in_use(rows, n_rows);
    float top = 0.f;
#pragma unroll 4
    for (int64_t m = threadIdx.x; m < R; m += 1024) {
        const float v = fabsf(dloss[m]);
        const int32_t t = target[m];
        top = v < INFINITY && v > top && t >= 0 && t < classes ? v : top;
    }
    top = group_max<64>(top);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int k = 0; k < 16; ++k)
        top = fmaxf(top, lds[k]);
    const float s = top > 0.f ? ldexpf(1.f, min(max(14 - ilogbf(top), -126), 126)) : 1.f;
    if (threadIdx.x == 0)
        scale[0] = s;
    for (int32_t k = threadIdx.x; k < K; k += 1024)
        unscale[k] = 1.f / s;
}

// db = the runs' partial sums added in order: 32 columns a workgroup, 32 threads each.  Bound by
// latency: 9,228 columns of 188 tiles of rows in 11 us.
template <class T>
__global__ __launch_bounds__(1024) void k_xent_db(const float *__restrict__ part, XentRuns r,
                                                  int32_t rows, const int32_t *n_rows, int32_t N,
                                                  const float *scale, T *__restrict__ db)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, k0 = threadIdx.x >> 5;
    const int64_t n = (int64_t)blockIdx.x * 32 + c;
    const int32_t tiles = (int32_t)(((int64_t)rows_in_use(rows, n_rows) + r.tile_rows - 1) /
                                    r.tile_rows);
    float a = 0.f;
    if (n < N)
#pragma unroll 4
        for (int k = k0; k < tiles * r.tile_runs; k += 32)
            a += part[(int64_t)k * N + n];
    lds[k0][c] = a;
    __syncthreads();
    if (k0 == 0 && n < N) {
        for (int k = 1; k < 32; ++k)
            a += lds[k][c];
        db[n] = from_f32<T>(scale ? a / scale[0] : a);
    }
}

// dx from its fp32 sums over the pieces.  Bound by memory: 8,192 x 2,048 to
// bf16 in 18 us (5.6 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_xent_dx(const float *__restrict__ sum, int32_t rows,
                                                 const int32_t *n_rows, int32_t K, int64_t wide,
                                                 int64_t ld, T *__restrict__ dx)
{
    const int32_t R = rows_in_use(rows, n_rows);
    const int64_t quads = wide / 4, n = R * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int32_t k = 4 * (int32_t)(i - m * quads);
        const f4 v = *reinterpret_cast<const f4 *>(sum + m * wide + k);
        Pack<T, 4> p;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p.v[j] = from_f32<T>(v[j]);
        T *to = dx + m * ld + k;
        if (k + 4 <= K)
            store_pack(to, p);
        else
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (k + j < K)
                    to[j] = p.v[j];
    }
}

// ---------------------------------------------------------------- host
// Classes of a piece: dz of one takes 512 MB at most (or 1,024 classes).  Of the multiples of 256
// up to there the one whose tiles of 256 x 256 fill their rounds of 256 CUs best, in the logits'
// product (with sums of K) and in dW's (with sums of the rows).  us of a training step, 8,192 rows
// x 65,537 x 2,048 bf16, in pieces of
//     4,096  8,192  13,312  16,384  16,640  21,760  32,768
//     7,338  6,825   7,520   6,921   7,334   7,304   6,931
// Smaller ones gain little and lose more where rows are many (32,768 rows x 32,768 x 1,024 bf16:
// 9,029 us with 128 MB, 8,310 with 256, 7,475 with 512) and in fp32 (12,000 rows x 9,228 x 100:
// 1,217 us in two pieces, 1,117 in one).
int32_t xent_piece(int32_t rows, int32_t N, int32_t K, int64_t most)
{
    if (N <= most)
        return N;
    const int64_t rt = cdiv(rows, 256), kt = cdiv(K, 256);
    int64_t best = most;
    double least = 1e300;
    for (int64_t n = most; n >= 1024 && 2 * n >= most; n -= 256) {
        const int64_t tiles = n / 256;
        const double cost = (double)(cdiv(tiles * rt, 256) * K + cdiv(tiles * kt, 256) * rows) /
                            (double)n;
        if (cost < 0.99 * least)
            least = cost, best = n;
    }
    return (int32_t)best;
}
// Parts of the sums of dx and dW in fp32, where the small tile takes them: workgroups by the
// thousand, five a CU, since a few more than CUs leave most of them idle for half of the time.
// 12,000 rows x 9,228 x 100 (376 tiles of dx): a training step with 1, 2, 4, 5, 8 and 12 parts
// 1,428, 1,202, 1,157, 1,129, 1,106 and 1,108 us.
int32_t xent_split(int64_t M, int64_t N, int64_t K, int code)
{
    const LinearPlan l = linear_plan(M, N, K, code);
    if (code != TGM_F32 || l.large)
        return l.large ? 0 : l.parts;
    const int64_t tiles = cdiv(M, 64) * cdiv(N, 64), steps = cdiv(K, 32);
    return (int32_t)std::max<int64_t>(l.parts, std::min<int64_t>({2048 / tiles, steps / 16, 16}));
}
size_t xent_split_bytes(int64_t M, int64_t N, int64_t K, int code)
{
    if (M <= 0 || K <= 0)
        return 0;
    const int32_t parts = xent_split(M, N, K, code);
    return parts > 1 ? (size_t)parts * M * ((N + 3) / 4 * 4) * 4
                     : linear_split_bytes(M, N, K, code);
}
struct XentPlan {
    int32_t piece, last;      // classes of every piece, and of the last one
    int64_t pieces, ld_dz;
    int32_t wide;             // columns of x's copy
    size_t dz, sum, scale, db, split, found, copy, all;   // bytes of the parts of the work space
};
size_t whole(size_t n) { return (n + 255) / 256 * 256; }
XentPlan xent_plan(int32_t rows, int32_t N, int32_t K, int code)
{
    XentPlan p{};
    const int64_t eb = elem_bytes(code), R = std::max(rows, 1);
    const int64_t most = std::max<int64_t>(((int64_t)512 << 20) / (R * eb) / 256 * 256, 1024);
    p.piece = xent_piece(rows, N, K, most);
    p.pieces = cdiv(N, p.piece);
    p.last = (int32_t)(N - (p.pieces - 1) * p.piece);
    p.ld_dz = cdiv(p.piece, 16) * 16;
    p.dz = whole((size_t)rows * p.ld_dz * eb);
    p.sum = p.pieces > 1 ? whole((size_t)rows * round_up(K, 4) * 4) : 0;
    p.scale = code == TGM_F16 ? whole((size_t)(64 + round_up(K, 4)) * 4) : 0;
    p.db = whole((size_t)xent_db_parts(rows, code) * p.piece * 4);
    for (int32_t n : {p.piece, p.last})
        p.split = std::max({p.split, xent_split_bytes(rows, K, n, code),
                            xent_split_bytes(n, K, rows, code)});
    p.wide = round_up(K, 16 / (int)eb);
    p.found = rows ? whole((1 + look_groups(rows)) * sizeof(int32_t)) : 0;
    p.copy = whole((size_t)rows * p.wide * eb);
    p.split = whole(p.split);
    p.all = p.dz + p.sum + p.scale + p.db + p.split + p.found + p.copy;
    return p;
}
size_t sums_bytes(int32_t rows, int32_t N)
{
    return whole((size_t)xent_parts(N) * rows * sizeof(f2)) + whole((size_t)rows * 4);
}

tgm_status_t xent_args(const tgm_xent_desc *d, int64_t *ld)
{
    if (!d || d->rows < 0 || d->N < 1 || d->N > kMaxDim || d->K < 1 || d->K > kMaxDim ||
        !wide_type(d->dtype))
        return TGM_EINVAL;
    // a launch has fewer than 2^32 threads, 256 a tile
    const int64_t side = d->dtype == TGM_F32 ? 64 : 128, most = (int64_t)1 << 24;
    const int64_t r = cdiv(d->rows, side), n = cdiv(d->N, side), k = cdiv(d->K, side);
    if (r * n >= most || r * k >= most || n * k >= most)
        return TGM_EINVAL;
    const int64_t given[4] = {d->ld_x, d->ld_w, d->ld_dx, d->ld_dw};
    for (int i = 0; i < 4; ++i)
        if ((ld[i] = stride_of(given[i], d->K)) < 0)
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

template <class T> constexpr auto sums_of = std::is_same_v<T, float> ? xent_sums_f32
                                            : std::is_same_v<T, bf16> ? xent_sums_bf16
                                                                      : xent_sums_f16;
template <class T> constexpr auto grad_of = std::is_same_v<T, float> ? xent_grad_f32
                                            : std::is_same_v<T, bf16> ? xent_grad_bf16
                                                                      : xent_grad_f16;
template <class T> constexpr auto dw_of = std::is_same_v<T, float> ? xent_dw_f32
                                          : std::is_same_v<T, bf16> ? xent_dw_bf16
                                                                    : xent_dw_f16;
template <class T> constexpr auto tile_of_type = std::is_same_v<T, float> ? linear_tile_f32
                                                 : std::is_same_v<T, bf16> ? linear_tile_bf16
                                                                           : linear_tile_f16;

template <class T>
tgm_status_t forward(const tgm_xent_desc *d, const int64_t *ld, const void *x, const void *W,
                     const void *bias, const int32_t *target, const int32_t *n_rows, float *loss,
                     float *lse, char *work, hipStream_t s)
{
    LinearProduct p{W, x, ld[1], ld[0], d->K, nullptr, {}, nullptr, s};
    p.o.M = d->rows, p.o.N = d->N, p.o.n_rows = n_rows;
    XentArgs e{};
    e.bias = bias, e.target = target, e.rows = d->rows, e.classes = d->N;
    e.part = (f2 *)work;
    e.at_target = (float *)(work + whole((size_t)xent_parts(d->N) * d->rows * sizeof(f2)));
    XentRuns r;
    TGM_TRY_STATUS(sums_of<T>(p, e, &r));
    // (a launch has fewer than 2^32 threads)
    TGM_LAUNCH(k_xent_loss, dim3((uint32_t)std::min<int64_t>(cdiv(d->rows, 16), 1 << 21)),
               dim3(1024), 0, s, e.part, r.columns, d->rows, d->N, n_rows, target, e.at_target, loss, lse);
    return TGM_OK;
}

template <class T>
tgm_status_t backward(const tgm_xent_desc *d, const int64_t *ld, const void *x, const void *W,
                      const void *bias, const int32_t *target, const float *lse,
                      const float *dloss, const int32_t *n_rows, void *dx, void *dW, void *db,
                      char *work, hipStream_t s)
{
    constexpr int code = TypeCode<T>::code;
    const XentPlan plan = xent_plan(d->rows, d->N, d->K, code);
    T *dz = (T *)work;
    float *sum = (float *)(work + plan.dz);
    float *scale = plan.scale ? (float *)(work + plan.dz + plan.sum) : nullptr;
    float *unscale = scale ? scale + 64 : nullptr;
    float *part = (float *)(work + plan.dz + plan.sum + plan.scale);
    float *split = (float *)(work + plan.dz + plan.sum + plan.scale + plan.db);
    int32_t *take = (int32_t *)((char *)split + plan.split), *found = take + 1;
    T *copy = (T *)((char *)take + plan.found);
    const int64_t wide = round_up(d->K, 4);
    if (dW && d->rows) {
        const uint32_t groups = look_groups(d->rows);
        TGM_LAUNCH((k_xent_look<T>), dim3(groups), dim3(256), 0, s, (const T *)x, ld[0], d->K,
                   target, lse, d->N, d->rows, n_rows, found);
        const int64_t vectors = (int64_t)d->rows * plan.wide * (int64_t)sizeof(T) / 16;
        TGM_LAUNCH((k_xent_keep<T>), dim3((uint32_t)std::min<int64_t>(cdiv(vectors, 256), 1024)),
                   dim3(256), 0, s, (const T *)x, ld[0], d->K, target, lse, d->N, d->rows, n_rows,
                   found, groups, take, copy, plan.wide);
    }
    if (scale)
        TGM_LAUNCH(k_xent_scale, dim3(1), dim3(1024), 0, s, dloss, target, n_rows, d->rows, d->N,
                   d->K, scale, unscale);
    for (int64_t i = 0; i < plan.pieces; ++i) {
        const int64_t n0 = i * plan.piece;
        const int32_t n = i + 1 < plan.pieces ? plan.piece : plan.last;
        const T *w = (const T *)W + n0 * ld[1];
        XentRuns r{0, 1, 0};
        if (d->rows) {
            LinearProduct p{w, x, ld[1], ld[0], d->K, nullptr, {}, nullptr, s};
            p.o.M = d->rows, p.o.N = n, p.o.n_rows = n_rows;
            XentArgs e{};
            e.bias = bias ? (const T *)bias + n0 : nullptr;
            e.target = target, e.rows = d->rows, e.classes = d->N, e.n_first = (int32_t)n0;
            e.lse = lse, e.dloss = dloss, e.scale = scale, e.dz = dz, e.ld_dz = plan.ld_dz;
            e.db = db ? part : nullptr;
            TGM_TRY_STATUS(grad_of<T>(p, e, &r));
        }
        if (db)
            TGM_LAUNCH((k_xent_db<T>), dim3((uint32_t)cdiv(n, 32)), dim3(1024), 0, s, part, r,
                       d->rows, n_rows, n, scale, (T *)db + n0);
        if (dx && d->rows) {
            LinearProduct p{w, dz, ld[1], plan.ld_dz, n, nullptr, {}, split, s};
            p.o.M = d->rows, p.o.N = d->K, p.o.n_rows = n_rows, p.o.sn = unscale;
            p.parts = xent_split(d->rows, d->K, n, code);
            if (plan.pieces == 1) {
                p.o.y = dx, p.o.ld_y = ld[2];
                TGM_TRY_STATUS(tile_of_type<T>(p, 1, code));
            } else {
                // the pieces' sums in fp32, rounded once at the end
                p.o.y = sum, p.o.ld_y = wide;
                p.o.res = i ? sum : nullptr, p.o.ld_res = wide;
                if constexpr (code == TGM_F32)
                    TGM_TRY_STATUS(linear_tile_f32(p, 1, code));
                else if constexpr (code == TGM_BF16)
                    TGM_TRY_STATUS(xent_dx_bf16(p));
                else
                    TGM_TRY_STATUS(xent_dx_f16(p));
                if (i + 1 == plan.pieces)
                    TGM_LAUNCH((k_xent_dx<T>),
                               dim3((uint32_t)std::min<int64_t>(
                                   cdiv((int64_t)d->rows * (wide / 4), 256), 1 << 14)),
                               dim3(256), 0, s, sum, d->rows, n_rows, d->K, wide, ld[2], (T *)dx);
            }
        }
        if (dW) {
            LinearProduct p{x, dz, ld[0], plan.ld_dz, d->rows, n_rows, {}, split, s};
            p.o.M = n, p.o.N = d->K, p.o.sn = unscale;
            p.parts = d->rows ? xent_split(n, d->K, d->rows, code) : 0;
            // dz's rows have whole vectors
            p.o.pad_m = round_up(n, 16 / (int)sizeof(T)) - n;
            p.o.y = (T *)dW + n0 * ld[3], p.o.ld_y = ld[3];
            if (d->rows)
                TGM_TRY_STATUS(dw_of<T>(p, copy, plan.wide, take));
            else
                TGM_TRY_STATUS(tile_of_type<T>(p, 2, code));
        }
    }
    return TGM_OK;
}

}  // namespace

extern "C" tgm_status_t tgm_xent_work_bytes(int32_t rows, int32_t N, int32_t K, int32_t dtype,
                                            int32_t backward, size_t *bytes)
{
    if (!bytes)
        return TGM_EINVAL;
    int64_t ld[4];
    tgm_xent_desc d{rows, N, K, dtype, 0, 0, 0, 0};
    TGM_TRY_STATUS(xent_args(&d, ld));
    *bytes = backward ? xent_plan(rows, N, K, dtype).all : rows ? sums_bytes(rows, N) : 0;
    return TGM_OK;
}

extern "C" tgm_status_t tgm_xent(const tgm_xent_desc *d, const void *x, const void *W,
                                 const void *bias, const int32_t *target, const int32_t *n_rows,
                                 float *loss, float *lse, void *work, size_t work_bytes,
                                 void *stream)
{
    int64_t ld[4];
    TGM_TRY_STATUS(xent_args(d, ld));
    if (!W || (d->rows && (!x || !target)) || (!loss && !lse && d->rows))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_xent_work_bytes(d->rows, d->N, d->K, d->dtype, 0, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    if (d->rows == 0)
        return TGM_OK;
    char *w = (char *)work;
    const hipStream_t s = as_stream(stream);
    switch (d->dtype) {
    case TGM_F32: return forward<float>(d, ld, x, W, bias, target, n_rows, loss, lse, w, s);
    case TGM_BF16: return forward<bf16>(d, ld, x, W, bias, target, n_rows, loss, lse, w, s);
    default: return forward<f16>(d, ld, x, W, bias, target, n_rows, loss, lse, w, s);
    }
}

extern "C" tgm_status_t tgm_xent_backward(const tgm_xent_desc *d, const void *x, const void *W,
                                          const void *bias, const int32_t *target,
                                          const float *lse, const float *dloss,
                                          const int32_t *n_rows, void *dx, void *dW, void *db,
                                          void *work, size_t work_bytes, void *stream)
{
    int64_t ld[4];
    TGM_TRY_STATUS(xent_args(d, ld));
    if (!W || (d->rows && (!x || !target || !lse || !dloss)))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_xent_work_bytes(d->rows, d->N, d->K, d->dtype, 1, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    if ((!dx || !d->rows) && !dW && !db)
        return TGM_OK;
    char *w = (char *)work;
    const hipStream_t s = as_stream(stream);
    switch (d->dtype) {
    case TGM_F32:
        return backward<float>(d, ld, x, W, bias, target, lse, dloss, n_rows, dx, dW, db, w, s);
    case TGM_BF16:
        return backward<bf16>(d, ld, x, W, bias, target, lse, dloss, n_rows, dx, dW, db, w, s);
    default:
        return backward<f16>(d, ld, x, W, bias, target, lse, dloss, n_rows, dx, dW, db, w, s);
    }
}
