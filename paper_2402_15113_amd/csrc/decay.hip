// Linear attention with a decay for each head along packed or padded sequences
// (tgm_decay_attn), its gradient (tgm_decay_attn_backward) and its single-row form
// (tgm_decay_attn_step).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "decay.h"

using namespace tgm;

namespace {

// The states behind the cells of the sequences that go on, from those of the cells alone: a
// thread follows EACH elements of a head's state along a sequence of more rows than a cell.  The
// cells have to be followed in order, so that what bounds it is how many loads are under way: 16 a
// thread, double buffered.  129 cells of 8 heads of 128 x 128 (135 MB): 31 us, 4.4 TB/s; 45 cells of 16
// heads of 64 x 128 under 64 sequences 17.
// Its workgroups go by sequences where there are no more than four to a cell, else by cells, in
// which those that begin and go on have to be searched for (by cells alone 89 and 29 us), and
// since most of many have nothing to follow, they are fewer, of 8 elements a thread (with 2: 34).
bool decay_by_sequence(const DecayRun &r) { return r.a.S <= 4 * r.all_cells; }

template <bool BY_SEQUENCE, int EACH>
__global__ __launch_bounds__(256) void k_decay_walk(DecayRun run)
{
    const DecayArgs &A = run.a;
    const int32_t h = blockIdx.y, size = A.p * A.r;
    const int32_t at = (int32_t)(blockIdx.z * 256 * EACH + threadIdx.x);
    const float keep = decay_pow(decay_log2(A.decay[h]), (float)run.cell);
    const int64_t C = run.cell, n = BY_SEQUENCE ? A.S : run.all_cells;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        DecaySeq q;
        if constexpr (BY_SEQUENCE) {
            q = decay_seq(A, (int32_t)i);
            if (q.e - q.b <= C)
                continue;
        } else {
            const DecayPiece piece = decay_piece_onward(run, i);
            q = piece.q;
            if (piece.hi <= piece.lo || (A.rev ? piece.hi != q.e : piece.lo != q.b))
                continue;   // no sequence begins here and goes on
        }
        const int64_t first = A.offsets ? q.b / C : q.b / A.L * run.cells;
        const int64_t last = A.offsets ? (q.e - 1) / C : first + (q.e - q.b - 1) / C;
        const int64_t left = last - first - 1;   // cells that it goes on to, but for its last
        if (left <= 0)
            continue;
        float *s = run.states + (h * run.all_cells + (A.rev ? last : first)) * (int64_t)size;
        const int64_t next = (A.rev ? -1 : 1) * (int64_t)size;
        int32_t mine[EACH];   // past the state's end: the last element again, which is not stored
        float v[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            mine[k] = min(at + 256 * k, size - 1), v[k] = s[mine[k]];
        auto along = [&](auto ahead) __attribute__((always_inline)) {
            constexpr int AHEAD = decltype(ahead)::value;
            float e[2][AHEAD][EACH];
            // cells c + 1 .. c + AHEAD, past the last one that one again
            auto load = [&](float (&to)[AHEAD][EACH], int64_t c) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const float *p = s + min(c + 1 + u, left) * next;
#pragma unroll
                    for (int k = 0; k < EACH; ++k)
                        to[u][k] = p[mine[k]];
                }
            };
            auto follow = [&](const float (&from)[AHEAD][EACH], int64_t c)
                __attribute__((always_inline)) {
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u)
                        if (c + 1 + u <= left) {
                            float *p = s + (c + 1 + u) * next;
#pragma unroll
                            for (int k = 0; k < EACH; ++k) {
                                v[k] = v[k] * keep + from[u][k];
                                if (at + 256 * k < size)
                                    p[mine[k]] = v[k];
                            }
                        }
                };
            // the next cells' loads go before these cells' stores, which are waited for in order
            load(e[0], 0);
            for (int64_t c = 0; c < left; c += 2 * AHEAD) {
                if (c + AHEAD < left)
                    load(e[1], c + AHEAD);
                follow(e[0], c);
                if (c + 2 * AHEAD < left)
                    load(e[0], c + 2 * AHEAD);
                if (c + AHEAD < left)
                    follow(e[1], c + AHEAD);
            }
        };
        if (left <= 2)
            along(std::integral_constant<int, 2>{});
        else
            along(std::integral_constant<int, 16 / EACH>{});
    }
}

// The pieces that have something to do, those of most rows first (by 32nds of a cell), for the
// results pass of sequences of uneven lengths: otherwise a long piece that begins last is waited
// for.  The order within a length is any, and no result depends on it.  One workgroup; bound by
// the latency of each thread's searches: 109 pieces 5 us.
constexpr int kOrderThreads = 1024, kOrderEach = 8, kOrderLengths = 33;
__global__ __launch_bounds__(kOrderThreads) void k_decay_order(DecayRun run, int32_t *order)
{
    __shared__ int32_t place[kOrderLengths + 1];
    if (threadIdx.x <= kOrderLengths)
        place[threadIdx.x] = 0;
    __syncthreads();
    int length[kOrderEach];   // 0: the longest; the last: nothing to do
#pragma unroll
    for (int u = 0; u < kOrderEach; ++u) {
        const int64_t id = u * kOrderThreads + threadIdx.x;
        if (id >= run.ids)
            continue;
        const DecayPiece p = decay_piece_alone(run, id);
        const int64_t rows = p.hi - p.lo;
        length[u] = rows > 0 ? kOrderLengths - 2 - (int)(32 * (rows - 1) / run.cell)
                    : decay_empty_here(run, p) ? kOrderLengths - 1
                                               : kOrderLengths;
        atomicAdd(&place[length[u]], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 0, n = 0; i <= kOrderLengths; ++i) {
            const int32_t here = place[i];
            place[i] = n;
            n += here;
        }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kOrderEach; ++u) {
        const int64_t id = u * kOrderThreads + threadIdx.x;
        if (id < run.ids)
            order[atomicAdd(&place[length[u]], 1)] =
                length[u] == kOrderLengths ? -1 : (int32_t)id;
    }
}

// The gradient of a head of k or v that several heads of q share: theirs added in order, for
// the rows of sequences.  Bound by memory: 65,536 rows of 16 heads of 128, four to one (604 MB):
// 125 us, 4.8 TB/s, 157 by single columns; of 64, 56 us and 83.
constexpr int kSharedRows = 16;
template <class T, int VEC>
__global__ __launch_bounds__(256) void k_decay_shared(const float *__restrict__ part, DecayArgs A,
                                                      int32_t heads, int32_t share, int32_t d,
                                                      int64_t ld, T *__restrict__ out)
{
    const int64_t ids = (A.rows + kSharedRows - 1) / kSharedRows + A.S;
    const uint32_t wide = (uint32_t)(heads * d / VEC), head = (uint32_t)(d / VEC);
    for (int64_t id = blockIdx.x; id < ids; id += gridDim.x) {
        const DecayPiece p = decay_piece(A, id, kSharedRows);
        const uint32_t n = (uint32_t)max(p.hi - p.lo, (int64_t)0) * wide;
        for (uint32_t i = threadIdx.x; i < n; i += 256) {
            const int64_t row = p.lo + i / wide;
            const uint32_t c = i % wide, h = c / head;
            const float *q = part + (row * heads + h) * (int64_t)share * d + (c - h * head) * VEC;
            Pack<float, VEC> s = load_pack<float, VEC>(q);
            for (int k = 1; k < share; ++k) {
                const Pack<float, VEC> v = load_pack<float, VEC>(q + (int64_t)k * d);
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    s.v[j] += v.v[j];
            }
            Pack<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                o.v[j] = from_f32<T>(s.v[j]);
            store_pack(out + row * ld + c * VEC, o);
        }
    }
}

// One row for each of n states of a table.  A workgroup has a head of one: a thread reads and
// writes VEC neighbouring columns of every G-th row of the state.  Bound by memory: 192 states of
// 16 heads of 128 x 128 (403 MB) 87 us, 4.6 TB/s.  600 of 2 heads of 50 x 50 (24 MB) take 9 us,
// three times what their bytes do: 13 rows a thread, each loaded when the one before is stored,
// since both are of the one table.
template <class T, int VEC, int LANES>
__global__ __launch_bounds__(256) void k_decay_step(const T *__restrict__ q,
                                                    const T *__restrict__ k,
                                                    const T *__restrict__ v,
                                                    const float *__restrict__ decay,
                                                    const int32_t *__restrict__ slots,
                                                    const int32_t *__restrict__ n_rows,
                                                    float *state, T *__restrict__ o,
                                                    tgm_decay_attn_desc d)
{
    constexpr int G = 256 / LANES, WIDE = LANES * VEC;
    __shared__ float part[G][WIDE];
    const int32_t n = rows_in_use((int32_t)d.rows, n_rows);
    const int32_t h = blockIdx.y, hk = h / (d.H / d.H_kv);
    const int c = threadIdx.x % LANES * VEC, g = threadIdx.x / LANES;
    const float a = decay_pow(decay_log2(decay[h]), 1.f);
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const int32_t slot = slots ? slots[row] : (int32_t)row;
        const bool kept = slot >= 0 && slot < d.S;
        float *st = state + ((int64_t)(kept ? slot : 0) * d.H + h) * (d.d_k * d.d_v);
        const T *pq = q + row * d.ld_q + h * d.d_k, *pk = k + row * d.ld_k + hk * d.d_k;
        const T *pv = v + row * d.ld_v + hk * d.d_v;
        float acc[VEC], vs[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            acc[j] = 0.f, vs[j] = c < d.d_v ? to_f32(pv[c + j]) : 0.f;
        if (c < d.d_v)
#pragma unroll 4
            for (int i = g; i < d.d_k; i += G) {
                Pack<float, VEC> s{};
                if (kept)
                    s = load_pack<float, VEC>(st + i * d.d_v + c);
                const float ki = to_f32(pk[i]), qi = to_f32(pq[i]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    s.v[j] = a * s.v[j] + ki * vs[j];
                    acc[j] += qi * s.v[j];
                }
                if (kept)
                    store_pack(st + i * d.d_v + c, s);
            }
        if (o) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                part[g][c + j] = acc[j];
            __syncthreads();
            for (int j = threadIdx.x; j < d.d_v; j += 256) {
                float s = part[0][j];
#pragma unroll
                for (int u = 1; u < G; ++u)
                    s += part[u][j];
                o[row * d.ld_o + h * d.d_v + j] = from_f32<T>(d.scale * s);
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------- host
size_t whole(size_t n) { return (n + 255) / 256 * 256; }

// Workgroups along x for n of them a head: a launch has fewer than 2^32 threads.
uint32_t across(int64_t n, int32_t H) { return (uint32_t)std::min<int64_t>(n, (1 << 22) / H); }

// Rows of a cell: sequences of no more are one workgroup's (a head of them), longer ones are
// divided, which costs a pass over y and z for the states and two over the states.
// A cell's rows come one chunk after another and the states pass is over C rows' time, while
// the states to write and walk go as rows H / C, so the best C grows as the root of rows H.
// us of a call, cells of 64, 256, 512, 1,024, 2,048 and 4,096 rows, bf16 heads of 128:
//     1,024 rows x 8        40     51     78     92
//     16,384 x 8           177     92    100    148    260
//     65,536 x 8           844    362    276    234    279
//     65,536 x 32        3,400  1,338  1,070    930    868
//     262,144 x 1          991    275    187    183    272
//     262,147 x 8                            932    860    840
// (the root is 128, 512, 1,024, 2,048, 768 and 2,048 there: 44, 102, 242, 860, 200 and 860 us.)
// Padded sequences fill the card without being divided from 256 heads of them on: 16 x 4,096
// rows of 32 heads 438 us whole, 700 in
// cells of 2,048, 878 of 1,024; of 16 heads 334, 373 and 450; but 4 x 4,096 rows of 32 heads
// (128 workgroups) 231 whole and 197 in cells of 1,024.
int32_t decay_cell(int64_t rows, int32_t S, int32_t H, bool packed)
{
    if (!packed && (int64_t)S * H >= 256)
        return (int32_t)std::max<int64_t>(1, rows / S);
    const int64_t root = (int64_t)std::sqrt(2.0 * (double)rows * H);
    return (int32_t)std::min<int64_t>(4096, std::max<int64_t>(64, cdiv(root, 64) * 64));
}
// Cells, and whether any sequence may have more than one.
struct DecayPlan {
    int32_t cell;
    int64_t cells, ids, padded_cells;
    bool divided;
};
DecayPlan decay_plan(int64_t rows, int32_t S, int32_t H, bool packed)
{
    DecayPlan p{};
    p.cell = decay_cell(rows, S, H, packed);
    if (packed) {
        p.cells = cdiv(rows, p.cell), p.ids = p.cells + S, p.divided = p.cells > 1;
    } else {
        const int64_t L = S ? rows / S : 0;
        p.padded_cells = std::max<int64_t>(1, cdiv(L, p.cell));
        p.cells = p.ids = p.padded_cells * S, p.divided = p.padded_cells > 1;
    }
    return p;
}
// Sequences of 16 rows or fewer are a wavefront's each, longer ones a workgroup's: us of a
// call, wavefronts and workgroups, 40,000 rows x 4 heads of 50 fp32 and of 64 bf16, padded
//     4 rows    246  313   246  301
//     16         63   83    57   70
//     17         94   86    80   68
//     32         64   55    53   40
// and packed, of lengths that vary, where the mean decides:
//     8         242  268   251  262
//     11        183  183   198  195
//     16        159  149   145  123
bool decay_brief(int64_t rows, int32_t S, bool packed)
{
    return rows <= (packed ? 10 : 16) * (int64_t)S;
}

// Bytes of the pieces' order, 0 where none is made: it costs a launch and pays where pieces of a
// chunk's rows and more come after each other on a CU.  us of a training step with and without:
//     65,536 rows of 16 heads of 64 and 128 bf16 in 64 sequences   1,506  1,797
//     65,536 x 4 heads of 64 in 200, fp32                            557    707
//     20,000 x 8 heads of 64 in 12, fp32                             419    484
//     40,000 x 4 heads of 64 in 833 (48 rows), fp32                  314    372
//     in 1,250 (32)                                                  373    388
//     in 1,666 (24)                                                  435    435
//     in 2,500 (16)                                                  554    539
size_t order_bytes(const DecayPlan &p, int64_t rows, int32_t S, int32_t H)
{
    return S > 1 && p.ids <= kOrderThreads * kOrderEach && p.ids * H > 256 && rows >= 32 * p.ids
               ? (size_t)p.ids * 4
               : 0;
}

// Bytes of the cells' states and of the pieces' order, whichever form the sequences have.
struct DecayBytes {
    size_t states, order;
};
DecayBytes decay_bytes(int64_t rows, int32_t S, int32_t H, int32_t d_k, int32_t d_v)
{
    size_t cells = 0, order = 0;
    auto add = [&](const DecayPlan &p) {
        cells = std::max(cells, p.divided ? (size_t)p.cells : 0);
        order = std::max(order, order_bytes(p, rows, S, H));
    };
    add(decay_plan(rows, S, H, true));
    if (S && rows % S == 0)
        add(decay_plan(rows, S, H, false));
    return DecayBytes{whole(cells * H * d_k * d_v * 4), whole(order)};
}

struct DecayCall {
    const tgm_decay_attn_desc *d;
    int64_t ld_q, ld_k, ld_v, ld_o, ld_dq, ld_dk, ld_dv;
    DecayRun run;   // the sequences, decays and sizes
    bool divided, ordered;
    hipStream_t s;
};

template <class T> tgm_status_t go(const DecayRun &r, int what, hipStream_t s)
{
    return std::is_same_v<T, float>  ? decay_f32(r, what, s)
           : std::is_same_v<T, bf16> ? decay_bf16(r, what, s)
                                     : decay_f16(r, what, s);
}

// The work space's parts, and the order.
tgm_status_t begin(const DecayCall &c, DecayRun *r, char *work, DecayBytes b)
{
    r->states = (float *)work;
    if (c.ordered) {
        TGM_LAUNCH(k_decay_order, dim3(1), dim3(kOrderThreads), 0, c.s, *r,
                   (int32_t *)(work + b.states));
        r->order = (int32_t *)(work + b.states);
    }
    return TGM_OK;
}
// The states behind the cells, into r.states.
template <class T> tgm_status_t states(const DecayCall &c, const DecayRun &r)
{
    if (!c.divided)
        return TGM_OK;
    TGM_TRY_STATUS(go<T>(r, 0, c.s));
    const bool by_sequence = decay_by_sequence(r);
    const int64_t n = by_sequence ? r.a.S : r.all_cells, size = (int64_t)r.a.p * r.a.r;
    const bool many = n * r.a.H * cdiv(size, 512) > 4096;
    const int64_t z = cdiv(size, many ? 2048 : 512);
    const dim3 grid(across(n, (int32_t)(r.a.H * z)), (uint32_t)r.a.H, (uint32_t)z);
    if (by_sequence && many)
        TGM_LAUNCH((k_decay_walk<true, 8>), grid, dim3(256), 0, c.s, r);
    else if (by_sequence)
        TGM_LAUNCH((k_decay_walk<true, 2>), grid, dim3(256), 0, c.s, r);
    else if (many)
        TGM_LAUNCH((k_decay_walk<false, 8>), grid, dim3(256), 0, c.s, r);
    else
        TGM_LAUNCH((k_decay_walk<false, 2>), grid, dim3(256), 0, c.s, r);
    return TGM_OK;
}

template <class T>
tgm_status_t forward(const DecayCall &c, const void *q, const void *k, const void *v,
                     const float *first, void *o, float *last, char *work, DecayBytes b)
{
    DecayRun r = c.run;
    DecayArgs &a = r.a;
    const int32_t share = a.H / c.d->H_kv;
    a.x = DecayIn{q, c.ld_q, 1}, a.y = DecayIn{k, c.ld_k, share};
    a.z = DecayIn{v, c.ld_v, share};
    a.p = c.d->d_k, a.r = c.d->d_v, a.out = o, a.ld_out = c.ld_o;
    a.first = first, a.last = last, a.lag0 = 1, a.c_y = 1.f, a.c_out = c.d->scale;
    TGM_TRY_STATUS(begin(c, &r, work, b));
    TGM_TRY_STATUS(states<T>(c, r));
    return go<T>(r, 1, c.s);
}

template <class T>
tgm_status_t backward(const DecayCall &c, const void *q, const void *k, const void *v,
                      const float *first, const void *dO, const float *dlast, void *dq, void *dk,
                      void *dv, float *dfirst, char *work, DecayBytes b)
{
    const tgm_decay_attn_desc *d = c.d;
    const int32_t share = d->H / d->H_kv;
    const DecayIn iq{q, c.ld_q, 1}, ik{k, c.ld_k, share}, iv{v, c.ld_v, share}, io{dO, c.ld_o, 1};
    DecayRun r = c.run;
    DecayArgs &a = r.a;
    TGM_TRY_STATUS(begin(c, &r, work, b));
    if (dq) {
        a.y = ik, a.z = iv, a.p = d->d_k, a.r = d->d_v;
        a.first = first, a.lag0 = 1, a.c_y = 1.f, a.c_out = d->scale;
        TGM_TRY_STATUS(states<T>(c, r));
        a.x = io, a.y = iv, a.z = ik, a.p = d->d_v, a.r = d->d_k, a.turned = 1;
        a.out = dq, a.ld_out = c.ld_dq;
        TGM_TRY_STATUS(go<T>(r, 1, c.s));
    }
    if (!dk && !dv && !dfirst)
        return TGM_OK;
    // the others run against the first one's order
    a.rev = !c.run.a.rev, a.first = dlast, a.lag0 = 0, a.c_y = d->scale, a.c_out = 1.f;
    a.x = ik, a.y = iq, a.z = io, a.p = d->d_k, a.r = d->d_v, a.turned = 0;
    TGM_TRY_STATUS(states<T>(c, r));
    float *part = (float *)(work + b.states + b.order);
    auto results = [&](void *out, int32_t width, int64_t ld) -> tgm_status_t {
        if (share == 1 || !out) {
            a.out = out, a.ld_out = ld;
            return go<T>(r, 1, c.s);
        }
        a.out = part, a.ld_out = (int64_t)a.H * width;
        TGM_TRY_STATUS(go<T>(r, 2, c.s));
        const int64_t ids = cdiv(a.rows, kSharedRows) + a.S;
        const dim3 grid((uint32_t)std::min<int64_t>(ids, 1 << 16));
        if (width % 4 == 0)
            TGM_LAUNCH((k_decay_shared<T, 4>), grid, dim3(256), 0, c.s, part, a, d->H_kv, share,
                       width, ld, (T *)out);
        else
            TGM_LAUNCH((k_decay_shared<T, 1>), grid, dim3(256), 0, c.s, part, a, d->H_kv, share,
                       width, ld, (T *)out);
        return TGM_OK;
    };
    if (dv || dfirst) {
        a.last = dfirst, a.lag1 = 1;
        TGM_TRY_STATUS(results(dv, d->d_v, c.ld_dv));
    }
    if (dk) {
        a.x = iv, a.y = io, a.z = iq, a.p = d->d_v, a.r = d->d_k, a.turned = 1;
        a.last = nullptr;
        TGM_TRY_STATUS(results(dk, d->d_k, c.ld_dk));
    }
    return TGM_OK;
}

bool decay_sizes(int64_t rows, int32_t S, int32_t H, int32_t H_kv, int32_t d_k, int32_t d_v,
                 int32_t dtype)
{
    return rows >= 0 && rows <= (int64_t)1 << 30 && S >= 0 && H >= 1 && H <= 4096 && H_kv >= 1 &&
           H % H_kv == 0 && d_k >= 1 && d_k <= kDecayMaxD && d_v >= 1 && d_v <= kDecayMaxD &&
           wide_type(dtype);
}

tgm_status_t decay_call(const tgm_decay_attn_desc *d, const float *decay, const int64_t *offsets,
                        const int32_t *length, void *stream, DecayCall *c)
{
    if (!d || !decay_sizes(d->rows, d->S, d->H, d->H_kv, d->d_k, d->d_v, d->dtype) || !decay)
        return TGM_EINVAL;
    c->d = d, c->s = as_stream(stream);
    c->ld_q = stride_of(d->ld_q, (int64_t)d->H * d->d_k);
    c->ld_k = stride_of(d->ld_k, (int64_t)d->H_kv * d->d_k);
    c->ld_v = stride_of(d->ld_v, (int64_t)d->H_kv * d->d_v);
    c->ld_o = stride_of(d->ld_o, (int64_t)d->H * d->d_v);
    c->ld_dq = stride_of(d->ld_dq, (int64_t)d->H * d->d_k);
    c->ld_dk = stride_of(d->ld_dk, (int64_t)d->H_kv * d->d_k);
    c->ld_dv = stride_of(d->ld_dv, (int64_t)d->H_kv * d->d_v);
    for (int64_t ld : {c->ld_q, c->ld_k, c->ld_v, c->ld_o, c->ld_dq, c->ld_dk, c->ld_dv})
        if (ld < 0)
            return TGM_EINVAL;
    DecayArgs &a = c->run.a;
    a.decay = decay, a.offsets = offsets, a.length = length;
    a.rows = d->rows, a.S = d->S, a.H = d->H, a.rev = d->reverse != 0;
    return TGM_OK;
}
// Padded sequences divide the rows.
tgm_status_t decay_lengths(DecayCall *c)
{
    DecayArgs &a = c->run.a;
    if (!a.offsets) {
        if (a.S == 0 ? a.rows != 0 : a.rows % a.S != 0)
            return TGM_EINVAL;
        a.L = a.S ? a.rows / a.S : 0;
    }
    const DecayPlan p = decay_plan(a.rows, a.S, a.H, a.offsets != nullptr);
    c->run.cell = p.cell, c->run.cells = p.padded_cells, c->run.ids = p.ids;
    c->run.all_cells = p.cells;
    c->divided = p.divided;
    c->ordered = (a.offsets || a.length) && order_bytes(p, a.rows, a.S, a.H);
    c->run.brief = decay_brief(a.rows, a.S, a.offsets != nullptr);
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

template <class T, int VEC, int LANES>
tgm_status_t go_step(const DecayCall &c, const void *q, const void *k, const void *v,
                     const int32_t *slots, const int32_t *n_rows, float *state, void *o)
{
    tgm_decay_attn_desc d = *c.d;
    d.ld_q = c.ld_q, d.ld_k = c.ld_k, d.ld_v = c.ld_v, d.ld_o = c.ld_o;
    TGM_LAUNCH((k_decay_step<T, VEC, LANES>),
               dim3(across(d.rows, d.H), (uint32_t)d.H), dim3(256), 0, c.s, (const T *)q,
               (const T *)k, (const T *)v, c.run.a.decay, slots, n_rows, state, (T *)o, d);
    return TGM_OK;
}
// As few lanes as hold a row of the state, for as many rows at once, and 16 bytes a lane where
// rows of d_v columns keep vectors whole: us of 2,048 states of 8 heads of 64 x 32, 64 x 64 and
// 64 x 128 bf16
//     8, 16 and 32 lanes of 4 columns      44  108  223
//     32 lanes of 4 columns                61  128  223
//     32, 64 and 128 lanes of 1 column     50  147  290
template <class T>
tgm_status_t pick_step(const DecayCall &c, const void *q, const void *k, const void *v,
                       const int32_t *slots, const int32_t *n_rows, float *state, void *o)
{
    const int r = c.d->d_v;
    if (r % 4 == 0)
        return r <= 32 ? go_step<T, 4, 8>(c, q, k, v, slots, n_rows, state, o)
             : r <= 64 ? go_step<T, 4, 16>(c, q, k, v, slots, n_rows, state, o)
                       : go_step<T, 4, 32>(c, q, k, v, slots, n_rows, state, o);
    return r <= 32 ? go_step<T, 1, 32>(c, q, k, v, slots, n_rows, state, o)
         : r <= 64 ? go_step<T, 1, 64>(c, q, k, v, slots, n_rows, state, o)
                   : go_step<T, 1, 128>(c, q, k, v, slots, n_rows, state, o);
}

}  // namespace

extern "C" tgm_status_t tgm_decay_attn_work_bytes(int64_t rows, int32_t S, int32_t H, int32_t H_kv,
                                                  int32_t d_k, int32_t d_v, int32_t dtype,
                                                  int32_t backward, size_t *bytes)
{
    if (!bytes || !decay_sizes(rows, S, H, H_kv, d_k, d_v, dtype))
        return TGM_EINVAL;
    const DecayBytes b = decay_bytes(rows, S, H, d_k, d_v);
    *bytes = b.states + b.order +
             (backward && H != H_kv ? whole((size_t)rows * H * std::max(d_k, d_v) * 4) : 0);
    return TGM_OK;
}

extern "C" tgm_status_t tgm_decay_attn(const tgm_decay_attn_desc *d, const void *q, const void *k,
                                       const void *v, const float *decay, const int64_t *offsets,
                                       const int32_t *length, const float *state, void *o,
                                       float *state_last, void *work, size_t work_bytes,
                                       void *stream)
{
    DecayCall c{};
    TGM_TRY_STATUS(decay_call(d, decay, offsets, length, stream, &c));
    TGM_TRY_STATUS(decay_lengths(&c));
    if ((d->rows && (!q || !k || !v || !o)) || (state && state == state_last))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_decay_attn_work_bytes(d->rows, d->S, d->H, d->H_kv, d->d_k, d->d_v, d->dtype,
                                             0, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    if (d->S == 0)   // packed rows of no sequence
        return TGM_OK;
    const DecayBytes b = decay_bytes(d->rows, d->S, d->H, d->d_k, d->d_v);
    char *w = (char *)work;
    switch (d->dtype) {
    case TGM_F32: return forward<float>(c, q, k, v, state, o, state_last, w, b);
    case TGM_BF16: return forward<bf16>(c, q, k, v, state, o, state_last, w, b);
    default: return forward<f16>(c, q, k, v, state, o, state_last, w, b);
    }
}

extern "C" tgm_status_t tgm_decay_attn_backward(
    const tgm_decay_attn_desc *d, const void *q, const void *k, const void *v, const float *decay,
    const int64_t *offsets, const int32_t *length, const float *state, const void *dO,
    const float *dstate_last, void *dq, void *dk, void *dv, float *dstate, void *work,
    size_t work_bytes, void *stream)
{
    DecayCall c{};
    TGM_TRY_STATUS(decay_call(d, decay, offsets, length, stream, &c));
    TGM_TRY_STATUS(decay_lengths(&c));
    if ((d->rows && (!q || !k || !v || !dO)) || (dstate && dstate == dstate_last))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_decay_attn_work_bytes(d->rows, d->S, d->H, d->H_kv, d->d_k, d->d_v, d->dtype,
                                             1, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    if (d->S == 0)
        return TGM_OK;
    char *w = (char *)work;
    const DecayBytes b = decay_bytes(d->rows, d->S, d->H, d->d_k, d->d_v);
    switch (d->dtype) {
    case TGM_F32:
        return backward<float>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w, b);
    case TGM_BF16:
        return backward<bf16>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w, b);
    default:
        return backward<f16>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w, b);
    }
}

extern "C" tgm_status_t tgm_decay_attn_step(const tgm_decay_attn_desc *d, const void *q,
                                            const void *k, const void *v, const float *decay,
                                            const int32_t *slots, const int32_t *n_rows,
                                            float *state, void *o, void *stream)
{
    DecayCall c{};
    TGM_TRY_STATUS(decay_call(d, decay, nullptr, nullptr, stream, &c));
    if (d->rows && (!q || !k || !v || !state))
        return TGM_EINVAL;
    if (d->rows == 0)
        return TGM_OK;
    switch (d->dtype) {
    case TGM_F32: return pick_step<float>(c, q, k, v, slots, n_rows, state, o);
    case TGM_BF16: return pick_step<bf16>(c, q, k, v, slots, n_rows, state, o);
    default: return pick_step<f16>(c, q, k, v, slots, n_rows, state, o);
    }
}
