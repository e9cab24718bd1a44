// Gated linear recurrence along packed or padded sequences (tgm_scan), its
// gradient and its single-row form.
//
// h_t = a_t h_(t-1) + (1 - a_t) x_t is an affine map of h_(t-1), so the rows of
// a tile of 32 compose to h_out = P h_in + Q with P the product of the gates.
// Three launches: every tile's (P, Q), the state that enters every tile, and
// the rows themselves.  A wavefront takes one tile and 64 V channels (V
// neighbouring ones a lane) with all of the tile's loads in flight; the tiles
// run over the rows as they lie, whatever sequences they belong to, so uneven
// lengths cost nothing.  Bound by memory: the operator has to read g and x and
// write y once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq.h"

using namespace tgm;

namespace {

constexpr int kRows = 32;   // rows of a tile
constexpr int kWaves = 4;   // wavefronts (tiles) of a workgroup

// The sequences, and their rows' division into tiles: packed sequences share
// tiles of consecutive rows; padded ones have tiles of their own (`chunks` of
// them), or share one in whole sequences (`per` of them) where they are short.
struct Seqs {
    const int64_t *offsets;
    const int32_t *length;
    int64_t rows, L;
    int32_t S, per, chunks, rev;
    int64_t tiles;
};

struct Tile {
    int64_t p0;   // its first row in the scan's order
    int32_t n;    // rows
};

__device__ __forceinline__ Tile tile_at(const Seqs &q, int64_t k)
{
    int64_t lo, n;
    if (q.offsets) {
        const int64_t l0 = k * kRows;
        n = min((int64_t)kRows, q.rows - l0);
        lo = q.rev ? q.rows - l0 - n : l0;
    } else if (q.per) {
        const int64_t s = k * q.per;
        n = min((int64_t)q.per, q.S - s) * q.L;
        lo = s * q.L;
    } else {
        const int64_t s = k / q.chunks, l0 = (k - s * q.chunks) * kRows;
        n = min((int64_t)kRows, q.L - l0);
        lo = s * q.L + (q.rev ? q.L - l0 - n : l0);
    }
    return Tile{q.rev ? lo + n - 1 : lo, (int32_t)n};
}

// How many of the ascending offsets[0 .. S) are <= v, by one wavefront: a
// 64-ary search.  Whatever the offsets hold, it ends and stays in [0, S].
__device__ __forceinline__ int32_t count_le(const int64_t *__restrict__ off, int32_t S, int64_t v)
{
    const int lane = threadIdx.x & 63;
    int32_t lo = 0, hi = S;
    while (hi - lo > kWave) {
        const int32_t step = (hi - lo + kWave - 1) / kWave;
        const int64_t probe = (int64_t)lo + (int64_t)(lane + 1) * step - 1;
        const int c = __popcll(__ballot(probe < hi && off[probe] <= v));
        lo += c * step;
        hi = min(lo + step, hi);
    }
    const int64_t idx = (int64_t)lo + lane;
    return lo + __popcll(__ballot(idx < hi && off[idx] <= v));
}

// What a tile's rows are: lane r < 32 holds row r's sequence, the masks have a
// bit for each row that lies in a sequence, is its first and is its last (in
// the scan's order).
struct RowInfo {
    int32_t seq;
    uint32_t valid, first, last;
};

__device__ __forceinline__ RowInfo rows_of(const Seqs &q, const Tile &t)
{
    const int r = threadIdx.x & 31;
    const int64_t p = q.rev ? t.p0 - min(r, t.n - 1) : t.p0 + min(r, t.n - 1);
    int64_t begin, end;
    int32_t s;
    if (q.offsets) {
        const int64_t p1 = q.rev ? t.p0 - (t.n - 1) : t.p0, p2 = q.rev ? t.p0 : t.p0 + (t.n - 1);
        int32_t lo = count_le(q.offsets, q.S, p1) - 1;
        int32_t hi = max(lo, count_le(q.offsets, q.S, p2) - 1);
        while (lo < hi) {   // the last sequence that begins at or before p
            const int32_t mid = lo + (hi - lo + 1) / 2;
            if (q.offsets[mid] <= p)
                lo = mid;
            else
                hi = mid - 1;
        }
        s = lo;
        begin = s >= 0 ? q.offsets[s] : 0;
        end = s >= 0 ? q.offsets[s + 1] : 0;
        if (q.length && s >= 0)
            end = min(end, begin + max(0, q.length[s]));
    } else {
        s = (int32_t)(p / q.L);
        begin = s * q.L;
        end = begin + (q.length ? min(q.L, (int64_t)max(0, q.length[s])) : q.L);
    }
    const bool in = r < t.n && s >= 0 && p >= begin && p < end;
    const bool head = in && p == begin, tail = in && p == end - 1;
    RowInfo i;
    i.seq = s;
    i.valid = (uint32_t)__ballot(in);
    i.first = (uint32_t)__ballot(q.rev ? tail : head);
    i.last = (uint32_t)__ballot(q.rev ? head : tail);
    return i;
}

// The gates.  exp(-|g|) lies in (0, 1], so neither gate loses its small values
// and infinite g gives 0 and 1.
struct Gate {
    float a, i;   // sigmoid(g), sigmoid(-g)
};
__device__ __forceinline__ Gate gate_of(float g)
{
    const float e = __expf(-fabsf(g));
    const float big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
    return g > 0.f ? Gate{big, small} : Gate{small, big};
}

// This lane's channels: block b of `width` ones, V a lane; the last lane of a
// block of odd width moves back by one and repeats its neighbour's.  Lanes past
// the block repeat its last one without storing: every lane stays active, so
// that another's sequence can be read from it.
struct Lane {
    int32_t ch;
    bool on;
};
template <int V> __device__ __forceinline__ Lane lane_at(int32_t D, int32_t width, int b)
{
    const int32_t c0 = b * width, c1 = min(D, c0 + width);
    const int32_t ch = c0 + V * (int32_t)(threadIdx.x & 63);
    return Lane{min(ch, c1 - V), ch < c1};
}

struct ScanArgs {
    Seqs q;
    int32_t D, width;
    const void *g, *x, *dy;
    const float *h0;      // backward: also the forward's
    const float *last;    // backward: dh_last
    void *y, *dg, *dx;
    float *h_last;        // backward: dh0
    float *carry;         // states entering the tiles
    float *agg;           // (P, Q) of the tiles; P = -1: nothing of the state before gets through
    float *back;          // backward: what is handed back into the tiles
    int64_t ld_g, ld_x, ld_y, ld_dg, ld_dx;
};

__device__ __forceinline__ int64_t tile_index()
{
    return ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kWaves + (threadIdx.x >> 6);
}

// Tile k's (P, Q) for every channel.  BWD: of the adjoint, whose rows run the
// other way: c_out = a (dy + c_in).
template <class T, int V, bool BWD>
__global__ __launch_bounds__(64 * kWaves) void k_scan_agg(ScanArgs A)
{
    const int64_t k = tile_index();
    if (k >= A.q.tiles)
        return;
    const Tile t = tile_at(A.q, k);
    const Lane c = lane_at<V>(A.D, A.width, blockIdx.z);
    const T *g = (const T *)A.g + c.ch, *x = (const T *)(BWD ? A.dy : A.x) + c.ch;
    const int64_t ld_x = BWD ? A.ld_y : A.ld_x;
    const RowInfo in = rows_of(A.q, t);
    float P[V], Q[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        P[v] = 1.f, Q[v] = 0.f;
    if (in.valid) {
#pragma unroll 8
        for (int j = 0; j < kRows; ++j) {
            const int r = BWD ? kRows - 1 - j : j;
            if (!((in.valid >> r) & 1))
                continue;
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            const Pack<T, V> pg = load_pack<T, V>(g + p * A.ld_g);
            const Pack<T, V> px = load_pack<T, V>(x + p * ld_x);
            const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
            const bool cut = ((BWD ? in.last : in.first) >> r) & 1;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate G = gate_of(to_f32(pg.v[v]));
                const float u = to_f32(px.v[v]);
                if (cut) {
                    const float *from = BWD ? A.last : A.h0;
                    P[v] = -1.f;
                    Q[v] = from ? from[(int64_t)s * A.D + c.ch + v] : 0.f;
                }
                P[v] = P[v] < 0.f ? -1.f : P[v] * G.a;
                Q[v] = BWD ? G.a * (u + Q[v]) : fmaf(G.a, Q[v], G.i * u);
            }
        }
    }
    if (c.on) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float *o = A.agg + (k * A.D + c.ch + v) * 2;
            o[0] = P[v];
            o[1] = Q[v];
        }
    }
}

// The state that enters each tile, one thread a channel.
template <bool BWD> __global__ __launch_bounds__(64) void k_scan_carry(ScanArgs A)
{
    const int32_t ch = blockIdx.x * 64 + threadIdx.x;
    if (ch >= A.D)
        return;
    float *to = BWD ? A.back : A.carry;
    float h = 0.f;
#pragma unroll 8
    for (int64_t j = 0; j < A.q.tiles; ++j) {
        const int64_t k = BWD ? A.q.tiles - 1 - j : j;
        const float *o = A.agg + (k * A.D + ch) * 2;
        const float P = o[0], Q = o[1];
        to[k * A.D + ch] = h;
        h = P < 0.f ? Q : fmaf(P, h, Q);
    }
}

template <class T, int V> __global__ __launch_bounds__(64 * kWaves) void k_scan_rows(ScanArgs A)
{
    const int64_t k = tile_index();
    if (k >= A.q.tiles)
        return;
    const Tile t = tile_at(A.q, k);
    const Lane c = lane_at<V>(A.D, A.width, blockIdx.z);
    const T *g = (const T *)A.g + c.ch, *x = (const T *)A.x + c.ch;
    T *y = (T *)A.y + c.ch;
    const RowInfo in = rows_of(A.q, t);
    if (!in.valid)
        return;
    float h[V];
    if (in.valid & ~in.first & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = A.carry[k * A.D + c.ch + v];
    }
    // y may be g or x: every row is loaded before the first one is stored
    Pack<T, V> pg[kRows], px[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((in.valid >> r) & 1) {
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            pg[r] = load_pack<T, V>(g + p * A.ld_g);
            px[r] = load_pack<T, V>(x + p * A.ld_x);
        }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((in.valid >> r) & 1) {
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
            Pack<T, V> py;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t at = (int64_t)s * A.D + c.ch + v;
                if ((in.first >> r) & 1)
                    h[v] = A.h0 ? A.h0[at] : 0.f;
                const Gate G = gate_of(to_f32(pg[r].v[v]));
                h[v] = fmaf(G.a, h[v], G.i * to_f32(px[r].v[v]));
                py.v[v] = from_f32<T>(h[v]);
                if (((in.last >> r) & 1) && A.h_last && c.on)
                    A.h_last[at] = h[v];
            }
            if (c.on)
                store_pack(y + p * A.ld_y, py);
        }
}

template <class T, int V>
__global__ __launch_bounds__(64 * kWaves) void k_scan_rows_bwd(ScanArgs A)
{
    const int64_t k = tile_index();
    if (k >= A.q.tiles)
        return;
    const Tile t = tile_at(A.q, k);
    const Lane c = lane_at<V>(A.D, A.width, blockIdx.z);
    const T *g = (const T *)A.g + c.ch, *x = (const T *)A.x + c.ch, *dy = (const T *)A.dy + c.ch;
    T *dg = (T *)A.dg + c.ch, *dx = (T *)A.dx + c.ch;
    const RowInfo in = rows_of(A.q, t);
    if (!in.valid)
        return;
    float h[V], e[V];
    if (in.valid & ~in.first & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = A.carry[k * A.D + c.ch + v];
    }
    const int32_t end = t.n - 1;
    if ((in.valid & ~in.last) >> end & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            e[v] = A.back[k * A.D + c.ch + v];
    }
    Pack<T, V> pg[kRows], px[kRows], py[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((in.valid >> r) & 1) {
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            pg[r] = load_pack<T, V>(g + p * A.ld_g);
            px[r] = load_pack<T, V>(x + p * A.ld_x);
            py[r] = load_pack<T, V>(dy + p * A.ld_y);
        }
    // the states before the rows again, as the forward call formed them
    float before[kRows][V];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((in.valid >> r) & 1) {
            const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if ((in.first >> r) & 1)
                    h[v] = A.h0 ? A.h0[(int64_t)s * A.D + c.ch + v] : 0.f;
                before[r][v] = h[v];
                const Gate G = gate_of(to_f32(pg[r].v[v]));
                h[v] = fmaf(G.a, h[v], G.i * to_f32(px[r].v[v]));
            }
        }
#pragma unroll
    for (int r = kRows - 1; r >= 0; --r)
        if ((in.valid >> r) & 1) {
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
            Pack<T, V> og, ox;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t at = (int64_t)s * A.D + c.ch + v;
                if ((in.last >> r) & 1)
                    e[v] = A.last ? A.last[at] : 0.f;
                e[v] += to_f32(py[r].v[v]);
                const Gate G = gate_of(to_f32(pg[r].v[v]));
                const float d = G.i * e[v];
                ox.v[v] = from_f32<T>(d);
                e[v] *= G.a;
                og.v[v] = from_f32<T>((before[r][v] - to_f32(px[r].v[v])) * G.a * d);
                if (((in.first >> r) & 1) && A.h_last && c.on)
                    A.h_last[at] = e[v];
            }
            if (c.on) {
                store_pack(dg + p * A.ld_dg, og);
                store_pack(dx + p * A.ld_dx, ox);
            }
        }
}

// A sequence without rows ends with the state that it starts from (backward:
// hands its end's gradient to its start): a wavefront looks 64 of them over.
__global__ __launch_bounds__(256) void k_scan_empty(Seqs q, int32_t D,
                                                    const float *__restrict__ from,
                                                    float *__restrict__ to)
{
    const int lane = threadIdx.x & 63;
    const int64_t waves = (int64_t)gridDim.x * 4;
    for (int64_t s0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 64; s0 < q.S;
         s0 += waves * 64) {
        const int64_t s = s0 + lane;
        bool none = false;
        if (s < q.S) {
            none = q.offsets ? q.offsets[s + 1] <= q.offsets[s] : q.L == 0;
            none |= q.length && q.length[s] <= 0;
        }
        for (uint64_t m = __ballot(none); m; m &= m - 1) {
            const int64_t at = (s0 + __ffsll((unsigned long long)m) - 1) * D;
            for (int32_t c = lane; c < D; c += 64)
                to[at + c] = from ? from[at + c] : 0.f;
        }
    }
}

template <class T, int V>
__global__ __launch_bounds__(256) void k_scan_step(const T *g, const T *x,
                                                   const int32_t *__restrict__ slots,
                                                   const int32_t *__restrict__ n_rows,
                                                   float *state, T *y, int32_t rows, int32_t S,
                                                   int32_t D, int32_t per, int64_t ld_g,
                                                   int64_t ld_x, int64_t ld_y)
{
    // `per` vectors of V channels a row; the last one moves back to the row's end
    const int64_t n = (int64_t)rows_in_use(rows, n_rows) * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
        const int64_t p = i / per;
        const int32_t e = (int32_t)(i - p * per) * V, ch = min(e, D - V), skip = e - ch;
        const int64_t s = slots ? (int64_t)slots[p] : p;
        const bool in = s >= 0 && s < S;
        const Pack<T, V> pg = load_pack<T, V>(g + p * ld_g + ch);
        const Pack<T, V> px = load_pack<T, V>(x + p * ld_x + ch);
        float *h = state + s * D + ch;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v >= skip) {   // a channel of the state has one owner: it is updated in place
                const Gate G = gate_of(to_f32(pg.v[v]));
                const float u = fmaf(G.a, in ? h[v] : 0.f, G.i * to_f32(px.v[v]));
                if (in)
                    h[v] = u;
                if (y)
                    y[p * ld_y + ch + v] = from_f32<T>(u);
            }
    }
}

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int kMaxD = 65536;

// Fills q's division into tiles; false where the sequences cannot be.
bool divide(Seqs *q, bool packed)
{
    q->L = 0, q->per = 0, q->chunks = 0, q->tiles = 0;
    if (q->rows < 0 || q->rows >= kMaxRows || q->S < 0)
        return false;
    if (packed) {
        q->tiles = cdiv(q->rows, kRows);
        return true;
    }
    if (q->S == 0)
        return q->rows == 0;
    if (q->rows % q->S)
        return false;
    q->L = q->rows / q->S;
    if (q->L == 0)
        return true;
    if (q->L <= kRows) {
        q->per = (int32_t)(kRows / q->L);
        q->tiles = cdiv(q->S, q->per);
    } else {
        q->chunks = (int32_t)cdiv(q->L, kRows);
        q->tiles = (int64_t)q->S * q->chunks;
    }
    return true;
}

int64_t most_tiles(int64_t rows, int32_t S)
{
    Seqs q{};
    q.rows = rows, q.S = S;
    int64_t n = divide(&q, true) ? q.tiles : -1;
    if (n >= 0 && divide(&q, false))
        n = std::max(n, q.tiles);
    return n;
}

// Channels a wavefront takes: pairs where there are over 64, as long as every
// block of an odd number of them keeps two.
int pick_width(int32_t D, int want, int32_t *width)
{
    if (want == 2 && D > 64) {
        const int32_t blocks = (int32_t)cdiv(D, 128);
        const int32_t w = round_up((int32_t)cdiv(D, blocks), 2);
        const int32_t rest = D - w * (blocks - 1);
        if (rest >= 2) {
            *width = w;
            return 2;
        }
    }
    *width = 64;
    return 1;
}

dim3 tile_grid(const ScanArgs &A)
{
    const int64_t wg = cdiv(A.q.tiles, kWaves), x = std::min<int64_t>(wg, 1 << 20);
    return dim3((uint32_t)x, (uint32_t)cdiv(wg, x), (uint32_t)cdiv(A.D, A.width));
}

template <class T, int V, bool BWD> tgm_status_t launch_scan(const ScanArgs &A, hipStream_t s)
{
    if (!A.q.tiles)
        return TGM_OK;
    const dim3 grid = tile_grid(A);
    if (!A.q.per) {   // short padded sequences lie inside their tiles
        TGM_LAUNCH((k_scan_agg<T, V, BWD>), grid, dim3(64 * kWaves), 0, s, A);
        TGM_LAUNCH((k_scan_carry<BWD>), dim3((uint32_t)cdiv(A.D, 64)), dim3(64), 0, s, A);
    }
    if (BWD)
        TGM_LAUNCH((k_scan_rows_bwd<T, V>), grid, dim3(64 * kWaves), 0, s, A);
    else
        TGM_LAUNCH((k_scan_rows<T, V>), grid, dim3(64 * kWaves), 0, s, A);
    return TGM_OK;
}

template <class T, bool BWD> tgm_status_t run_scan(ScanArgs A, hipStream_t s)
{
    // a lane of fp32 pairs would hold more rows than registers in the gradient
    const int V = pick_width(A.D, BWD && sizeof(T) == 4 ? 1 : 2, &A.width);
    return V == 2 ? launch_scan<T, 2, BWD>(A, s) : launch_scan<T, 1, BWD>(A, s);
}

tgm_status_t empties(const ScanArgs &A, const float *from, hipStream_t s)
{
    if (A.h_last && A.q.S && (A.q.offsets || A.q.length || A.q.L == 0))
        TGM_LAUNCH(k_scan_empty, dim3((uint32_t)std::min<int64_t>(cdiv(A.q.S, 256), 4096)),
                   dim3(256), 0, s, A.q, A.D, from, A.h_last);
    return TGM_OK;
}

tgm_status_t scan_args(const tgm_scan_desc *d, const void *g, const void *x,
                       const int64_t *offsets, const int32_t *length, const float *h0,
                       ScanArgs *A)
{
    if (!d || d->D < 1 || d->D > kMaxD || !wide_type(d->dtype))
        return TGM_EINVAL;
    A->q.offsets = offsets, A->q.length = length;
    A->q.rows = d->rows, A->q.S = d->S, A->q.rev = d->reverse != 0;
    if (!divide(&A->q, offsets != nullptr))
        return TGM_EINVAL;
    A->D = d->D;
    A->ld_g = stride_of(d->ld_g, d->D);
    A->ld_x = stride_of(d->ld_x, d->D);
    A->ld_y = stride_of(d->ld_y, d->D);
    A->ld_dg = stride_of(d->ld_dg, d->D);
    A->ld_dx = stride_of(d->ld_dx, d->D);
    if (A->ld_g < 0 || A->ld_x < 0 || A->ld_y < 0 || A->ld_dg < 0 || A->ld_dx < 0)
        return TGM_EINVAL;
    if (d->rows && (!g || !x))
        return TGM_EINVAL;
    A->g = g, A->x = x, A->h0 = h0;
    return TGM_OK;
}

// Splits the work space: the tiles' maps, and their states (`carry` or `back`).
tgm_status_t take_work(ScanArgs *A, void *work, size_t work_bytes, float **states)
{
    const size_t need = (size_t)A->q.tiles * A->D * 12;
    if (!need || A->q.per)
        return TGM_OK;
    if (!work || ((uintptr_t)work & 15))
        return TGM_EINVAL;
    if (work_bytes < need)
        return TGM_ESIZE;
    A->agg = (float *)work;
    if (!*states)
        *states = A->agg + (size_t)A->q.tiles * A->D * 2;
    return TGM_OK;
}

}  // namespace

extern "C" tgm_status_t tgm_scan_carry_rows(int64_t rows, int32_t S, int32_t packed, int64_t *n)
{
    Seqs q{};
    q.rows = rows, q.S = S;
    if (!n || !divide(&q, packed != 0))
        return TGM_EINVAL;
    *n = q.tiles;
    return TGM_OK;
}

extern "C" tgm_status_t tgm_scan_work_bytes(int64_t rows, int32_t D, int32_t S, size_t *bytes)
{
    const int64_t n = most_tiles(rows, S);
    if (!bytes || n < 0 || D < 1 || D > kMaxD)
        return TGM_EINVAL;
    *bytes = (size_t)n * D * 12;
    return TGM_OK;
}

extern "C" tgm_status_t tgm_scan(const tgm_scan_desc *d, const void *g, const void *x,
                                 const int64_t *offsets, const int32_t *length, const float *h0,
                                 void *y, float *h_last, float *carry, void *work,
                                 size_t work_bytes, void *stream)
{
    ScanArgs A{};
    TGM_TRY_STATUS(scan_args(d, g, x, offsets, length, h0, &A));
    if (d->rows && !y)
        return TGM_EINVAL;
    A.y = y, A.h_last = h_last, A.carry = carry;
    TGM_TRY_STATUS(take_work(&A, work, work_bytes, &A.carry));
    const hipStream_t s = as_stream(stream);
    TGM_TRY_STATUS(empties(A, h0, s));
    switch (d->dtype) {
    case TGM_F32: return run_scan<float, false>(A, s);
    case TGM_BF16: return run_scan<bf16, false>(A, s);
    default: return run_scan<f16, false>(A, s);
    }
}

extern "C" tgm_status_t tgm_scan_backward(const tgm_scan_desc *d, const void *g, const void *x,
                                          const int64_t *offsets, const int32_t *length,
                                          const float *h0, const float *carry, const void *dy,
                                          const float *dh_last, void *dg, void *dx, float *dh0,
                                          void *work, size_t work_bytes, void *stream)
{
    ScanArgs A{};
    TGM_TRY_STATUS(scan_args(d, g, x, offsets, length, h0, &A));
    if (d->rows && (!dy || !dg || !dx || !carry))
        return TGM_EINVAL;
    A.dy = dy, A.dg = dg, A.dx = dx, A.last = dh_last, A.h_last = dh0;
    A.carry = const_cast<float *>(carry);   // read only: the states go to `back`
    TGM_TRY_STATUS(take_work(&A, work, work_bytes, &A.back));
    const hipStream_t s = as_stream(stream);
    TGM_TRY_STATUS(empties(A, dh_last, s));
    switch (d->dtype) {
    case TGM_F32: return run_scan<float, true>(A, s);
    case TGM_BF16: return run_scan<bf16, true>(A, s);
    default: return run_scan<f16, true>(A, s);
    }
}

extern "C" tgm_status_t tgm_scan_step(const tgm_scan_desc *d, const void *g, const void *x,
                                      const int32_t *slots, const int32_t *n_rows, float *state,
                                      void *y, void *stream)
{
    if (!d || d->rows < 0 || d->rows >= kMaxRows || d->S < 0 || d->D < 1 || d->D > kMaxD ||
        !wide_type(d->dtype))
        return TGM_EINVAL;
    const int64_t ld_g = stride_of(d->ld_g, d->D), ld_x = stride_of(d->ld_x, d->D),
                  ld_y = stride_of(d->ld_y, d->D);
    if (ld_g < 0 || ld_x < 0 || ld_y < 0 || (d->rows && (!g || !x)) || (d->S && !state))
        return TGM_EINVAL;
    if (d->rows == 0)
        return TGM_OK;
    const hipStream_t s = as_stream(stream);
    auto go = [&](auto t, auto v) -> tgm_status_t {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        const int32_t per = (int32_t)cdiv(d->D, V);
        const int64_t wg = std::min<int64_t>(cdiv(d->rows * per, 256), 1 << 16);
        TGM_LAUNCH((k_scan_step<T, V>), dim3((uint32_t)wg), dim3(256), 0, s, (const T *)g,
                   (const T *)x, slots, n_rows, state, (T *)y, (int32_t)d->rows, d->S, d->D, per,
                   ld_g, ld_x, ld_y);
        return TGM_OK;
    };
    using One = std::integral_constant<int, 1>;
    using Four = std::integral_constant<int, 4>;
    const bool one = d->D < 4;
    switch (d->dtype) {
    case TGM_F32: return one ? go(float{}, One{}) : go(float{}, Four{});
    case TGM_BF16: return one ? go(bf16{}, One{}) : go(bf16{}, Four{});
    default: return one ? go(f16{}, One{}) : go(f16{}, Four{});
    }
}
