// Gated linear recurrence along packed or padded sequences (tgm_scan), its
// gradient and its single-row form.
//
// h_t = a_t h_(t-1) + (1 - a_t) x_t is an affine map of h_(t-1), so the rows of
// a tile of 32 compose to h_out = P h_in + Q with P the product of the gates,
// and tiles compose likewise.  One pass over the data: a wavefront takes one
// tile and 64 V channels (V neighbouring ones a lane), a workgroup 8 tiles in a
// row; rows stay in registers between the tile's map and its states, so g and x
// are read once and y is written once, which is what bounds the operator.
// Between workgroups the states go along a chain (below).  The tiles run over
// the rows as they lie, whatever sequences they belong to, so uneven lengths
// cost nothing.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq.h"

using namespace tgm;

namespace {

constexpr int kRows = 32;   // rows of a tile
constexpr int kWaves = 8;   // wavefronts (tiles) of a workgroup

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
    int32_t D, width, blocks;   // channels, those of a wavefront, wavefronts for a row
    int32_t groups;             // workgroups along the rows
    const void *g, *x, *dy;
    const float *h0;      // backward: also the forward's
    const float *last;    // backward: dh_last
    void *y, *dg, *dx;
    float *h_last;        // backward: dh0
    float *carry;         // states entering the tiles (may be null in the forward)
    uint64_t *maps, *states;    // [groups x D]: the chain's words
    int32_t *ticket;            // [blocks]
    int64_t ld_g, ld_x, ld_y, ld_dg, ld_dx;
};

// ---------------------------------------------------------------- the chain
// A map (P, Q) is one 64-bit word, P in the upper half: a word is written and
// read whole, so no other ordering is needed.  P = -1 stands for a map that
// ignores the state before (a sequence begins inside it), all bits set for a
// word that is not there yet (a computed NaN never has them all set).
//
// Workgroups take their places in the rows' order by a counter as they start.
// The first of each channel block's chain is its runner: it composes the
// others' maps in order and hands every workgroup the state before its rows,
// 32 words a load.  A workgroup writes its map without waiting for anyone, and
// the runner waits only for the lowest place whose map is missing, which a
// workgroup that has started holds or the next one to start will hold; so
// every wait ends, however few workgroups run at once.
constexpr uint64_t kAbsent = ~(uint64_t)0;

__device__ __forceinline__ uint64_t word_of(float P, float Q)
{
    const uint32_t p = P != P ? 0x7fc00000u : __float_as_uint(P);
    return (uint64_t)p << 32 | __float_as_uint(Q);
}
__device__ __forceinline__ uint64_t word_load(const uint64_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void word_store(uint64_t *p, uint64_t w)
{
    __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float upper(uint64_t w) { return __uint_as_float((uint32_t)(w >> 32)); }
__device__ __forceinline__ float lower(uint64_t w) { return __uint_as_float((uint32_t)w); }

// (P, Q) after (p, q): the map of both.
__device__ __forceinline__ void compose(float &P, float &Q, float p, float q)
{
    Q = p < 0.f ? q : fmaf(p, Q, q);
    P = p < 0.f || P < 0.f ? -1.f : P * p;
}

__device__ void run_chain(const ScanArgs &A, int b)
{
    constexpr int kAhead = 32;
    const int32_t c0 = b * A.width, c1 = min(A.D, c0 + A.width);
    const int32_t ch = c0 + (int32_t)threadIdx.x;
    if ((int)(threadIdx.x & ~63u) + c0 >= c1)   // one wavefront for every 64 channels
        return;
    const uint64_t *maps = A.maps + min(ch, c1 - 1);
    uint64_t *states = A.states + min(ch, c1 - 1);
    float h = 0.f;
    for (int32_t done = 0; done < A.groups;) {
        uint64_t w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            w[i] = word_load(maps + (int64_t)min(done + i, A.groups - 1) * A.D);
        const int32_t from = done;
        bool ready = true;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            ready = ready && __all(w[i] != kAbsent);
            if (ready && from + i < A.groups) {
                word_store(states + (int64_t)(from + i) * A.D, word_of(-1.f, h));
                const float p = upper(w[i]);
                h = p < 0.f ? lower(w[i]) : fmaf(p, h, lower(w[i]));
                ++done;
            }
        }
        if (done == from)
            __builtin_amdgcn_s_sleep(2);
    }
}

// This workgroup's place and channel block; false: it was a runner and is done.
__device__ __forceinline__ bool take_place(const ScanArgs &A, int &place, int &b)
{
    __shared__ int32_t t;
    b = (int)(blockIdx.x % (uint32_t)A.blocks);
    place = (int)(blockIdx.x / (uint32_t)A.blocks);
    if (!A.ticket)
        return true;
    if (threadIdx.x == 0)
        t = __hip_atomic_fetch_add(A.ticket + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    place = t - 1;
    if (place < 0) {
        run_chain(A, b);
        return false;
    }
    return true;
}

// The state before this wavefront's tile, from its and its workgroup's maps:
// `need` where its first row continues a sequence.  P, Q: the tile's map.
template <int V>
__device__ __forceinline__ void enter(const ScanArgs &A, int place, const Lane &c, bool need,
                                      const float (&P)[V], const float (&Q)[V], float (&h)[V])
{
    __shared__ f2 maps[kWaves][64 * V];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int v = 0; v < V; ++v)
        maps[w][lane * V + v] = f2{P[v], Q[v]};
    __syncthreads();
    float p[V], q[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        p[v] = 1.f, q[v] = 0.f;
    for (int u = 0; u < w; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const f2 m = maps[u][lane * V + v];
            compose(p[v], q[v], m.x, m.y);
        }
    if (A.ticket && w == kWaves - 1 && c.on) {   // the workgroup's map, as soon as it is known
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float ap = p[v], aq = q[v];
            compose(ap, aq, P[v], Q[v]);
            word_store(A.maps + (int64_t)place * A.D + c.ch + v, word_of(ap, aq));
        }
    }
    if (!need)
        return;
    float before[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        before[v] = 0.f;
    // a sequence that begins in the workgroup before this tile cuts every channel alike
    if (A.ticket && place > 0 && __any(p[0] >= 0.f || p[0] != p[0])) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint64_t *at = A.states + (int64_t)place * A.D + c.ch + v;
            uint64_t s = word_load(at);
            while (__any(s == kAbsent)) {
                __builtin_amdgcn_s_sleep(1);
                s = word_load(at);
            }
            before[v] = lower(s);
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        h[v] = p[v] < 0.f ? q[v] : fmaf(p[v], before[v], q[v]);
}

// ---------------------------------------------------------------- the passes
// ALONE: no sequence leaves its tile (short padded ones).
template <class T, int V, bool ALONE>
__global__ __launch_bounds__(64 * kWaves) void k_scan(ScanArgs A)
{
    int place, b;
    if (!take_place(A, place, b))
        return;
    const int64_t k = (int64_t)place * kWaves + (threadIdx.x >> 6);
    const bool some = k < A.q.tiles;
    if (ALONE && !some)
        return;
    const Tile t = tile_at(A.q, some ? k : 0);
    const Lane c = lane_at<V>(A.D, A.width, b);
    const T *g = (const T *)A.g + c.ch, *x = (const T *)A.x + c.ch;
    T *y = (T *)A.y + c.ch;
    RowInfo in = rows_of(A.q, t);
    if (!some)
        in.valid = in.first = in.last = 0;
    // y may be g or x: every row is loaded before the first one is stored
    Pack<T, V> pg[kRows], px[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((in.valid >> r) & 1) {
            const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
            pg[r] = load_pack<T, V>(g + p * A.ld_g);
            px[r] = load_pack<T, V>(x + p * A.ld_x);
        }
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        h[v] = 0.f;
    if constexpr (!ALONE) {
        float P[V], Q[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            P[v] = 1.f, Q[v] = 0.f;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if ((in.valid >> r) & 1) {
                if ((in.first >> r) & 1) {
                    const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        P[v] = -1.f;
                        Q[v] = A.h0 ? A.h0[(int64_t)s * A.D + c.ch + v] : 0.f;
                    }
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Gate G = gate_of(to_f32(pg[r].v[v]));
                    P[v] = P[v] < 0.f ? -1.f : P[v] * G.a;
                    Q[v] = fmaf(G.a, Q[v], G.i * to_f32(px[r].v[v]));
                }
            }
        const bool need = in.valid & ~in.first & 1;
        enter<V>(A, place, c, need, P, Q, h);
        if (need && A.carry && c.on) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                A.carry[k * A.D + c.ch + v] = h[v];
        }
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

// The gradient's pass, tiles and rows in the other order: a row hands a e back
// to the one before it, with e = dy + what it was handed itself.
template <class T, int V, bool ALONE>
__global__ __launch_bounds__(64 * kWaves) void k_scan_bwd(ScanArgs A)
{
    int place, b;
    if (!take_place(A, place, b))
        return;
    const int64_t k = A.q.tiles - 1 - ((int64_t)place * kWaves + (threadIdx.x >> 6));
    const bool some = k >= 0;
    if (ALONE && !some)
        return;
    const Tile t = tile_at(A.q, some ? k : 0);
    const Lane c = lane_at<V>(A.D, A.width, b);
    const T *g = (const T *)A.g + c.ch, *x = (const T *)A.x + c.ch, *dy = (const T *)A.dy + c.ch;
    T *dg = (T *)A.dg + c.ch, *dx = (T *)A.dx + c.ch;
    RowInfo in = rows_of(A.q, t);
    if (!some)
        in.valid = in.first = in.last = 0;
    float h[V], e[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        h[v] = e[v] = 0.f;
    if (in.valid & ~in.first & 1) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = A.carry[k * A.D + c.ch + v];
    }
    Pack<T, V> pg[kRows], py[kRows];
    float d[kRows][V];   // x, then (h_(t-1) - x) a (1 - a)
    {
        Pack<T, V> px[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if ((in.valid >> r) & 1) {
                const int64_t p = A.q.rev ? t.p0 - r : t.p0 + r;
                pg[r] = load_pack<T, V>(g + p * A.ld_g);
                px[r] = load_pack<T, V>(x + p * A.ld_x);
                py[r] = load_pack<T, V>(dy + p * A.ld_y);
            }
        // the states before the rows again, as the forward call formed them
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if ((in.valid >> r) & 1) {
                const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if ((in.first >> r) & 1)
                        h[v] = A.h0 ? A.h0[(int64_t)s * A.D + c.ch + v] : 0.f;
                    const Gate G = gate_of(to_f32(pg[r].v[v]));
                    const float u = to_f32(px[r].v[v]);
                    d[r][v] = (h[v] - u) * (G.a * G.i);
                    h[v] = fmaf(G.a, h[v], G.i * u);
                }
            }
    }
    if constexpr (!ALONE) {
        float P[V], Q[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            P[v] = 1.f, Q[v] = 0.f;
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r)
            if ((in.valid >> r) & 1) {
                if ((in.last >> r) & 1) {
                    const int32_t s = __builtin_amdgcn_readlane(in.seq, r);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        P[v] = -1.f;
                        Q[v] = A.last ? A.last[(int64_t)s * A.D + c.ch + v] : 0.f;
                    }
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Gate G = gate_of(to_f32(pg[r].v[v]));
                    P[v] = P[v] < 0.f ? -1.f : P[v] * G.a;
                    Q[v] = G.a * (to_f32(py[r].v[v]) + Q[v]);
                }
            }
        const bool need = ((in.valid & ~in.last) >> (t.n - 1)) & 1;
        enter<V>(A, place, c, need, P, Q, e);
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
                ox.v[v] = from_f32<T>(G.i * e[v]);
                og.v[v] = from_f32<T>(d[r][v] * e[v]);
                e[v] *= G.a;
                if (((in.first >> r) & 1) && A.h_last && c.on)
                    A.h_last[at] = e[v];
            }
            if (c.on) {
                store_pack(dg + p * A.ld_dg, og);
                store_pack(dx + p * A.ld_dx, ox);
            }
        }
}

// Before a pass: no word of the chain is there and no place is taken; and a
// sequence without rows ends with the state that it starts from (backward:
// hands its end's gradient to its start), which a wavefront does for 64 of them.
__global__ __launch_bounds__(256) void k_scan_begin(Seqs q, int32_t D,
                                                    const float *__restrict__ from, float *to,
                                                    uint64_t *words, int64_t n, int32_t *ticket,
                                                    int32_t blocks)
{
    const int64_t threads = (int64_t)gridDim.x * 256, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = id; i < n; i += threads)
        words[i] = kAbsent;
    if (ticket && id < blocks)
        ticket[id] = 0;
    if (!to)
        return;
    const int lane = threadIdx.x & 63;
    for (int64_t s0 = id - lane; s0 < q.S; s0 += threads) {
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

constexpr int64_t kMaxRows = ((int64_t)1 << 30) + 1;
constexpr int64_t kMaxGrid = ((int64_t)1 << 32) / (64 * kWaves);   // threads of a launch: 32 bits
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

template <class T, int V, bool BWD> tgm_status_t launch_scan(const ScanArgs &A, hipStream_t s)
{
    // a runner more for every chain
    const dim3 grid((uint32_t)(((int64_t)A.groups + (A.ticket ? 1 : 0)) * A.blocks));
    const dim3 block(64 * kWaves);
    if (BWD) {
        if (A.q.per)
            TGM_LAUNCH((k_scan_bwd<T, V, true>), grid, block, 0, s, A);
        else
            TGM_LAUNCH((k_scan_bwd<T, V, false>), grid, block, 0, s, A);
    } else {
        if (A.q.per)
            TGM_LAUNCH((k_scan<T, V, true>), grid, block, 0, s, A);
        else
            TGM_LAUNCH((k_scan<T, V, false>), grid, block, 0, s, A);
    }
    return TGM_OK;
}

// Lays the chain out in the work space: maps and states, [groups x D] words
// each, and the places' counters.
size_t chain_bytes(int64_t groups, int64_t D) { return (size_t)groups * D * 16 + 2048 * 4; }

template <class T, bool BWD>
tgm_status_t run_scan(ScanArgs A, void *work, size_t work_bytes, hipStream_t s)
{
    // a lane of fp32 pairs would hold more rows than registers in the gradient
    const int V = pick_width(A.D, BWD && sizeof(T) == 4 ? 1 : 2, &A.width);
    A.blocks = (int32_t)cdiv(A.D, A.width);
    A.groups = (int32_t)cdiv(A.q.tiles, kWaves);
    if (((int64_t)A.groups + 1) * A.blocks >= kMaxGrid)
        return TGM_EINVAL;
    if (A.q.rows) {
        if (!work || ((uintptr_t)work & 15))
            return TGM_EINVAL;
        if (work_bytes < chain_bytes(cdiv(most_tiles(A.q.rows, A.q.S), kWaves), A.D))
            return TGM_ESIZE;
    }
    int64_t words = 0;
    if (!A.q.per && A.groups > 1) {
        words = (int64_t)A.groups * A.D * 2;
        A.maps = (uint64_t *)work;
        A.states = A.maps + words / 2;
        A.ticket = (int32_t *)(A.maps + words);
    }
    const bool empty = A.h_last && A.q.S && (A.q.offsets || A.q.length || A.q.L == 0);
    if (words || empty) {
        const int64_t wg = std::min<int64_t>(cdiv(std::max<int64_t>(words, A.q.S), 256), 2048);
        TGM_LAUNCH(k_scan_begin, dim3((uint32_t)wg), dim3(256), 0, s, A.q, A.D,
                   BWD ? A.last : A.h0, empty ? A.h_last : nullptr, A.maps, words, A.ticket,
                   A.blocks);
    }
    if (!A.q.tiles)
        return TGM_OK;
    return V == 2 ? launch_scan<T, 2, BWD>(A, s) : launch_scan<T, 1, BWD>(A, s);
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
    *bytes = n ? chain_bytes(cdiv(n, kWaves), D) : 0;
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
    const hipStream_t s = as_stream(stream);
    switch (d->dtype) {
    case TGM_F32: return run_scan<float, false>(A, work, work_bytes, s);
    case TGM_BF16: return run_scan<bf16, false>(A, work, work_bytes, s);
    default: return run_scan<f16, false>(A, work, work_bytes, s);
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
    A.carry = const_cast<float *>(carry);   // read only here
    const hipStream_t s = as_stream(stream);
    switch (d->dtype) {
    case TGM_F32: return run_scan<float, true>(A, work, work_bytes, s);
    case TGM_BF16: return run_scan<bf16, true>(A, work, work_bytes, s);
    default: return run_scan<f16, true>(A, work, work_bytes, s);
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
