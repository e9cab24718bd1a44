// Gated linear recurrence along packed or padded sequences (tgm_scan), its
// gradient and its single-row form.
//
// h_t = a_t h_(t-1) + (1 - a_t) x_t is an affine map of h_(t-1), so the rows of
// a tile of 32 compose to h_out = P h_in + Q with P the product of the gates,
// and tiles compose likewise.  One pass over the data: a wavefront takes one
// tile and 64 V channels (V neighbouring ones a lane), a workgroup several tiles in a
// row; rows stay in registers between the tile's map and its states, so g and x
// are read once and y is written once, which is what bounds the operator.
// Between workgroups the states go along a chain (below).  The tiles run over
// the rows as they lie, whatever sequences they belong to, so uneven lengths
// cost nothing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "scan_places.h"
#include "seq.h"

using namespace tgm;

namespace {

constexpr int kRows = 32;   // rows of a tile
// Wavefronts (tiles) of a workgroup, so that two or more workgroups' rows fit a
// CU's registers: 128 a lane forward, 256 in the gradient.  One history of
// 1,000,003 rows of 128 bf16 channels: 224 us with 8 (361 with 4: twice the maps
// for its chain, 293 with 10: one workgroup a CU); the gradient of 131,072 rows
// of 512: 203 us with 4, 246 with 8 (one workgroup a CU).
constexpr int kWaves = 8, kWavesBwd = 4;

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

__device__ __forceinline__ int64_t row_at(const Seqs &q, const Tile &t, int r)
{
    return q.rev ? t.p0 - r : t.p0 + r;
}

__device__ __forceinline__ RowInfo info_of(const Seqs &q, int32_t s, int64_t p, int64_t begin,
                                           int64_t end, bool in)
{
    in = in && p >= begin && p < end;
    const bool head = in && p == begin, tail = in && p == end - 1;
    RowInfo i;
    i.seq = s;
    i.valid = (uint32_t)__ballot(in);
    i.first = (uint32_t)__ballot(q.rev ? tail : head);
    i.last = (uint32_t)__ballot(q.rev ? head : tail);
    return i;
}

__device__ __forceinline__ RowInfo rows_padded(const Seqs &q, const Tile &t)
{
    const int r = threadIdx.x & 31;
    const int64_t p = row_at(q, t, min(r, t.n - 1));
    const int32_t s = (int32_t)(p / q.L);
    const int64_t begin = s * q.L;
    const int64_t end = begin + (q.length ? min(q.L, (int64_t)max(0, q.length[s])) : q.L);
    return info_of(q, s, p, begin, end, r < t.n);
}

__device__ __forceinline__ RowInfo rows_packed(const Seqs &q, const Tile &t)
{
    const int lane = threadIdx.x & 63, r = lane & 31;
    const int64_t p = row_at(q, t, min(r, t.n - 1));
    const int64_t p1 = q.rev ? t.p0 - (t.n - 1) : t.p0, p2 = q.rev ? t.p0 : t.p0 + (t.n - 1);
    const int32_t n = count_le(q.offsets, q.S, p1);   // sequences that begin up to the tile
    // the beginnings after those, 64 of them in the lanes, and the one before
    const bool at = lane <= q.S - n;
    const int64_t next = at ? q.offsets[n + lane] : INT64_MAX;
    const int64_t here = n > 0 ? q.offsets[n - 1] : 0;
    int32_t s;
    int64_t begin, end;
    if (__popcll(__ballot(lane < q.S - n && next <= p2)) < 64) {
        int c = 0;   // those up to p
#pragma unroll
        for (int step = 32; step; step >>= 1) {
            const int64_t v = __shfl(next, c + step - 1);
            c += c + step - 1 < q.S - n && v <= p ? step : 0;
        }
        s = n - 1 + c;
        const int64_t before = __shfl(next, max(c - 1, 0));
        begin = c ? before : here;
        end = __shfl(next, c);
    } else {   // more than 64 begin inside the tile: empty ones among them
        int32_t lo = n - 1, hi = max(lo, count_le(q.offsets, q.S, p2) - 1);
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
    }
    if (q.length && s >= 0)
        end = min(end, begin + max(0, q.length[s]));
    return info_of(q, s, p, begin, end, r < t.n && s >= 0);
}

// The gates.  exp(-|g|) lies in (0, 1], so neither gate loses its small values
// and infinite g gives 0 and 1.  A gate below 2^-126, where the exponential ends, is 0.
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
// This lane's elements of a row of a dense array.
template <class T> __device__ __forceinline__ T *in_row(T *X, int64_t p, int64_t ld, int32_t ch)
{
    return X + p * ld + (uint32_t)ch;
}
// A tile's rows of a matrix: one 64-bit base, the wavefront's, and an offset of
// 32 bits for row r of the scan's order (32 rows of less than 2^24 elements).
template <class T> struct Rows {
    char *base;
    uint32_t first, step;
    __device__ __forceinline__ Rows(const void *X, const Seqs &q, const Tile &t, int64_t ld)
    {
        const int64_t lo = q.rev ? t.p0 - (t.n - 1) : t.p0;
        base = (char *)const_cast<void *>(X) + lo * ld * (int64_t)sizeof(T);
        const uint32_t b = (uint32_t)ld * (uint32_t)sizeof(T);
        first = q.rev ? (uint32_t)(t.n - 1) * b : 0u;
        step = q.rev ? 0u - b : b;
    }
    __device__ __forceinline__ T *at(int r, int32_t ch) const
    {
        return reinterpret_cast<T *>(base + (first + (uint32_t)r * step)) + (uint32_t)ch;
    }
};
__device__ __forceinline__ int wave_id()
{
    return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
}

// A row's elements in a lane, as they came: between the passes over a tile they
// stay packed, which the compiler is kept from undoing (unpacked 16-bit
// elements take twice the registers).
template <class T, int V> struct Held {
    Pack<T, V> v;
    __device__ __forceinline__ float at(int i) const { return to_f32(v.v[i]); }
    __device__ __forceinline__ void keep() {}
};
template <class T> struct HeldPair {
    uint32_t w;
    __device__ __forceinline__ float at(int i) const
    {
        const uint16_t u = (uint16_t)(w >> (16 * i));
        return to_f32(__builtin_bit_cast(T, u));
    }
    __device__ __forceinline__ void keep() { asm volatile("" : "+v"(w)); }
};
template <> struct Held<f16, 2> : HeldPair<f16> {};
template <> struct Held<bf16, 2> : HeldPair<bf16> {};
template <class T, int V> __device__ __forceinline__ Held<T, V> hold(const T *p)
{
    using HeldT = Held<T, V>;
    return __builtin_bit_cast(HeldT, load_pack<T, V>(p));
}

// The states that a tile's sequences start from (or hand back from), one for
// each row in `mask`: the first two are loaded ahead, before the rows are gone
// through; the others, in tiles of short sequences, when met.
template <int V> struct Starts {
    float v0[V], v1[V];
    __device__ __forceinline__ void load(const float *X, uint32_t mask, int32_t seq, int32_t D,
                                         int32_t ch)
    {
        one(v0, X, mask, seq, D, ch);
        one(v1, X, mask & (mask - 1), seq, D, ch);
    }
    // that of row r of the mask
    __device__ __forceinline__ void get(float (&h)[V], const float *X, uint32_t mask, int r,
                                        int32_t seq, int32_t D, int32_t ch) const
    {
        const int j = __builtin_popcount(mask & ((1u << r) - 1));
        float other[V];
#pragma unroll
        for (int u = 0; u < V; ++u)
            other[u] = 0.f;
        if (j >= 2)
            one(other, X, mask & ~((1u << r) - 1), seq, D, ch);
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const float a = v0[u], b = v1[u];
            h[u] = j == 0 ? a : j == 1 ? b : other[u];
        }
    }

private:
    static __device__ __forceinline__ void one(float (&to)[V], const float *X, uint32_t mask,
                                               int32_t seq, int32_t D, int32_t ch)
    {
#pragma unroll
        for (int u = 0; u < V; ++u)
            to[u] = 0.f;
        if (X && mask) {
            const float *x = in_row(X, __builtin_amdgcn_readlane(seq, __builtin_ctz(mask)), D, ch);
#pragma unroll
            for (int u = 0; u < V; ++u)
                to[u] = x[u];
        }
    }
};

struct ScanArgs {
    Seqs q;
    int32_t D, width, blocks;   // channels, those of a wavefront, wavefronts for a row
    int32_t groups;             // workgroups along the rows
    uint32_t tasks;             // workgroups for those and for the chains
    int32_t spare;              // workgroups for the sequences without rows
    bool backward;
    const void *g, *x, *dy;
    const float *h0;      // backward: also the forward's
    const float *last;    // backward: dh_last
    void *y, *dg, *dx;
    float *h_last;        // backward: dh0
    float *carry;         // states entering the tiles (may be null in the forward)
    uint64_t *maps, *states;    // [groups x D]: the chain's words
    int32_t *ticket;            // [kMaxRunners] tasks taken; null without a chain
    int64_t ld_g, ld_x, ld_y, ld_dg, ld_dx;
};

// ---------------------------------------------------------------- the chain
// A map (P, Q) is one 64-bit word, P in the upper half: a word is written and
// read whole, so no other ordering is needed.  P = -1 stands for a map that
// ignores the state before (a sequence begins inside it), all bits set for a
// word that is not there yet (a computed NaN never has them all set).
//
// Workgroups take their tasks in the rows' order by a counter as they start.  The
// first are runners: each composes the maps of a chain (64 channels') in order and hands
// every workgroup the state before its rows.  A workgroup writes its map without
// waiting for anyone, and what it waits for itself comes from places below its own
// and from its runner, which have all started.  A runner waits for places that may not
// have; the order of the tasks (scan_places.h) bounds how many do so at once, and so
// every wait ends.
//
// P is zero where a gate is, and nowhere else: a product that falls below the smallest
// number is kLeast instead, so that an infinite state stays infinite (zero times it is
// NaN) wherever its rows fall into tiles.
constexpr float kLeast = 0x1p-149f;
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

// (P, Q) after (p, q): the map of both, but for the product, which lift() makes kLeast
// where it is zero and `low`, the lowest p of all (1 before the first), is not.
__device__ __forceinline__ void compose(float &P, float &Q, float &low, float p, float q)
{
    Q = p < 0.f ? q : fmaf(p, Q, q);
    P = p < 0.f || P < 0.f ? -1.f : P * p;
    low = fminf(low, p);
}
__device__ __forceinline__ float lift(float P, float low)
{
    return P == 0.f && low > 0.f ? kLeast : P;
}
// P of a tile, which the pass over its rows has only multiplied: where it is zero and
// no gate of the rows in `valid` is.  lowest(r, v): row r's gate, or what it grows with;
// is_zero(its lowest one): whether that gate is zero.
template <int V, class L, class Z>
__device__ __forceinline__ void lift_tile(float (&P)[V], uint32_t valid, L lowest, Z is_zero)
{
    if (__builtin_expect(!__any(P[0] == 0.f || P[V - 1] == 0.f), 1))
        return;
    float least[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        least[v] = INFINITY;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
        if ((valid >> r) & 1)
#pragma unroll
            for (int v = 0; v < V; ++v)
                least[v] = fminf(least[v], lowest(r, v));
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (P[v] == 0.f && !is_zero(least[v]))
            P[v] = kLeast;
}

// A runner takes 64 channels, `part` of block b.  Its wavefronts take a block of 16 maps
// each at a time: a block that is there is composed on its own, the state before each
// block comes from the maps of the blocks before it, and the states inside follow one
// by one: the same operations whichever words were there at which look, so results do
// not depend on timing.  With W = 1 a wavefront is a runner by itself.
template <int W> __device__ __forceinline__ void run_chain(const ScanArgs &A, int b, int part)
{
    constexpr int kBlock = 16;
    __shared__ f2 block[2][W][64];
    __shared__ int32_t there[2][W];
    const int lane = threadIdx.x & 63, u = W > 1 ? wave_id() : 0;
    const int32_t c0 = b * A.width + 64 * part, c1 = min(A.D, (b + 1) * A.width);
    const uint32_t ch = (uint32_t)min(c0 + lane, c1 - 1);
    float base = 0.f;             // the state before the first block not done
    int32_t at = 0, known = 0;    // the first map of that block; how many of it are done
    uint64_t w[kBlock];
    auto fetch = [&](uint64_t (&to)[kBlock], int32_t first) __attribute__((always_inline)) {
        const uint64_t *maps = A.maps + (int64_t)min(first, A.groups - 1) * A.D + ch;
        const int32_t left = max(1, min(kBlock, A.groups - first));
#pragma unroll
        for (int i = 0; i < kBlock; ++i)
            to[i] = word_load(maps + (uint64_t)((uint32_t)min(i, left - 1) * (uint32_t)A.D));
    };
    for (int turn = 0; at < A.groups; turn ^= 1) {
        const int32_t first = at + kBlock * u, left = min(kBlock, A.groups - first);
        fetch(w, first);
        uint32_t absent = 0;   // bit i: word i is not there for every lane
#pragma unroll
        for (int i = 0; i < kBlock; ++i)
            absent |= __ballot((uint32_t)(w[i] >> 32) == ~0u) ? 1u << i : 0u;
        const int n = left <= 0 ? 0 : absent ? min(left, __builtin_ctz(absent)) : left;
        f2 m[W];
        int32_t count[W];
        float P = 1.f, Q = 0.f, low = 1.f;
        if (n == kBlock)
#pragma unroll
            for (int i = 0; i < kBlock; ++i)
                compose(P, Q, low, upper(w[i]), lower(w[i]));
        P = lift(P, low);
        if constexpr (W == 1) {
            m[0] = f2{P, Q}, count[0] = n;
        } else {
            block[turn][u][lane] = f2{P, Q};
            if (lane == 0)
                there[turn][u] = n;
            lds_barrier();   // one a turn: two turns' words are apart
#pragma unroll
            for (int k = 0; k < W; ++k)
                m[k] = block[turn][k][lane], count[k] = there[turn][k];
        }
        float h = base;
        int32_t whole = 0, rest = 0;   // blocks there from the first on; of the one after
#pragma unroll
        for (int k = 0; k < W; ++k)
            if (whole == k) {
                rest = __builtin_amdgcn_readfirstlane(count[k]);
                if (rest == kBlock) {
                    ++whole;
                    rest = 0;
                    base = m[k].x < 0.f ? m[k].y : fmaf(m[k].x, base, m[k].y);
                    h = k < u ? base : h;
                }
            }
        if (u <= whole) {   // the state before this wavefront's block is known
            uint64_t *states = A.states + (int64_t)first * A.D + ch;
            const int done = u ? 0 : known;
            auto next = [&](int i) __attribute__((always_inline)) {
                const float p = upper(w[i]), q = lower(w[i]);
                h = p < 0.f ? q : fmaf(p, h, q);
            };
            auto hand = [&](int i) __attribute__((always_inline)) {
                word_store(states + (uint64_t)((uint32_t)i * (uint32_t)A.D), word_of(-1.f, h));
            };
            if (n == kBlock && !done) {
#pragma unroll
                for (int i = 0; i < kBlock; ++i) {
                    hand(i);
                    next(i);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kBlock; ++i)
                    if (i < n) {
                        if (i >= done)
                            hand(i);
                        next(i);
                    }
            }
        }
        if (!whole && rest <= known)
            __builtin_amdgcn_s_sleep(1);
        at += kBlock * whole;
        known = rest;
        if (at + rest >= A.groups)
            break;
    }
}

// A sequence without rows ends with the state that it starts from (backward: hands
// its end's gradient to its start): the workgroups past the tiles', a wavefront
// for 8 sequences at a time.
template <int W> __device__ void pass_on(const ScanArgs &A, int64_t wg)
{
    constexpr int kSeqs = 8;
    const float *from = A.backward ? A.last : A.h0;
    const int lane = threadIdx.x & 63;
    for (int64_t s0 = (wg * W + wave_id()) * kSeqs; s0 < A.q.S;
         s0 += (int64_t)A.spare * W * kSeqs) {
        const int64_t s = s0 + lane;
        bool none = false;
        if (lane < kSeqs && s < A.q.S) {
            none = A.q.offsets ? A.q.offsets[s + 1] <= A.q.offsets[s] : A.q.L == 0;
            none |= A.q.length && A.q.length[s] <= 0;
        }
        for (uint64_t m = __ballot(none); m; m &= m - 1) {
            const int64_t at = (s0 + __ffsll((unsigned long long)m) - 1) * A.D;
            for (int32_t c = lane; c < A.D; c += 64)
                A.h_last[at + c] = from ? from[at + c] : 0.f;
        }
    }
}

// This workgroup's place and channel block; false: it had another task, and is done.
template <int V, int W, bool ALONE>
__device__ __forceinline__ bool take_place(const ScanArgs &A, int &place, int &b)
{
    __shared__ int32_t t;
    if (blockIdx.x >= A.tasks) {
        pass_on<W>(A, blockIdx.x - A.tasks);
        return false;
    }
    b = (int)(blockIdx.x % (uint32_t)A.blocks);
    place = (int)(blockIdx.x / (uint32_t)A.blocks);
    if (ALONE || !A.ticket)
        return true;
    const ScanTasks all{A.blocks, A.groups, V, W};
    if (threadIdx.x == 0)
        t = __hip_atomic_fetch_add(A.ticket + (all.narrow() ? b : 0), 1, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    place = __builtin_amdgcn_readfirstlane(t) - V;
    if (all.narrow()) {
        if (place < 0)   // V runners
            run_chain<W>(A, b, place + V);
        return place >= 0;
    }
    const ScanTask task = wide_task(all, (uint32_t)(place + V));
    b = task.block, place = task.place;
    if (place < 0) {
        const int chain = (-1 - place) * W + wave_id();
        b += chain / V;
        if (b < min(A.blocks, task.block + all.deep()) &&
            b * A.width + 64 * (chain % V) < min(A.D, (b + 1) * A.width))
            run_chain<1>(A, b, chain % V);
        return false;
    }
    return true;
}

// The state before this wavefront's tile, from its and its workgroup's maps:
// `need` where its first row continues a sequence.  P, Q: the tile's map.
template <int V, int W>
__device__ __forceinline__ void enter(const ScanArgs &A, int place, const Lane &c, bool need,
                                      const float (&P)[V], const float (&Q)[V], float (&h)[V])
{
    __shared__ f2 maps[W][64 * V];
    __shared__ float state[64 * V];
    __shared__ bool wanted;
    const int lane = threadIdx.x & 63, w = wave_id();
#pragma unroll
    for (int v = 0; v < V; ++v)
        maps[w][lane * V + v] = f2{P[v], Q[v]};
    if (threadIdx.x == 0)
        wanted = need && A.ticket && place > 0;
    __syncthreads();
    float p[V], q[V], low[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        p[v] = 1.f, q[v] = 0.f, low[v] = 1.f;
    for (int u = 0; u < w; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const f2 m = maps[u][lane * V + v];
            compose(p[v], q[v], low[v], m.x, m.y);
        }
    if (A.ticket && w == W - 1 && c.on) {   // the workgroup's map, as soon as it is known
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float ap = p[v], aq = q[v], al = low[v];
            compose(ap, aq, al, P[v], Q[v]);
            word_store(A.maps + (int64_t)place * A.D + c.ch + v, word_of(lift(ap, al), aq));
        }
    }
    if (__builtin_amdgcn_readfirstlane((int)wanted)) {
        // One wavefront looks for the state: eight would take the memory's time.  Where a
        // sequence begins in the rows of the place before, its map has the state, without
        // the runner's doing: 4,000 short sequences, 44,001 rows of 100 fp32: 29.6 us forward
        // and 41 back, 33.9 and 48.6 without.
        if (w == 0) {
            const int64_t at = (int64_t)place * A.D + c.ch;
            const uint64_t *states = A.states + at, *before = A.maps + (at - A.D);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                uint64_t m = word_load(before + v), s = word_load(states + v);
                while (__any(s == kAbsent && !(upper(m) < 0.f))) {
                    __builtin_amdgcn_s_sleep(4);
                    if (__any(m == kAbsent))
                        m = word_load(before + v);
                    s = word_load(states + v);
                }
                if (upper(m) < 0.f)
                    s = m;
                state[lane * V + v] = lower(s);
            }
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = state[lane * V + v];
    }
    if (need)
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = p[v] < 0.f ? q[v] : fmaf(lift(p[v], low[v]), h[v], q[v]);
}

// ---------------------------------------------------------------- the passes
// ALONE: no sequence leaves its tile (short padded ones).  Bound by memory: 12,000 padded
// sequences of 10 rows, 100 fp32 channels (144 MB): 31 us, 4.6 TB/s; by the chain's hand-over
// besides where there is one: 1,000,003 rows of 128 bf16 (768 MB): 216 to 228 us, 3.4 TB/s;
// 131,072 of 512 (403 MB, and the carries): 126 us, 3.2 TB/s.
template <class T, int V, int W, bool ALONE>
__global__ __launch_bounds__(64 * W, 4) void k_scan(ScanArgs A)
{
    int place, b;
    if (!take_place<V, W, ALONE>(A, place, b))
        return;
    const int64_t k = (int64_t)place * W + wave_id();
    const bool some = k < A.q.tiles;
    if (ALONE && !some)
        return;
    const Tile t = tile_at(A.q, some ? k : 0);
    const Lane c = lane_at<V>(A.D, A.width, b);
    // All loads go out at once, without a branch between them: packed rows before
    // the search for their sequences; a padded row of no sequence is another one
    // again.  y may be g or x: every row is loaded before the first is stored.
    RowInfo in{};
    uint32_t wanted = ~0u >> (kRows - t.n);
    if (some && !A.q.offsets) {
        in = rows_padded(A.q, t);
        wanted = in.valid;
    }
    if (ALONE && !wanted)
        return;
    const int other = wanted ? __builtin_ctz(wanted) : 0;
    const Rows<const T> gs(A.g, A.q, t, A.ld_g), xs(A.x, A.q, t, A.ld_x);
    const Rows<T> ys(A.y, A.q, t, A.ld_y);
    Held<T, V> pg[kRows], px[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int from = (wanted >> r) & 1 ? r : other;
        pg[r] = hold<T, V>(gs.at(from, c.ch));
        px[r] = hold<T, V>(xs.at(from, c.ch));
    }
    if (some && A.q.offsets)
        in = rows_packed(A.q, t);
    Starts<V> starts;
    starts.load(A.h0, in.first, in.seq, A.D, c.ch);
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        h[v] = 0.f;
    // most tiles of long sequences are plain: no row of them begins or ends one
    const bool plain = in.valid == ~0u && !in.first && !in.last;
    // fp32 rows' registers hold the gate and (1 - a) x from here on; 16-bit ones have no
    // room for them and form the gates twice.  44,001 rows of 100: 27.7 us, 29.6 with them
    // formed twice.
    constexpr bool KEEP = !ALONE && sizeof(T) == 4;
    if constexpr (KEEP)
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gate G = gate_of(pg[r].at(v));
                pg[r].v.v[v] = G.a;
                px[r].v.v[v] *= G.i;
            }
    if constexpr (!ALONE) {
        float P[V], Q[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            P[v] = 1.f, Q[v] = 0.f;
        auto map = [&](auto is_plain) __attribute__((always_inline)) {
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if (is_plain || ((in.valid >> r) & 1)) {
                    if (!is_plain && ((in.first >> r) & 1))
                        starts.get(Q, A.h0, in.first, r, in.seq, A.D, c.ch);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        float a, entry;
                        if constexpr (KEEP) {
                            a = pg[r].at(v), entry = px[r].at(v);
                        } else {
                            const Gate G = gate_of(pg[r].at(v));
                            a = G.a, entry = G.i * px[r].at(v);
                        }
                        P[v] *= a;
                        Q[v] = fmaf(a, Q[v], entry);
                    }
                }
        };
        if (plain)
            map(std::true_type{});
        else
            map(std::false_type{});
        if (in.first)
#pragma unroll
            for (int v = 0; v < V; ++v)
                P[v] = -1.f;
        else
            lift_tile<V>(P, in.valid, [&](int r, int v) { return pg[r].at(v); },
                     [](float a) { return (KEEP ? a : gate_of(a).a) == 0.f; });
        const bool need = in.valid & ~in.first & 1;
        enter<V, W>(A, place, c, need, P, Q, h);
        if (need && A.carry && c.on) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                in_row(A.carry, k, A.D, c.ch)[v] = h[v];
        }
    }
    auto rows = [&](auto is_plain) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (is_plain || ((in.valid >> r) & 1)) {
                if (!is_plain && ((in.first >> r) & 1))
                    starts.get(h, A.h0, in.first, r, in.seq, A.D, c.ch);
                Pack<T, V> py;
                pg[r].keep(), px[r].keep();
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if constexpr (KEEP) {
                        h[v] = fmaf(pg[r].at(v), h[v], px[r].at(v));
                    } else {
                        const Gate G = gate_of(pg[r].at(v));
                        h[v] = fmaf(G.a, h[v], G.i * px[r].at(v));
                    }
                    py.v[v] = from_f32<T>(h[v]);
                }
                if (c.on)
                    store_pack(ys.at(r, c.ch), py);
                if (!is_plain && ((in.last >> r) & 1) && A.h_last && c.on) {
                    float *to = in_row(A.h_last, __builtin_amdgcn_readlane(in.seq, r), A.D, c.ch);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        to[v] = h[v];
                }
            }
    };
    if (plain)
        rows(std::true_type{});
    else
        rows(std::false_type{});
}

// The gradient's pass, tiles in the other order: a row hands a e back to the
// one before it, with e = dy + what it was handed itself.  Five rows a row where the
// pass forward has three, so half as many wavefronts fit a CU: 131,072 rows of 512 bf16
// (671 MB): 203 us, 3.3 TB/s.
template <class T, int V, int W, bool ALONE>
__global__ __launch_bounds__(64 * W, 2) void k_scan_bwd(ScanArgs A)
{
    int place, b;
    if (!take_place<V, W, ALONE>(A, place, b))
        return;
    const int64_t k = A.q.tiles - 1 - ((int64_t)place * W + wave_id());
    const bool some = k >= 0;
    if (ALONE && !some)
        return;
    const Tile t = tile_at(A.q, some ? k : 0);
    const Lane c = lane_at<V>(A.D, A.width, b);
    RowInfo in{};
    uint32_t wanted = ~0u >> (kRows - t.n);
    if (some && !A.q.offsets) {
        in = rows_padded(A.q, t);
        wanted = in.valid;
    }
    if (ALONE && !wanted)
        return;
    const int other = wanted ? __builtin_ctz(wanted) : 0;
    const Rows<const T> gs(A.g, A.q, t, A.ld_g), xs(A.x, A.q, t, A.ld_x), dys(A.dy, A.q, t, A.ld_y);
    const Rows<T> dgs(A.dg, A.q, t, A.ld_dg), dxs(A.dx, A.q, t, A.ld_dx);
    // kept between the passes: g, dy and (h_(t-1) - x) a; the gates are formed twice (kept,
    // they would take the registers of a third wavefront: 44,001 rows of 100 fp32, 46 us
    // where this takes 41)
    float d[kRows][V];
    float h[V], e[V], P[V], Q[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        h[v] = e[v] = Q[v] = 0.f, P[v] = 1.f;
    Starts<V> ends;
    Held<T, V> pg[kRows], px[kRows], py[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {   // as in k_scan
        const int from = (wanted >> r) & 1 ? r : other;
        pg[r] = hold<T, V>(gs.at(from, c.ch));
        px[r] = hold<T, V>(xs.at(from, c.ch));
        py[r] = hold<T, V>(dys.at(from, c.ch));
    }
    if (some && A.q.offsets)
        in = rows_packed(A.q, t);
    const bool plain = in.valid == ~0u && !in.first && !in.last;
    Starts<V> starts;
    starts.load(A.h0, in.first, in.seq, A.D, c.ch);
    ends.load(A.last, in.last, in.seq, A.D, c.ch);
    if (in.valid & ~in.first & 1) {
        const float *from = in_row(A.carry, k, A.D, c.ch);
#pragma unroll
        for (int v = 0; v < V; ++v)
            h[v] = from[v];
    }
    // the states before the rows again, as the forward call formed them, and
    // what the tile hands back: the sum over its first sequence's rows of dy
    // times the gates up to the row, and the end's share
    auto map = [&](auto is_plain) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (is_plain || ((in.valid >> r) & 1)) {
                if (!is_plain && ((in.first >> r) & 1))
                    starts.get(h, A.h0, in.first, r, in.seq, A.D, c.ch);
                const bool open = is_plain || !(in.last & ((1u << r) - 1));
                float end[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    end[v] = 0.f;
                if (!ALONE && !is_plain && open && ((in.last >> r) & 1))
                    ends.get(end, A.last, in.last, r, in.seq, A.D, c.ch);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Gate G = gate_of(pg[r].at(v));
                    const float u = px[r].at(v);
                    d[r][v] = (h[v] - u) * G.a;
                    h[v] = fmaf(G.a, h[v], G.i * u);
                    if (!ALONE && open) {
                        P[v] *= G.a;
                        Q[v] = fmaf(P[v], py[r].at(v) + end[v], Q[v]);
                    }
                }
            }
    };
    if (plain)
        map(std::true_type{});
    else
        map(std::false_type{});
    if constexpr (!ALONE) {
        // an infinite dy times a product that fell to zero
        if (__builtin_expect(__any((P[0] == 0.f && Q[0] != Q[0]) ||
                                   (P[V - 1] == 0.f && Q[V - 1] != Q[V - 1])), 0)) {
            const uint32_t open = in.valid & (in.last ^ (in.last - 1));   // up to the first end
#pragma unroll
            for (int v = 0; v < V; ++v)
                P[v] = 1.f, Q[v] = 0.f;
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if ((open >> r) & 1) {
                    float end[V];
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        end[v] = 0.f;
                    if ((in.last >> r) & 1)
                        ends.get(end, A.last, in.last, r, in.seq, A.D, c.ch);
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const float a = gate_of(pg[r].at(v)).a;
                        P[v] = fmaf(P[v], a, P[v] > 0.f && a > 0.f ? kLeast : 0.f);
                        Q[v] = fmaf(P[v], py[r].at(v) + end[v], Q[v]);
                    }
                }
        }
        if (in.last)
#pragma unroll
            for (int v = 0; v < V; ++v)
                P[v] = -1.f;
        else
            lift_tile<V>(P, in.valid, [&](int r, int v) { return pg[r].at(v); },
                     [](float g) { return gate_of(g).a == 0.f; });
        const bool need = ((in.valid & ~in.last) >> (t.n - 1)) & 1;
        enter<V, W>(A, place, c, need, P, Q, e);
    }
    auto rows = [&](auto is_plain) __attribute__((always_inline)) {
#pragma unroll
        for (int r = kRows - 1; r >= 0; --r)
            if (is_plain || ((in.valid >> r) & 1)) {
                if (!is_plain && ((in.last >> r) & 1))
                    ends.get(e, A.last, in.last, r, in.seq, A.D, c.ch);
                pg[r].keep(), py[r].keep();
                Pack<T, V> og, ox;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    e[v] += py[r].at(v);
                    const Gate G = gate_of(pg[r].at(v));
                    const float back = G.i * e[v];
                    ox.v[v] = from_f32<T>(back);
                    og.v[v] = from_f32<T>(d[r][v] * back);
                    e[v] *= G.a;
                }
                if (c.on) {
                    store_pack(dgs.at(r, c.ch), og);
                    store_pack(dxs.at(r, c.ch), ox);
                }
                if (!is_plain && ((in.first >> r) & 1) && A.h_last && c.on) {
                    float *to = in_row(A.h_last, __builtin_amdgcn_readlane(in.seq, r), A.D, c.ch);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        to[v] = e[v];
                }
            }
    };
    if (plain)
        rows(std::true_type{});
    else
        rows(std::false_type{});
}

// Before a pass with a chain: none of its words is there and no task is taken (5 us).
__global__ __launch_bounds__(256) void k_scan_begin(uint64_t *words, int64_t n, int32_t *ticket)
{
    const int64_t threads = (int64_t)gridDim.x * 256, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = id; i < n; i += threads)
        words[i] = kAbsent;
    if (id < kMaxRunners)
        ticket[id] = 0;
}

// One row of each slot's sequence, elementwise: bound by the launch (600 rows of 100: 4 us).
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

// Whether a launch has fewer than 2^32 threads: forward, with the runners and the workgroups
// for sequences without rows, and so in the gradient, whose workgroups are half as wide
// and at most twice as many.  T ceil(D / 64) <= 2^26 - 2^15 does in every type.
bool fits(int64_t tiles, int32_t blocks)
{
    return (cdiv(tiles, kWaves) + 2) * blocks + 256 < ((int64_t)1 << 32) / (64 * kWaves);
}
static_assert(kWaves == 2 * kWavesBwd, "");

int64_t most_tiles(int64_t rows, int32_t S)
{
    Seqs q{};
    q.rows = rows, q.S = S;
    int64_t n = divide(&q, true) ? q.tiles : -1;
    if (n >= 0 && divide(&q, false))
        n = std::max(n, q.tiles);
    return n;
}

// Channels a wavefront takes: one a lane of 32 bits; of 16 bits pairs where there are over
// 64, as long as every block of an odd number of them keeps two.  Pairs against single
// ones, bf16, forward and back, us: 131,072 x 512: 129 and 206, 147 and 214; 1,000,000 x
// 128: 220 and 374, 282 and 395.
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

template <class T, int V, int W, bool BWD>
tgm_status_t launch_scan(const ScanArgs &A, hipStream_t s)
{
    const dim3 grid(A.tasks + (uint32_t)A.spare), block(64 * W);
    if constexpr (BWD) {
        if (A.q.per)
            TGM_LAUNCH((k_scan_bwd<T, V, W, true>), grid, block, 0, s, A);
        else
            TGM_LAUNCH((k_scan_bwd<T, V, W, false>), grid, block, 0, s, A);
    } else {
        if (A.q.per)
            TGM_LAUNCH((k_scan<T, V, W, true>), grid, block, 0, s, A);
        else
            TGM_LAUNCH((k_scan<T, V, W, false>), grid, block, 0, s, A);
    }
    return TGM_OK;
}

// The chain in the work space: maps and states, [groups x D] words each, and the
// counters of tasks, with room to 8 KiB.
size_t chain_bytes(int64_t groups, int64_t D) { return (size_t)groups * D * 16 + 8192; }

template <class T, bool BWD>
tgm_status_t run_scan(ScanArgs A, void *work, size_t work_bytes, hipStream_t s)
{
    const int V = pick_width(A.D, sizeof(T) == 4 ? 1 : 2, &A.width);
    constexpr int W = BWD ? kWavesBwd : kWaves;
    A.blocks = (int32_t)cdiv(A.D, A.width);
    A.groups = (int32_t)cdiv(A.q.tiles, W);
    if (!fits(A.q.tiles, A.blocks))
        return TGM_EINVAL;
    if (A.q.rows) {
        if (!work || ((uintptr_t)work & 15))
            return TGM_EINVAL;
        if (work_bytes < chain_bytes(cdiv(most_tiles(A.q.rows, A.q.S), kWavesBwd), A.D))
            return TGM_ESIZE;
    }
    int64_t words = 0;
    if (!A.q.per && A.groups > 1) {
        words = (int64_t)A.groups * A.D * 2;
        A.maps = (uint64_t *)work;
        A.states = A.maps + words / 2;
        A.ticket = (int32_t *)(A.maps + words);
    }
    A.backward = BWD;
    A.tasks = (uint32_t)(words ? ScanTasks{A.blocks, A.groups, V, W}.all()
                               : (int64_t)A.groups * A.blocks);
    if (A.h_last && A.q.S && (A.q.offsets || A.q.length || A.q.L == 0))
        A.spare = (int32_t)std::min<int64_t>(cdiv(A.q.S, 8 * W), 256);
    if (words)
        TGM_LAUNCH(k_scan_begin, dim3((uint32_t)std::min<int64_t>(cdiv(words, 256), 1024)),
                   dim3(256), 0, s, A.maps, words, A.ticket);
    if (!A.q.tiles && !A.spare)
        return TGM_OK;
    if constexpr (sizeof(T) == 2)
        if (V == 2)
            return launch_scan<T, 2, W, BWD>(A, s);
    return launch_scan<T, 1, W, BWD>(A, s);
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
    // the fewest tiles and channel blocks of any call of this size
    if (!bytes || n < 0 || D < 1 || D > kMaxD ||
        !fits(cdiv(rows, kRows), (int32_t)cdiv(D, 128)))
        return TGM_EINVAL;
    *bytes = n ? chain_bytes(cdiv(n, kWavesBwd), D) : 0;
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
