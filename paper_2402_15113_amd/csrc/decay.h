// What the kernels of the linear attention with a decay for each head (tgm_decay_attn)
// share.
//
// The operator and each of its gradients is one recurrence over three matrices' rows,
//   S_t = a S_(t-1) + c_y y_t z_t^T,   out_t = c_out x_t S_t,
// along every sequence or against it:
//   o:   x, y, z = q, k, v            from the first state
//   dq:  x, y, z = do, v, k           from its transpose
//   dk:  x, y, z = v, do, q           backwards, from the transpose of the last state's gradient
//   dv:  x, y, z = k, q, do           backwards, from the last state's gradient
#pragma once

#include "seq.h"

namespace tgm {

constexpr int kDecayMaxD = 128;

// A matrix of rows and the head that head h of the recurrence reads: h / share.
struct DecayIn {
    const void *p;
    int64_t ld;
    int32_t share;
};

struct DecayArgs {
    DecayIn x, y, z;         // p, p and r columns a head
    void *out;               // null: states only
    int64_t ld_out;
    const float *decay;      // [H]: log a
    const int64_t *offsets;  // null: sequences of L rows
    const int32_t *length;
    const float *first;      // states [S x H x dk x dv] before the first rows; may be null
    float *last;             // states after the last ones; may be null
    int64_t rows, L;
    int32_t S, H, p, r;
    int32_t turned;          // the states in memory are S^T, [r x p]
    int32_t rev;             // from each sequence's last row to its first
    int32_t lag0;            // the first state's weight at the first row: a^lag0 (0 or 1)
    int32_t lag1;            // the last state is a^lag1 S (0 or 1)
    float c_y, c_out;
};

// Rows b .. e - 1 of sequence s; empty where its offsets make no sense.
struct DecaySeq {
    int64_t b, e;
};
__device__ __forceinline__ DecaySeq decay_seq(const DecayArgs &a, int32_t s)
{
    int64_t b, e;
    if (a.offsets) {
        b = min(max(a.offsets[s], (int64_t)0), a.rows);
        e = min(max(a.offsets[s + 1], b), a.rows);
    } else {
        b = s * a.L;
        e = b + a.L;
    }
    if (a.length)
        e = min(e, b + max(0, a.length[s]));
    return DecaySeq{b, e};
}

// Where a sequence begins, for the search below.
__device__ __forceinline__ int64_t decay_begin(const DecayArgs &a, int32_t s)
{
    return a.offsets ? min(max(a.offsets[s], (int64_t)0), a.rows) : s * a.L;
}

// The cell of C rows that row b (0 .. rows, at most 2^30) is in.
__device__ __forceinline__ int64_t decay_cell_of(int64_t b, int32_t C)
{
    return (uint32_t)b / (uint32_t)C;
}

// lo and how many sequences of lo .. hi - 1 have key(s) <= v, by one wavefront: a 64-ary search,
// whose last 256 are looked at together.  Keys ascend where the offsets make sense; whatever
// they hold, it ends and stays in [lo, hi].
template <class Key>
__device__ __forceinline__ int32_t decay_count(int32_t lo, int32_t hi, int64_t v, Key key)
{
    constexpr int LAST = 4;
    const int lane = threadIdx.x & 63;
    while (hi - lo > LAST * kWave) {
        const int32_t step = (int32_t)(((int64_t)hi - lo + kWave - 1) / kWave);
        const int64_t probe = (int64_t)lo + (int64_t)(lane + 1) * step - 1;
        const int c =
            __popcll(__ballot(probe < hi && key((int32_t)min(probe, (int64_t)hi - 1)) <= v));
        lo += c * step;
        hi = (int32_t)min((int64_t)lo + step, (int64_t)hi);
    }
    if (hi <= lo)
        return lo;
    int64_t k[LAST];
#pragma unroll
    for (int u = 0; u < LAST; ++u)
        k[u] = key((int32_t)min((int64_t)lo + u * kWave + lane, (int64_t)hi - 1));
    int32_t n = 0;
#pragma unroll
    for (int u = 0; u < LAST; ++u)
        n += __popcll(__ballot((int64_t)lo + u * kWave + lane < hi && k[u] <= v));
    return lo + n;
}

// The rows that sequence `s` has in cell `cell` of C consecutive rows: piece `id` of
// cdiv(rows, C) + S.  A path through cells and sequences, which goes to the next sequence
// or to the next cell at every step, meets every pair that has rows in common, and every
// sequence in the cell where it begins: sequence s begins at step cell(begin) + s, and these
// steps ascend.  No list of pieces has to be made, whatever the offsets on the device are.
struct DecayPiece {
    int32_t s;
    int64_t cell, lo, hi;   // hi <= lo: no rows
    DecaySeq q;
};
// The sequences whose first step may be the last one up to step `id`: lo .. hi - 1.  (A sequence's
// first step is its own number and at most as many cells more.)
struct DecaySteps {
    int32_t lo, hi;
};
__device__ __forceinline__ DecaySteps decay_steps(const DecayArgs &a, int64_t id, int32_t C)
{
    const int64_t cells = decay_cell_of(a.rows + C - 1, C);
    return DecaySteps{(int32_t)min(max(id - cells, (int64_t)0), (int64_t)a.S),
                      (int32_t)min(id + 1, (int64_t)a.S)};
}
// Sequence s's first step.
__device__ __forceinline__ int64_t decay_step_of(const DecayArgs &a, int32_t s, int32_t C)
{
    return decay_cell_of(decay_begin(a, s), C) + s;
}
// n sequences have begun at step id or before.
__device__ __forceinline__ DecayPiece decay_piece(const DecayArgs &a, int64_t id, int32_t C,
                                                  int32_t n)
{
    DecayPiece p{max(n - 1, 0), -1, 0, 0, {0, 0}};
    if (n < 1)   // before the first sequence
        return p;
    p.cell = id - p.s;
    p.q = decay_seq(a, p.s);
    p.lo = max(p.q.b, p.cell * C);
    p.hi = min(p.q.e, (p.cell + 1) * C);
    return p;
}
__device__ __forceinline__ DecayPiece decay_piece(const DecayArgs &a, int64_t id, int32_t C)
{
    const DecaySteps t = decay_steps(a, id, C);
    return decay_piece(a, id, C, decay_count(t.lo, t.hi, id, [&](int32_t s) {
                           return decay_step_of(a, s, C);
                       }));
}

struct DecayRun {
    DecayArgs a;
    float *states;      // [H x all_cells x dk x dv]: the state behind each cell's rows (in the
                        // recurrence's order) where a sequence goes on to the next cell
    int32_t cell;       // rows of a cell
    int64_t all_cells;
    int64_t cells;      // of a padded sequence, 0 for packed ones
    int64_t ids;        // pieces
    const int32_t *order;   // [ids], the pieces with rows, long ones first, then -1; may be null
    bool brief;         // sequences of few rows for the most part
};

// A sequence of no more than a cell's rows is one piece, which the cell that it begins in has.
__device__ __forceinline__ DecayPiece decay_whole(const DecayRun &r, DecayPiece p)
{
    if (p.q.e - p.q.b <= r.cell) {
        const bool here = decay_cell_of(p.q.b, r.cell) == p.cell;
        p.lo = here ? p.q.b : 0, p.hi = here ? p.q.e : 0;
    }
    return p;
}
__device__ __forceinline__ DecayPiece decay_padded_piece(const DecayRun &r, int64_t id)
{
    DecayPiece p;
    p.s = (int32_t)(id / r.cells), p.cell = id;
    p.q = decay_seq(r.a, p.s);
    const int64_t k = id - p.s * r.cells;
    p.lo = p.q.b + k * r.cell;
    p.hi = min(p.q.e, p.lo + r.cell);
    return p;
}
// Piece `id` of the sequences: whole sequences, and longer ones by cells.  Packed sequences
// share a grid of cells, padded ones have cells of their own.
__device__ __forceinline__ DecayPiece decay_piece_of(const DecayRun &r, int64_t id)
{
    return r.a.offsets ? decay_whole(r, decay_piece(r.a, id, r.cell)) : decay_padded_piece(r, id);
}
// The same by a single thread.
__device__ __forceinline__ DecayPiece decay_piece_alone(const DecayRun &r, int64_t id)
{
    if (!r.a.offsets)
        return decay_padded_piece(r, id);
    DecaySteps t = decay_steps(r.a, id, r.cell);
    while (t.lo < t.hi) {
        const int32_t mid = t.lo + (t.hi - t.lo) / 2;
        if (decay_step_of(r.a, mid, r.cell) <= id)
            t.lo = mid + 1;
        else
            t.hi = mid;
    }
    return decay_whole(r, decay_piece(r.a, id, r.cell, t.lo));
}
// The piece of cell `id` that goes on to the next cell (in the recurrence's order), if there is
// one: at most one sequence of more than a cell's rows has its last (backwards: first) row and
// the next.
__device__ __forceinline__ DecayPiece decay_piece_onward(const DecayRun &r, int64_t id)
{
    const DecayArgs &a = r.a;
    DecayPiece p;
    if (a.offsets) {
        const int64_t row = a.rev ? id * r.cell : min((id + 1) * r.cell, a.rows) - 1;
        const int32_t n =
            decay_count(0, a.S, row, [&](int32_t s) { return decay_begin(a, s); });
        p = DecayPiece{max(n - 1, 0), id, 0, 0, {0, 0}};
        if (n < 1)
            return p;
        p.q = decay_seq(a, p.s);
        p.lo = max(p.q.b, id * r.cell), p.hi = min(p.q.e, (id + 1) * r.cell);
    } else {
        p = decay_padded_piece(r, id);
    }
    if (p.q.e - p.q.b <= r.cell || (a.rev ? p.lo == p.q.b : p.hi == p.q.e))
        p.lo = p.hi = 0;
    return p;
}
// Whether a sequence without rows is the piece's to look after.
__device__ __forceinline__ bool decay_empty_here(const DecayRun &r, const DecayPiece &p)
{
    return p.q.e <= p.q.b && (r.a.offsets ? p.cell == decay_cell_of(p.q.b, r.cell)
                                           : p.cell == p.s * r.cells);
}

// what: 0 states, 1 results of the inputs' type, 2 results in fp32
tgm_status_t decay_f32(const DecayRun &r, int what, hipStream_t s);
tgm_status_t decay_bf16(const DecayRun &r, int what, hipStream_t s);
tgm_status_t decay_f16(const DecayRun &r, int what, hipStream_t s);

// a^n from log2 a, which is kept finite so that a^0 is 1 also where a is 0.
__device__ __forceinline__ float decay_log2(float g)
{
    const float g2 = g * 1.44269504088896340736f;
    return g2 < -1e30f ? -1e30f : g2;
}
__device__ __forceinline__ float decay_pow(float g2, float n)
{
    return __builtin_amdgcn_exp2f(n * g2);
}

}  // namespace tgm
