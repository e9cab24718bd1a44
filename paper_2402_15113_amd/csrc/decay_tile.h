// The recurrence of csrc/decay.h by chunks of C rows, on the matrix cores.  Within a chunk,
// with n rows and i, s counted from its first,
//   out_i = c_out a^(i + 1) x_i S  +  c_out c_y sum_(s <= i) a^(i - s) (x_i . y_s) z_s,
//   S    <- a^n S + c_y sum_s a^(n - 1 - s) y_s z_s^T,
// which is four products instead of C steps.
//
// A workgroup has a head of a piece of a sequence and goes from chunk to chunk.  Its
// wavefronts share the state by columns: each keeps its columns of S (fp32, all p rows) in
// registers, where the matrix instructions leave them in just the places that the next
// product's operand has them in, so S never goes through LDS.  What they exchange are the
// weights a^(i - s) (x_i . y_s), a row of 16 i each, through LDS.
//
// 16-bit inputs: the weights and S are rounded once for the products that make out of them. S
// itself takes a^(n - 1 - s) z_s in parts, so that no error of 16 bits is carried along: three of
// bf16, whose sum is the fp32 product, or two of fp16, whose sum is off by 2^-23 of it.  fp16 is
// narrow, so its numbers come times powers of two: one for a row of weights, one for a column of S
// (a lane has one column of S and of z), one for a column of z, whose second parts have another
// 2^12.  What is below 2^-27 of the largest of its row of weights or column of S loses bits to
// fp16's smallest steps; of a column of z, what is below 2^-29 of its largest in the chunk.
//
// What bounds it: the chain from chunk to chunk (loads, weights, results, state, two exchanges
// through LDS), of which 16 wavefronts a CU do not hide all; q, k, v and o pass once here and k and
// v once more for the states.  bf16, 262,147 rows of 8 heads of 128: results 553 us at least and
// 624 in the median (2.1 GB, 3.9 TB/s), states 265 and 291 (1.1 GB, 4.1 TB/s); 65,536 rows of 16
// heads of 64 and 128 in 64 sequences, at least: results 266 us, dq 152, dv 293 and dk 174 (fp32,
// for four heads each), states 54.  fp32, 262,147 rows of 8 heads of 128: results 1,558 us at least
// (171 G operations, 110 TFLOP/s), states 692 (99 TFLOP/s); 4,000 sequences of 11 rows of 2 heads
// of 50 with their states 80 (200 MB).
#pragma once

#include <type_traits>

#include "decay.h"
#include "linear.h"

namespace tgm {

typedef short d4s __attribute__((ext_vector_type(4)));

// C rows of W columns in LDS.  Rows are so much longer than they have to be that both kinds
// of read meet different banks: 16 bytes of 8 neighbouring rows, and (16 bits) 32 bytes of 4,
// or (32 bits) 64 bytes of every 4th of 16.
template <class T, int C, int W> struct DecayTile {
    static constexpr int VEC = 16 / (int)sizeof(T);
    static constexpr int PITCH = W * (int)sizeof(T) + (sizeof(T) == 2 ? 32 : 16);
    static constexpr int BYTES = C * PITCH;

    // 16 bytes along a row: the fragment of rows r0 .. r0 + 15 for step ks of 4 VEC columns
    static __device__ __forceinline__ Frag<T> along(const char *t, int r0, int ks, int i, int q)
    {
        Frag<T> f;
        f.v = *reinterpret_cast<const Pack<T, VEC> *>(__builtin_assume_aligned(
            t + (r0 + i) * PITCH + 16 * (4 * ks + q), 16));
        return f;
    }
    // The transposed fragment: lane i of 16 has column c0 + i, for step ks of 4 VEC rows; of
    // 16-bit ones a lane has rows 4 q + r and 16 + 4 q + r of 32, so that the lanes that read
    // together have 8 neighbouring rows, in banks of their own.
    static __device__ __forceinline__ Frag<T> across(const char *t, int c0, int ks, int i, int q)
    {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 rows of 16 elements; lane i gets the i-th column of them
            typedef __attribute__((address_space(3))) d4s *lds_d4;
            d4s v[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const char *p =
                    t + (32 * ks + 16 * u + 4 * q + (i >> 2)) * PITCH + 2 * (c0 + 4 * (i & 3));
                v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_d4)(__attribute__((address_space(3))) void *)const_cast<char *>(p));
            }
            __builtin_memcpy(&f.v, v, sizeof(v));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                f.v.v[j] = *reinterpret_cast<const T *>(t + (16 * ks + 4 * q + j) * PITCH +
                                                        4 * (c0 + i));
        }
        return f;
    }
    // x and the weights lie in another order, 16-bit columns 16 h + 4 q + r of every 32 at 8 q +
    // 4 h + r: the order in which a lane holds two blocks of the state, and the rows of z, so
    // that `along` reads what their products take.  x's columns as they are, for the product
    // with y:
    static __device__ __forceinline__ Frag<T> along_x(const char *t, int r0, int ks, int i, int q)
    {
        if constexpr (sizeof(T) == 4) {
            return along(t, r0, ks, i, q);
        } else {
            const char *p = t + (r0 + i) * PITCH + 64 * ks + 32 * (q & 1) + 8 * (q >> 1);
            const uint64_t lo = *reinterpret_cast<const uint64_t *>(p);
            const uint64_t hi = *reinterpret_cast<const uint64_t *>(p + 16);
            Frag<T> f;
            __builtin_memcpy(&f.v, &lo, 8);
            __builtin_memcpy((char *)&f.v + 8, &hi, 8);
            return f;
        }
    }
};

typedef unsigned d4u __attribute__((ext_vector_type(4), may_alias));
typedef d4u d4u_any __attribute__((aligned(1)));

// A chunk's rows of one matrix in memory: n of them, row i of the chunk at i ld from `base`,
// or at (n - 1 - i) ld where the recurrence runs backwards.  63 rows of 2^24 fp32 columns are
// below 2^32 bytes, so a lane keeps 32 bits for a row's place.
struct DecayRows {
    const char *base;
    uint32_t ld;      // bytes
    int32_t n, rev;
    __device__ __forceinline__ uint32_t at(int i) const
    {
        return (uint32_t)(rev ? n - 1 - i : i) * ld;
    }
};

// A tile on its way from memory: rows past n and columns past the head's width are zeros.
template <class T, int C, int W, int TH> struct DecayLoad {
    using Tile = DecayTile<T, C, W>;
    static constexpr int VEC = Tile::VEC, PER = W / VEC, N = (C * PER + TH - 1) / TH;
    static constexpr bool EVEN = C * PER % TH == 0;   // else the last threads have none
    d4u v[N];   // of a vector type, which the compiler loads as one (a Pack it takes apart)

    __device__ __forceinline__ void load(const DecayRows &r, int width)
    {
        // (formed anew: the places of three forms of a load would stay in registers)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        if (r.n == C && width == W) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid;
                if (EVEN || e < C * PER)
                    v[u] = *reinterpret_cast<const d4u_any *>(
                        r.base + (r.at(e / PER) + (uint32_t)(e % PER * 16)));
            }
        } else if (width % VEC == 0) {
            // past the ends: the last one again, for zeros
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid, row = e / PER, c = e % PER * VEC;
                v[u] = *reinterpret_cast<const d4u_any *>(
                    r.base + (r.at(min(row, r.n - 1)) +
                              (uint32_t)(min(c, width - VEC) * (int)sizeof(T))));
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid, row = e / PER, c = e % PER * VEC;
                if (row >= r.n || c >= width)
                    v[u] = d4u{0, 0, 0, 0};
            }
        } else if (width > VEC) {
            // the last vector of a row moves back to its end, and its elements forward
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid, row = e / PER, c = e % PER * VEC;
                v[u] = *reinterpret_cast<const d4u_any *>(
                    r.base + (r.at(min(row, r.n - 1)) +
                              (uint32_t)(min(c, width - VEC) * (int)sizeof(T))));
            }
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid, row = e / PER, c = e % PER * VEC;
                const int back = max(0, c - (width - VEC));
                v[u] = __builtin_bit_cast(d4u, __builtin_bit_cast(unsigned __int128, v[u]) >>
                                                   (8 * (int)sizeof(T) * min(back, VEC - 1)));
                if (row >= r.n || c >= width)
                    v[u] = d4u{0, 0, 0, 0};
            }
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int e = u * TH + tid, row = e / PER, c = e % PER * VEC;
                v[u] = d4u{0, 0, 0, 0};
                if (row < r.n && c == 0)
                    v[u] = part(reinterpret_cast<const T *>(r.base + r.at(row)), width);
            }
        }
    }
    // the first `some` < VEC elements of a vector
    static __device__ __forceinline__ d4u part(const T *from, int some)
    {
        d4u r{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < VEC - 1; ++j)
            if (j < some) {
                if constexpr (sizeof(T) == 4)
                    r[j] = __builtin_bit_cast(unsigned, from[j]);
                else
                    r[j / 2] |= (unsigned)__builtin_bit_cast(uint16_t, from[j]) << (16 * (j & 1));
            }
        return r;
    }
    // Waits for the loads, here and not behind stores that follow.
    __device__ __forceinline__ void arrive() const
    {
#pragma unroll
        for (int u = 0; u < N; ++u)
            asm volatile("" ::"v"(v[u]));
    }
    // X: in x's order
    template <bool X> __device__ __forceinline__ void store(char *t) const
    {
        int tid = threadIdx.x;   // formed anew, as in load
        asm volatile("" : "+v"(tid));
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int e = u * TH + tid, m = e % PER;
            char *row = t + e / PER * Tile::PITCH;
            if (!EVEN && e >= C * PER)
                continue;
            if constexpr (X && sizeof(T) == 2) {
                // columns 8 m .. + 7 of every 32: h = m / 2, q = 2 (m % 2) and the next
                typedef unsigned d2u __attribute__((ext_vector_type(2), may_alias));
                char *to = row + 64 * (m >> 2) + 32 * (m & 1) + 8 * ((m >> 1) & 1);
                *reinterpret_cast<d2u *>(to) = d2u{v[u].x, v[u].y};
                *reinterpret_cast<d2u *>(to + 16) = d2u{v[u].z, v[u].w};
            } else {
                *reinterpret_cast<d4u *>(__builtin_assume_aligned(row + 16 * m, 16)) = v[u];
            }
        }
    }
};

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }
// The power of two that brings a largest absolute value (finite, or 0) to 2^13 .. 2^14: fp16 has
// all its bits from there down to 2^-14.
__device__ __forceinline__ float half_scale(float top)
{
    return top > 0.f ? ldexpf(1.f, min(max(13 - ilogbf(top), -126), 100)) : 1.f;
}
// 1 / v of a power of two from 2^-126 to 2^126.
__device__ __forceinline__ float one_over(float v)
{
    return __uint_as_float(0x7f000000u - __float_as_uint(v));
}
// The largest of the four lanes that hold a column.
__device__ __forceinline__ float column_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
// What fp16's second part is held times besides: its smallest steps are 2^-36, not 2^-24.
constexpr float kLowPart = 4096.f;

// Which piece and head workgroup `id` takes: every XCD (id % 8) runs of all heads of a
// piece, whose rows lie side by side and which may share k and v.
struct DecayPlace {
    int64_t piece;
    int32_t head;
};
__device__ __forceinline__ DecayPlace decay_place(int64_t id, int64_t ids, int32_t H)
{
    const int64_t whole = ids / 8 * 8;
    if (id < whole * H) {
        const int64_t m = id / 8;
        return DecayPlace{m / H * 8 + id % 8, (int32_t)(m % H)};
    }
    const int64_t m = id - whole * H;
    return DecayPlace{whole + m / H, (int32_t)(m % H)};
}

// Rows of a chunk: 32, so that two workgroups a CU fit its registers, and 64 for the states alone
// of few 16-bit columns.  us with chunks of 32 and of 64 rows, bf16: results of 262,147 rows of 8
// heads of 128 x 128 711 and 780, of 65,536 rows of 16 heads of 64 x 128 333 and 336; states of
// the latter 114 and 81.
template <class T, int P, bool OUT> constexpr int decay_chunk()
{
    return !OUT && sizeof(T) == 2 && P <= 64 ? 64 : 32;
}

// Wavefronts of a SIMD that registers are kept for: two workgroups of 512 threads or four of 256
// fit a CU; three of those with 128 x 64 columns in fp32 and fp16, which would not be kept in 128
// registers.  us with 3 and 4: 262,144 rows of 8 heads of 128 x 64 fp32 1,338 and 1,377; a training
// step of 65,536 rows of 8 heads of 64 and 128 in 64 sequences fp16 834 and 907, of 16 heads, 4 of
// k and v, bf16 1,375 and 1,361.  With 4, kernels of 128 columns spill vector registers around
// their pieces: bf16 45 (128 x 64) and 36 (128 x 128), fp16 19 to 21 and fp32 13 (128 x 128).
template <class T, int P, int R, bool OUT> constexpr int decay_waves()
{
    return OUT && P == 128 && R == 64 && TypeCode<T>::code != TGM_BF16 ? 3 : 4;
}

// OUT: x and the results; without, the pieces' states alone (for sequences that go on).
template <class T, class O, int P, int R, bool OUT>
__global__ __launch_bounds__(4 * R, (decay_waves<T, P, R, OUT>())) void k_decay(DecayRun run)
{
    constexpr int C = decay_chunk<T, P, OUT>(), NW = R / 16, TH = 64 * NW, TB = C / 16;
    constexpr int STEP = 64 / (int)sizeof(T);       // elements of a fragment's sum
    constexpr int BLOCKS = STEP / 16;               // blocks of 16 in them
    constexpr int KP = P / STEP, PB = P / 16, VEC = 16 / (int)sizeof(T);
    constexpr bool F16 = TypeCode<T>::code == TGM_F16, F32 = sizeof(T) == 4;
    constexpr int PARTS = F32 ? 1 : F16 ? 2 : 3, GROUP = PB < 4 ? PB : 4;
    using TX = DecayTile<T, C, P>;
    using TZ = DecayTile<T, C, R>;
    using TW = DecayTile<T, C, C>;
    __shared__ __attribute__((aligned(16))) char lx[OUT ? TX::BYTES : 16], ly[TX::BYTES],
        lz[TZ::BYTES], lw[OUT ? TW::BYTES : 16];
    // c_out c_y a^d at C + d for the distances d >= 0 within a chunk, zeros below
    __shared__ float by_distance[OUT ? 2 * C : 1];
    __shared__ float row_scale[F16 ? C : 1];
    const DecayArgs &A = run.a;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int lane_row = lane & 15, lane_group = lane >> 4, r0 = 16 * w;
    // element e of a fragment of z is row STEP k + 4 g + row_of(e)
    auto row_of = [](int e) { return e < 4 ? e : 12 + e; };
    constexpr int LAST = F32 ? 3 : 19;
    // the state's row that element j of block pb of a lane is, q its group of 16
    auto state_row = [](int pb, int j, int q) { return 16 * pb + 4 * q + j; };
    const int64_t ids = OUT ? run.ids : run.all_cells, all = ids * A.H;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
        const DecayPlace place = decay_place(at, ids, A.H);
        const int64_t id = OUT && run.order ? run.order[place.piece] : place.piece;
        if (id < 0)
            continue;
        const DecayPiece piece = OUT ? decay_piece_of(run, id) : decay_piece_onward(run, id);
        const int32_t h = place.head;
        const bool empty = OUT && decay_empty_here(run, piece);
        const int64_t rows = piece.hi - piece.lo;
        const bool begins = empty || (A.rev ? piece.hi == piece.q.e : piece.lo == piece.q.b);
        const bool ends =
            OUT && (empty || (A.rev ? piece.lo == piece.q.b : piece.hi == piece.q.e));
        if (rows <= 0 && !(empty && A.last))
            continue;
        const float decay = decay_log2(A.decay[h]);
        const int64_t size = (int64_t)A.p * A.r;

        // rows t0 .. t0 + n - 1 of the piece, in the recurrence's order
        auto rows_of = [&](const void *p, int64_t ld, int64_t head, int bytes, int64_t t0, int n)
            __attribute__((always_inline)) {
                const int64_t low = A.rev ? piece.hi - t0 - n : piece.lo + t0;
                return DecayRows{(const char *)p + (low * ld + head) * bytes,
                                 (uint32_t)(ld * bytes), n, A.rev};
            };
        DecayLoad<T, C, P, TH> vx, vy;
        DecayLoad<T, C, R, TH> vz;
        auto fetch = [&](int64_t t0) __attribute__((always_inline)) {
            const int n = (int)min((int64_t)C, rows - t0);
            constexpr int B = sizeof(T);
            if constexpr (OUT)
                vx.load(rows_of(A.x.p, A.x.ld, (int64_t)(h / A.x.share) * A.p, B, t0, n), A.p);
            vy.load(rows_of(A.y.p, A.y.ld, (int64_t)(h / A.y.share) * A.p, B, t0, n), A.p);
            vz.load(rows_of(A.z.p, A.z.ld, (int64_t)(h / A.z.share) * A.r, B, t0, n), A.r);
        };
        if (rows > 0)
            fetch(0);

        // ---- the state before the piece
        f4 st[PB];
        const float *from = nullptr;
        if (begins)
            from = A.first ? A.first + ((int64_t)piece.s * A.H + h) * size : nullptr;
        else if (OUT)
            from = run.states + (h * run.all_cells + piece.cell + (A.rev ? 1 : -1)) * size;
        const int col = r0 + lane_row;
        // where element (r, col) of a state lies: 32 bits, formed where it is used (all of
        // them would stay in registers for the next piece)
        const uint32_t s_col = (uint32_t)col * (A.turned ? (uint32_t)A.p : 1u) * 4u;
        const uint32_t s_row = (A.turned ? 1u : (uint32_t)A.r) * 4u;
        int q = lane_group;
        asm volatile("" : "+v"(q));
#pragma unroll
        for (int pb = 0; pb < PB; ++pb)
            st[pb] = f4{0.f, 0.f, 0.f, 0.f};
        // (turned: 4 rows of a column are neighbours.  By single elements a training step of 1,000 x
        // 40 rows of 4 heads of 128 x 104 fp16 took 1,115 us, so 843; with fp16's scales by columns
        // 876.)
        if (from && A.turned) {
#pragma unroll
            for (int pb = 0; pb < PB; ++pb) {
                const int r = state_row(pb, 0, q);
                const float *at = reinterpret_cast<const float *>(
                    reinterpret_cast<const char *>(from) + (s_col + (uint32_t)r * 4u));
                if (col < A.r && r + 4 <= A.p)
                    __builtin_memcpy(&st[pb], at, 16);
                else if (col < A.r)
#pragma unroll
                    for (int j = 0; j < 3; ++j)
                        if (r + j < A.p)
                            st[pb][j] = at[j];
            }
        } else if (from && col < A.r)
#pragma unroll
            for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = state_row(pb, j, q);
                    const float v = *reinterpret_cast<const float *>(
                        reinterpret_cast<const char *>(from) +
                        (s_col + (uint32_t)min(r, A.p - 1) * s_row));
                    st[pb][j] = r < A.p ? v : 0.f;
                }
        // of whole chunks as a lane's factor times one that all lanes share
        float lane_weight[C / STEP], shared_weight[VEC];
#pragma unroll
        for (int k = 0; k < C / STEP; ++k)
            lane_weight[k] =
                A.c_y * decay_pow(decay, (float)(C - LAST - 1 - STEP * k - 4 * lane_group));
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            shared_weight[e] = __builtin_bit_cast(
                float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(
                           int, decay_pow(decay, (float)(LAST - row_of(e))))));
        lds_barrier();   // no one reads the last piece's chunks any more
        if constexpr (OUT) {
            for (int i = threadIdx.x; i < 2 * C; i += TH)
                by_distance[i] =
                    i < C ? 0.f : A.c_out * A.c_y * decay_pow(decay, (float)(i - C));
        }
        bool some = from != nullptr;     // a state that is not all zeros
        int lag = begins ? A.lag0 : 1;   // its weight at the chunk's first row: a^lag

        // The weights of a chunk of NB blocks of 16 rows (the last may be shorter); NB is known
        // so that no branch stands between a fragment's read and its product.  What follows
        // from a lane's place is formed anew in every chunk: all of it would stay in
        // registers, several times over.
        auto scores = [&](auto blocks) __attribute__((always_inline)) {
            constexpr int NB = decltype(blocks)::value;
            int i16 = lane_row, g = lane_group;
            asm volatile("" : "+v"(i16), "+v"(g));
            // rows 16 b .. + 15 and NS blocks of s a wavefront
            constexpr int NS = F16 || NW < NB * 2 ? NB : NW >= NB * NB ? 1 : NB * NB / NW;
            constexpr int TASKS = NB * (NB / NS);
            auto task_of = [&](int task) __attribute__((always_inline)) {
                const int b = task % NB, s0 = task / NB * NS;
                f4 acc[NS];
#pragma unroll
                for (int s = 0; s < NS; ++s)
                    acc[s] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KP; ++k) {
                    const Frag<T> fx = TX::along_x(lx, 16 * b, k, i16, g);
#pragma unroll
                    for (int s = 0; s < NS; ++s)
                        acc[s] = mfma(TX::along(ly, 16 * (s0 + s), k, i16, g), fx, acc[s]);
                }
                float top = 0.f;
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // row i16 of block b, column 4 g + j of block s0 + s (a product
                        // with a later row is none, whatever it is)
                        const int d = 16 * (b - s0 - s) + i16 - (4 * g + j);
                        acc[s][j] = d >= 0 ? acc[s][j] * by_distance[C + d] : 0.f;
                        if constexpr (F16)
                            top = finite(acc[s][j]) ? fmaxf(top, fabsf(acc[s][j])) : top;
                    }
                float scale = 1.f;
                if constexpr (F16) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    scale = half_scale(top);
                    if (g == 0)
                        row_scale[16 * b + i16] = 1.f / scale;
                }
                // columns 16 s + 4 g .. + 3, in their order
                auto to = [&](int s) __attribute__((always_inline)) {
                    return reinterpret_cast<Pack<T, 4> *>(__builtin_assume_aligned(
                        lw + (16 * b + i16) * TW::PITCH +
                            (F32 ? 16 * s + 4 * g : 32 * (s >> 1) + 8 * g + 4 * (s & 1)) *
                                (int)sizeof(T),
                        4 * sizeof(T)));
                };
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    Pack<T, 4> q;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        q.v[j] = from_f32<T>(F16 ? acc[s][j] * scale : acc[s][j]);
                    *to(s0 + s) = q;
                }
                if constexpr (NB % BLOCKS) {   // the rest of a fragment's sum
                    Pack<T, 4> q;
                    __builtin_memset(&q, 0, sizeof(q));
                    *to(NB) = q;
                }
            };
            if constexpr (TASKS == NW)
                task_of(w);
            else
#pragma unroll 1
                for (int task = w; task < TASKS; task += NW)
                    task_of(task);
        };

        // The results of n rows and the state behind them.
        auto rest = [&](auto blocks, auto full, int64_t t0, int n, bool more)
            __attribute__((always_inline)) {
            constexpr int NB = decltype(blocks)::value, KC = (NB + BLOCKS - 1) / BLOCKS;
            int i16 = lane_row, g = lane_group;
            asm volatile("" : "+v"(i16), "+v"(g));

            // ---- this wavefront's columns of z
            Frag<T> z[KC];
#pragma unroll
            for (int k = 0; k < KC; ++k)
                z[k] = TZ::across(lz, r0, k, i16, g);

            if constexpr (OUT) {
                f4 o[NB];
                bool spoilt = false;
                // of the state's column that the lane has.  (Formed without a state too, registers
                // spill, and a training step of 4,000 sequences of 11 rows takes 435 us for 340.)
                float s_scale = 1.f;
                if (F16 && some) {
                    float top = 0.f;
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float v = fabsf(st[pb][j]);
                            top = v < INFINITY ? fmaxf(top, v) : top;
                        }
                    s_scale = half_scale(column_max(top));
                }
                // A weight of zero does not keep what is not finite in a later row of the
                // chunk from a row's sum.  The last block's sums show whether there may be any:
                // then such elements of z count as zero, and are added where they belong.
#pragma unroll 1
                for (;;) {
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        o[b] = f4{0.f, 0.f, 0.f, 0.f};
                    if (some) {
#pragma unroll
                        for (int k = 0; k < KP; ++k) {
                            Frag<T> s;
#pragma unroll
                            for (int e = 0; e < VEC; ++e) {
                                const float v = st[BLOCKS * k + e / 4][e % 4];
                                s.v.v[e] = from_f32<T>(F16 ? v * s_scale : v);
                            }
#pragma unroll
                            for (int b = 0; b < NB; ++b)
                                o[b] = mfma(s, TX::along(lx, 16 * b, k, i16, g), o[b]);
                        }
                        if constexpr (F16)   // 1 over the scales of the four columns that o has
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float back = __shfl(one_over(s_scale), 4 * g + j);
#pragma unroll
                                for (int b = 0; b < NB; ++b)
                                    o[b][j] *= back;
                            }
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            const float f =
                                A.c_out * decay_pow(decay, (float)(16 * b + i16 + lag));
                            o[b] *= f;
                        }
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        f4 c = F16 ? f4{0.f, 0.f, 0.f, 0.f} : o[b];
#pragma unroll
                        for (int k = 0; k < KC; ++k)
                            if (BLOCKS * k <= b)
                                c = mfma(z[k], TW::along(lw, 16 * b, k, i16, g), c);
                        o[b] = F16 ? o[b] + c * row_scale[16 * b + i16] : c;
                    }
                    float seen = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        seen += o[NB - 1][j] * 0.f;
                    if (spoilt || !__any(seen != 0.f))   // NaN where one is not finite
                        break;
#pragma unroll
                    for (int k = 0; k < KC; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            if (!finite(to_f32(z[k].v.v[e])))
                                spoilt = true, z[k].v.v[e] = from_f32<T>(0.f);
                    spoilt = __any(spoilt);
                    if (!spoilt)
                        break;
                }
                if (spoilt) {
#pragma unroll 1
                    for (int s = 0; s < n; ++s) {
                        const int place =
                            F32 ? s : (s & ~31) + 8 * ((s >> 2) & 3) + 4 * ((s >> 4) & 1) + (s & 3);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float v = to_f32(*reinterpret_cast<const T *>(
                                lz + s * TZ::PITCH + (r0 + 4 * g + j) * (int)sizeof(T)));
                            if (finite(v))
                                continue;
#pragma unroll
                            for (int b = 0; b < NB; ++b)
                                if (16 * b + i16 >= s)
                                    o[b][j] += v * to_f32(*reinterpret_cast<const T *>(
                                                       lw + (16 * b + i16) * TW::PITCH +
                                                       place * (int)sizeof(T)));
                        }
                    }
#pragma unroll
                    for (int k = 0; k < KC; ++k)
                        z[k] = TZ::across(lz, r0, k, i16, g);
                }
                // the next chunk is there: its wait would be for these stores too
                if (more)
                    vx.arrive(), vy.arrive(), vz.arrive();
                if (A.out) {
                    const DecayRows to_rows =
                        rows_of(A.out, A.ld_out, (int64_t)h * A.r + r0, sizeof(O), t0, n);
                    const int c = r0 + 4 * g;
                    auto to = [&](int b) __attribute__((always_inline)) {
                        return reinterpret_cast<O *>(
                            const_cast<char *>(to_rows.base) +
                            (to_rows.at(16 * b + i16) + 4 * g * (uint32_t)sizeof(O)));
                    };
                    if (c + 4 <= A.r) {
#pragma unroll
                        for (int b = 0; b < NB; ++b) {
                            Pack<O, 4> q;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                q.v[j] = from_f32<O>(o[b][j]);
                            if (full || 16 * b + i16 < n)
                                store_pack(to(b), q);
                        }
                    } else if (c < A.r) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
                            if (16 * b + i16 < n)
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    if (c + j < A.r)
                                        to(b)[j] = from_f32<O>(o[b][j]);
                    }
                }
            }

            // ---- the state behind the chunk, where anyone reads it
            if (more || !OUT || (ends && A.last)) {
                // c_y a^(n - 1 - s) for row s of element e of z[k]
                auto weight = [&](int k, int e) __attribute__((always_inline)) {
                    if constexpr (full)
                        return lane_weight[k] * shared_weight[e];
                    else
                        return A.c_y * decay_pow(decay, (float)max(0, n - 1 - STEP * k - 4 * g -
                                                                          row_of(e)));
                };
                float z_scale = 1.f;
                if constexpr (F16) {
                    float top = 0.f;
#pragma unroll
                    for (int k = 0; k < KC; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const float v = fabsf(to_f32(z[k].v.v[e]) * weight(k, e));
                            top = v < INFINITY ? fmaxf(top, v) : top;
                        }
                    z_scale = half_scale(column_max(top));
                }
                const float whole = decay_pow(decay, (float)(n - 1 + lag));
                if (!F16 && some)
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb)
                        st[pb] *= whole;
                // (products into one block wait for each other)
                if constexpr (F16) {
                    // both parts' sums apart, for their scales, which the state may not hold
                    constexpr int PAIR = GROUP / 2;
                    const float back = one_over(z_scale), keep = some ? whole : 0.f;
                    Frag<T> high_part[KC], low_part[KC];
#pragma unroll
                    for (int k = 0; k < KC; ++k)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const float v = to_f32(z[k].v.v[e]) * weight(k, e) * z_scale;
                            high_part[k].v.v[e] = from_f32<T>(v);
                            low_part[k].v.v[e] =
                                from_f32<T>((v - to_f32(high_part[k].v.v[e])) * kLowPart);
                        }
#pragma unroll
                    for (int p2 = 0; p2 < PB; p2 += PAIR) {
                        f4 high[PAIR], low[PAIR];
#pragma unroll
                        for (int i = 0; i < PAIR; ++i)
                            high[i] = low[i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < KC; ++k) {
                            Frag<T> f[PAIR];
#pragma unroll
                            for (int i = 0; i < PAIR; ++i)
                                f[i] = TX::across(ly, 16 * (p2 + i), k, i16, g);
#pragma unroll
                            for (int i = 0; i < PAIR; ++i)
                                low[i] = mfma(f[i], low_part[k], low[i]);
#pragma unroll
                            for (int i = 0; i < PAIR; ++i)
                                high[i] = mfma(f[i], high_part[k], high[i]);
                        }
#pragma unroll
                        for (int i = 0; i < PAIR; ++i)
                            st[p2 + i] = st[p2 + i] * keep + (high[i] + low[i] / kLowPart) * back;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < KC; ++k) {
                        Frag<T> part[PARTS];
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            float v = to_f32(z[k].v.v[e]) * weight(k, e);
#pragma unroll
                            for (int u = 0; u < PARTS; ++u) {
                                part[u].v.v[e] = from_f32<T>(v);
                                if (u + 1 < PARTS)
                                    v -= to_f32(part[u].v.v[e]);
                            }
                        }
#pragma unroll
                        for (int p4 = 0; p4 < PB; p4 += GROUP) {
                            Frag<T> f[GROUP];
#pragma unroll
                            for (int i = 0; i < GROUP; ++i) {
                                const int pb = p4 + i;
                                f[i] = TX::across(ly, 16 * pb, k, i16, g);
                            }
#pragma unroll
                            for (int u = 0; u < PARTS; ++u)
#pragma unroll
                                for (int i = 0; i < GROUP; ++i)
                                    st[p4 + i] = mfma(f[i], part[u], st[p4 + i]);
                        }
                    }
                }
                some = true;
            }
            lag = 1;
        };

        auto put = [&]() __attribute__((always_inline)) {
            if constexpr (OUT)
                vx.template store<true>(lx);
            vy.template store<false>(ly);
            vz.template store<false>(lz);
        };
        using All = std::integral_constant<int, TB>;
        using Half = std::integral_constant<int, TB / 2>;
        using One = std::integral_constant<int, 1>;
        // by the blocks that n rows have
        auto by_blocks = [&](int n, auto f) __attribute__((always_inline)) {
            if (n > C / 2)
                f(All{});
            else if (n > 16)
                f(Half{});
            else
                f(One{});
        };
        if (rows > 0)
            put();
        lds_barrier();
        int64_t t0 = 0;
#pragma unroll 1
        for (; t0 + C < rows; t0 += C) {
            fetch(t0 + C);
            if constexpr (OUT) {
                scores(All{});
                lds_barrier();
            }
            rest(All{}, std::true_type{}, t0, C, true);
            lds_barrier();
            put();
            lds_barrier();
        }
        if constexpr (OUT) {
            if (rows > 0)
                by_blocks((int)(rows - t0), [&](auto nb) { scores(nb); });
            lds_barrier();
        }
        if (rows > 0) {
            const int n = (int)(rows - t0);
            by_blocks(n, [&](auto nb) { rest(nb, std::false_type{}, t0, n, false); });
        }

        // ---- the state behind the piece
        float *to = nullptr;
        float f = 1.f;
        if (!OUT)
            to = run.states + (h * run.all_cells + piece.cell) * size;
        else if (ends && A.last) {
            to = A.last + ((int64_t)piece.s * A.H + h) * size;
            if (A.lag1 && !empty)
                f = decay_pow(decay, 1.f);
        }
        asm volatile("" : "+v"(q));
        if (to && col < A.r)
#pragma unroll
            for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = state_row(pb, j, q);
                    if (r < A.p)
                        *reinterpret_cast<float *>(reinterpret_cast<char *>(to) +
                                                   (s_col + (uint32_t)r * s_row)) = f * st[pb][j];
                }
    }
}

// Between a wavefront's lanes' writes to LDS and its other lanes' reads of them, and back: LDS
// serves a wavefront in order, only the compiler has to be kept from moving them.
__device__ __forceinline__ void exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Short sequences: a wavefront has a head of a piece and all columns of its state, and chunks of 16
// rows.  The weights a^(i - s) (x_i . y_s) of 16 rows are left by the matrix instructions where the
// next product takes them; LDS, of which every wavefront has its own, turns y and z; no wavefront
// waits for another.  Bound by each sequence's loads, several thousand instructions and stores, one
// after another, of which the 8 wavefronts a CU that a state in registers leaves room for (211
// vector registers, 241 scalar ones in lanes of others) do not cover all; the state is kept there
// also where there is none before and one chunk is all.  12,000 sequences of 10 rows of 2 heads of
// 50 fp32 with their states (431 MB) in 163 us, 2.6 TB/s; without the states behind them 83.
// (States moved through LDS, 16 bytes a lane side by side: 177 us.)
template <class T, class O, int P, int R>
__global__ __launch_bounds__(256, 2) void k_decay_short(DecayRun run)
{
    constexpr int STEP = 64 / (int)sizeof(T), BLOCKS = STEP / 16, KP = P / STEP, PB = P / 16;
    constexpr int CB = R / 16, VEC = 16 / (int)sizeof(T), B = sizeof(T);
    constexpr bool F16 = TypeCode<T>::code == TGM_F16, F32 = sizeof(T) == 4;
    constexpr int PARTS = F32 ? 1 : F16 ? 2 : 3;
    using TY = DecayTile<T, 16, P>;
    using TZ = DecayTile<T, 16, R>;
    __shared__ __attribute__((aligned(16))) char lds[4][TY::BYTES + TZ::BYTES];
    const DecayArgs &A = run.a;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    char *ly = lds[w], *lz = ly + TY::BYTES;
    const int64_t all = run.ids * A.H;
    for (int64_t at = (int64_t)blockIdx.x * 4 + w; at < all; at += (int64_t)gridDim.x * 4) {
        // (formed anew: what follows from it would stay in registers)
        int i16 = lane & 15, g = lane >> 4;
        asm volatile("" : "+v"(i16), "+v"(g));
        const DecayPlace place = decay_place(at, run.ids, A.H);
        const DecayPiece piece = decay_piece_of(run, place.piece);
        const int32_t h = place.head;
        const bool empty = decay_empty_here(run, piece);
        const int64_t rows = piece.hi - piece.lo;
        const bool begins = empty || (A.rev ? piece.hi == piece.q.e : piece.lo == piece.q.b);
        const bool ends = empty || (A.rev ? piece.lo == piece.q.b : piece.hi == piece.q.e);
        if (rows <= 0 && !(empty && A.last))
            continue;
        const float decay = decay_log2(A.decay[h]);
        const int64_t size = (int64_t)A.p * A.r;
        const float *from = nullptr;
        if (begins)
            from = A.first ? A.first + ((int64_t)piece.s * A.H + h) * size : nullptr;
        else
            from = run.states + (h * run.all_cells + piece.cell + (A.rev ? 1 : -1)) * size;
        // Element (r, c) of a state: what all lanes share is the base, so that a lane keeps one
        // place for each block of columns.
        const uint32_t s_col = (A.turned ? (uint32_t)A.p : 1u) * 4u;
        const uint32_t s_row = (A.turned ? 1u : (uint32_t)A.r) * 4u;
        auto each = [&](auto f) __attribute__((always_inline)) {
            uint32_t lane_at[CB];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                lane_at[cb] = (uint32_t)(16 * cb + i16) * s_col + (uint32_t)(4 * g) * s_row;
#pragma unroll
            for (int pb = 0; pb < PB; ++pb) {
                const bool whole = 16 * pb + 16 <= A.p;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
                    if (16 * cb + i16 < A.r)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (whole || 16 * pb + 4 * g + j < A.p)
                                f(pb, cb, j, (size_t)(16 * pb + j) * s_row, lane_at[cb]);
            }
        };
        f4 st[PB][CB];
#pragma unroll
        for (int pb = 0; pb < PB; ++pb)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                st[pb][cb] = f4{0.f, 0.f, 0.f, 0.f};
        if (from && A.turned) {   // 4 rows of a column are neighbours
#pragma unroll
            for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const int r = 16 * pb + 4 * g, c = 16 * cb + i16;
                    const float *p = from + (c * A.p + r);
                    if (c < A.r && r + 4 <= A.p)
                        __builtin_memcpy(&st[pb][cb], p, 16);
                    else if (c < A.r)
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (r + j < A.p)
                                st[pb][cb][j] = p[j];
                }
        } else if (from)
            each([&](int pb, int cb, int j, size_t base, uint32_t mine)
                     __attribute__((always_inline)) {
                         st[pb][cb][j] = *reinterpret_cast<const float *>(
                             reinterpret_cast<const char *>(from) + base + mine);
                     });
        // Where one chunk is all, the state behind it is formed with rows and columns exchanged:
        // then a lane has 4 columns of a row, which are neighbours in memory.
        const bool exchanged = rows > 0 && rows <= 16 && ends && A.last && !A.turned;
        bool some = from != nullptr;
        int lag = begins ? A.lag0 : 1;

        auto rows_of = [&](const void *p, int64_t ld, int64_t head, int bytes, int64_t t0, int n)
            __attribute__((always_inline)) {
                const int64_t low = A.rev ? piece.hi - t0 - n : piece.lo + t0;
                return DecayRows{(const char *)p + (low * ld + head) * bytes,
                                 (uint32_t)(ld * bytes), n, A.rev};
            };
        // columns 16 b + 4 g .. + 3 of row i16 for all b, zeros where there are none
        auto fetch = [&](auto &v, const DecayRows &r, int width) __attribute__((always_inline)) {
            constexpr int N = sizeof(v) / sizeof(v[0]);
            __builtin_memset(&v, 0, sizeof(v));
            if (i16 < r.n) {
                const char *row = r.base + (r.at(i16) + (uint32_t)(4 * g * B));
#pragma unroll
                for (int b = 0; b < N; ++b) {
                    const T *from4 = reinterpret_cast<const T *>(row + 16 * b * B);
                    if (16 * b + 16 <= width || 16 * b + 4 * g + 4 <= width)
                        v[b] = load_pack<T, 4>(from4);
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (16 * b + 4 * g + j < width)
                                v[b].v[j] = from4[j];
                }
            }
        };
        // the fragment for step k: 16-bit columns 16 h + 4 g + r of 32, the state's order
        auto along = [&](const Pack<T, 4> *v, int k) __attribute__((always_inline)) {
            Frag<T> f;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                f.v.v[e] = v[BLOCKS * k + e / 4].v[e % 4];
            return f;
        };
        // the transposed one: column c0 + i16, rows 4 g .. + 3
        auto across = [&](const char *t, int pitch, int c0) __attribute__((always_inline)) {
            Frag<T> f;
            __builtin_memset(&f, 0, sizeof(f));
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    f.v.v[j] =
                        *reinterpret_cast<const T *>(t + (4 * g + j) * pitch + 4 * (c0 + i16));
            } else {
                typedef __attribute__((address_space(3))) d4s *lds_d4;
                const char *p = t + (4 * g + (i16 >> 2)) * pitch + 2 * (c0 + 4 * (i16 & 3));
                const d4s v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_d4)(__attribute__((address_space(3))) void *)const_cast<char *>(p));
                __builtin_memcpy(&f.v, &v, sizeof(v));
            }
            return f;
        };
#pragma unroll 1
        for (int64_t t0 = 0; t0 < rows; t0 += 16) {
            const int n = (int)min((int64_t)16, rows - t0);
            const bool more = t0 + 16 < rows;
            const DecayRows rx = rows_of(A.x.p, A.x.ld, (int64_t)(h / A.x.share) * A.p, B, t0, n);
            const DecayRows ry = rows_of(A.y.p, A.y.ld, (int64_t)(h / A.y.share) * A.p, B, t0, n);
            const DecayRows rz = rows_of(A.z.p, A.z.ld, (int64_t)(h / A.z.share) * A.r, B, t0, n);
            Pack<T, 4> px[PB], py[PB], pz[CB];
            fetch(px, rx, A.p);
            fetch(py, ry, A.p);
            fetch(pz, rz, A.r);
            exchange();   // (no lane reads the last chunk any more)
#pragma unroll
            for (int b = 0; b < PB; ++b)
                *reinterpret_cast<Pack<T, 4> *>(__builtin_assume_aligned(
                    ly + i16 * TY::PITCH + (16 * b + 4 * g) * B, 4 * B)) = py[b];
#pragma unroll
            for (int b = 0; b < CB; ++b)
                *reinterpret_cast<Pack<T, 4> *>(__builtin_assume_aligned(
                    lz + i16 * TZ::PITCH + (16 * b + 4 * g) * B, 4 * B)) = pz[b];
            exchange();
            Frag<T> x[KP], z[CB];
#pragma unroll
            for (int k = 0; k < KP; ++k)
                x[k] = along(px, k);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                z[cb] = across(lz, TZ::PITCH, 16 * cb);
            const bool onward = more || (ends && A.last);   // the state behind the chunk is read

            // ---- the weights of row i16 and rows 4 g .. + 3
            f4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KP; ++k)
                acc = mfma(along(py, k), x[k], acc);
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = i16 - (4 * g + j);
                const float f = A.c_out * A.c_y * decay_pow(decay, (float)max(d, 0));
                acc[j] = d >= 0 ? acc[j] * f : 0.f;
                if constexpr (F16)
                    top = finite(acc[j]) ? fmaxf(top, fabsf(acc[j])) : top;
            }
            float w_scale = 1.f;
            if constexpr (F16) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                w_scale = half_scale(top);
            }
            Frag<T> wf;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                wf.v.v[e] = from_f32<T>(e >= 4 ? 0.f : F16 ? acc[e % 4] * w_scale : acc[e % 4]);

            // ---- the results
            f4 o[CB];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                o[cb] = f4{0.f, 0.f, 0.f, 0.f};
            if (some) {
                float s_scale[CB];   // of the lane's columns
                if constexpr (F16)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        float most = 0.f;
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float v = fabsf(st[pb][cb][j]);
                                most = v < INFINITY ? fmaxf(most, v) : most;
                            }
                        s_scale[cb] = half_scale(column_max(most));
                    }
#pragma unroll
                for (int k = 0; k < KP; ++k)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        Frag<T> s;
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const float v = st[BLOCKS * k + e / 4][cb][e % 4];
                            s.v.v[e] = from_f32<T>(F16 ? v * s_scale[cb] : v);
                        }
                        o[cb] = mfma(s, x[k], o[cb]);
                    }
                const float f = A.c_out * decay_pow(decay, (float)(i16 + lag));
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    if constexpr (F16)   // 1 over the scales of the four columns that o has
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            o[cb][j] *= __shfl(one_over(s_scale[cb]), 4 * g + j);
                    o[cb] *= f;
                }
            }
            // what is not finite in z counts as zero, and is added where it belongs (k_decay)
            bool spoilt = false;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    spoilt |= !finite(to_f32(z[cb].v.v[j]));
            spoilt = __any(spoilt);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                Frag<T> c = z[cb];
                if (spoilt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (!finite(to_f32(c.v.v[j])))
                            c.v.v[j] = from_f32<T>(0.f);
                if constexpr (F16) {
                    const f4 p = mfma(c, wf, f4{0.f, 0.f, 0.f, 0.f});
                    o[cb] += p * (1.f / w_scale);
                } else {
                    o[cb] = mfma(c, wf, o[cb]);
                }
            }
            if (spoilt)
#pragma unroll 1
                for (int s = 0; s < n; ++s) {
                    const float w0 = __shfl(acc[0], 16 * (s >> 2) + i16);
                    const float w1 = __shfl(acc[1], 16 * (s >> 2) + i16);
                    const float w2 = __shfl(acc[2], 16 * (s >> 2) + i16);
                    const float w3 = __shfl(acc[3], 16 * (s >> 2) + i16);
                    const float ws = s & 2 ? (s & 1 ? w3 : w2) : s & 1 ? w1 : w0;
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int c = 16 * cb + 4 * g + j;
                            if (c < A.r) {
                                const float v = to_f32(
                                    *reinterpret_cast<const T *>(lz + s * TZ::PITCH + c * B));
                                if (!finite(v) && i16 >= s)
                                    o[cb][j] += v * ws;
                            }
                        }
                }
            if (A.out && i16 < n) {
                const DecayRows ro =
                    rows_of(A.out, A.ld_out, (int64_t)h * A.r, sizeof(O), t0, n);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    const int c = 16 * cb + 4 * g;
                    O *to = reinterpret_cast<O *>(const_cast<char *>(ro.base) +
                                                  (ro.at(i16) + (uint32_t)(c * (int)sizeof(O))));
                    Pack<O, 4> q;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        q.v[j] = from_f32<O>(o[cb][j]);
                    if (c + 4 <= A.r)
                        store_pack(to, q);
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (c + j < A.r)
                                to[j] = q.v[j];
                }
            }

            // ---- the state behind the chunk
            if (onward) {
                float v[CB][4], most[CB], z_scale[CB];
#pragma unroll
                for (int cb = 0; cb < CB; ++cb)
                    most[cb] = 0.f, z_scale[cb] = 1.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float f = A.c_y * decay_pow(decay, (float)max(0, n - 1 - (4 * g + j)));
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        v[cb][j] = to_f32(z[cb].v.v[j]) * f;
                        if constexpr (F16)
                            most[cb] =
                                finite(v[cb][j]) ? fmaxf(most[cb], fabsf(v[cb][j])) : most[cb];
                    }
                }
                if constexpr (F16)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
                        z_scale[cb] = half_scale(column_max(most[cb]));
                const float whole = decay_pow(decay, (float)(n - 1 + lag));
                Frag<T> yt[PB];
#pragma unroll
                for (int pb = 0; pb < PB; ++pb)
                    yt[pb] = across(ly, TY::PITCH, 16 * pb);
                if (some && !exchanged)   // (F16 too: its parts' sums are apart)
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb)
                            st[pb][cb] *= whole;
                float *to = A.last + ((int64_t)piece.s * A.H + h) * size;
                const float f = A.lag1 ? decay_pow(decay, 1.f) : 1.f;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    Frag<T> part[PARTS];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        float u = e >= 4 ? 0.f : F16 ? v[cb][e % 4] * z_scale[cb] : v[cb][e % 4];
#pragma unroll
                        for (int k = 0; k < PARTS; ++k) {
                            part[k].v.v[e] = from_f32<T>(u);
                            if (k + 1 < PARTS)
                                u -= to_f32(part[k].v.v[e]);
                            if constexpr (F16)
                                u *= kLowPart;
                        }
                    }
                    f4 high[PB], low[PB];   // F16: the parts' sums, for their scales
                    if (!exchanged) {
                        if constexpr (F16) {
                            const float back = one_over(z_scale[cb]);
#pragma unroll
                            for (int pb = 0; pb < PB; ++pb)
                                low[pb] = mfma(yt[pb], part[1], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int pb = 0; pb < PB; ++pb)
                                high[pb] = mfma(yt[pb], part[0], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int pb = 0; pb < PB; ++pb)
                                st[pb][cb] += (high[pb] + low[pb] / kLowPart) * back;
                        } else {
#pragma unroll
                            for (int k = 0; k < PARTS; ++k)
#pragma unroll
                                for (int pb = 0; pb < PB; ++pb)
                                    st[pb][cb] = mfma(yt[pb], part[k], st[pb][cb]);
                        }
                        continue;
                    }
                    const int c = 16 * cb + 4 * g;
                    f4 r[PB], back;   // 1 over the scales of the lane's four columns
                    if constexpr (F16)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            back[j] = __shfl(one_over(z_scale[cb]), 4 * g + j);
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb) {
                        const int row = 16 * pb + i16;
                        r[pb] = f4{0.f, 0.f, 0.f, 0.f};
                        if (from && row < A.p) {
                            const float *p = from + (row * A.r + c);
                            if (c + 4 <= A.r)
                                __builtin_memcpy(&r[pb], p, 16);
                            else
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    if (c + j < A.r)
                                        r[pb][j] = p[j];
                            r[pb] *= whole;
                        }
                    }
                    if constexpr (F16) {
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb)
                            low[pb] = mfma(part[1], yt[pb], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb)
                            high[pb] = mfma(part[0], yt[pb], f4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb)
                            r[pb] += (high[pb] + low[pb] / kLowPart) * back;
                    } else {
#pragma unroll
                        for (int k = 0; k < PARTS; ++k)
#pragma unroll
                            for (int pb = 0; pb < PB; ++pb)
                                r[pb] = mfma(part[k], yt[pb], r[pb]);
                    }
#pragma unroll
                    for (int pb = 0; pb < PB; ++pb) {
                        const int row = 16 * pb + i16;
                        float *p = to + (row * A.r + c);
                        r[pb] *= f;
                        if (row < A.p) {
                            if (c + 4 <= A.r)
                                __builtin_memcpy(p, &r[pb], 16);
                            else
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    if (c + j < A.r)
                                        p[j] = r[pb][j];
                        }
                    }
                }
                some = true;
            }
            lag = 1;
        }
        if (ends && A.last && !exchanged) {
            char *to = reinterpret_cast<char *>(A.last + ((int64_t)piece.s * A.H + h) * size);
            const float f = A.lag1 && !empty ? decay_pow(decay, 1.f) : 1.f;
            each([&](int pb, int cb, int j, size_t base, uint32_t mine)
                     __attribute__((always_inline)) {
                         *reinterpret_cast<float *>(to + base + mine) = f * st[pb][cb][j];
                     });
        }
    }
}

template <class T, class O, int P, int R, bool OUT>
tgm_status_t launch_decay(const DecayRun &r, hipStream_t s)
{
    constexpr int TH = 4 * R;
    const int64_t n = std::min<int64_t>((OUT ? r.ids : r.all_cells) * r.a.H, 1 << 22);
    if (n > 0)
        TGM_LAUNCH((k_decay<T, O, P, R, OUT>), dim3((uint32_t)n), dim3(TH), 0, s, r);
    return TGM_OK;
}
template <class T, class O, int P, int R>
tgm_status_t launch_short(const DecayRun &r, hipStream_t s)
{
    const int64_t n = std::min<int64_t>(cdiv(r.ids * r.a.H, 4), 1 << 22);
    if (n > 0)
        TGM_LAUNCH((k_decay_short<T, O, P, R>), dim3((uint32_t)n), dim3(256), 0, s, r);
    return TGM_OK;
}
// The smallest tile that a head fits.  us in tiles of 32 x 32, 64 x 64 and 128 x 128, 262,144 rows
// of 8 heads in one sequence: of 32 x 32 bf16 252, 400 and 920, fp32 423, 843 and 2,319; of 64 x
// 64 bf16 498 and 1,014, fp32 838 and 2,399; of 64 x 128 (its own tile first) bf16 825 and 1,019,
// of 128 x 64 707 and 956.  Short sequences of 32 x 32 with their states: bf16 750 and 1,497.
template <class T, class O, bool OUT> tgm_status_t pick_decay(const DecayRun &r, hipStream_t s)
{
    const int p = r.a.p, q = r.a.r;
    if constexpr (OUT)
        if (r.brief && p <= 64 && q <= 64)
            return p <= 32 && q <= 32 ? launch_short<T, O, 32, 32>(r, s)
                                      : launch_short<T, O, 64, 64>(r, s);
    if (p <= 32 && q <= 32)
        return launch_decay<T, O, 32, 32, OUT>(r, s);
    if (p <= 64)
        return q <= 64 ? launch_decay<T, O, 64, 64, OUT>(r, s)
                       : launch_decay<T, O, 64, 128, OUT>(r, s);
    return q <= 64 ? launch_decay<T, O, 128, 64, OUT>(r, s)
                   : launch_decay<T, O, 128, 128, OUT>(r, s);
}
// what: 0 states, 1 results of type T, 2 results in fp32
template <class T> tgm_status_t run_decay(const DecayRun &r, int what, hipStream_t s)
{
    if (what == 0)
        return pick_decay<T, float, false>(r, s);
    if constexpr (sizeof(T) == 2)
        if (what == 2)
            return pick_decay<T, float, true>(r, s);
    return pick_decay<T, T, true>(r, s);
}

}  // namespace tgm
