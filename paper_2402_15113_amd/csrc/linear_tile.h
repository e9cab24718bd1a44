// The tiled product of tgm_linear: C[m, n] = sum_k P(n, k) Q(m, k).
//
// A workgroup takes BN columns and BM rows of C.  The sum goes in steps of 128
// bytes of an operand's row (64 elements of 16 bits), two steps' tiles in LDS.  A
// step has two halves, each with its fragments in registers: while one half is
// multiplied the other half's fragments (or the next step's first) are read, and
// the tile that was read last is refilled, a piece after every few matrix
// instructions: a wavefront issues in order, and LDS takes all wavefronts' reads of
// a half at 4 cycles each, so that reads issued at once left the matrix cores idle
// for half of the time.  Bound by the matrix cores for large products: 8 bit, 16,384 x
// 4,096 x 8,192: 414 to 432 us, 2.6 PFLOP/s; bf16, 8,192 x 8,192 x 8,192: 763 to 797 us, 1.4
// PFLOP/s; fp32, 8,192 x 4,096 x 2,048: 983 us, 140 TFLOP/s.
#pragma once

#include <algorithm>
#include <type_traits>

#include "linear.h"

namespace tgm {

typedef short s4v __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));

// An operand's tile in LDS: X elements along the output, 128 bytes along the sum.
// KC (contiguous along the sum): X rows of 128 bytes; else a row of X elements for
// every k.  16-byte chunks change places within a row, so that the lanes of a
// read meet different banks.
template <class T, bool KC, int X> struct LdsTile {
    static constexpr int VEC = 16 / (int)sizeof(T), BK = 128 / (int)sizeof(T);
    static constexpr int kPow2 = X * sizeof(T) <= 256 ? 256 : X * sizeof(T) <= 512 ? 512 : 1024;
    static constexpr int PITCH = KC ? 128 : kPow2;
    static constexpr int ROWS = KC ? X : BK;
    static constexpr int CHUNKS = KC ? 8 : X * (int)sizeof(T) / 16;
    static constexpr int BYTES = ROWS * PITCH;
    static_assert(KC || sizeof(T) > 1, "");

    static __device__ __forceinline__ int turn(int row)
    {
        if (KC)
            return row & 7;
        if (sizeof(T) == 2)   // the 16 rows of a transposing read: k & 3, k >> 3
            return 2 * (((row & 3) | ((row >> 3) & 3) << 2) & (PITCH / 32 - 1));
        return 4 * ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int chunk)
    {
        return row * PITCH + ((chunk ^ turn(row)) << 4);
    }

    // The fragment of rows (columns) x0 .. x0 + 15 in half c of the step.
    static __device__ __forceinline__ Frag<T> read(const char *lds, int x0, int c)
    {
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        Frag<T> f;
        if constexpr (KC) {
            f.v = *reinterpret_cast<const Pack<T, VEC> *>(
                __builtin_assume_aligned(lds + at(x0 + i, 4 * c + q), 16));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 rows of 16 elements; lane i gets column i
            typedef __attribute__((address_space(3))) s4v *lds_s4;
            s4v v[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int k = 32 * c + 8 * q + 4 * t + (i >> 2), x = x0 + 4 * (i & 3);
                const char *p = lds + at(k, x >> 3) + 8 * (i & 1);
                v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s4)(__attribute__((address_space(3))) void *)const_cast<char *>(p));
            }
            __builtin_memcpy(&f.v, v, sizeof(v));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                f.v.v[j] = *reinterpret_cast<const T *>(
                    lds + at(16 * c + 4 * q + j, (x0 + i) >> 2) + 4 * (i & 3));
        }
        return f;
    }
    // For the 32 x 32 x 64 instruction of 8-bit values: rows x0 .. x0 + 31, 32 bytes a
    // lane.
    static __device__ __forceinline__ i8v read32(const char *lds, int x0, int c)
    {
        const int lane = threadIdx.x & 63, i = lane & 31, q = lane >> 5;
        typedef int i4v __attribute__((ext_vector_type(4)));
        const i4v a = *reinterpret_cast<const i4v *>(
            __builtin_assume_aligned(lds + at(x0 + i, 4 * c + q), 16));
        const i4v b = *reinterpret_cast<const i4v *>(
            __builtin_assume_aligned(lds + at(x0 + i, 4 * c + q + 2), 16));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// One operand on its way into LDS.  DIRECT: 16 bytes a lane straight into LDS,
// where its base and rows lie on 16 bytes; else through registers, at any
// alignment.  TH threads.
template <class T, bool KC, int X, int TH, bool DIRECT> struct Operand {
    using Lds = LdsTile<T, KC, X>;
    static constexpr int VEC = Lds::VEC, BK = Lds::BK;
    static constexpr int NR = (Lds::ROWS * Lds::CHUNKS + TH - 1) / TH;   // chunks a thread
    static constexpr int ND = (Lds::BYTES + TH * 16 - 1) / (TH * 16);    // direct loads a thread
    static_assert(Lds::BYTES % 1024 == 0, "");

    const T *base;
    int64_t ld;
    int32_t x0, n;              // the tile's first row (column) and how many the operand has
    uint32_t off[DIRECT ? ND : 1];
    // of a vector type, which the compiler loads as one (a Pack it takes apart)
    typedef unsigned u4v __attribute__((ext_vector_type(4), may_alias));
    typedef u4v u4v_any __attribute__((aligned(1)));
    u4v v[DIRECT ? 1 : NR];

    __device__ __forceinline__ void init(const T *p, int64_t ld_, int32_t x0_, int32_t n_)
    {
        base = p, ld = ld_, x0 = x0_, n = n_;
        if constexpr (DIRECT) {
            // chunk e of LDS, in the order that a wavefront's lanes fill it
#pragma unroll
            for (int u = 0; u < ND; ++u) {
                const int e = (u * (TH / 64) + (int)(threadIdx.x >> 6)) * 64 + (threadIdx.x & 63);
                const int row = e / (Lds::PITCH / 16);
                const int c = (e % (Lds::PITCH / 16)) ^ Lds::turn(row);
                // past the edge: the last one again, whose results are not kept
                off[u] = KC ? (uint32_t)(min(x0 + row, n - 1) - x0) * (uint32_t)(ld * sizeof(T)) +
                                  16u * c
                            : (uint32_t)row * (uint32_t)(ld * sizeof(T)) +
                                  (uint32_t)(min(x0 + c * VEC, n - VEC) - x0) * (uint32_t)sizeof(T);
                // a register of its own: a product's upper half would stay with it
                asm volatile("" : "+v"(off[u]));
            }
        }
    }
    // the u-th of the ND loads of a whole step from k on into `lds`, without waiting
    // for it; `from` as from_k(k)
    __device__ __forceinline__ const char *from_k(int64_t k) const
    {
        return reinterpret_cast<const char *>(KC ? base + (int64_t)x0 * ld + k
                                                 : base + k * ld + x0);
    }
    __device__ __forceinline__ void direct(char *lds, const char *from, int u) const
    {
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds +
                            1024u * (u * (TH / 64) +
                                     __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)));
        if (Lds::BYTES % (TH * 16) && u == ND - 1 &&
            1024 * (u * (TH / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6))) >=
                Lds::BYTES)
            return;   // a wavefront past the tile's end
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :
                     : "s"(to), "v"(off[u]), "s"(from)
                     : "memory", "m0");
    }
    // Whether a step from k on can be loaded by vectors: a whole one, of rows that hold
    // one.  Others go by elements (tail).
    __device__ __forceinline__ bool by_vectors(int64_t k, int64_t K) const
    {
        return k + BK <= K && (KC || n >= VEC);
    }
    __device__ __forceinline__ void load(int64_t k)
    {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int u = 0; u < NR; ++u) {
                const int e = min(u * TH + (int)threadIdx.x, Lds::ROWS * Lds::CHUNKS - 1);
                const int row = e / Lds::CHUNKS, x = x0 + e % Lds::CHUNKS * VEC;
                if (KC) {
                    v[u] = *reinterpret_cast<const u4v_any *>(
                        base + (int64_t)min(x0 + row, n - 1) * ld + k + e % Lds::CHUNKS * VEC);
                } else {
                    // past the edge: the last vector, moved up to the columns asked for
                    const int back = max(0, x - (n - VEC));
                    v[u] = *reinterpret_cast<const u4v_any *>(base + (k + row) * ld + (x - back));
                    if (back)
                        v[u] = __builtin_bit_cast(u4v, back < VEC
                                   ? __builtin_bit_cast(unsigned __int128, v[u]) >>
                                         (8 * (int)sizeof(T) * back)
                                   : (unsigned __int128)0);
                }
            }
        }
    }
    __device__ __forceinline__ void store(char *lds) const
    {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int u = 0; u < NR; ++u) {
                const int e = u * TH + (int)threadIdx.x;
                if (Lds::ROWS * Lds::CHUNKS % TH == 0 || e < Lds::ROWS * Lds::CHUNKS)
                    *reinterpret_cast<u4v *>(
                        lds + Lds::at(e / Lds::CHUNKS, e % Lds::CHUNKS)) = v[u];
            }
        }
    }
    // The last, partial step at once: zeros past K.  By vectors where none of them
    // straddles K (or the operand's edge), else by elements, several on their way
    // together.
    __device__ __forceinline__ void tail(char *lds, int64_t k, int64_t K) const
    {
        if (KC ? K % VEC == 0 : n % VEC == 0) {
#pragma unroll 2
            for (int u = 0; u < NR; ++u) {
                const int e = u * TH + (int)threadIdx.x;
                const int row = min(e / Lds::CHUNKS, Lds::ROWS - 1), c = e % Lds::CHUNKS;
                const int32_t x = x0 + (KC ? row : c * VEC);
                const int64_t kk = k + (KC ? c * VEC : row);
                // past the ends: the last one again
                const T *from = KC ? base + (int64_t)min(x, n - 1) * ld + min(kk, K - VEC)
                                   : base + min(kk, K - 1) * ld + min(x, n - VEC);
                Pack<T, VEC> r = load_pack<T, VEC>(from);
                if (kk >= K)
                    __builtin_memset(&r, 0, sizeof(r));
                if (e < Lds::ROWS * Lds::CHUNKS)
                    *reinterpret_cast<Pack<T, VEC> *>(
                        __builtin_assume_aligned(lds + Lds::at(row, c), 16)) = r;
            }
            return;
        }
        constexpr int PER = KC ? BK : Lds::CHUNKS * VEC, MANY = 8;
        constexpr int ALL = Lds::ROWS * PER;
#pragma unroll 1
        for (int e0 = threadIdx.x; e0 < ALL; e0 += MANY * TH) {
            T v[MANY];
#pragma unroll
            for (int j = 0; j < MANY; ++j) {
                const int e = min(e0 + j * TH, ALL - 1), row = e / PER, i = e % PER;
                const int64_t kk = min(k + (KC ? i : row), K - 1);
                v[j] = KC ? base[(int64_t)min(x0 + row, n - 1) * ld + kk]
                          : base[kk * ld + min(x0 + i, n - 1)];
            }
#pragma unroll
            for (int j = 0; j < MANY; ++j) {
                const int e = e0 + j * TH, row = e / PER, i = e % PER;
                if (k + (KC ? i : row) >= K)
                    __builtin_memset(&v[j], 0, sizeof(T));
                if (e < ALL)
                    *reinterpret_cast<T *>(lds + Lds::at(row, i / VEC) +
                                           i % VEC * (int)sizeof(T)) = v[j];
            }
        }
    }
};

// Between a wavefront's lanes' writes to LDS and its other lanes' reads of them, and back:
// LDS serves a wavefront in order, so that only the compiler has to be kept from moving
// them (no instruction).
__device__ __forceinline__ void lanes_exchange()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Which tile workgroup `id` takes: every XCD (id % 8) a run of neighbouring tiles,
// 8 rows of tiles deep, so that its L2 holds what they share.
struct TileAt {
    int32_t n, m, part;
};
__device__ __forceinline__ TileAt tile_of(uint32_t id, int32_t tn, int32_t tm, int32_t parts)
{
    const uint32_t total = (uint32_t)tn * tm * parts, each = total / 8;
    if (id < each * 8)
        id = (id % 8) * each + id / 8;
    const uint32_t tiles = (uint32_t)tn * tm, part = id / tiles, t = id - part * tiles;
    const uint32_t band = t / (8u * tn), r = t - band * 8u * tn;
    const uint32_t deep = min(8u, (uint32_t)tm - band * 8u);
    return TileAt{(int32_t)(r / deep), (int32_t)(band * 8 + r % deep), (int32_t)part};
}

// One half step's fragments of a wavefront, and their products.
template <class T, class O, class LP, class LQ, int NA, int MA> struct Half {
    Frag<T> p[NA], q[MA];
    using Acc = f4;
    static constexpr int SIDE = 16;
    // piece a of NA
    __device__ __forceinline__ void read(const char *lp, const char *lq, int wn, int wm, int c,
                                         int a)
    {
        p[a] = LP::read(lp, wn + 16 * a, c);
#pragma unroll
        for (int b = a * MA / NA; b < (a + 1) * MA / NA; ++b)
            q[b] = LQ::read(lq, wm + 16 * b, c);
    }
    // used: blocks of columns that C has (the others' products are left out)
    __device__ __forceinline__ void multiply(Acc (&acc)[NA][MA], int a, int used) const
    {
        if constexpr (sizeof(T) == 4) {
            // a quarter of the sum for every block: four instructions in a row on one
            // block would wait for each other
            static_assert(NA == 4, "");
#pragma unroll
            for (int i = 0; i < NA; ++i)
                if (i < used)
#pragma unroll
                    for (int b = 0; b < MA; ++b)
                        acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                            p[i].v.v[a], q[b].v.v[a], acc[i][b], 0, 0, 0);
        } else {
#pragma unroll
            for (int b = 0; b < MA; ++b)
                if constexpr (sizeof(T) == 1)
                    acc[a][b] = mfma_wide(p[a], q[b], acc[a][b]);
                else
                    acc[a][b] = mfma(p[a], q[b], acc[a][b]);
        }
    }
};
// 8-bit operands: blocks of 32 x 32, 64 k an instruction, which runs at twice the rate
// of those for 32 k.
template <class T, class O, class LP, class LQ, int NA, int MA> struct Half8 {
    i8v p[NA], q[MA];
    using Acc = f16v;
    static constexpr int SIDE = 32;
    __device__ __forceinline__ void read(const char *lp, const char *lq, int wn, int wm, int c,
                                         int a)
    {
        p[a] = LP::read32(lp, wn + 32 * a, c);
#pragma unroll
        for (int b = a * MA / NA; b < (a + 1) * MA / NA; ++b)
            q[b] = LQ::read32(lq, wm + 32 * b, c);
    }
    __device__ __forceinline__ void multiply(Acc (&acc)[NA][MA], int a, int) const
    {
        // block scales of 1 (the exponent 127)
#pragma unroll
        for (int b = 0; b < MA; ++b)
            acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                p[a], q[b], acc[a][b], 0, 0, 0, 127, 0, 127);
    }
};

template <class T, class O, bool PK, bool QK, int BN, int BM, int NW, int MW, bool DIRECT>
__global__ __launch_bounds__(64 * NW * MW, 2) void k_linear_tile(
    const T *__restrict__ P, const T *__restrict__ Q, int64_t ld_p, int64_t ld_q, int32_t K_,
    LinearOut o, const int32_t *k_rows, float *work, int32_t tn, int32_t tm, int32_t parts)
{
    constexpr int TH = 64 * NW * MW;
    constexpr bool BIG = sizeof(T) == 1 && sizeof(O) != 4;
    constexpr int SIDE = BIG ? 32 : 16, NA = BN / NW / SIDE, MA = BM / MW / SIDE;
    using OP = Operand<T, PK, BN, TH, DIRECT>;
    using OQ = Operand<T, QK, BM, TH, DIRECT>;
    using LP = typename OP::Lds;
    using LQ = typename OQ::Lds;
    using H = std::conditional_t<BIG, Half8<T, O, LP, LQ, NA, MA>, Half<T, O, LP, LQ, NA, MA>>;
    constexpr int BK = OP::BK;
    __shared__ __attribute__((aligned(1024))) char lds[2][LP::BYTES + LQ::BYTES];
    const TileAt t = tile_of(blockIdx.x, tn, tm, parts);
    const int32_t M = rows_in_use(o.M, o.n_rows), n0 = t.n * BN, m0 = t.m * BM;
    if (m0 >= M)
        return;
    const int64_t K = rows_in_use(K_, k_rows);
    const int64_t steps = (K + BK - 1) / BK, per = (steps + parts - 1) / parts;
    const int64_t s0 = t.part * per;
    const int32_t ns = (int32_t)max((int64_t)0, min(steps - s0, per));
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wn = (w % NW) * (BN / NW), wm = (w / NW) * (BM / MW);

    const int used = min(NA, (o.N - n0 - wn + SIDE - 1) / SIDE);
    OP p;
    OQ q;
    p.init(P, ld_p, n0, o.N);
    q.init(Q, ld_q, m0, M);
    // Steps that come whole, by vectors; the others go first, by their elements: behind
    // the loop their code would take registers from it.
    const int32_t quick = p.by_vectors(0, BK) && q.by_vectors(0, BK)
                              ? (int32_t)min((int64_t)ns, max((int64_t)0, K / BK - s0)) : 0;
    auto slow = [&](int32_t s) __attribute__((always_inline)) {
        const int64_t k = (s0 + s) * BK;
        p.tail(lds[0], k, K);
        q.tail(lds[0] + LP::BYTES, k, K);
        lds_barrier();
    };
    if (quick < ns)
        slow(quick);
    typename H::Acc acc[NA][MA];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int b = 0; b < MA; ++b)
            acc[a][b] = typename H::Acc(0.f);
    if (quick < ns) {
#pragma unroll 1
        for (int32_t s = quick;;) {
            H h;
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int a = 0; a < NA; ++a)
                    h.read(lds[0], lds[0] + LP::BYTES, wn, wm, c, a);
#pragma unroll
                for (int a = 0; a < NA; ++a)
                    h.multiply(acc, a, used);
            }
            lds_barrier();
            if constexpr (DIRECT) {   // one partial step at most
                break;
            } else {
                if (++s >= ns)
                    break;
                slow(s);
            }
        }
    }

    // Step s into its tile.  DIRECT: on its way there; else into registers (fetch) and
    // from there (put).
    auto fill = [&](int32_t s) __attribute__((always_inline)) {
        const int64_t k = (s0 + s) * BK;
        char *to = lds[s & 1];
        const char *fp = p.from_k(k), *fq = q.from_k(k);
#pragma unroll
        for (int u = 0; u < OP::ND; ++u)
            p.direct(to, fp, u);
#pragma unroll
        for (int u = 0; u < OQ::ND; ++u)
            q.direct(to + LP::BYTES, fq, u);
    };
    auto fetch = [&](int32_t s) __attribute__((always_inline)) {
        p.load((s0 + s) * BK), q.load((s0 + s) * BK);
    };
    auto put = [&](int32_t s) __attribute__((always_inline)) {
        char *to = lds[s & 1];
        p.store(to), q.store(to + LP::BYTES);
    };
    auto arrive = [&]() __attribute__((always_inline)) {
        // by the builtin, which the compiler counts: behind an asm it would wait once
        // more for what it has itself loaded before
        if constexpr (DIRECT)
            __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
        lds_barrier();
    };
    H h0, h1;
    // Step s; NEXT: one follows; MORE: another one follows that, and is called for.
    auto step = [&](int32_t s, auto next, auto more) __attribute__((always_inline)) {
        const char *lp = lds[s & 1];
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            h1.read(lp, lp + LP::BYTES, wn, wm, 1, a);
            h0.multiply(acc, a, used);
            issue_fence();
        }
        const char *ln = lds[(s + 1) & 1];
        if constexpr (next) {
            // the next step's tile is there, and no one reads this one's any more
            if constexpr (!DIRECT)
                put(s + 1);
            arrive();
            if constexpr (!DIRECT && more)
                fetch(s + 2);
        }
        const int64_t k = (s0 + s + 2) * BK;
        const char *fp = p.from_k(k), *fq = q.from_k(k);
        char *to = lds[s & 1];
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            if constexpr (DIRECT && more) {
                constexpr int ND = OP::ND + OQ::ND;
#pragma unroll
                for (int u = a * ND / NA; u < (a + 1) * ND / NA; ++u)
                    if (u < OP::ND)
                        p.direct(to, fp, u);
                    else
                        q.direct(to + LP::BYTES, fq, u - OP::ND);
            }
            if constexpr (next)
                h0.read(ln, ln + LP::BYTES, wn, wm, 0, a);
            h1.multiply(acc, a, used);
            issue_fence();
        }
    };
    if (quick > 0) {
        if constexpr (DIRECT) {
            fill(0);
        } else {
            fetch(0);
            put(0);
        }
        arrive();
        if (quick > 1) {
            if constexpr (DIRECT)
                fill(1);
            else
                fetch(1);
        }
#pragma unroll
        for (int a = 0; a < NA; ++a)
            h0.read(lds[0], lds[0] + LP::BYTES, wn, wm, 0, a);
        using yes = std::true_type;
        using no = std::false_type;
        int32_t s = 0;
        for (; s + 2 < quick; ++s)
            step(s, yes{}, yes{});
        if (s + 1 < quick)
            step(s++, yes{}, no{});
        step(s, no{}, no{});
    }

    constexpr int LANES = SIDE, QUADS = BIG ? 4 : 1;
    auto sums = [&](int a, int b, int u) __attribute__((always_inline)) {
        if constexpr (BIG)
            return f4{acc[a][b][4 * u], acc[a][b][4 * u + 1], acc[a][b][4 * u + 2],
                      acc[a][b][4 * u + 3]};
        else
            return acc[a][b];
    };
    const int32_t n1 = n0 + wn + 4 * (lane / LANES), m1 = m0 + wm + lane % LANES;
    if (work) {
        const int32_t wide = (o.N + 3) & ~3;
#pragma unroll
        for (int b = 0; b < MA; ++b)
            if (m1 + SIDE * b < M)
#pragma unroll
                for (int a = 0; a < NA; ++a)
#pragma unroll
                    for (int u = 0; u < QUADS; ++u) {
                        const int32_t n = n1 + SIDE * a + 8 * u;
                        if (n < o.N)
                            *reinterpret_cast<f4 *>(
                                work + ((int64_t)t.part * o.M + m1 + SIDE * b) * wide + n) =
                                sums(a, b, u);
                    }
        return;
    }
    // A lane holds four columns of a row; through LDS, a block of SIDE rows and CW
    // columns at a time, it gets eight of them, and eight lanes a whole 128-byte line (of
    // 16-bit results) where the wavefront wrote quarters of 16 lines.  A block's residual
    // is loaded before any of it is stored: the compiler, which cannot tell it from
    // y, would wait for every load in turn.
    constexpr int CW = BN / NW < 64 ? BN / NW : 64, PITCH = CW + 4, LPR = CW / 8;
    constexpr int PASS = 64 / LPR, PASSES = SIDE / PASS;   // rows at a time
    static_assert(sizeof(lds) >= NW * MW * SIDE * PITCH * sizeof(float), "");
    lds_barrier();   // no one reads a tile any more
    float *mine = reinterpret_cast<float *>(&lds[0][0]) + w * (SIDE * PITCH);
    const int row = lane / LPR, col = lane % LPR * 8;
#pragma unroll
    for (int cc = 0; cc < BN / NW / CW; ++cc) {
        const int32_t n = n0 + wn + cc * CW + col;
        Columns<O, 8> columns;
        columns.load(o, n);
        Pack<O, 8> res[MA][PASSES];
        float sm[MA][PASSES];
#pragma unroll
        for (int b = 0; b < MA; ++b)
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int32_t m = m0 + wm + SIDE * b + PASS * i + row;
                sm[b][i] = o.sm && m < M ? o.sm[m] : 1.f;
                if (o.res && m < M && columns.left > 0)
                    res[b][i] = columns.residual(o, m, n);
            }
#pragma unroll
        for (int b = 0; b < MA; ++b) {
#pragma unroll
            for (int a = 0; a < CW / SIDE; ++a)
#pragma unroll
                for (int u = 0; u < QUADS; ++u)
                    *reinterpret_cast<f4 *>(mine + lane % LANES * PITCH + SIDE * a +
                                            4 * (lane / LANES) + 8 * u) =
                        sums(cc * (CW / SIDE) + a, b, u);
            lanes_exchange();
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int32_t m = m0 + wm + SIDE * b + PASS * i + row;
                const float *sum = mine + (PASS * i + row) * PITCH + col;
                const f4 *from = reinterpret_cast<const f4 *>(sum);
                const f4 c0 = from[0], c1 = from[1];
                float v[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
                if (m < M && columns.left > 0)
                    columns.finish(o, m, n, v, sm[b][i], res[b][i]);
            }
            lanes_exchange();
        }
    }
}

// The parts' sums added in order.  Bound by memory: two parts of 4,096 x 2,048, to bf16
// (84 MB): 16 us, 5.2 TB/s.
template <class O>
__global__ __launch_bounds__(256) void k_linear_join(const float *__restrict__ work, LinearOut o,
                                                     int32_t parts)
{
    const int32_t M = rows_in_use(o.M, o.n_rows), quads = (o.N + 3) / 4, wide = 4 * quads;
    const int64_t n = (int64_t)M * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / quads;
        const int32_t c = 4 * (int32_t)(i - m * quads);
        f4 a = *reinterpret_cast<const f4 *>(work + m * wide + c);
        for (int z = 1; z < parts; ++z)
            a += *reinterpret_cast<const f4 *>(work + ((int64_t)z * o.M + m) * wide + c);
        finish<O>(o, m, c, a);
    }
}

// ---------------------------------------------------------------- host
template <class T, bool KC> inline bool lies_on_16(const void *X, int64_t ld, int64_t n)
{
    constexpr int VEC = 16 / (int)sizeof(T);
    return ((uintptr_t)X & 15) == 0 && ld % VEC == 0 && ld * (int64_t)sizeof(T) < (1 << 23) &&
           (KC || n % VEC == 0);
}
template <class T, bool PK, bool QK> inline bool direct(const LinearProduct &p)
{
    return lies_on_16<T, PK>(p.P, p.ld_p, p.o.N) && lies_on_16<T, QK>(p.Q, p.ld_q, p.o.M);
}

template <class T, class O, bool PK, bool QK, int BN, int BM, int NW, int MW, bool DIRECT>
tgm_status_t launch_tile(const LinearProduct &p, int parts)
{
    const int64_t tn = cdiv(p.o.N, BN), tm = cdiv(p.o.M, BM), wg = tn * tm * parts;
    if (wg * (64 * NW * MW) >= (int64_t)1 << 32)
        return TGM_EINVAL;
    float *work = parts > 1 ? p.work : nullptr;
    TGM_LAUNCH((k_linear_tile<T, O, PK, QK, BN, BM, NW, MW, DIRECT>), dim3((uint32_t)wg),
               dim3(64 * NW * MW), 0, p.s, (const T *)p.P, (const T *)p.Q, p.ld_p, p.ld_q, p.K, p.o,
               p.k_rows, work, (int32_t)tn, (int32_t)tm, parts);
    if (parts > 1)
        TGM_LAUNCH((k_linear_join<O>),
                   dim3((uint32_t)std::min<int64_t>(cdiv((int64_t)p.o.M * cdiv(p.o.N, 4), 256),
                                                    1 << 14)),
                   dim3(256), 0, p.s, p.work, p.o, parts);
    return TGM_OK;
}

}  // namespace tgm
