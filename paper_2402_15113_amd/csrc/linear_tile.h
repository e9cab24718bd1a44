// The tiled product of tgm_linear: C[m, n] = sum_k P(n, k) Q(m, k).
//
// A workgroup takes BN columns and BM rows of C.  The sum goes in steps of 128
// bytes of an operand's row (64 elements of 16 bits), two steps' tiles in LDS:
// while one is multiplied the next one arrives.  Bound by the matrix cores for
// large products; a step of a 256 x 256 tile reads LDS for about three quarters
// of the time that its matrix instructions take.
#pragma once

#include <algorithm>

#include "linear.h"

namespace tgm {

typedef short s4v __attribute__((ext_vector_type(4)));

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

    // The fragment of rows (columns) x0 .. x0 + 15 and the c-th 64 bytes of the sum.
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
};

// One operand on its way into LDS.  DIRECT: 16 bytes a lane straight into LDS,
// where its base and rows lie on 16 bytes; else through registers, at any
// alignment.  TH threads.
template <class T, bool KC, int X, int TH, bool DIRECT> struct Operand {
    using Lds = LdsTile<T, KC, X>;
    static constexpr int VEC = Lds::VEC, BK = Lds::BK;
    static constexpr int NR = (Lds::ROWS * Lds::CHUNKS + TH - 1) / TH;   // chunks a thread
    static constexpr int ND = Lds::BYTES / (TH * 16);                    // direct loads a thread
    static_assert(!DIRECT || Lds::BYTES % (TH * 16) == 0, "");

    const T *base;
    int64_t ld;
    int32_t x0, n;              // the tile's first row (column) and how many the operand has
    uint32_t off[DIRECT ? ND : 1];
    Pack<T, VEC> v[DIRECT ? 1 : NR];

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
            }
        }
    }
    // a whole step from k on into `lds`, without waiting for it
    __device__ __forceinline__ void direct(char *lds, int64_t k) const
    {
        const char *from = reinterpret_cast<const char *>(KC ? base + (int64_t)x0 * ld + k
                                                             : base + k * ld + x0);
#pragma unroll
        for (int u = 0; u < ND; ++u) {
            const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds +
                                1024u * (u * (TH / 64) +
                                         __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)));
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :
                         : "s"(to), "v"(off[u]), "s"(from)
                         : "memory", "m0");
        }
    }
    __device__ __forceinline__ Pack<T, VEC> chunk(int row, int c, int64_t k, int64_t K,
                                                  bool whole) const
    {
        Pack<T, VEC> r;
        if (KC) {
            const T *p = base + (int64_t)min(x0 + row, n - 1) * ld + k + c * VEC;
            if (whole || k + (c + 1) * VEC <= K)
                return load_pack<T, VEC>(p);
            __builtin_memset(&r, 0, sizeof(r));
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (k + c * VEC + j < K)
                    r.v[j] = p[j];
        } else {
            const int32_t x = x0 + c * VEC;
            const T *p = base + (k + row) * ld + x;
            if ((whole || k + row < K) && x + VEC <= n)
                return load_pack<T, VEC>(p);
            __builtin_memset(&r, 0, sizeof(r));
            if (whole || k + row < K)
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (x + j < n)
                        r.v[j] = p[j];
        }
        return r;
    }
    // the step from k on (up to K: zeros past it) through registers
    __device__ __forceinline__ void load(int64_t k, int64_t K)
    {
        const bool whole = k + BK <= K;
        if constexpr (!DIRECT) {
#pragma unroll
            for (int u = 0; u < NR; ++u) {
                const int e = min(u * TH + (int)threadIdx.x, Lds::ROWS * Lds::CHUNKS - 1);
                v[u] = chunk(e / Lds::CHUNKS, e % Lds::CHUNKS, k, K, whole);
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
                    *reinterpret_cast<Pack<T, VEC> *>(__builtin_assume_aligned(
                        lds + Lds::at(e / Lds::CHUNKS, e % Lds::CHUNKS), 16)) = v[u];
            }
        }
    }
    // the last, partial step at once
    __device__ __forceinline__ void tail(char *lds, int64_t k, int64_t K) const
    {
        for (int e = threadIdx.x; e < Lds::ROWS * Lds::CHUNKS; e += TH)
            *reinterpret_cast<Pack<T, VEC> *>(__builtin_assume_aligned(
                lds + Lds::at(e / Lds::CHUNKS, e % Lds::CHUNKS), 16)) =
                chunk(e / Lds::CHUNKS, e % Lds::CHUNKS, k, K, false);
    }
};

__device__ __forceinline__ f4 mfma_e4m3(const Frag<e4m3> &p0, const Frag<e4m3> &p1,
                                        const Frag<e4m3> &q0, const Frag<e4m3> &q1, f4 c)
{
    typedef int i8v __attribute__((ext_vector_type(8)));
    struct Two {
        Frag<e4m3> a, b;
    };
    // 128 k at once, at twice the rate of 32; block scales of 1 (the exponent 127)
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
        __builtin_bit_cast(i8v, Two{p0, p1}), __builtin_bit_cast(i8v, Two{q0, q1}), c, 0, 0, 0,
        127, 0, 127);
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

template <class T, class O, bool PK, bool QK, int BN, int BM, int NW, int MW, bool DIRECT>
__global__ __launch_bounds__(64 * NW * MW) void k_linear_tile(
    const T *__restrict__ P, const T *__restrict__ Q, int64_t ld_p, int64_t ld_q, int32_t K_,
    LinearOut o, const int32_t *k_rows, float *work, int32_t tn, int32_t tm, int32_t parts)
{
    constexpr int TH = 64 * NW * MW, NA = BN / NW / 16, MA = BM / MW / 16;
    using OP = Operand<T, PK, BN, TH, DIRECT>;
    using OQ = Operand<T, QK, BM, TH, DIRECT>;
    constexpr int BK = OP::BK;
    __shared__ __attribute__((aligned(1024))) char lds[2][OP::Lds::BYTES + OQ::Lds::BYTES];
    const TileAt t = tile_of(blockIdx.x, tn, tm, parts);
    const int32_t M = rows_in_use(o.M, o.n_rows), n0 = t.n * BN, m0 = t.m * BM;
    if (m0 >= M)
        return;
    const int64_t K = rows_in_use(K_, k_rows);
    const int64_t steps = (K + BK - 1) / BK, per = (steps + parts - 1) / parts;
    const int64_t s0 = t.part * per, ns = max((int64_t)0, min(steps - s0, per));
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int wn = (w % NW) * (BN / NW), wm = (w / NW) * (BM / MW);

    OP p;
    OQ q;
    p.init(P, ld_p, n0, o.N);
    q.init(Q, ld_q, m0, M);
    f4 acc[NA][MA];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int b = 0; b < MA; ++b)
            acc[a][b] = f4{0.f, 0.f, 0.f, 0.f};

    auto fill = [&](int64_t s) __attribute__((always_inline)) {   // direct
        const int64_t k = (s0 + s) * BK;
        char *to = lds[s & 1];
        if (k + BK <= K) {
            p.direct(to, k);
            q.direct(to + OP::Lds::BYTES, k);
        } else {
            p.tail(to, k, K);
            q.tail(to + OP::Lds::BYTES, k, K);
        }
    };
    if (ns > 0) {
        if constexpr (DIRECT) {
            fill(0);
        } else {
            p.load(s0 * BK, K), q.load(s0 * BK, K);
            p.store(lds[0]), q.store(lds[0] + OP::Lds::BYTES);
        }
    }
    for (int64_t s = 0; s < ns; ++s) {
        // this step's tiles are there and no one reads the other ones any more
        if constexpr (DIRECT)
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        if (s + 1 < ns) {
            if constexpr (DIRECT)
                fill(s + 1);
            else
                p.load((s0 + s + 1) * BK, K), q.load((s0 + s + 1) * BK, K);
        }
        const char *lp = lds[s & 1], *lq = lp + OP::Lds::BYTES;
        if constexpr (sizeof(T) == 1 && sizeof(O) != 4) {
            Frag<T> fq[MA][2];
#pragma unroll
            for (int b = 0; b < MA; ++b)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    fq[b][c] = OQ::Lds::read(lq, wm + 16 * b, c);
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const Frag<T> f0 = OP::Lds::read(lp, wn + 16 * a, 0);
                const Frag<T> f1 = OP::Lds::read(lp, wn + 16 * a, 1);
#pragma unroll
                for (int b = 0; b < MA; ++b)
                    acc[a][b] = mfma_e4m3(f0, f1, fq[b][0], fq[b][1], acc[a][b]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                Frag<T> fq[MA];
#pragma unroll
                for (int b = 0; b < MA; ++b)
                    fq[b] = OQ::Lds::read(lq, wm + 16 * b, c);
#pragma unroll
                for (int a = 0; a < NA; ++a) {
                    const Frag<T> f = OP::Lds::read(lp, wn + 16 * a, c);
#pragma unroll
                    for (int b = 0; b < MA; ++b)
                        if constexpr (sizeof(T) == 1)
                            acc[a][b] = mfma_wide(f, fq[b], acc[a][b]);
                        else
                            acc[a][b] = mfma(f, fq[b], acc[a][b]);
                }
            }
        }
        if constexpr (!DIRECT)
            if (s + 1 < ns)
                p.store(lds[(s + 1) & 1]), q.store(lds[(s + 1) & 1] + OP::Lds::BYTES);
    }

    const int32_t wide = (o.N + 3) & ~3;
#pragma unroll
    for (int b = 0; b < MA; ++b) {
        const int32_t m = m0 + wm + 16 * b + (lane & 15);
        if (m < M)
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const int32_t n = n0 + wn + 16 * a + 4 * (lane >> 4);
                if (n < o.N) {
                    if (work)
                        *reinterpret_cast<f4 *>(work + ((int64_t)t.part * o.M + m) * wide + n) =
                            acc[a][b];
                    else
                        finish<O>(o, m, n, acc[a][b]);
                }
            }
    }
}

// The parts' sums added in order.
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

template <class T, class O, bool PK, bool QK, int BN, int BM, int NW, int MW>
tgm_status_t launch_tile(const LinearProduct &p, int parts)
{
    const int32_t tn = (int32_t)cdiv(p.o.N, BN), tm = (int32_t)cdiv(p.o.M, BM);
    const dim3 grid((uint32_t)((int64_t)tn * tm * parts)), block(64 * NW * MW);
    float *work = parts > 1 ? p.work : nullptr;
    if (lies_on_16<T, PK>(p.P, p.ld_p, p.o.N) && lies_on_16<T, QK>(p.Q, p.ld_q, p.o.M))
        TGM_LAUNCH((k_linear_tile<T, O, PK, QK, BN, BM, NW, MW, true>), grid, block, 0, p.s,
                   (const T *)p.P, (const T *)p.Q, p.ld_p, p.ld_q, p.K, p.o, p.k_rows, work, tn,
                   tm, parts);
    else
        TGM_LAUNCH((k_linear_tile<T, O, PK, QK, BN, BM, NW, MW, false>), grid, block, 0, p.s,
                   (const T *)p.P, (const T *)p.Q, p.ld_p, p.ld_q, p.K, p.o, p.k_rows, work, tn,
                   tm, parts);
    if (parts > 1)
        TGM_LAUNCH((k_linear_join<O>),
                   dim3((uint32_t)std::min<int64_t>(cdiv((int64_t)p.o.M * cdiv(p.o.N, 4), 256),
                                                    1 << 14)),
                   dim3(256), 0, p.s, p.work, p.o, parts);
    return TGM_OK;
}

}  // namespace tgm
