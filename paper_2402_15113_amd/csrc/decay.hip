// Linear attention with a decay for each head along packed or padded sequences
// (tgm_decay_attn), its gradient (tgm_decay_attn_backward) and its single-row form
// (tgm_decay_attn_step).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "decay.h"

using namespace tgm;

namespace {

// Row by row: a workgroup has a sequence's head, its state in registers, 256 / RW groups of
// threads with every (256 / RW)-th of the state's rows and a column each.
constexpr int kRowThreads = 256;
template <class T, class O, int RW>
__global__ __launch_bounds__(kRowThreads) void k_decay_rows(DecayArgs A)
{
    constexpr int G = kRowThreads / RW, NI = kDecayMaxD / G;
    __shared__ float xs[kDecayMaxD], ys[kDecayMaxD], part[G][RW];
    const int j = threadIdx.x % RW, g = threadIdx.x / RW;
    const int32_t h = blockIdx.y;
    const float decay = A.decay[h], a = decay_pow(decay, 1.f);
    const bool col = j < A.r;
    for (int64_t s = blockIdx.x; s < A.S; s += gridDim.x) {
        const DecaySeq q = decay_seq(A, (int32_t)s);
        const int64_t n = q.e - q.b, at = (s * A.H + h) * (int64_t)(A.p * A.r);
        float st[NI];
#pragma unroll
        for (int u = 0; u < NI; ++u) {
            const int i = g + u * G;
            st[u] = A.first && col && i < A.p
                        ? A.first[at + (A.turned ? (int64_t)j * A.p + i : (int64_t)i * A.r + j)]
                        : 0.f;
        }
        for (int64_t t = 0; t < n; ++t) {
            const int64_t row = A.rev ? q.e - 1 - t : q.b + t;
            const float f = t == 0 && A.lag0 == 0 ? 1.f : a;
            if ((int)threadIdx.x < A.p) {
                const T *y = (const T *)A.y.p + row * A.y.ld + (int64_t)(h / A.y.share) * A.p;
                const T *x = (const T *)A.x.p + row * A.x.ld + (int64_t)(h / A.x.share) * A.p;
                ys[threadIdx.x] = A.c_y * to_f32(y[threadIdx.x]);
                xs[threadIdx.x] = to_f32(x[threadIdx.x]);
            }
            const T *z = (const T *)A.z.p + row * A.z.ld + (int64_t)(h / A.z.share) * A.r;
            const float zj = col ? to_f32(z[j]) : 0.f;
            __syncthreads();
            float o = 0.f;
#pragma unroll
            for (int u = 0; u < NI; ++u) {
                const int i = g + u * G;
                if (i < A.p) {
                    st[u] = f * st[u] + ys[i] * zj;
                    o += xs[i] * st[u];
                }
            }
            part[g][j] = o;
            __syncthreads();
            if (A.out && g == 0 && col) {
                for (int k = 1; k < G; ++k)
                    o += part[k][j];
                ((O *)A.out)[row * A.ld_out + (int64_t)h * A.r + j] = from_f32<O>(A.c_out * o);
            }
        }
        if (A.last) {
            const float f = A.lag1 && (n || A.lag0) ? a : 1.f;
#pragma unroll
            for (int u = 0; u < NI; ++u) {
                const int i = g + u * G;
                if (col && i < A.p)
                    A.last[at + (A.turned ? (int64_t)j * A.p + i : (int64_t)i * A.r + j)] =
                        f * st[u];
            }
        }
        __syncthreads();
    }
}

// The gradient of a head of k or v that several heads of q share: theirs added in order, for
// the rows of sequences.  Bound by memory.
constexpr int kSharedRows = 16;
template <class T>
__global__ __launch_bounds__(256) void k_decay_shared(const float *__restrict__ part, DecayArgs A,
                                                      int32_t heads, int32_t share, int32_t d,
                                                      int64_t ld, T *__restrict__ out)
{
    const int64_t ids = (A.rows + kSharedRows - 1) / kSharedRows + A.S, wide = (int64_t)heads * d;
    for (int64_t id = blockIdx.x; id < ids; id += gridDim.x) {
        const DecayPiece p = decay_piece(A, id, kSharedRows);
        for (int64_t i = threadIdx.x; i < (p.hi - p.lo) * wide; i += 256) {
            const int64_t row = p.lo + i / wide;
            const int32_t c = (int32_t)(i % wide), h = c / d;
            const float *q = part + (row * heads + h) * (int64_t)share * d + (c - h * d);
            float s = q[0];
            for (int k = 1; k < share; ++k)
                s += q[(int64_t)k * d];
            out[row * ld + c] = from_f32<T>(s);
        }
    }
}

// One row for each of n states of a table.  A workgroup has a head of one: a thread reads
// and writes VEC neighbouring columns of every G-th row of the state.  Bound by memory.
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
    const float a = decay_pow(decay[h], 1.f);
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

template <class T, class O> tgm_status_t go_rows(const DecayArgs &a, hipStream_t s)
{
    const dim3 grid(across(a.S, a.H), (uint32_t)a.H);
    if (a.S == 0)
        return TGM_OK;
    if (a.r <= 32)
        TGM_LAUNCH((k_decay_rows<T, O, 32>), grid, dim3(kRowThreads), 0, s, a);
    else if (a.r <= 64)
        TGM_LAUNCH((k_decay_rows<T, O, 64>), grid, dim3(kRowThreads), 0, s, a);
    else
        TGM_LAUNCH((k_decay_rows<T, O, 128>), grid, dim3(kRowThreads), 0, s, a);
    return TGM_OK;
}

struct DecayCall {
    const tgm_decay_attn_desc *d;
    int64_t ld_q, ld_k, ld_v, ld_o, ld_dq, ld_dk, ld_dv;
    DecayArgs a;   // the sequences, decays and sizes
    hipStream_t s;
};

template <class T>
tgm_status_t forward(DecayCall &c, const void *q, const void *k, const void *v, const float *first,
                     void *o, float *last)
{
    DecayArgs a = c.a;
    const int32_t share = a.H / c.d->H_kv;
    a.x = DecayIn{q, c.ld_q, 1}, a.y = DecayIn{k, c.ld_k, share};
    a.z = DecayIn{v, c.ld_v, share};
    a.p = c.d->d_k, a.r = c.d->d_v, a.out = o, a.ld_out = c.ld_o;
    a.first = first, a.last = last, a.lag0 = 1, a.c_y = 1.f, a.c_out = c.d->scale;
    return go_rows<T, T>(a, c.s);
}

template <class T>
tgm_status_t backward(DecayCall &c, const void *q, const void *k, const void *v,
                      const float *first, const void *dO, const float *dlast, void *dq, void *dk,
                      void *dv, float *dfirst, char *work)
{
    const tgm_decay_attn_desc *d = c.d;
    const int32_t share = d->H / d->H_kv;
    const DecayIn iq{q, c.ld_q, 1}, ik{k, c.ld_k, share}, iv{v, c.ld_v, share}, io{dO, c.ld_o, 1};
    DecayArgs a = c.a;
    if (dq) {
        a.x = io, a.y = iv, a.z = ik, a.p = d->d_v, a.r = d->d_k, a.turned = 1;
        a.out = dq, a.ld_out = c.ld_dq, a.first = first, a.last = nullptr, a.lag0 = 1;
        a.c_y = 1.f, a.c_out = d->scale;
        TGM_TRY_STATUS((go_rows<T, T>(a, c.s)));
    }
    // the others run against the first one's order
    a.rev = !c.a.rev, a.first = dlast, a.lag0 = 0, a.c_y = d->scale, a.c_out = 1.f;
    auto go = [&](void *out, int32_t width, int64_t ld) -> tgm_status_t {
        if (share == 1 || !out) {
            a.out = out, a.ld_out = ld;
            return go_rows<T, T>(a, c.s);
        }
        a.out = work, a.ld_out = (int64_t)a.H * width;
        TGM_TRY_STATUS((go_rows<T, float>(a, c.s)));
        const int64_t ids = cdiv(a.rows, kSharedRows) + a.S;
        TGM_LAUNCH((k_decay_shared<T>), dim3((uint32_t)std::min<int64_t>(ids, 1 << 16)),
                   dim3(256), 0, c.s, (const float *)work, a, d->H_kv, share, width, ld, (T *)out);
        return TGM_OK;
    };
    if (dk) {
        a.x = iv, a.y = io, a.z = iq, a.p = d->d_v, a.r = d->d_k, a.turned = 1;
        a.last = nullptr;
        TGM_TRY_STATUS(go(dk, d->d_k, c.ld_dk));
    }
    if (dv || dfirst) {
        a.x = ik, a.y = iq, a.z = io, a.p = d->d_k, a.r = d->d_v, a.turned = 0;
        a.last = dfirst, a.lag1 = 1;
        TGM_TRY_STATUS(go(dv, d->d_v, c.ld_dv));
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
    c->a.decay = decay, c->a.offsets = offsets, c->a.length = length;
    c->a.rows = d->rows, c->a.S = d->S, c->a.H = d->H, c->a.rev = d->reverse != 0;
    return TGM_OK;
}
// Padded sequences divide the rows.
tgm_status_t decay_lengths(DecayCall *c)
{
    if (c->a.offsets)
        return TGM_OK;
    if (c->a.S == 0 ? c->a.rows != 0 : c->a.rows % c->a.S != 0)
        return TGM_EINVAL;
    c->a.L = c->a.S ? c->a.rows / c->a.S : 0;
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
               (const T *)k, (const T *)v, c.a.decay, slots, n_rows, state, (T *)o, d);
    return TGM_OK;
}
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
    *bytes = backward && H != H_kv ? whole((size_t)rows * H * std::max(d_k, d_v) * 4) : 0;
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
    if (d->rows && (!q || !k || !v || !o))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_decay_attn_work_bytes(d->rows, d->S, d->H, d->H_kv, d->d_k, d->d_v, d->dtype,
                                             0, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    switch (d->dtype) {
    case TGM_F32: return forward<float>(c, q, k, v, state, o, state_last);
    case TGM_BF16: return forward<bf16>(c, q, k, v, state, o, state_last);
    default: return forward<f16>(c, q, k, v, state, o, state_last);
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
    if (d->rows && (!q || !k || !v || !dO))
        return TGM_EINVAL;
    size_t need = 0;
    TGM_TRY_STATUS(tgm_decay_attn_work_bytes(d->rows, d->S, d->H, d->H_kv, d->d_k, d->d_v, d->dtype,
                                             1, &need));
    TGM_TRY_STATUS(check_work(need, work, work_bytes));
    char *w = (char *)work;
    switch (d->dtype) {
    case TGM_F32:
        return backward<float>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w);
    case TGM_BF16:
        return backward<bf16>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w);
    default:
        return backward<f16>(c, q, k, v, state, dO, dstate_last, dq, dk, dv, dstate, w);
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
