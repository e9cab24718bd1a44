// What the kernels of the cross entropy over classes (tgm_xent) share.
#pragma once

#include "linear.h"

namespace tgm {

// A product's logits, of columns n_first .. n_first + N - 1 of all classes, on their way
// into sums (XentSums) or into their gradient (XentGrad).
struct XentArgs {
    const void *bias;        // of the product's columns; may be null
    const int32_t *target;   // [rows]
    int32_t rows, classes, n_first;
    // sums
    f2 *part;                // [parts x rows]: the largest logit of a run of columns, and the
                             // sum of exponentials relative to it
    float *at_target;        // [rows]
    // gradient
    const float *lse, *dloss;
    const float *scale;      // a power of two that dz is held times; may be null
    void *dz;
    int64_t ld_dz;
    float *db;               // [parts x N] partial sums of columns; may be null
};

// Runs of columns that the sums come in, and of rows that db's do, at most; the tiles of
// csrc/xent_tile.h hold runs of 64 columns or more, and of 64 rows (fp32: 16) or more.
inline int64_t xent_parts(int64_t N) { return cdiv(N, 128) * 2; }
inline int64_t xent_db_parts(int64_t rows, int code)
{
    return code == TGM_F32 ? cdiv(rows, 64) * 4 : cdiv(rows, 256) * 4;
}
// What a launch came to: runs of columns, rows to a run of db's and runs to a tile.
struct XentRuns {
    int32_t columns, tile_rows, tile_runs;
};

tgm_status_t xent_sums_f32(const LinearProduct &p, const XentArgs &e, XentRuns *r);
tgm_status_t xent_sums_bf16(const LinearProduct &p, const XentArgs &e, XentRuns *r);
tgm_status_t xent_sums_f16(const LinearProduct &p, const XentArgs &e, XentRuns *r);
tgm_status_t xent_grad_f32(const LinearProduct &p, const XentArgs &e, XentRuns *r);
tgm_status_t xent_grad_bf16(const LinearProduct &p, const XentArgs &e, XentRuns *r);
tgm_status_t xent_grad_f16(const LinearProduct &p, const XentArgs &e, XentRuns *r);
// dx of a piece of the classes in fp32, added to what is there.
tgm_status_t xent_dx_bf16(const LinearProduct &p);
tgm_status_t xent_dx_f16(const LinearProduct &p);
// dW, of another x (dense rows of ld, on 16 bytes) where *take is not zero.
tgm_status_t xent_dw_f32(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take);
tgm_status_t xent_dw_bf16(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take);
tgm_status_t xent_dw_f16(const LinearProduct &p, const void *x, int64_t ld, const int32_t *take);

}  // namespace tgm
