/*
 * Internal interface of the operators on the loaded layout: what their entry points (cfa_ops.cu)
 * hand to the kernels of the products (cfa_matmul.cu), of the choice of experts (cfa_route.cu) and
 * of the sorting of tokens by expert (cfa_sort.cu).  Not part of the C ABI.
 */
#ifndef CFA_OPS_H
#define CFA_OPS_H

#include <cuda_runtime.h>
#include <stdint.h>

#include "cfa.h"
#include "cfa_internal.h"

/*
 * y = act(x w^T + bias) + residual for one or several groups of x's rows, each with its own w.
 *
 * One group: `tokens` rows of x.  Several (n_groups > 1 or offs given): group g owns the rows
 * [offs[g], offs[g + 1]) of x, y and residual (offs in device memory, offs[n_groups] <= tokens), and
 * its weight starts at row g * w_rows of w.
 * gated: w holds w_rows / 2 gate rows and as many up rows, y has w_rows / 2 columns.
 */
typedef struct cfa_matmul {
    const void *x, *w, *bias, *residual;
    void *y;
    const int32_t *offs;
    /* ids: the choices from which offs was counted, if the kernel is to count for itself: then it needs
     * offs only as a mark.  w_ready: w and the choices (without ids: offs) are in memory when the
     * launch starts, although the launch before it may not have ended */
    const int32_t *ids;
    int32_t n_ids, first, w_ready;
    int64_t tokens, w_rows, cols;
    int64_t x_stride, w_stride, r_stride, y_stride; /* elements */
    int32_t n_groups;
    int32_t f16;      /* 1: binary16, 0: bf16 (x, w; bias, residual and y unless f32) */
    int32_t bias_f32, y_f32;
    int64_t bias_up;  /* gated: where the up rows' bias starts, in elements */
    int32_t act, gated;
    int32_t exact;    /* 1: the sums are rounded as fp32 results are to be */
    int32_t lose;     /* self-test, 1: the loads are not issued, 2: the epilogue gives up */
    int32_t busy;     /* groups that can hold rows at all (host's bound) */
    int64_t likely;   /* rows to expect in all groups, at most `tokens` */
} cfa_matmul;

/* The pairs (token, choice) sorted by expert. */
typedef struct cfa_sort {
    const int32_t *ids; /* [pairs] */
    int64_t pairs;
    int32_t top_k, first, experts;
    int32_t *hist;      /* [cfa_sort_blocks(pairs), experts] */
    int32_t *offs;      /* [experts + 1] out: where each expert's rows start */
    int32_t *place;     /* [pairs] out: a pair's row, -1 if its expert is elsewhere */
} cfa_sort;

/* All of these enqueue on `stream` and return a CUDA error. `early`: may start before the kernel
 * before it on the stream has ended, and waits inside; `release`: its dependents may do so. */
cudaError_t cfa_launch_matmul(const cfa_matmul *m, int early, int release, cudaStream_t stream);
/* CTAs in which a wait has run out, and those of them whose loads in flight did not end either: counted
 * up on the device and never set back, so that no reader takes anything from another. */
typedef struct cfa_op_counts {
    uint32_t ran_out, in_flight;
} cfa_op_counts;
/* What has been counted since *seen, which becomes `now`: 0 nothing, 1 waits that ran out, 2 loads in
 * flight too.  Lower counts than those seen are a new start of the device's. */
static inline int cfa_op_news(cfa_op_counts *seen, cfa_op_counts now)
{
    if ((int32_t)(now.ran_out - seen->ran_out) < 0 || (int32_t)(now.in_flight - seen->in_flight) < 0)
        seen->ran_out = seen->in_flight = 0;
    const int word = now.in_flight != seen->in_flight ? 2 : now.ran_out != seen->ran_out ? 1 : 0;
    *seen = now;
    return word;
}
/* The current device's news since the calling thread last asked. */
cudaError_t cfa_matmul_status(int *word);
cudaError_t cfa_matmul_selftest(int *word);
cudaError_t cfa_launch_route(const cfa_route_args *a, cudaStream_t stream);
/* Rows of hist that the sort of so many pairs needs. */
int64_t cfa_sort_blocks(int64_t pairs);
/* The sort, and the tokens' rows of x into their places in xs (rows of `hidden` elements). */
cudaError_t cfa_launch_sort(const cfa_sort *s, const void *x, int64_t x_stride, int64_t hidden,
                            void *xs, cudaStream_t stream);
/* y[t] = residual[t] + sum_j weights[t, j] part[place[t, j]]. */
typedef struct cfa_combine {
    const float *part; /* [rows, hidden] */
    const float *weights;
    const int32_t *place;
    const void *residual;
    void *y;
    int64_t tokens, hidden, r_stride, y_stride;
    int32_t top_k, f16;
} cfa_combine;
cudaError_t cfa_launch_combine(const cfa_combine *c, cudaStream_t stream);
/* Rows of cols 2-byte elements onto rows of to_stride (a multiple of 8) elements at a 16-byte aligned
 * address, the rest of each row zeros: up to three matrices, none empty. */
typedef struct cfa_rows {
    const void *from;
    void *to;
    int64_t from_stride, to_stride, rows, cols;
} cfa_rows;
cudaError_t cfa_launch_realign(const cfa_rows *m, int n, cudaStream_t stream);

cudaError_t cfa_launch_norm(const cfa_norm_args *a, cudaStream_t stream);
cudaError_t cfa_launch_append(const cfa_append_args *a, cudaStream_t stream);
cudaError_t cfa_launch_logprobs(const cfa_logprobs_args *a, cudaStream_t stream);

#define CFA_ATTEND_BLOCKS 152 /* of a launch, one to an SM */
typedef struct cfa_attend_work {
    cfa_attend_args a;
    int32_t group, row_tiles; /* query heads of a key head; tiles of a sequence and key head */
    int32_t nt;               /* a tile has 8 nt rows */
    uint32_t group_inverse;   /* 2^32 / group, rounded up */
    float *parts;             /* [CFA_ATTEND_BLOCKS][2] partials */
    unsigned long long *marks; /* [CFA_ATTEND_BLOCKS][2]: the partials that are there */
    unsigned long long number; /* of the call, its mark; not 0 */
} cfa_attend_work;
cudaError_t cfa_launch_attend_bf16(const cfa_attend_work *w, cudaStream_t stream);
cudaError_t cfa_launch_attend_f16(const cfa_attend_work *w, cudaStream_t stream);
cudaError_t cfa_launch_attend_bf16_f8(const cfa_attend_work *w, cudaStream_t stream);
cudaError_t cfa_launch_attend_f16_f8(const cfa_attend_work *w, cudaStream_t stream);

#endif /* CFA_OPS_H */
