/*
 * Entry points of the operators on the loaded layout: they check every argument, carve the
 * workspace and enqueue the kernels.  Nothing is allocated and nothing is read back.
 */
#include <cstdarg>
#include <cstdio>

#include "cfa_ops.h"

namespace {

constexpr uint64_t kAlign = 256; /* of the workspace and its parts */

cfa_status refuse(cfa_status st, const char *fmt, ...)
{
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    cfa_internal_set_error(msg);
    return st;
}

cfa_status cuda_result(const char *what, cudaError_t e)
{
    if (e == cudaSuccess) return CFA_OK;
    return refuse(CFA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

/* Bytes from the first element of a matrix to its last; false if they do not fit 62 bits. */
bool extent(int64_t rows, int64_t cols, int64_t stride, uint64_t size, uint64_t *bytes)
{
    *bytes = 0;
    if (rows == 0 || cols == 0) return true;
    const unsigned __int128 n =
        ((unsigned __int128)(rows - 1) * (uint64_t)(rows > 1 ? stride : 0) + (uint64_t)cols) * size;
    if (n >> 62) return false;
    *bytes = (uint64_t)n;
    return true;
}

bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    const uint64_t p = (uint64_t)(uintptr_t)a, q = (uint64_t)(uintptr_t)b;
    return na && nb && p < q + nb && q < p + na;
}

bool off_grid(const void *p, uint64_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

uint64_t aligned(uint64_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

bool is_half(int32_t dtype) { return dtype == CFA_DTYPE_BF16 || dtype == CFA_DTYPE_F16; }

constexpr int64_t kMost = 1ll << 31; /* rows, columns and strides stay below this */

bool size_ok(int64_t n, int64_t least) { return n >= least && n < kMost; }

/* ---- linear ---- */

bool on_tma_grid(const void *p, int64_t rows, int64_t stride)
{
    return !off_grid(p, 16) && (rows <= 1 || stride % 8 == 0);
}

/* A weight off the grid is moved and multiplied in slices that stay in L2, through the same part of
 * the workspace: moved as a whole it would be written to memory and read again. */
constexpr uint64_t kSliceBytes = 72ull << 20;
constexpr int64_t kSliceRows = 256; /* slices are multiples of this many columns of y */

struct LinearPlan {
    bool move_x, move_w;
    int64_t row;          /* elements of a moved row */
    int64_t slice;        /* columns of y per slice of a moved w (all of them if it stays) */
    uint64_t x_bytes, w_bytes;
};

cfa_status linear_plan(const cfa_linear_args *a, LinearPlan *p)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_linear: NULL arguments");
    if (!is_half(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_linear: x and w are bf16 or f16");
    if (!size_ok(a->tokens, 0) || !size_ok(a->rows, 1) || !size_ok(a->cols, 1))
        return refuse(CFA_ERR_INVAL, "cfa_linear: %lld tokens, %lld rows, %lld columns",
                      (long long)a->tokens, (long long)a->rows, (long long)a->cols);
    if ((a->tokens > 1 && (a->x_stride < a->cols || a->x_stride >= kMost)) ||
        (a->rows > 1 && (a->w_stride < a->cols || a->w_stride >= kMost)))
        return refuse(CFA_ERR_INVAL, "cfa_linear: row strides %lld, %lld of rows of %lld",
                      (long long)a->x_stride, (long long)a->w_stride, (long long)a->cols);
    if (off_grid(a->x, 2) || off_grid(a->w, 2))
        return refuse(CFA_ERR_ALIGN, "cfa_linear: x or w is off its element grid");
    p->row = (a->cols + 7) / 8 * 8;
    p->move_x = !on_tma_grid(a->x, a->tokens, a->x_stride);
    p->move_w = !on_tma_grid(a->w, a->rows, a->w_stride);
    p->x_bytes = p->move_x ? aligned((uint64_t)a->tokens * p->row * 2) : 0;
    const int64_t halves = a->flags & CFA_LINEAR_GATED ? 2 : 1;
    p->slice = (a->rows + halves - 1) / halves;
    if (p->move_w) {
        const int64_t fit = (int64_t)(kSliceBytes / ((uint64_t)p->row * 2 * halves)) / kSliceRows *
                            kSliceRows;
        if (p->slice > fit) p->slice = fit > kSliceRows ? fit : kSliceRows;
        if (p->slice * halves > a->rows) p->slice = (a->rows + halves - 1) / halves;
        p->w_bytes = aligned((uint64_t)(p->slice * halves) * p->row * 2);
    }
    return CFA_OK;
}

} // namespace

extern "C" cfa_status cfa_linear_workspace(const cfa_linear_args *a, uint64_t *bytes)
{
    if (!bytes) return refuse(CFA_ERR_INVAL, "cfa_linear_workspace: NULL output");
    LinearPlan p = {};
    const cfa_status st = linear_plan(a, &p);
    *bytes = st ? 0 : p.x_bytes + p.w_bytes;
    return st;
}

extern "C" cfa_status cfa_linear_async(const cfa_linear_args *a, cfa_stream stream_)
{
    LinearPlan p = {};
    const cfa_status st = linear_plan(a, &p);
    if (st) return st;
    const bool gated = a->flags & CFA_LINEAR_GATED;
    if ((a->flags & ~CFA_LINEAR_GATED) || a->reserved)
        return refuse(CFA_ERR_INVAL, "cfa_linear: unknown flags");
    if (a->activation < CFA_ACT_NONE || a->activation > CFA_ACT_SILU)
        return refuse(CFA_ERR_INVAL, "cfa_linear: unknown activation %d", a->activation);
    if (a->y_dtype != a->dtype && a->y_dtype != CFA_DTYPE_F32)
        return refuse(CFA_ERR_DTYPE, "cfa_linear: y is of x's dtype or f32");
    if (a->bias && a->bias_dtype != a->dtype && a->bias_dtype != CFA_DTYPE_F32)
        return refuse(CFA_ERR_DTYPE, "cfa_linear: the bias is of x's dtype or f32");
    if (gated && a->rows % 2)
        return refuse(CFA_ERR_INVAL, "cfa_linear: %lld rows are no gate and up halves",
                      (long long)a->rows);
    const int64_t outs = gated ? a->rows / 2 : a->rows;
    if (a->tokens > 1 && (a->y_stride < outs || a->y_stride >= kMost ||
                          (a->residual && (a->residual_stride < outs ||
                                           a->residual_stride >= kMost))))
        return refuse(CFA_ERR_INVAL, "cfa_linear: row strides of y or the residual below %lld",
                      (long long)outs);
    if (a->tokens == 0) return CFA_OK;
    if (!a->x || !a->w || !a->y) return refuse(CFA_ERR_INVAL, "cfa_linear: NULL x, w or y");
    const uint64_t ys = a->y_dtype == CFA_DTYPE_F32 ? 4 : 2;
    if (off_grid(a->y, ys) || (a->residual && off_grid(a->residual, ys)) ||
        (a->bias && off_grid(a->bias, a->bias_dtype == CFA_DTYPE_F32 ? 4 : 2)))
        return refuse(CFA_ERR_ALIGN, "cfa_linear: y, residual or bias is off its element grid");
    uint64_t nx, nw, ny, nr;
    if (!extent(a->tokens, a->cols, a->x_stride, 2, &nx) ||
        !extent(a->rows, a->cols, a->w_stride, 2, &nw) ||
        !extent(a->tokens, outs, a->y_stride, ys, &ny) ||
        !extent(a->tokens, outs, a->residual_stride, ys, &nr))
        return refuse(CFA_ERR_INVAL, "cfa_linear: a matrix is too large");
    const uint64_t nb = (uint64_t)a->rows * (a->bias_dtype == CFA_DTYPE_F32 ? 4 : 2);
    const bool in_place = a->residual == a->y &&
                          (a->tokens <= 1 || a->residual_stride == a->y_stride);
    if (overlap(a->y, ny, a->x, nx) || overlap(a->y, ny, a->w, nw) ||
        (a->bias && overlap(a->y, ny, a->bias, nb)) ||
        (a->residual && !in_place && overlap(a->y, ny, a->residual, nr)))
        return refuse(CFA_ERR_OVERLAP, "cfa_linear: y overlaps an input");
    const uint64_t need = p.x_bytes + p.w_bytes;
    if (need) {
        if (!a->workspace || a->workspace_bytes < need)
            return refuse(CFA_ERR_INVAL, "cfa_linear: the workspace must hold %llu bytes",
                          (unsigned long long)need);
        if (off_grid(a->workspace, kAlign))
            return refuse(CFA_ERR_ALIGN, "cfa_linear: the workspace must be 256-byte aligned");
        if (overlap(a->workspace, need, a->x, nx) || overlap(a->workspace, need, a->w, nw) ||
            overlap(a->workspace, need, a->y, ny) ||
            (a->bias && overlap(a->workspace, need, a->bias, nb)) ||
            (a->residual && overlap(a->workspace, need, a->residual, nr)))
            return refuse(CFA_ERR_OVERLAP, "cfa_linear: the workspace overlaps an operand");
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    cfa_matmul m = {};
    m.x = a->x;
    m.x_stride = a->x_stride;
    m.tokens = m.likely = a->tokens;
    m.cols = a->cols;
    m.r_stride = a->residual_stride;
    m.y_stride = a->y_stride;
    m.n_groups = m.busy = 1;
    m.f16 = a->dtype == CFA_DTYPE_F16;
    m.bias_f32 = a->bias && a->bias_dtype == CFA_DTYPE_F32;
    m.bias_up = outs;
    m.y_f32 = m.exact = a->y_dtype == CFA_DTYPE_F32;
    m.act = a->activation;
    m.gated = gated;
    uint8_t *ws = static_cast<uint8_t *>(a->workspace), *wws = ws + p.x_bytes;
    cudaError_t e = cudaSuccess;
    for (int64_t c = 0; !e && c < outs; c += p.slice) {
        const int64_t n = outs - c < p.slice ? outs - c : p.slice;
        cfa_rows move[3];
        int moves = 0;
        if (p.move_x && c == 0) {
            move[moves++] = {a->x, ws, a->x_stride, p.row, a->tokens, a->cols};
            m.x = ws;
            m.x_stride = p.row;
        }
        m.w = a->w;
        m.w_stride = a->w_stride;
        m.w_rows = a->rows;
        if (p.move_w) {
            const uint16_t *w = static_cast<const uint16_t *>(a->w);
            move[moves++] = {w + c * a->w_stride, wws, a->w_stride, p.row, n, a->cols};
            if (gated)
                move[moves++] = {w + (outs + c) * a->w_stride, wws + n * p.row * 2, a->w_stride,
                                 p.row, n, a->cols};
            m.w = wws;
            m.w_stride = p.row;
            m.w_rows = gated ? 2 * n : n;
        }
        if (moves) e = cfa_launch_realign(move, moves, stream);
        m.bias = a->bias ? static_cast<const uint8_t *>(a->bias) + c * (m.bias_f32 ? 4 : 2)
                         : nullptr;
        m.residual = a->residual ? static_cast<const uint8_t *>(a->residual) + c * ys : nullptr;
        m.y = static_cast<uint8_t *>(a->y) + c * ys;
        if (!e) e = cfa_launch_matmul(&m, 1, 0, stream);
    }
    return cuda_result("cfa_linear", e);
}

/* ---- route ---- */

extern "C" cfa_status cfa_route_async(const cfa_route_args *a, cfa_stream stream)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_route: NULL arguments");
    if (!is_half(a->dtype) && a->dtype != CFA_DTYPE_F32)
        return refuse(CFA_ERR_DTYPE, "cfa_route: logits are bf16, f16 or f32");
    if (!size_ok(a->tokens, 0) || a->experts < 1 || a->experts > CFA_ROUTE_MAX_EXPERTS)
        return refuse(CFA_ERR_INVAL, "cfa_route: %lld tokens, %d experts", (long long)a->tokens,
                      a->experts);
    if (a->top_k < 1 || a->top_k > a->experts || a->top_k > CFA_ROUTE_MAX_TOP_K)
        return refuse(CFA_ERR_INVAL, "cfa_route: top_k %d of %d experts", a->top_k, a->experts);
    if (a->groups < 1 || a->groups > 32 || a->experts % a->groups || a->top_groups < 1 ||
        a->top_groups > a->groups)
        return refuse(CFA_ERR_INVAL, "cfa_route: %d of %d groups of %d experts", a->top_groups,
                      a->groups, a->experts);
    if ((a->scoring != CFA_SCORE_SOFTMAX && a->scoring != CFA_SCORE_SIGMOID) ||
        (a->flags & ~CFA_ROUTE_RENORMALIZE))
        return refuse(CFA_ERR_INVAL, "cfa_route: unknown scoring or flags");
    if (a->tokens > 1 && (a->logits_stride < a->experts || a->logits_stride >= kMost))
        return refuse(CFA_ERR_INVAL, "cfa_route: row stride %lld of rows of %d",
                      (long long)a->logits_stride, a->experts);
    if (a->tokens == 0) return CFA_OK;
    if (!a->logits || !a->weights || !a->ids)
        return refuse(CFA_ERR_INVAL, "cfa_route: NULL logits, weights or ids");
    const uint64_t es = a->dtype == CFA_DTYPE_F32 ? 4 : 2;
    if (off_grid(a->logits, es) || off_grid(a->weights, 4) || off_grid(a->ids, 4) ||
        (a->bias && off_grid(a->bias, 4)))
        return refuse(CFA_ERR_ALIGN, "cfa_route: a pointer is off its element grid");
    uint64_t nl;
    const uint64_t no = (uint64_t)a->tokens * a->top_k * 4, nb = (uint64_t)a->experts * 4;
    if (!extent(a->tokens, a->experts, a->logits_stride, es, &nl))
        return refuse(CFA_ERR_INVAL, "cfa_route: the logits are too large");
    if (overlap(a->weights, no, a->ids, no) || overlap(a->weights, no, a->logits, nl) ||
        overlap(a->ids, no, a->logits, nl) ||
        (a->bias && (overlap(a->weights, no, a->bias, nb) || overlap(a->ids, no, a->bias, nb))))
        return refuse(CFA_ERR_OVERLAP, "cfa_route: an output overlaps another operand");
    return cuda_result("cfa_route", cfa_launch_route(a, reinterpret_cast<cudaStream_t>(stream)));
}

/* ---- experts ---- */

namespace {

constexpr int64_t kCounted = 4096; /* choices that the first product's CTAs count for themselves */

struct ExpertsPlan {
    int64_t pairs;
    uint64_t hist, offs, place, xs, mid, part, total; /* offsets into the workspace */
};

cfa_status experts_plan(const cfa_experts_args *a, ExpertsPlan *p)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_experts: NULL arguments");
    if (!is_half(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_experts: x and weights are bf16 or f16");
    if (!size_ok(a->tokens, 0) || !size_ok(a->hidden, 1) || !size_ok(a->inter, 1) ||
        a->experts < 1 || a->experts > CFA_EXPERTS_MAX || a->first_expert < 0 || a->top_k < 1 ||
        a->top_k > CFA_ROUTE_MAX_TOP_K)
        return refuse(CFA_ERR_INVAL,
                      "cfa_experts: %lld tokens, %lld hidden, %lld inter, %d experts from %d, "
                      "top_k %d", (long long)a->tokens, (long long)a->hidden, (long long)a->inter,
                      a->experts, a->first_expert, a->top_k);
    if (a->hidden % 8 || a->inter % 8)
        return refuse(CFA_ERR_ALIGN, "cfa_experts: hidden and inter must be multiples of 8");
    p->pairs = a->tokens * a->top_k;
    if (p->pairs >= kMost || a->experts * a->inter * 2 >= kMost || a->experts * a->hidden >= kMost)
        return refuse(CFA_ERR_INVAL, "cfa_experts: too many rows");
    const uint64_t n = (uint64_t)p->pairs;
    uint64_t at = 0;
    auto part = [&at](uint64_t bytes) {
        const uint64_t o = at;
        at += aligned(bytes);
        return o;
    };
    p->hist = part((uint64_t)cfa_sort_blocks(p->pairs) * a->experts * 4);
    p->offs = part((uint64_t)(a->experts + 1) * 4);
    p->place = part(n * 4);
    p->xs = part(n * a->hidden * 2);
    p->mid = part(n * a->inter * 2);
    p->part = part(n * a->hidden * 4);
    p->total = at;
    return CFA_OK;
}

} // namespace

extern "C" cfa_status cfa_experts_workspace(const cfa_experts_args *a, uint64_t *bytes)
{
    if (!bytes) return refuse(CFA_ERR_INVAL, "cfa_experts_workspace: NULL output");
    ExpertsPlan p = {};
    const cfa_status st = experts_plan(a, &p);
    *bytes = st ? 0 : p.total;
    return st;
}

extern "C" cfa_status cfa_experts_async(const cfa_experts_args *a, cfa_stream stream_)
{
    ExpertsPlan p = {};
    const cfa_status st = experts_plan(a, &p);
    if (st) return st;
    const bool gated = a->flags & CFA_EXPERTS_GATED;
    if (a->flags & ~CFA_EXPERTS_GATED) return refuse(CFA_ERR_INVAL, "cfa_experts: unknown flags");
    if (a->activation < CFA_ACT_NONE || a->activation > CFA_ACT_SILU)
        return refuse(CFA_ERR_INVAL, "cfa_experts: unknown activation %d", a->activation);
    if (a->tokens > 1 &&
        (a->x_stride < a->hidden || a->x_stride >= kMost || a->y_stride < a->hidden ||
         a->y_stride >= kMost ||
         (a->residual && (a->residual_stride < a->hidden || a->residual_stride >= kMost))))
        return refuse(CFA_ERR_INVAL, "cfa_experts: row strides of rows of %lld",
                      (long long)a->hidden);
    if (a->tokens == 0) return CFA_OK;
    if (!a->x || !a->w13 || !a->w2 || !a->ids || !a->weights || !a->y || !a->workspace)
        return refuse(CFA_ERR_INVAL, "cfa_experts: NULL pointer");
    if (off_grid(a->x, 2) || off_grid(a->y, 2) || (a->residual && off_grid(a->residual, 2)) ||
        off_grid(a->ids, 4) || off_grid(a->weights, 4))
        return refuse(CFA_ERR_ALIGN, "cfa_experts: a pointer is off its element grid");
    if (off_grid(a->w13, 16) || off_grid(a->w2, 16))
        return refuse(CFA_ERR_ALIGN, "cfa_experts: w13 and w2 must be 16-byte aligned");
    if (off_grid(a->workspace, kAlign))
        return refuse(CFA_ERR_ALIGN, "cfa_experts: the workspace must be 256-byte aligned");
    if (a->workspace_bytes < p.total)
        return refuse(CFA_ERR_INVAL, "cfa_experts: the workspace must hold %llu bytes",
                      (unsigned long long)p.total);
    uint64_t nx, nr, ny;
    const int64_t rows13 = gated ? 2 * a->inter : a->inter;
    uint64_t n13, n2;
    if (!extent(a->tokens, a->hidden, a->x_stride, 2, &nx) ||
        !extent(a->tokens, a->hidden, a->residual_stride, 2, &nr) ||
        !extent(a->tokens, a->hidden, a->y_stride, 2, &ny) ||
        !extent(a->experts * rows13, a->hidden, a->hidden, 2, &n13) ||
        !extent(a->experts * a->hidden, a->inter, a->inter, 2, &n2))
        return refuse(CFA_ERR_INVAL, "cfa_experts: a matrix is too large");
    const uint64_t np = (uint64_t)p.pairs * 4;
    const bool in_place = a->residual == a->y &&
                          (a->tokens <= 1 || a->residual_stride == a->y_stride);
    const struct {
        const void *p;
        uint64_t n;
    } in[] = {{a->w13, n13}, {a->w2, n2}, {a->ids, np}, {a->weights, np}, {a->x, nx},
              {a->residual, a->residual ? nr : 0}};
    for (const auto &o : in) {
        if (overlap(a->workspace, p.total, o.p, o.n))
            return refuse(CFA_ERR_OVERLAP, "cfa_experts: the workspace overlaps an operand");
        if (o.p == a->residual && in_place) continue;
        if (overlap(a->y, ny, o.p, o.n))
            return refuse(CFA_ERR_OVERLAP, "cfa_experts: y overlaps an input");
    }
    if (overlap(a->workspace, p.total, a->y, ny))
        return refuse(CFA_ERR_OVERLAP, "cfa_experts: the workspace overlaps an operand");

    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    cfa_sort s = {};
    s.ids = a->ids;
    s.pairs = p.pairs;
    s.top_k = a->top_k;
    s.first = a->first_expert;
    s.experts = a->experts;
    s.hist = reinterpret_cast<int32_t *>(ws + p.hist);
    s.offs = reinterpret_cast<int32_t *>(ws + p.offs);
    s.place = reinterpret_cast<int32_t *>(ws + p.place);
    cudaError_t e = cfa_launch_sort(&s, a->x, a->x_stride, a->hidden, ws + p.xs, stream);
    cfa_matmul m = {};
    m.offs = s.offs;
    m.tokens = p.pairs;
    m.n_groups = a->experts;
    m.busy = (int32_t)(p.pairs < a->experts ? p.pairs : a->experts);
    /* Experts before the first are other ranks': their share of the pairs is not here.  How many come
     * behind the last is not known, so that lower ranks are cut for more rows than come (32 of 128
     * experts, 512 tokens: 70.5, 68.7, 66.6 and 68.0 us on ranks 0 to 3).  A guess for the cut alone. */
    m.likely = p.pairs * a->experts / ((int64_t)a->first_expert + a->experts);
    if (m.likely < m.busy) m.likely = m.busy;
    m.f16 = a->dtype == CFA_DTYPE_F16;
    m.x = ws + p.xs;
    m.x_stride = a->hidden;
    m.w = a->w13;
    m.w_rows = rows13;
    m.cols = m.w_stride = a->hidden;
    /* The activated values are rounded to x's type: the tensor cores take the second product's operands
     * in 16 bits, and in 32 they would be split in two and multiplied twice.  Against 64 bits the result
     * is off by 1.4 times what its own rounding makes (bf16 0.0024 instead of 0.0017); in f16 values
     * above 65,504 become infinite. */
    m.y = ws + p.mid;
    m.y_stride = a->inter;
    m.act = a->activation;
    m.gated = gated;
    /* The sort's launch lets this one start once all before the call has ended, and this one the
     * next once the sort has: their weights are there before what they multiply them with. */
    m.w_ready = 1;
    if (p.pairs <= kCounted) {
        m.ids = a->ids;
        m.n_ids = (int32_t)p.pairs;
        m.first = a->first_expert;
    } else {
        m.w_ready = 0;
    }
    if (!e) e = cfa_launch_matmul(&m, 1, 1, stream);
    m.ids = nullptr;
    m.w_ready = 1;
    m.x = m.y;
    m.x_stride = a->inter;
    m.w = a->w2;
    m.w_rows = a->hidden;
    m.cols = m.w_stride = a->inter;
    /* The products of each choice stay in fp32 until they are summed; not `exact`, since the sum is
     * rounded to 16 bits, a thousand times what the accumulator's truncation costs. */
    m.y = ws + p.part;
    m.y_stride = a->hidden;
    m.y_f32 = 1;
    m.act = CFA_ACT_NONE;
    m.gated = 0;
    if (!e) e = cfa_launch_matmul(&m, 1, 1, stream);
    cfa_combine c = {};
    c.part = reinterpret_cast<const float *>(ws + p.part);
    c.weights = a->weights;
    c.place = s.place;
    c.residual = a->residual;
    c.y = a->y;
    c.tokens = a->tokens;
    c.hidden = a->hidden;
    c.r_stride = a->residual_stride;
    c.y_stride = a->y_stride;
    c.top_k = a->top_k;
    c.f16 = m.f16;
    if (!e) e = cfa_launch_combine(&c, stream);
    return cuda_result("cfa_experts", e);
}

extern "C" cfa_status cfa_op_status(void)
{
    int word = 0;
    const cudaError_t e = cfa_matmul_status(&word);
    if (e) return cuda_result("cfa_op_status", e);
    if (!word) return CFA_OK;
    return refuse(word == 1 ? CFA_ERR_DEVICE : CFA_ERR_SUSPECT,
                  word == 1 ? "a product's wait ran out: its result is not valid"
                            : "a product's wait ran out, and loads in flight did not end");
}

extern "C" cfa_status cfa_selftest_op_timeout(int device, int *status_word)
{
    if (!status_word) return refuse(CFA_ERR_INVAL, "cfa_selftest_op_timeout: NULL output");
    int prev = 0;
    cudaError_t e = cudaGetDevice(&prev);
    if (!e && device >= 0) e = cudaSetDevice(device);
    if (!e) {
        e = cfa_matmul_selftest(status_word);
        if (device >= 0) cudaSetDevice(prev);
    }
    return cuda_result("cfa_selftest_op_timeout", e);
}
