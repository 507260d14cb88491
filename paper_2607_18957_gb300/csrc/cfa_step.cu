/*
 * Entry points of the operators of a decoding step around the products: they check every argument and
 * enqueue the kernels.  Nothing is allocated and nothing is read back.
 */
#include <atomic>
#include <chrono>
#include <cmath>

#include "cfa_checks.h"

using namespace cfa_checks;

namespace {

uint64_t size_of(int32_t dtype) { return dtype == CFA_DTYPE_F32 ? 4 : 2; }

bool is_value(int32_t dtype) { return is_half(dtype) || dtype == CFA_DTYPE_F32; }

/* Whether a scale of exponents is finite in powers of two as well, times k (infinite, it would make NaN of a
 * difference of 0). */
bool exponents_ok(float scale, float k)
{
    const float two = scale * 1.4426950408889634f;
    return std::isfinite(two) && std::isfinite(two * k);
}

} // namespace

/* ---- norm ---- */

extern "C" cfa_status cfa_norm_async(const cfa_norm_args *a, cfa_stream stream)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_norm: NULL arguments");
    if (!is_value(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_norm: x is bf16, f16 or f32");
    if (a->weight_dtype != a->dtype && a->weight_dtype != CFA_DTYPE_F32)
        return refuse(CFA_ERR_DTYPE, "cfa_norm: the weights are of x's dtype or f32");
    if (!size_ok(a->tokens, 0) || a->cols < 1 || a->cols > CFA_NORM_MAX_COLS)
        return refuse(CFA_ERR_INVAL, "cfa_norm: %lld tokens, %lld columns", (long long)a->tokens,
                      (long long)a->cols);
    if (a->activation < CFA_ACT_NONE || a->activation > CFA_ACT_SILU)
        return refuse(CFA_ERR_INVAL, "cfa_norm: unknown activation %d", a->activation);
    if (a->flags || a->reserved) return refuse(CFA_ERR_INVAL, "cfa_norm: unknown flags");
    if (!std::isfinite(a->scale) || !std::isfinite(a->offset) || !(a->eps >= 0.0f) ||
        !std::isfinite(a->eps))
        return refuse(CFA_ERR_INVAL, "cfa_norm: scale %g, offset %g, eps %g", a->scale, a->offset,
                      a->eps);
    const struct {
        const void *p;
        int64_t stride;
        bool out;
    } m[] = {{a->x, a->x_stride, false},       {a->residual, a->residual_stride, false},
             {a->gate, a->gate_stride, false}, {a->y, a->y_stride, true},
             {a->h, a->h_stride, true}};
    const bool one_gate = a->gate && a->gate_stride == 0;
    if (a->tokens > 1)
        for (const auto &o : m)
            if (o.p && !(one_gate && o.p == a->gate && !o.out) &&
                (o.stride < a->cols || o.stride >= kMost))
                return refuse(CFA_ERR_INVAL, "cfa_norm: row stride %lld of rows of %lld",
                              (long long)o.stride, (long long)a->cols);
    if (a->tokens == 0) return CFA_OK;
    if (!a->x || !a->weight || !a->y) return refuse(CFA_ERR_INVAL, "cfa_norm: NULL x, weight or y");
    const uint64_t es = size_of(a->dtype), ws = size_of(a->weight_dtype);
    for (const auto &o : m)
        if (off_grid(o.p, es)) return refuse(CFA_ERR_ALIGN, "cfa_norm: a matrix is off its element grid");
    if (off_grid(a->weight, ws) || off_grid(a->post_weight, ws))
        return refuse(CFA_ERR_ALIGN, "cfa_norm: a weight is off its element grid");
    uint64_t n[5];
    for (int i = 0; i < 5; ++i) {
        n[i] = 0;
        const bool one = i == 2 && one_gate;
        if (m[i].p && !extent(one ? 1 : a->tokens, a->cols, m[i].stride, es, &n[i]))
            return refuse(CFA_ERR_INVAL, "cfa_norm: a matrix is too large");
    }
    const uint64_t nw = (uint64_t)a->cols * ws;
    for (int i = 3; i < 5; ++i) { /* a row is read before it is written, by the same threads */
        for (int j = 0; j < 3; ++j) {
            const bool in_place = m[i].p == m[j].p && !(j == 2 && one_gate && a->tokens > 1) &&
                                  (a->tokens <= 1 || m[i].stride == m[j].stride);
            if (!in_place && overlap(m[i].p, n[i], m[j].p, n[j]))
                return refuse(CFA_ERR_OVERLAP, "cfa_norm: an output overlaps an input");
        }
        if (overlap(m[i].p, n[i], a->weight, nw) ||
            overlap(m[i].p, n[i], a->post_weight, a->post_weight ? nw : 0))
            return refuse(CFA_ERR_OVERLAP, "cfa_norm: an output overlaps a weight");
    }
    if (overlap(a->y, n[3], a->h, n[4])) return refuse(CFA_ERR_OVERLAP, "cfa_norm: y overlaps h");
    return cuda_result("cfa_norm", cfa_launch_norm(a, reinterpret_cast<cudaStream_t>(stream)));
}

/* ---- the paged cache ---- */

namespace {

struct Cache {
    const void *p;
    int64_t page, token, head; /* strides */
    uint64_t bytes;            /* from the first value to the last */
};

/* Checks the strides of a cache and counts its bytes. */
cfa_status cache_ok(const char *who, Cache *c, int64_t pages, int64_t page_size, int64_t heads,
                    int64_t dim, uint64_t size)
{
    const struct {
        int64_t n, stride;
    } d[] = {{pages, c->page}, {page_size, c->token}, {heads, c->head}};
    unsigned __int128 last = (uint64_t)dim;
    for (const auto &x : d) {
        if (x.n > 1 && (x.stride < dim || x.stride >> 40))
            return refuse(CFA_ERR_INVAL, "%s: cache stride %lld", who, (long long)x.stride);
        last += (unsigned __int128)(x.n > 1 ? (uint64_t)(x.n - 1) * (uint64_t)x.stride : 0);
    }
    if (pages == 0) last = 0;
    if (last * size >> 62) return refuse(CFA_ERR_INVAL, "%s: a cache is too large", who);
    c->bytes = (uint64_t)last * size;
    return CFA_OK;
}

cfa_status scales_ok(const char *who, int32_t dtype, int32_t cache_dtype, float k, float v)
{
    if (cache_dtype != dtype && cache_dtype != CFA_DTYPE_F8_E4M3)
        return refuse(CFA_ERR_DTYPE, "%s: the cache is of x's dtype or f8_e4m3", who);
    if (!(k > 0.0f) || !std::isfinite(k) || !(v > 0.0f) || !std::isfinite(v))
        return refuse(CFA_ERR_INVAL, "%s: scales %g, %g", who, k, v);
    if (cache_dtype == dtype && (k != 1.0f || v != 1.0f))
        return refuse(CFA_ERR_INVAL, "%s: only a cache in 8 bits has scales", who);
    return CFA_OK;
}

} // namespace

/* ---- append ---- */

extern "C" cfa_status cfa_append_async(const cfa_append_args *a, cfa_stream stream)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_append: NULL arguments");
    if (!is_half(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_append: qkv is bf16 or f16");
    cfa_status st = scales_ok("cfa_append", a->dtype, a->cache_dtype, a->k_scale, a->v_scale);
    if (st) return st;
    if (!size_ok(a->tokens, 0) || a->heads < 0 || a->kv_heads < 1 || a->heads > 8192 ||
        a->kv_heads > 8192 || a->pages < 0 || a->page_size < 1)
        return refuse(CFA_ERR_INVAL, "cfa_append: %lld tokens, %d and %d heads, %d pages of %d",
                      (long long)a->tokens, a->heads, a->kv_heads, a->pages, a->page_size);
    if (a->head_dim < 8 || a->head_dim > CFA_HEAD_DIM_MAX || a->head_dim % 8)
        return refuse(CFA_ERR_INVAL, "cfa_append: heads of %d", a->head_dim);
    if (a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 2)
        return refuse(CFA_ERR_INVAL, "cfa_append: %d of %d values turn", a->rotary_dim, a->head_dim);
    if (a->flags & ~CFA_APPEND_INTERLEAVED) return refuse(CFA_ERR_INVAL, "cfa_append: unknown flags");
    if (a->rotary_dim && !std::isfinite(a->magnitude))
        return refuse(CFA_ERR_INVAL, "cfa_append: magnitude %g", a->magnitude);
    const int64_t q_cols = (int64_t)a->heads * a->head_dim;
    const int64_t cols = q_cols + 2 * (int64_t)a->kv_heads * a->head_dim;
    if (a->tokens > 1 && (a->qkv_stride < cols || a->qkv_stride >= kMost ||
                          (a->q && (a->q_stride < q_cols || a->q_stride >= kMost))))
        return refuse(CFA_ERR_INVAL, "cfa_append: row strides %lld, %lld of rows of %lld, %lld",
                      (long long)a->qkv_stride, (long long)a->q_stride, (long long)cols,
                      (long long)q_cols);
    const uint64_t cs = a->cache_dtype == CFA_DTYPE_F8_E4M3 ? 1 : 2;
    Cache k = {a->k_cache, a->k_page_stride, a->k_token_stride, a->k_head_stride, 0};
    Cache v = {a->v_cache, a->v_page_stride, a->v_token_stride, a->v_head_stride, 0};
    if ((st = cache_ok("cfa_append", &k, a->pages, a->page_size, a->kv_heads, a->head_dim, cs)) ||
        (st = cache_ok("cfa_append", &v, a->pages, a->page_size, a->kv_heads, a->head_dim, cs)))
        return st;
    if (a->tokens == 0) return CFA_OK;
    if (!a->qkv || !a->slots || (a->pages && (!a->k_cache || !a->v_cache)))
        return refuse(CFA_ERR_INVAL, "cfa_append: NULL qkv, slots or cache");
    if (a->rotary_dim ? !a->positions || !a->frequencies : a->positions || a->frequencies)
        return refuse(CFA_ERR_INVAL, "cfa_append: positions and frequencies belong to values that turn");
    if (off_grid(a->qkv, 2) || off_grid(a->q, 2) || off_grid(a->k_cache, cs) ||
        off_grid(a->v_cache, cs) || off_grid(a->positions, 4) || off_grid(a->slots, 4) ||
        off_grid(a->frequencies, 8))
        return refuse(CFA_ERR_ALIGN, "cfa_append: a pointer is off its element grid");
    uint64_t nx, nq = 0;
    if (!extent(a->tokens, cols, a->qkv_stride, 2, &nx) ||
        (a->q && !extent(a->tokens, q_cols, a->q_stride, 2, &nq)))
        return refuse(CFA_ERR_INVAL, "cfa_append: a matrix is too large");
    const uint64_t n4 = (uint64_t)a->tokens * 4, nf = (uint64_t)a->rotary_dim * 4;
    const bool in_place = a->q == a->qkv && (a->tokens <= 1 || a->q_stride == a->qkv_stride);
    const struct {
        const void *p;
        uint64_t n;
    } in[] = {{a->qkv, nx}, {a->slots, n4}, {a->positions, a->positions ? n4 : 0},
              {a->frequencies, nf}},
      out[] = {{a->q, nq}, {k.p, k.bytes}, {v.p, v.bytes}};
    for (const auto &o : out)
        for (const auto &i : in)
            if (!(o.p == a->q && i.p == a->qkv && in_place) && overlap(o.p, o.n, i.p, i.n))
                return refuse(CFA_ERR_OVERLAP, "cfa_append: an output overlaps an input");
    /* keys and values may lie in one buffer, page by page, so that their ends do not tell */
    if (overlap(a->q, nq, k.p, k.bytes) || overlap(a->q, nq, v.p, v.bytes) ||
        (k.bytes && k.p == v.p))
        return refuse(CFA_ERR_OVERLAP, "cfa_append: q, the keys and the values overlap");
    return cuda_result("cfa_append", cfa_launch_append(a, reinterpret_cast<cudaStream_t>(stream)));
}

/* ---- attend ---- */

namespace {

constexpr int64_t kMostKeys = 1ll << 30; /* of a sequence */
constexpr int64_t kMostRows = 1 << 18;   /* new tokens times query heads of a key head */

struct AttendPlan {
    cfa_attend_work w;
    uint64_t marks, total; /* bytes */
};

/* A number that no other call has and that memory does not hold by chance: a counter from a start that
 * differs by process, mixed over 64 bits (one to one, so that no two counts give the same). */
unsigned long long call_number()
{
    static std::atomic<unsigned long long> next{
        (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() << 20 ^
        (unsigned long long)(uintptr_t)&next};
    unsigned long long x = next.fetch_add(1, std::memory_order_relaxed);
    x = (x ^ x >> 30) * 0xBF58476D1CE4E5B9ull;
    x = (x ^ x >> 27) * 0x94D049BB133111EBull;
    x ^= x >> 31;
    return x ? x : 1;
}

cfa_status attend_plan(const cfa_attend_args *a, AttendPlan *p)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_attend: NULL arguments");
    if (!is_half(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_attend: q is bf16 or f16");
    if (a->head_dim != 64 && a->head_dim != 96 && a->head_dim != 128 && a->head_dim != 256)
        return refuse(CFA_ERR_INVAL, "cfa_attend: heads of %d: 64, 96, 128 or 256", a->head_dim);
    if (a->heads < 1 || a->heads > 8192 || a->kv_heads < 1 || a->heads % a->kv_heads ||
        a->new_tokens < 1 || (int64_t)a->new_tokens * (a->heads / a->kv_heads) > kMostRows)
        return refuse(CFA_ERR_INVAL, "cfa_attend: %d heads over %d, %d new tokens", a->heads,
                      a->kv_heads, a->new_tokens);
    p->w = {};
    p->w.a = *a;
    p->w.group = a->heads / a->kv_heads;
    const int64_t rows = (int64_t)p->w.group * a->new_tokens;
    p->w.nt = rows <= 8 || a->head_dim > 128 ? 1 : 2; /* 16 rows of 256 dims do not fit the registers */
    const int64_t row_tiles = (rows + 8 * p->w.nt - 1) / (8 * p->w.nt);
    p->w.group_inverse = (uint32_t)(((1ull << 32) + p->w.group - 1) / p->w.group);
    p->w.row_tiles = (int32_t)row_tiles;
    /* a partial: O of 8 nt rows, their maxima and sums */
    const uint64_t part = 4ull * (8 * p->w.nt) * (a->head_dim + 2);
    p->marks = aligned(sizeof(unsigned long long) * 2 * CFA_ATTEND_BLOCKS);
    p->total = p->marks + aligned(part * 2 * CFA_ATTEND_BLOCKS);
    return CFA_OK;
}

} // namespace

extern "C" cfa_status cfa_attend_workspace(const cfa_attend_args *a, uint64_t *bytes)
{
    if (!bytes) return refuse(CFA_ERR_INVAL, "cfa_attend_workspace: NULL output");
    AttendPlan p;
    const cfa_status st = attend_plan(a, &p);
    *bytes = st ? 0 : p.total;
    return st;
}

extern "C" cfa_status cfa_attend_async(const cfa_attend_args *a, cfa_stream stream_)
{
    AttendPlan p;
    cfa_status st = attend_plan(a, &p);
    if (st) return st;
    st = scales_ok("cfa_attend", a->dtype, a->cache_dtype, a->k_scale, a->v_scale);
    if (st) return st;
    if (!size_ok(a->sequences, 0) || a->max_pages < 0 || a->cache_pages < 1 || a->page_size < 1 ||
        (int64_t)a->max_pages * a->page_size > kMostKeys)
        return refuse(CFA_ERR_INVAL, "cfa_attend: %lld sequences of %d pages of %d, %d in the cache",
                      (long long)a->sequences, a->max_pages, a->page_size, a->cache_pages);
    if (a->window < 0 || a->window > kMostKeys || a->flags || !exponents_ok(a->scale, a->k_scale))
        return refuse(CFA_ERR_INVAL, "cfa_attend: window %d, scale %g, flags %u", a->window, a->scale,
                      a->flags);
    const int64_t slots = (int64_t)a->max_pages * a->page_size / 32 + 1;
    const int64_t tiles = (int64_t)p.w.row_tiles * a->kv_heads;
    if (slots * a->sequences >> 31 || (unsigned __int128)(slots * a->sequences) * (uint64_t)tiles >> 40)
        return refuse(CFA_ERR_INVAL, "cfa_attend: %lld sequences are too many", (long long)a->sequences);
    const int64_t cols = (int64_t)a->heads * a->head_dim, rows = a->sequences * a->new_tokens;
    if (rows > 1 && (a->q_stride < cols || a->q_stride >= kMost || a->out_stride < cols ||
                     a->out_stride >= kMost))
        return refuse(CFA_ERR_INVAL, "cfa_attend: row strides %lld, %lld of rows of %lld",
                      (long long)a->q_stride, (long long)a->out_stride, (long long)cols);
    if (a->sequences > 1 && (a->pages_stride < a->max_pages || a->pages_stride >= kMost))
        return refuse(CFA_ERR_INVAL, "cfa_attend: row stride %lld of %d pages",
                      (long long)a->pages_stride, a->max_pages);
    const uint64_t cs = a->cache_dtype == CFA_DTYPE_F8_E4M3 ? 1 : 2;
    Cache k = {a->k_cache, a->k_page_stride, a->k_token_stride, a->k_head_stride, 0};
    Cache v = {a->v_cache, a->v_page_stride, a->v_token_stride, a->v_head_stride, 0};
    if ((st = cache_ok("cfa_attend", &k, a->cache_pages, a->page_size, a->kv_heads, a->head_dim, cs)) ||
        (st = cache_ok("cfa_attend", &v, a->cache_pages, a->page_size, a->kv_heads, a->head_dim, cs)))
        return st;
    if (a->sequences == 0) return CFA_OK;
    if (!a->q || !a->k_cache || !a->v_cache || !a->lengths || (!a->pages && a->max_pages) || !a->out ||
        !a->workspace)
        return refuse(CFA_ERR_INVAL, "cfa_attend: NULL pointer");
    uint64_t grid = 0;
    for (const Cache *c : {&k, &v}) {
        grid |= (uint64_t)(uintptr_t)c->p;
        if (a->cache_pages > 1) grid |= (uint64_t)c->page * cs;
        if (a->page_size > 1) grid |= (uint64_t)c->token * cs;
        if (a->kv_heads > 1) grid |= (uint64_t)c->head * cs;
    }
    grid |= (uint64_t)(uintptr_t)a->q | (uint64_t)(uintptr_t)a->out;
    if (rows > 1) grid |= (uint64_t)(a->q_stride | a->out_stride) * 2;
    if (grid & 15)
        return refuse(CFA_ERR_ALIGN, "cfa_attend: q, out or a cache is off the 16-byte grid");
    if (off_grid(a->pages, 4) || off_grid(a->lengths, 4) || off_grid(a->lse, 4))
        return refuse(CFA_ERR_ALIGN, "cfa_attend: a pointer is off its element grid");
    if (off_grid(a->workspace, kAlign))
        return refuse(CFA_ERR_ALIGN, "cfa_attend: the workspace must be 256-byte aligned");
    if (a->workspace_bytes < p.total)
        return refuse(CFA_ERR_INVAL, "cfa_attend: the workspace must hold %llu bytes",
                      (unsigned long long)p.total);
    uint64_t nq, no, np;
    if (!extent(rows, cols, a->q_stride, 2, &nq) || !extent(rows, cols, a->out_stride, 2, &no) ||
        !extent(a->sequences, a->max_pages, a->pages_stride, 4, &np))
        return refuse(CFA_ERR_INVAL, "cfa_attend: a matrix is too large");
    const uint64_t nl = a->lse ? (uint64_t)rows * a->heads * 4 : 0, n4 = (uint64_t)a->sequences * 4;
    const struct {
        const void *p;
        uint64_t n;
    } m[] = {{a->out, no},        {a->lse, nl},   {a->workspace, p.total}, {a->q, nq}, {k.p, k.bytes},
             {v.p, v.bytes}, {a->pages, np}, {a->lengths, n4}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 8; ++j)
            if (overlap(m[i].p, m[i].n, m[j].p, m[j].n))
                return refuse(CFA_ERR_OVERLAP,
                              "cfa_attend: an output or the workspace overlaps another operand");
    p.w.marks = static_cast<unsigned long long *>(a->workspace);
    p.w.number = call_number();
    p.w.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(a->workspace) + p.marks);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    const bool f16 = a->dtype == CFA_DTYPE_F16;
    const cudaError_t e = cs == 1 ? (f16 ? cfa_launch_attend_f16_f8(&p.w, stream)
                                         : cfa_launch_attend_bf16_f8(&p.w, stream))
                                  : (f16 ? cfa_launch_attend_f16(&p.w, stream)
                                         : cfa_launch_attend_bf16(&p.w, stream));
    return cuda_result("cfa_attend", e);
}

/* ---- logprobs ---- */

extern "C" cfa_status cfa_logprobs_async(const cfa_logprobs_args *a, cfa_stream stream)
{
    if (!a) return refuse(CFA_ERR_INVAL, "cfa_logprobs: NULL arguments");
    if (!is_value(a->dtype)) return refuse(CFA_ERR_DTYPE, "cfa_logprobs: logits are bf16, f16 or f32");
    if (!size_ok(a->rows, 0) || !size_ok(a->cols, 1))
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: %lld rows, %lld columns", (long long)a->rows,
                      (long long)a->cols);
    if (a->top < 0 || a->top > CFA_LOGPROBS_MAX_TOP || a->top > a->cols)
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: top %d of %lld", a->top, (long long)a->cols);
    if (!(a->scale > 0.0f) || !exponents_ok(a->scale, 1.0f) || a->flags)
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: scale %g, flags %u", a->scale, a->flags);
    if (a->rows > 1 && (a->stride < a->cols || a->stride >= kMost))
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: row stride %lld of rows of %lld",
                      (long long)a->stride, (long long)a->cols);
    if (a->rows == 0) return CFA_OK;
    if (!a->logits || !a->tokens || !a->logprobs || !a->entropy ||
        (a->top && (!a->top_logprobs || !a->top_ids)))
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: NULL pointer");
    const uint64_t es = size_of(a->dtype);
    if (off_grid(a->logits, es) || off_grid(a->tokens, 4) || off_grid(a->logprobs, 4) ||
        off_grid(a->entropy, 4) || off_grid(a->top_logprobs, 4) || off_grid(a->top_ids, 4))
        return refuse(CFA_ERR_ALIGN, "cfa_logprobs: a pointer is off its element grid");
    uint64_t nx;
    if (!extent(a->rows, a->cols, a->stride, es, &nx))
        return refuse(CFA_ERR_INVAL, "cfa_logprobs: the logits are too large");
    const uint64_t n = (uint64_t)a->rows * 4, nt = n * a->top;
    const struct {
        const void *p;
        uint64_t n;
    } m[] = {{a->logprobs, n}, {a->entropy, n},  {a->top_logprobs, nt},
             {a->top_ids, nt}, {a->logits, nx}, {a->tokens, n}};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 6; ++j)
            if (overlap(m[i].p, m[i].n, m[j].p, m[j].n))
                return refuse(CFA_ERR_OVERLAP, "cfa_logprobs: an output overlaps another operand");
    return cuda_result("cfa_logprobs", cfa_launch_logprobs(a, reinterpret_cast<cudaStream_t>(stream)));
}
