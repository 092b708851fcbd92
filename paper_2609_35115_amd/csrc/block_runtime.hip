// C ABI of a block's operators of dc_flow.h: argument checks, and the launches of
// norm_kernels.hip, linear_kernels.hip and paged_kernels.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "block_internal.h"
#include "dc_flow.h"
#include "linear_plan.h"
#include "paged_plan.h"

using namespace dcb;

namespace {

thread_local char g_error[256] = "";

dc_status fail(dc_status code, const char* what, const char* why)
{
    std::snprintf(g_error, sizeof(g_error), "%s%s", what, why);
    return code;
}

dc_status done(hipError_t e, const char* where)
{
    if (e == hipSuccess) return DC_OK;
    if (e == hipErrorInvalidConfiguration) return fail(DC_ERANGE, "", "the call has too many rows for a launch");
    std::snprintf(g_error, sizeof(g_error), "%s: %s", where, hipGetErrorString(e));
    return DC_EDEVICE;
}

constexpr int64_t kMaxRows = (int64_t)1 << 30;   // tokens of a call (with their heads, of an attention call)
constexpr int32_t kMaxWidth = 16384;             // of a norm: eight waves of 32 elements a lane
constexpr int32_t kMaxSide = 1 << 24;            // a Linear layer's n_in, n_out

#define CHECK(cond, code, why) \
    do {                       \
        if (!(cond)) return fail(code, "", why); \
    } while (0)
#define CHECK_OF(cond, code, what, why) \
    do {                                \
        if (!(cond)) return fail(code, what, why); \
    } while (0)
#define PASS(x)                               \
    do {                                      \
        const dc_status st_ = (x);            \
        if (st_ != DC_OK) return st_;         \
    } while (0)

bool known(int32_t dtype) { return dtype == DC_F32 || dtype == DC_BF16; }
int64_t size_of(int32_t dtype) { return dtype == DC_BF16 ? 2 : 4; }

dc_status check_call(const dc_call* c)
{
    CHECK(c, DC_EINVAL, "call is NULL");
    CHECK(c->batch >= 1 && c->n >= 0, DC_EINVAL, "the call's batch must be >= 1 and n >= 0");
    CHECK((int64_t)c->batch * c->n <= kMaxRows, DC_ERANGE, "the call has too many rows");
    return DC_OK;
}

// A row set of a call of n tokens (no data is needed for n = 0).
dc_status check_rows(const dc_rows* r, int32_t n, const char* what)
{
    CHECK_OF(r && (r->data || n == 0), DC_EINVAL, what, ": NULL");
    CHECK_OF(known(r->dtype), DC_EINVAL, what, ": dtype must be DC_F32 or DC_BF16");
    CHECK_OF((uintptr_t)r->data % size_of(r->dtype) == 0, DC_EINVAL, what, ": not aligned to its elements");
    return DC_OK;
}
// Results: every row has a place of its own.
dc_status check_out(const dc_rows* r, const dc_call* c, const char* what)
{
    PASS(check_rows(r, c->n, what));
    CHECK_OF((r->stride_b || c->batch <= 1) && (r->stride_t || c->n <= 1), DC_EINVAL, what, ": rows that overlap each other's");
    return DC_OK;
}

Rows rows(const dc_rows* r) { return r ? Rows{r->data, r->stride_b, r->stride_t, r->dtype == DC_BF16} : Rows{}; }

dc_status check_norm(const dc_norm* m, const char* what)
{
    CHECK_OF(m->kind == DC_NORM_RMS || m->kind == DC_NORM_LAYER, DC_EINVAL, what, ": kind must be DC_NORM_RMS or DC_NORM_LAYER");
    CHECK_OF(m->eps >= 0.0f && std::isfinite(m->eps), DC_EINVAL, what, ": eps must be >= 0 and finite");
    CHECK_OF((uintptr_t)m->gain % 4 == 0 && (uintptr_t)m->bias % 4 == 0, DC_EINVAL, what, ": not aligned to its elements");
    return DC_OK;
}
NormSpec norm(const dc_norm* m) { return m ? NormSpec{m->kind, m->eps, m->gain, m->bias} : NormSpec{}; }

dc_status check_layer(const dc_linear_layer* l)
{
    CHECK(l, DC_EINVAL, "layer is NULL");
    CHECK(l->n_in >= 1 && l->n_out >= 1, DC_EINVAL, "the layer's n_in and n_out must be >= 1");
    CHECK(l->n_in <= kMaxSide && l->n_out <= kMaxSide, DC_ERANGE, "the layer's n_in and n_out must be <= 2^24");
    CHECK(known(l->dtype), DC_EINVAL, "the layer's dtype must be DC_F32 or DC_BF16");
    CHECK(l->act == DC_ACT_NONE || l->act == DC_ACT_GELU || l->act == DC_ACT_SILU, DC_EINVAL, "the layer's act is unknown");
    return DC_OK;
}

dc_status check_paged(const dc_paged* c)
{
    CHECK(c, DC_EINVAL, "cache is NULL");
    CHECK(c->abi_version == DC_PAGED_ABI_VERSION, DC_EVERSION, "abi_version mismatch");
    CHECK(c->batch >= 1 && c->heads >= 1, DC_EINVAL, "the cache's batch and heads must be >= 1");
    CHECK(c->head_dim == 64 || c->head_dim == 128, DC_EINVAL, "head_dim must be 64 or 128");
    CHECK(known(c->dtype), DC_EINVAL, "dtype must be DC_F32 or DC_BF16");
    CHECK(c->page_size >= 1 && (c->page_size & (c->page_size - 1)) == 0, DC_EINVAL, "page_size must be a power of two");
    CHECK(c->pages >= 1 && c->table_pages >= 1, DC_EINVAL, "the pool and the table need pages");
    CHECK((int64_t)c->page_size * c->table_pages <= (int64_t)1 << 30, DC_ERANGE, "page_size * table_pages must be <= 2^30");
    CHECK((int64_t)c->batch * c->heads <= (int64_t)1 << 26, DC_ERANGE, "batch * heads must be <= 2^26");
    return DC_OK;
}
dc_status check_pool(const dc_paged* c)
{
    PASS(check_paged(c));
    CHECK(c->table && (uintptr_t)c->table % 4 == 0, DC_EINVAL, "the table is NULL or not aligned to its elements");
    const int64_t per = 16 / size_of(c->dtype), most = ((int64_t)1 << 32) * per;
    for (int v = 0; v < 2; v++) {
        const void* data = v ? c->v : c->k;
        const char* what = v ? "v" : "k";
        CHECK_OF(data && (uintptr_t)data % 16 == 0, DC_EINVAL, what, ": the pool is NULL or not aligned to 16 bytes");
        for (int64_t s : {v ? c->v_stride_page : c->k_stride_page, v ? c->v_stride_t : c->k_stride_t, v ? c->v_stride_h : c->k_stride_h}) {
            CHECK_OF(s >= 0 && s % per == 0, DC_EINVAL, what, ": the pool's strides must be >= 0 and keep rows aligned to 16 bytes");
            CHECK_OF(s < most, DC_ERANGE, what, ": the pool's strides must be below 2^36 bytes");
        }
    }
    return DC_OK;
}

Paged paged(const dc_paged* c)
{
    const int64_t per = 16 / size_of(c->dtype);
    auto units = [&](int64_t s) { return (uint32_t)(s / per); };
    return Paged{c->table, c->table_stride, (char*)c->k, (char*)c->v,
                 units(c->k_stride_page), units(c->k_stride_t), units(c->k_stride_h),
                 units(c->v_stride_page), units(c->v_stride_t), units(c->v_stride_h),
                 c->batch, c->heads, c->head_dim, c->dtype == DC_BF16,
                 __builtin_ctz((unsigned)c->page_size), c->pages, c->page_size * c->table_pages};
}

PagedPlan plan(const dc_paged* c, int32_t n, int32_t group, int32_t window, int32_t sinks)
{
    return plan_paged(c->head_dim, c->dtype == DC_BF16, (int64_t)c->batch * c->heads, n, group, c->page_size * c->table_pages, window, sinks);
}

dc_status check_span(const dc_span* s, const dc_paged* c)
{
    CHECK(s && s->pos, DC_EINVAL, "span or its pos is NULL");
    CHECK(s->batch == c->batch, DC_EINVAL, "the span and the cache differ in batch");
    CHECK(s->n >= 0, DC_EINVAL, "the span's n must be >= 0");
    return DC_OK;
}

dc_status check_heads(const dc_head_rows* r, int32_t n, int32_t dtype, const char* what)
{
    CHECK_OF(r && r->heads >= 1 && (r->data || n == 0), DC_EINVAL, what, ": NULL or no heads");
    CHECK_OF((uintptr_t)r->data % size_of(dtype) == 0, DC_EINVAL, what, ": not aligned to its elements");
    return DC_OK;
}

// Rows of a call: heads * batch * n.  (Quotients: the product may not fit 64 bits.)
dc_status check_size(int64_t heads, int32_t batch, int32_t n)
{
    CHECK(heads <= kMaxRows / batch && (n == 0 || heads * batch <= kMaxRows / n), DC_ERANGE, "the call has too many rows");
    return DC_OK;
}

HeadsOf heads(const dc_head_rows* r) { return HeadsOf{r->data, r->stride_b, r->stride_t, r->stride_h, r->heads}; }

}  // namespace

extern "C" {

const char* dc_block_last_error(void) { return g_error; }

dc_status dc_norm_residual(const dc_call* call, int32_t width, const dc_rows* x, float x_scale, const dc_rows* h,
                           const dc_norm* post, const dc_rows* gate, const dc_rows* r_out, const dc_norm* pre,
                           const dc_rows* scale, const dc_rows* shift, const dc_rows* y_out, void* hip_stream)
{
    PASS(check_call(call));
    CHECK(width >= 1, DC_EINVAL, "width must be >= 1");
    CHECK(width <= kMaxWidth, DC_ERANGE, "width must be <= 16384");
    CHECK(std::isfinite(x_scale), DC_EINVAL, "x_scale must be finite");
    PASS(check_rows(x, call->n, "x"));
    CHECK(h || (!post && !gate), DC_EINVAL, "post and gate go with h");
    CHECK(y_out || (!pre && !scale && !shift), DC_EINVAL, "pre, scale and shift go with y_out");
    CHECK(r_out || y_out, DC_EINVAL, "r_out and y_out are NULL");
    if (h) PASS(check_rows(h, call->n, "h"));
    if (post) PASS(check_norm(post, "post"));
    if (pre) PASS(check_norm(pre, "pre"));
    if (gate) PASS(check_rows(gate, call->n, "gate"));
    if (scale) PASS(check_rows(scale, call->n, "scale"));
    if (shift) PASS(check_rows(shift, call->n, "shift"));
    if (r_out) {
        PASS(check_out(r_out, call, "r_out"));
        CHECK(r_out->dtype == x->dtype, DC_EINVAL, "r_out must have x's dtype");
    }
    if (y_out) {
        PASS(check_out(y_out, call, "y_out"));
        CHECK(!h || y_out->dtype == h->dtype, DC_EINVAL, "y_out must have h's dtype");
    }
    if (call->n == 0) return DC_OK;
    NormParams p{};
    p.x = rows(x);
    p.h = rows(h);
    p.gate = rows(gate);
    p.r = rows(r_out);
    p.scale = rows(scale);
    p.shift = rows(shift);
    p.y = rows(y_out);
    p.post = norm(post);
    p.pre = norm(pre);
    p.call = Call{call->lens, call->batch, call->n};
    p.width = width;
    p.x_scale = x_scale;
    return done(launch_norm(p, (hipStream_t)hip_stream), "dc_norm_residual");
}

int64_t dc_linear_workspace(const dc_linear_layer* layer, int32_t batch, int32_t n)
{
    const dc_call call{nullptr, batch, n};
    if (check_layer(layer) != DC_OK || check_call(&call) != DC_OK || n == 0) return 0;
    return plan_linear((int64_t)batch * n, layer->n_out, layer->n_in, layer->glu != 0, layer->dtype == DC_BF16).ws_bytes;
}

dc_status dc_linear(const dc_call* call, const dc_linear_layer* layer, const dc_rows* x, const dc_rows* gate,
                    const dc_rows* residual, float residual_scale, const dc_rows* out, void* workspace,
                    int64_t workspace_bytes, void* hip_stream)
{
    PASS(check_call(call));
    PASS(check_layer(layer));
    const int64_t es = size_of(layer->dtype);
    CHECK(layer->weight && (uintptr_t)layer->weight % es == 0, DC_EINVAL, "the weight is NULL or not aligned to its elements");
    CHECK((uintptr_t)layer->bias % 4 == 0, DC_EINVAL, "the bias is not aligned to its elements");
    CHECK(layer->stride >= layer->n_in, DC_EINVAL, "the weight's stride must be >= n_in");
    PASS(check_rows(x, call->n, "x"));
    CHECK(x->dtype == layer->dtype, DC_EINVAL, "x must have the weight's dtype");
    if (gate) PASS(check_rows(gate, call->n, "gate"));
    if (residual) PASS(check_rows(residual, call->n, "residual"));
    PASS(check_out(out, call, "out"));
    CHECK(std::isfinite(residual_scale), DC_EINVAL, "residual_scale must be finite");
    if (call->n == 0) return DC_OK;
    LinearParams p{};
    p.w = layer->weight;
    p.bias = layer->bias;
    p.wstride = layer->stride;
    p.K = layer->n_in;
    p.N = layer->n_out;
    p.bf16 = layer->dtype == DC_BF16;
    p.act = layer->act;
    p.glu = layer->glu ? 1 : 0;
    p.x = rows(x);
    p.gate = rows(gate);
    p.res = rows(residual);
    p.out = rows(out);
    p.res_scale = residual_scale;
    p.call = Call{call->lens, call->batch, call->n};
    p.M = call->batch * call->n;
    const int64_t per = 16 / es;
    p.wide = (uintptr_t)p.w % 16 == 0 && (uintptr_t)x->data % 16 == 0 && layer->stride % per == 0 && layer->n_in % per == 0 &&
             x->stride_b % per == 0 && x->stride_t % per == 0;
    const LinearPlan plan = plan_linear(p.M, p.N, p.K, p.glu, p.bf16);
    CHECK(plan.ws_bytes == 0 || (workspace && workspace_bytes >= plan.ws_bytes && (uintptr_t)workspace % 16 == 0), DC_EINVAL,
          "workspace is NULL, too small or not 16-byte aligned");
    p.splits = plan.splits;
    p.ws = (float*)workspace;
    return done(launch_linear(p, plan, (hipStream_t)hip_stream), "dc_linear");
}

dc_status dc_paged_append(const dc_paged* c, const dc_span* span, const dc_head_rows* k, const dc_head_rows* v,
                          void* hip_stream)
{
    PASS(check_pool(c));
    PASS(check_span(span, c));
    PASS(check_heads(k, span->n, c->dtype, "k"));
    PASS(check_heads(v, span->n, c->dtype, "v"));
    CHECK(k->heads == c->heads && v->heads == c->heads, DC_EINVAL, "k and v need the cache's heads");
    PASS(check_size(c->heads, span->batch, span->n));
    if (span->n == 0) return DC_OK;
    PagedParams p{};
    p.c = paged(c);
    p.k = heads(k);
    p.v = heads(v);
    p.pos = span->pos;
    p.lens = span->lens;
    p.n = span->n;
    return done(launch_append(p, (hipStream_t)hip_stream), "dc_paged_append");
}

int64_t dc_paged_workspace(const dc_paged* c, int32_t q_heads, int32_t n, int32_t window, int32_t sinks)
{
    if (check_paged(c) != DC_OK || q_heads < 1 || q_heads % c->heads != 0 || n < 1 || window < 0 || sinks < 0) return 0;
    if (check_size(q_heads, c->batch, n) != DC_OK) return 0;
    return plan(c, n, q_heads / c->heads, window, sinks).ws_bytes;
}

dc_status dc_paged_attend(const dc_paged* c, const dc_span* span, const dc_head_rows* q, const dc_head_rows* out,
                          int32_t window, int32_t sinks, int32_t causal, float scale, void* workspace,
                          int64_t workspace_bytes, void* hip_stream)
{
    PASS(check_pool(c));
    PASS(check_span(span, c));
    PASS(check_heads(q, span->n, c->dtype, "q"));
    PASS(check_heads(out, span->n, c->dtype, "out"));
    CHECK(q->heads % c->heads == 0 && out->heads == q->heads, DC_EINVAL,
          "q's heads must be a multiple of the cache's, and out's the same");
    CHECK(window >= 0 && sinks >= 0, DC_EINVAL, "window and sinks must be >= 0");
    const float scale_log2 = scale * 1.4426950408889634f;
    CHECK(std::isfinite(scale_log2), DC_EINVAL, "scale and scale * log2(e) must be finite");
    PASS(check_size(q->heads, span->batch, span->n));
    if (span->n == 0) return DC_OK;
    PagedParams p{};
    p.c = paged(c);
    p.q = heads(q);
    p.o = heads(out);
    p.pos = span->pos;
    p.lens = span->lens;
    p.n = span->n;
    p.group = q->heads / c->heads;
    p.window = window;
    p.sinks = window ? sinks : 0;
    p.causal = causal ? 1 : 0;
    p.scale_log2 = scale_log2;
    const PagedPlan pl = plan(c, p.n, p.group, window, sinks);
    CHECK(pl.ws_bytes == 0 || (workspace && workspace_bytes >= pl.ws_bytes && (uintptr_t)workspace % 16 == 0), DC_EINVAL,
          "workspace is NULL, too small or not 16-byte aligned");
    p.splits = pl.splits;
    p.ws = (float*)workspace;
    return done(launch_attend(p, pl, (hipStream_t)hip_stream), "dc_paged_attend");
}

}  // extern "C"
