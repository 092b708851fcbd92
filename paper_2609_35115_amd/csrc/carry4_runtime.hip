// C ABI of the attention operators of dc_flow.h: argument checks, and the
// launches of carry4_kernels.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

#include "carry4_internal.h"
#include "dc_flow.h"

using namespace dcf;

namespace {

thread_local char g_error[256] = "";

dc_status fail(dc_status code, const char* why)
{
    std::snprintf(g_error, sizeof(g_error), "%s", why);
    return code;
}

dc_status done(hipError_t e, const char* where)
{
    if (e == hipSuccess) return DC_OK;
    if (e == hipErrorInvalidConfiguration) return fail(DC_ERANGE, "the call has too many rows for a launch");
    std::snprintf(g_error, sizeof(g_error), "%s: %s", where, hipGetErrorString(e));
    return DC_EDEVICE;
}

constexpr int64_t kMaxSlots = 1 << 24;             // byte offsets inside a region fit 32 bits
constexpr int64_t kMaxThreads = (int64_t)1 << 34;   // of a call's rows: rows and blocks fit 31 bits

#define CHECK(cond, code, why) \
    do {                       \
        if (!(cond)) return fail(code, why); \
    } while (0)
#define PASS(x)                               \
    do {                                      \
        const dc_status st_ = (x);            \
        if (st_ != DC_OK) return st_;         \
    } while (0)

dc_status check_shape(const dc_carry4* c)
{
    CHECK(c, DC_EINVAL, "carry is NULL");
    CHECK(c->abi_version == DC_CARRY4_ABI_VERSION, DC_EVERSION, "abi_version mismatch");
    CHECK(c->batch >= 1 && c->heads >= 1, DC_EINVAL, "the carry's batch and heads must be >= 1");
    CHECK(c->head_dim == 64 || c->head_dim == 128, DC_EINVAL, "head_dim must be 64 or 128");
    CHECK(c->sinks >= 0 && c->ring >= 1, DC_EINVAL, "need sinks >= 0 and ring >= 1");
    CHECK((int64_t)c->sinks + c->ring <= kMaxSlots, DC_ERANGE, "sinks + ring must be <= 2^24");
    CHECK((int64_t)c->batch * c->heads <= (int64_t)1 << 26, DC_ERANGE, "batch * heads must be <= 2^26");
    return DC_OK;
}

dc_status check_carry(const dc_carry4* c)
{
    PASS(check_shape(c));
    CHECK(c->data, DC_EINVAL, "the carry's data is NULL");
    CHECK((uintptr_t)c->data % 256 == 0, DC_EINVAL, "the carry's data must be 256-byte aligned");
    return DC_OK;
}

dc_status check_span(const dc_span* s)
{
    CHECK(s && s->pos, DC_EINVAL, "span or its pos is NULL");
    CHECK(s->batch >= 1 && s->n >= 0, DC_EINVAL, "the span's batch must be >= 1 and n >= 0");
    return DC_OK;
}

dc_status check_dtype(int32_t dtype)
{
    CHECK(dtype == DC_F32 || dtype == DC_BF16, DC_EINVAL, "dtype must be DC_F32 or DC_BF16");
    return DC_OK;
}

// A row set of a call of n tokens (no data is needed for n = 0).
dc_status check_rows(const dc_head_rows* r, int64_t n, int32_t dtype, const char* what)
{
    char why[96];
    const int64_t es = dtype == DC_BF16 ? 2 : 4;
    std::snprintf(why, sizeof(why), "%s: NULL, no heads, or not aligned to its elements", what);
    CHECK(r && r->heads >= 1 && (r->data || n == 0) && (uintptr_t)r->data % es == 0, DC_EINVAL, why);
    return DC_OK;
}

HeadRows rows(const dc_head_rows* r) { return HeadRows{r->data, r->stride_b, r->stride_t, r->stride_h, r->heads, 0, nullptr, 0, 0}; }

bool wide(const dc_head_rows* r, int32_t dtype)
{
    const int64_t per = dtype == DC_BF16 ? 8 : 4;   // elements of 16 bytes
    return (uintptr_t)r->data % 16 == 0 && r->stride_b % per == 0 && r->stride_t % per == 0 && r->stride_h % per == 0;
}

Carry4 carry(const dc_carry4* c)
{
    return Carry4{(uint8_t*)c->data, carry4_region(c->sinks + c->ring, c->head_dim), c->heads, c->head_dim, c->sinks, c->ring};
}

Spans spans(const dc_span* s, int sinks) { return Spans{s->pos, s->lens, s->sinks, 1, s->n, sinks}; }

dc_status check_norm(const dc_qk_norm* m, int32_t head_dim)
{
    CHECK(m, DC_EINVAL, "norm is NULL");
    CHECK(m->n_freqs >= 0 && m->n_freqs % 8 == 0 && 2 * (int64_t)m->n_freqs <= head_dim, DC_EINVAL,
          "n_freqs must be a multiple of 8 with 2 n_freqs <= head_dim");
    CHECK(m->freqs || m->n_freqs == 0, DC_EINVAL, "freqs is NULL");
    CHECK(m->eps >= 0.0f && std::isfinite(m->eps), DC_EINVAL, "eps must be >= 0 and finite");
    return DC_OK;
}

void set_norm(HeadsParams& p, const dc_qk_norm* m)
{
    p.norm = 1;
    p.q_gain = m->q_gain;
    p.k_gain = m->k_gain;
    p.freqs = m->freqs;
    p.rot = 2 * m->n_freqs;
    p.interleaved = m->interleaved ? 1 : 0;
    p.eps = m->eps;
}

// Rows of a call: heads * batch * n.  (Quotients: the product may not fit 64 bits.)
dc_status check_size(int64_t heads, int32_t batch, int32_t n, int32_t head_dim)
{
    const int64_t most = kMaxThreads / (head_dim / 4);
    CHECK(heads <= most / batch && (n == 0 || heads * batch <= most / n), DC_ERANGE, "the call has too many rows");
    return DC_OK;
}

}  // namespace

extern "C" {

const char* dc_carry4_last_error(void) { return g_error; }

dc_status dc_qk_norm_rope(const dc_qk_norm* norm, const dc_span* span, int32_t head_dim, int32_t dtype,
                          const dc_head_rows* q, const dc_head_rows* k, const dc_head_rows* q_out,
                          const dc_head_rows* k_out, void* hip_stream)
{
    PASS(check_span(span));
    PASS(check_dtype(dtype));
    CHECK(head_dim == 64 || head_dim == 128, DC_EINVAL, "head_dim must be 64 or 128");
    PASS(check_norm(norm, head_dim));
    PASS(check_rows(q, span->n, dtype, "q"));
    PASS(check_rows(k, span->n, dtype, "k"));
    PASS(check_rows(q_out, span->n, dtype, "q_out"));
    PASS(check_rows(k_out, span->n, dtype, "k_out"));
    CHECK(q_out->heads == q->heads && k_out->heads == k->heads, DC_EINVAL, "outputs need as many heads as their inputs");
    PASS(check_size((int64_t)q->heads + k->heads, span->batch, span->n, head_dim));
    if (span->n == 0) return DC_OK;
    HeadsParams p{};
    p.q = rows(q);
    p.k = rows(k);
    p.q_out = rows(q_out);
    p.k_out = rows(k_out);
    p.wide_in = wide(q, dtype) && wide(k, dtype);
    p.wide_out = wide(q_out, dtype) && wide(k_out, dtype);
    set_norm(p, norm);
    p.sp = spans(span, 0);
    p.sp.sinks = nullptr;
    p.entries = span->batch;
    return done(launch_heads(p, head_dim, dtype == DC_BF16, (hipStream_t)hip_stream), "dc_qk_norm_rope");
}

int64_t dc_carry4_bytes(const dc_carry4* c)
{
    if (check_shape(c) != DC_OK) return 0;
    return (int64_t)c->batch * c->heads * carry4_region(c->sinks + c->ring, c->head_dim);
}

dc_status dc_carry4_append(const dc_carry4* c, const dc_qk_norm* norm, const dc_span* span, int32_t dtype,
                           const dc_head_rows* q, const dc_head_rows* k, const dc_head_rows* v,
                           const dc_head_rows* q_out, void* hip_stream)
{
    PASS(check_carry(c));
    PASS(check_span(span));
    PASS(check_dtype(dtype));
    CHECK(span->batch == c->batch, DC_EINVAL, "the span and the carry differ in batch");
    PASS(check_rows(k, span->n, dtype, "k"));
    PASS(check_rows(v, span->n, dtype, "v"));
    CHECK(k->heads == c->heads && v->heads == c->heads, DC_EINVAL, "k and v need the carry's heads");
    int64_t heads = 2 * (int64_t)c->heads;
    if (norm) {
        PASS(check_norm(norm, c->head_dim));
        PASS(check_rows(q, span->n, dtype, "q"));
        PASS(check_rows(q_out, span->n, dtype, "q_out"));
        CHECK(q_out->heads == q->heads, DC_EINVAL, "outputs need as many heads as their inputs");
        heads += q->heads;
    } else {
        CHECK(!q && !q_out, DC_EINVAL, "q and q_out go with norm");
    }
    PASS(check_size(heads, span->batch, span->n, c->head_dim));
    if (span->n == 0) return DC_OK;
    HeadsParams p{};
    p.k = rows(k);
    p.v = rows(v);
    p.wide_in = wide(k, dtype) && wide(v, dtype);
    if (norm) {
        p.q = rows(q);
        p.q_out = rows(q_out);
        p.wide_in = p.wide_in && wide(q, dtype);
        p.wide_out = wide(q_out, dtype);
        set_norm(p, norm);
    }
    p.c = carry(c);
    p.sp = spans(span, c->sinks);
    p.entries = span->batch;
    return done(launch_heads(p, c->head_dim, dtype == DC_BF16, (hipStream_t)hip_stream), "dc_carry4_append");
}

int64_t dc_carry4_workspace(const dc_carry4* c, int32_t q_heads, int32_t n, int32_t window)
{
    if (check_shape(c) != DC_OK || q_heads < 1 || q_heads % c->heads != 0 || n < 1 || window < 0) return 0;
    if (check_size(q_heads, c->batch, n, c->head_dim) != DC_OK) return 0;
    int64_t bytes[2] = {0, 0};   // of fp32 and of bf16 rows
    for (int bf16 = 0; bf16 < 2; bf16++) attend4_splits(carry(c), c->batch, n, q_heads / c->heads, window, bf16, bytes + bf16);
    return std::max(bytes[0], bytes[1]);
}

dc_status dc_carry4_attend(const dc_carry4* c, const dc_span* span, int32_t dtype, const dc_head_rows* q,
                           const dc_head_rows* out, int32_t window, int32_t causal, float scale, void* workspace,
                           int64_t workspace_bytes, void* hip_stream)
{
    PASS(check_carry(c));
    PASS(check_span(span));
    PASS(check_dtype(dtype));
    CHECK(span->batch == c->batch, DC_EINVAL, "the span and the carry differ in batch");
    PASS(check_rows(q, span->n, dtype, "q"));
    PASS(check_rows(out, span->n, dtype, "out"));
    CHECK(q->heads % c->heads == 0 && out->heads == q->heads, DC_EINVAL,
          "q's heads must be a multiple of the carry's, and out's the same");
    CHECK(window >= (causal ? 1 : 0), DC_EINVAL, "window must be >= 1 (causal) or >= 0");
    // (a call that begins among the first tokens puts up to `sinks` of its own there)
    CHECK((int64_t)window + span->n - (causal ? 1 : 0) <= (int64_t)c->ring + c->sinks, DC_ERANGE,
          "the window and the call's tokens do not fit the carry");
    const float scale_log2 = scale * 1.4426950408889634f;
    CHECK(std::isfinite(scale_log2), DC_EINVAL, "scale and scale * log2(e) must be finite");
    PASS(check_size(q->heads, span->batch, span->n, c->head_dim));
    if (span->n == 0) return DC_OK;
    Attend4Params p{};
    p.q = rows(q);
    p.o = rows(out);
    p.c = carry(c);
    p.sp = spans(span, c->sinks);
    p.entries = span->batch;
    p.group = q->heads / c->heads;
    p.window = window;
    p.causal = causal ? 1 : 0;
    p.scale_log2 = scale_log2;
    p.wide_in = wide(q, dtype);
    p.wide_out = wide(out, dtype);
    int64_t need = 0;
    p.splits = attend4_splits(p.c, p.entries, span->n, p.group, window, dtype == DC_BF16, &need);
    CHECK(need == 0 || (workspace && workspace_bytes >= need && (uintptr_t)workspace % 16 == 0), DC_EINVAL,
          "workspace is NULL, too small or not 16-byte aligned");
    p.ws = (float*)workspace;
    return done(launch_attend4(p, dtype == DC_BF16, (hipStream_t)hip_stream), "dc_carry4_attend");
}

dc_status dc_carry4_read(const dc_carry4* c, const dc_span* span, int32_t dtype, const dc_head_rows* k,
                         const dc_head_rows* v, void* hip_stream)
{
    PASS(check_carry(c));
    PASS(check_span(span));
    PASS(check_dtype(dtype));
    CHECK(span->batch == c->batch, DC_EINVAL, "the span and the carry differ in batch");
    PASS(check_rows(k, span->n, dtype, "k"));
    PASS(check_rows(v, span->n, dtype, "v"));
    CHECK(k->heads == c->heads && v->heads == c->heads, DC_EINVAL, "k and v need the carry's heads");
    PASS(check_size(2 * (int64_t)c->heads, span->batch, span->n, c->head_dim));
    if (span->n == 0) return DC_OK;
    Read4Params p{};
    p.c = carry(c);
    p.sp = spans(span, c->sinks);
    p.k = rows(k);
    p.v = rows(v);
    p.wide = wide(k, dtype) && wide(v, dtype);
    p.entries = span->batch;
    return done(launch_read4(p, dtype == DC_BF16, (hipStream_t)hip_stream), "dc_carry4_read");
}

}  // extern "C"
