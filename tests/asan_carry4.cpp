// Host-side driver of the attention operators and the flow decoder's options for
// a sanitized build without a GPU: sizes, refusals and plans at ordinary and
// extreme values, and dc_flow_init_opt over valid and invalid options.  A call
// that every check lets pass ends at its launch, or at the first device
// allocation, with DC_EDEVICE or DC_ENOMEM; pointers are never read.  Prints
// one line per failed expectation and exits non-zero if any failed.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>
#include <vector>

#include "carry4_plan.h"
#include "dc_flow.h"

static int g_failures = 0;
static int g_calls = 0;

static void expect(bool ok, const char* what, long long detail)
{
    g_calls++;
    if (!ok) {
        std::printf("FAILED: %s (%lld)\n", what, detail);
        g_failures++;
    }
}

static const int32_t kMax = std::numeric_limits<int32_t>::max();
static void* const kPtr = reinterpret_cast<void*>((uintptr_t)1 << 20);

static bool refused(dc_status s) { return s == DC_EINVAL || s == DC_ERANGE || s == DC_EVERSION; }
static bool passed(dc_status s) { return s == DC_EDEVICE || s == DC_ERANGE; }   // (DC_ERANGE: past a launch's blocks)

static dc_head_rows rows(int32_t heads, int64_t stride = 64) { return dc_head_rows{kPtr, stride, stride, stride, heads}; }

static void operators()
{
    const int32_t values[] = {std::numeric_limits<int32_t>::min(), -1, 0, 1, 2, 3, 7, 56, 1000, 1 << 15, (1 << 24) - 1, 1 << 24, 1 << 26, kMax - 1, kMax};
    const int64_t strides[] = {0, 64, -64, (int64_t)1 << 40, std::numeric_limits<int64_t>::max(), std::numeric_limits<int64_t>::min()};
    dc_qk_norm norm{nullptr, nullptr, static_cast<float*>(kPtr), 32, 0, 1e-6f};
    for (int32_t batch : values)
        for (int32_t heads : values)
            for (int32_t slots : values)
                for (int32_t D : {64, 128, 96, kMax}) {
                    const dc_carry4 c{DC_CARRY4_ABI_VERSION, batch, heads, D, slots > 5 ? 5 : 0, slots > 5 ? slots - 5 : slots, kPtr};
                    const bool ok = batch >= 1 && heads >= 1 && (D == 64 || D == 128) && slots >= 1 && slots <= 1 << 24 && (int64_t)batch * heads <= 1 << 26;
                    const int64_t bytes = dc_carry4_bytes(&c);
                    expect(ok ? bytes >= (int64_t)batch * heads * slots * (D + D / 16) : bytes == 0, "carry bytes", bytes);
                    for (int32_t n : values)
                        for (int32_t q : {1, 3, 8, 1 << 20, kMax}) {
                            const int32_t window = n > 7 ? n : 7;
                            const int64_t ws = dc_carry4_workspace(&c, q, n, window);
                            expect(ws >= 0 && (ok || ws == 0), "workspace", ws);
                            if (!ok || D == 128) continue;
                            const dc_span s{static_cast<int64_t*>(kPtr), nullptr, nullptr, batch, n};
                            const dc_head_rows qr = rows(q), kr = rows(heads);
                            const dc_status a = dc_carry4_attend(&c, &s, DC_BF16, &qr, &qr, window, 1, 0.125f, kPtr, ws, nullptr);
                            expect(n == 0 && a == DC_OK ? true : refused(a) || passed(a), "attend", a);
                            const dc_status b = dc_carry4_append(&c, &norm, &s, DC_F32, &qr, &kr, &kr, &qr, nullptr);
                            expect(n == 0 ? b == DC_OK || refused(b) : refused(b) || passed(b), "append", b);
                            const dc_status r = dc_carry4_read(&c, &s, DC_F32, &kr, &kr, nullptr);
                            expect(n == 0 ? r == DC_OK || refused(r) : refused(r) || passed(r), "read", r);
                        }
                }
    for (int32_t batch : values)
        for (int32_t n : values)
            for (int32_t q : values)
                for (int64_t stride : strides) {
                    const dc_span s{static_cast<int64_t*>(kPtr), nullptr, nullptr, batch, n};
                    const dc_head_rows a = rows(q, stride), b = rows(kMax, stride);
                    const dc_status x = dc_qk_norm_rope(&norm, &s, 128, DC_BF16, &a, &a, &a, &a, nullptr);
                    expect(n == 0 ? x == DC_OK || refused(x) : refused(x) || passed(x), "norm", x);
                    const dc_status y = dc_qk_norm_rope(&norm, &s, 64, DC_F32, &a, &b, &a, &b, nullptr);
                    expect(n == 0 ? y == DC_OK || refused(y) : refused(y) || passed(y), "norm of many heads", y);
                }
    // texts: one for each refusal, of the calling thread
    expect(dc_carry4_attend(nullptr, nullptr, 0, nullptr, nullptr, 0, 0, 0, nullptr, 0, nullptr) == DC_EINVAL, "NULL", 0);
    expect(std::strlen(dc_carry4_last_error()) > 0, "error text", 0);
    for (float eps : {-1.0f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()}) {
        dc_qk_norm m = norm;
        m.eps = eps;
        const dc_span s{static_cast<int64_t*>(kPtr), nullptr, nullptr, 1, 1};
        const dc_head_rows a = rows(1);
        expect(dc_qk_norm_rope(&m, &s, 64, DC_F32, &a, &a, &a, &a, nullptr) == DC_EINVAL, "eps", 0);
    }
}

// The rules over the range of what the calls accept: a shape that exists, splits
// that leave no more blocks than a launch has, 32 bits of keys.
static void plans()
{
    for (int D : {64, 128})
        for (int64_t regions : {1ll, 7ll, 256ll, 5000ll, 1ll << 20, 1ll << 26})
            for (int n : {1, 2, 17, 56, 1000, 1 << 20, 1 << 30})
                for (int group : {1, 8, 56, 1 << 16})
                    for (int slots : {1, 33, 458, 100000, 1 << 24})
                        for (int window : {0, 1, 100, 1 << 24, kMax})
                            for (bool bf16 : {false, true}) {
                                if (regions * n > 1 << 30 || regions * n * group > 1 << 30) continue;
                                const dcf::Plan4 p = dcf::plan4(D, slots / 2, slots - slots / 2, regions, n, group, window, bf16);
                                expect(p.rows == 16 || p.rows == 64 || (p.rows == 128 && bf16), "rows of a block", p.rows);
                                expect(p.splits >= 1 && p.splits <= 512, "splits", p.splits);
                                const int64_t blocks = regions * (((int64_t)n * group + p.rows - 1) / p.rows);
                                expect(p.splits == 1 || blocks * p.splits < 1 << 20, "blocks of a split call", blocks * p.splits);
                            }
}

static dc_flow_cfg flow_cfg(bool real)
{
    dc_flow_cfg c{};
    c.abi_version = DC_FLOW_ABI_VERSION;
    if (real) {
        c.n_mel = 80, c.dim = 512, c.heads = 8, c.depth = 2, c.mlp = 2048, c.t_dim = 256, c.n_steps = 3;
        c.f_prompt = 302, c.f_retained = 100, c.f_chunk = 50, c.f_call = 56;
    } else {
        c.n_mel = 16, c.dim = 128, c.heads = 2, c.depth = 2, c.mlp = 256, c.t_dim = 32, c.n_steps = 4;
        c.f_prompt = 24, c.f_retained = 16, c.f_chunk = 8, c.f_call = 10;
    }
    c.batch = 1;
    c.dtype = DC_F32;
    c.cfg_rate = 0.7f;
    c.temperature = 1.0f;
    return c;
}

static void options()
{
    for (int shape = 0; shape < 4; shape++)
        for (int dt = 0; dt < 2; dt++)
            for (int batch : {1, 2, 16, 128})
                for (int carry : {0, 4})
                    for (int rope : {-1, 0, 16, 64}) {   // -1: no norm
                        dc_flow_cfg c = flow_cfg(shape == 1);
                        if (shape == 2) c.f_prompt = 4096, c.f_chunk = c.f_call = 4096, c.f_retained = 6 * 4096, c.batch = 1;
                        if (shape == 3) c.f_prompt = 1, c.f_chunk = 1, c.f_call = 1, c.f_retained = 0;
                        c.dtype = dt ? DC_BF16 : DC_F32;
                        if (shape != 2) c.batch = batch;
                        const dc_flow_opt o{DC_FLOW_OPT_VERSION, carry, rope >= 0, rope > 0 ? rope : 0, 10000.0f, 1e-6f};
                        const int64_t n = dc_flow_blob_floats_opt(&c, &o);
                        expect(n == dc_flow_blob_floats(&c) + (rope >= 0 ? (int64_t)c.depth * 128 : 0), "blob size", n);
                        std::vector<float> blob((size_t)n, 0.5f);
                        dc_flow_state* s = reinterpret_cast<dc_flow_state*>(&blob);
                        const dc_status st = dc_flow_init_opt(blob.data(), (size_t)n * 4, &c, &o, &s);
                        expect((st == DC_ENOMEM || st == DC_EDEVICE) && !s, "valid options", st);
                        expect(std::strlen(dc_flow_last_error(nullptr)) > 0, "error text", st);
                        expect(dc_flow_init_opt(blob.data(), (size_t)(n - 1) * 4, &c, &o, &s) == DC_EINVAL && !s, "short blob", 0);
                    }
    const dc_flow_cfg c = flow_cfg(false);
    const dc_flow_opt good{DC_FLOW_OPT_VERSION, 4, 1, 32, 10000.0f, 1e-6f};
    std::vector<float> blob((size_t)dc_flow_blob_floats_opt(&c, &good), 0.0f);
    auto bad = [&](dc_flow_opt o, const char* what, dc_status want) {
        dc_flow_state* s = nullptr;
        expect(dc_flow_init_opt(blob.data(), blob.size() * 4, &c, &o, &s) == want && !s, what, 0);
        if (want == DC_EINVAL) expect(dc_flow_blob_floats_opt(&c, &o) == 0, what, 1);
    };
    auto with = [&](auto set) { dc_flow_opt o = good; set(o); return o; };
    bad(with([](dc_flow_opt& o) { o.abi_version = 9; }), "options' version", DC_EVERSION);
    for (int v : {-4, 1, 8, (int)kMax}) bad(with([&](dc_flow_opt& o) { o.carry_bits = v; }), "carry_bits", DC_EINVAL);
    for (int v : {-1, 0, 2, (int)kMax}) bad(with([&](dc_flow_opt& o) { o.qk_norm = v; }), "qk_norm", DC_EINVAL);
    for (int v : {-16, 8, 65, 80, (int)kMax, (int)std::numeric_limits<int32_t>::min()}) bad(with([&](dc_flow_opt& o) { o.rope_dims = v; }), "rope_dims", DC_EINVAL);
    for (float v : {0.0f, -1.0f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()})
        bad(with([&](dc_flow_opt& o) { o.rope_base = v; }), "rope_base", DC_EINVAL);
    for (float v : {-1e-6f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()})
        bad(with([&](dc_flow_opt& o) { o.qk_eps = v; }), "qk_eps", DC_EINVAL);
    dc_flow_state* s = nullptr;
    expect(dc_flow_init_opt(blob.data(), blob.size() * 4, nullptr, &good, &s) == DC_EINVAL, "NULL cfg", 0);
    expect(dc_flow_init_opt(nullptr, blob.size() * 4, &c, &good, &s) == DC_EINVAL, "NULL blob", 0);
    expect(dc_flow_init_opt(blob.data(), blob.size() * 4, &c, &good, nullptr) == DC_EINVAL, "NULL out", 0);
    expect(dc_flow_blob_floats_opt(nullptr, &good) == 0, "size of NULL", 0);
}

int main()
{
    plans();
    operators();
    options();
    std::printf("checks %d failures %d\n", g_calls, g_failures);
    return g_failures ? 1 : 0;
}
