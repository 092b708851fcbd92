// Host-side driver of a block's operators for a sanitized build without a GPU:
// sizes, refusals and plans at ordinary and extreme values.  A call that every
// check lets pass ends at its launch with DC_EDEVICE; pointers are never read.
// Prints one line per failed expectation and exits non-zero if any failed.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <limits>

#include "dc_flow.h"
#include "linear_plan.h"
#include "paged_plan.h"

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

static const int32_t kMax = std::numeric_limits<int32_t>::max(), kMin = std::numeric_limits<int32_t>::min();
static const int64_t kLong = std::numeric_limits<int64_t>::max();
static void* const kPtr = reinterpret_cast<void*>((uintptr_t)1 << 20);

static bool refused(dc_status s) { return s == DC_EINVAL || s == DC_ERANGE || s == DC_EVERSION; }
static bool passed(dc_status s) { return s == DC_EDEVICE || s == DC_ERANGE; }   // (DC_ERANGE: past a launch's threads)
static void call(dc_status s, int32_t n, const char* what) { expect(refused(s) || (n == 0 ? s == DC_OK : passed(s)), what, s); }

static const int32_t kSizes[] = {kMin, -1, 0, 1, 2, 7, 64, 1000, 1 << 14, (1 << 14) + 1, 1 << 24, (1 << 24) + 1, 1 << 30, kMax};

static void norms_and_products()
{
    const int64_t strides[] = {0, 1, 64, -64, (int64_t)1 << 40, kLong, std::numeric_limits<int64_t>::min()};
    for (int32_t batch : kSizes)
        for (int32_t n : kSizes)
            for (int32_t w : kSizes)
                for (int64_t s : strides)
                    for (int32_t dt : {0, 1, 2}) {
                        const dc_call c{nullptr, batch, n};
                        const dc_rows x{kPtr, s, s, dt}, y{kPtr, 64, 1 << 20, DC_BF16};
                        const dc_norm m{DC_NORM_LAYER, 1e-6f, static_cast<float*>(kPtr), static_cast<float*>(kPtr)};
                        call(dc_norm_residual(&c, w, &x, 1.0f, &y, &m, &x, &x, &m, &x, &x, &y, nullptr), n, "norm");
                        call(dc_norm_residual(&c, w, &x, 0.5f, nullptr, nullptr, nullptr, &x, nullptr, nullptr, nullptr, nullptr, nullptr), n, "norm of x");
                        const dc_linear_layer l{kPtr, nullptr, s, w, 40, dt, DC_ACT_SILU, 1}, k{kPtr, nullptr, kLong, 72, w, dt, DC_ACT_GELU, 0};
                        for (const dc_linear_layer& q : {l, k}) {
                            const int64_t ws = dc_linear_workspace(&q, batch, n);
                            expect(ws >= 0, "workspace", ws);
                            call(dc_linear(&c, &q, &x, &y, &x, 1.0f, &y, kPtr, ws, nullptr), n, "product");
                        }
                    }
    expect(dc_linear(nullptr, nullptr, nullptr, nullptr, nullptr, 1.0f, nullptr, nullptr, 0, nullptr) == DC_EINVAL, "NULL", 0);
    expect(std::strlen(dc_block_last_error()) > 0, "error text", 0);
}

static void caches()
{
    for (int32_t batch : kSizes)
        for (int32_t heads : {kMin, 0, 1, 3, 1 << 20, kMax})
            for (int32_t page : {kMin, 0, 1, 3, 16, 1 << 20, 1 << 30, kMax})
                for (int32_t per : {kMin, 0, 1, 5, 1 << 10, 1 << 30, kMax})
                    for (int64_t s : {(int64_t)0, (int64_t)64, (int64_t)-64, (int64_t)1 << 33, ((int64_t)1 << 35) - 8, kLong}) {
                        const dc_paged c{DC_PAGED_ABI_VERSION, batch, heads, 64, DC_BF16, page, 9, per, static_cast<int32_t*>(kPtr), kLong, kPtr, kPtr, s, s, s, s, 64, s};
                        for (int32_t n : {kMin, 0, 1, 17, 1 << 20, kMax})
                            for (int32_t q : {1, 3, kMax}) {
                                const int32_t window = n > 5 ? n : 0;
                                const int64_t ws = dc_paged_workspace(&c, q, n, window, kMax);
                                expect(ws >= 0, "workspace", ws);
                                const dc_span sp{static_cast<int64_t*>(kPtr), nullptr, nullptr, batch, n};
                                const dc_head_rows a{kPtr, s, s, s, q}, b{kPtr, kLong, kLong, 64, heads};
                                call(dc_paged_attend(&c, &sp, &a, &a, window, kMax, 1, 0.1f, kPtr, ws, nullptr), n, "attend");
                                call(dc_paged_append(&c, &sp, &b, &b, nullptr), n, "append");
                            }
                    }
    expect(dc_paged_attend(nullptr, nullptr, nullptr, nullptr, 0, 0, 0, 0, nullptr, 0, nullptr) == DC_EINVAL, "NULL", 0);
}

// The rules over the range of what the calls accept: kernels that exist, splits that
// leave no more blocks than a launch has.
static void plans()
{
    for (int64_t M : {1ll, 16ll, 17ll, 33ll, 64ll, 65ll, 4096ll, 1ll << 20, 1ll << 30})
        for (int N : {1, 7, 64, 1000, 1 << 20, 1 << 24})
            for (int K : {1, 9, 64, 4096, 1 << 20, 1 << 24})
                for (int glu : {0, 1})
                    for (int bf16 : {0, 1}) {
                        const dcb::LinearPlan p = dcb::plan_linear(M, N, K, glu, bf16);
                        const dcb::LinearCost& c = dcb::kLinearCost[bf16][p.kind];
                        expect(p.kind >= 0 && p.kind < dcb::kLinearKinds && c.bm > 0, "kind", p.kind);
                        expect(p.splits >= 1 && p.splits <= 8 && (p.splits > 1) == (p.ws_bytes > 0), "splits", p.splits);
                        const int64_t bc = dcb::linear_columns(p.kind, c.bn, glu), tiles = (M + c.bm - 1) / c.bm * ((N + bc - 1) / bc);
                        expect(p.splits == 1 || tiles * p.splits <= 4096, "blocks", tiles * p.splits);
                        expect(p.kind != dcb::kTile256 || K % 8 == 0, "whole chunks", K);
                    }
    for (int D : {64, 128})
        for (int bf16 : {0, 1})
            for (int64_t regions : {1ll, 300ll, 1ll << 20, 1ll << 26})
                for (int n : {1, 2, 17, 1000, 1 << 20, 1 << 30})
                    for (int group : {1, 3, 64, 1 << 16})
                        for (int limit : {1, 31, 100000, 1 << 30})
                            for (int window : {0, 1, 5000, (int)kMax}) {
                                if (regions * n > 1 << 30 || regions * n * group > 1 << 30) continue;
                                const dcb::PagedPlan p = dcb::plan_paged(D, bf16, regions, n, group, limit, window, kMax);
                                expect(p.rows == 16 || p.rows == 64 || (p.rows == 128 && bf16), "rows of a block", p.rows);
                                expect(p.splits >= 1 && p.splits <= 64 && (p.splits > 1) == (p.ws_bytes > 0), "splits", p.splits);
                                const int64_t blocks = regions * (((int64_t)n * group + p.rows - 1) / p.rows);
                                expect(p.splits == 1 || blocks * p.splits <= 6000, "blocks of a split call", blocks * p.splits);
                            }
}

int main()
{
    plans();
    norms_and_products();
    caches();
    std::printf("checks %d failures %d\n", g_calls, g_failures);
    return g_failures ? 1 : 0;
}
