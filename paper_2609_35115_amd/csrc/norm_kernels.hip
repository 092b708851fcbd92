// gfx950 kernel of a block's norms: the residual add with the norm after a
// sublayer and its gate, and the modulated norm before the next one.
#include <algorithm>
#include <type_traits>

#include "block_internal.h"
#include "dc_flow.h"
#include "norm_plan.h"

namespace dcb {

// A factor or addend of every element of a row: (gate or 1 + scale) times gain, and
// bias times the same plus shift.
enum { kPostFactor, kPostAddend, kPreFactor, kPreAddend };

// r = x_scale x + gate post(h), y = pre(r) (1 + scale) + shift.
//
// A row's elements lie in NV vectors of eight consecutive ones a thread (vector
// t + i threads), so that the row is read once and both norms work on registers.
// LANES 0: a block of up to eight waves has a row; else LANES lanes of a wave have
// one (64 / LANES rows a wave, side by side), and there is no barrier.  Blocks or
// waves walk several rows, the next one loaded while this one is worked on.  Gains,
// biases and modulations are folded into a factor and an addend of each norm.  With
// KEEP they wait in LDS, written and read by the same thread, until the entry
// changes (where a modulation depends on it); else (a modulation for each token, or
// more than LDS holds) they are read at their use.  The mean is subtracted before
// squares are summed: no cancellation.
//
// What bounds it: HBM, at the rate of a copy (5.1 TB/s) where rows are long and many:
// 16,384 rows of 4,096 bf16 (537 MB) 100 us, 5.4 TB/s; fp32 with a bf16 sublayer (805 MB)
// 154 us; rows of 1,024 (134 MB, past the caches) 30 us, 4.5.  Rows not aligned to 16
// bytes pay for lines that two loads share (30,005 of 2,576 124 us, of 2,572 128, of
// 2,571 132; with a modulation for each entry 156).  Modulations for each token are read
// as rows are (8,192 of 4,096 with three: bf16, 470 MB, 115 us; fp32, 671 MB, 131);
// factors that LDS does not hold, again for every row (8,192 bf16 of 8,192 with all four
// arrays 161 us, 3.3 TB/s; 2,000 fp32 of 16,384 161).  Few rows: the launch, the loads'
// latency and each sum's (4 of 1,024 4.7 us in a graph).
template <bool RB, bool HB, int NV, int LANES, bool KEEP, bool REST>
__global__ __launch_bounds__(LANES ? 256 : 512) void norm_kernel(const NormParams p)
{
    constexpr bool ONE = LANES != 0;
    constexpr int ROWS = ONE ? 64 / (ONE ? LANES : 1) : 1;   // rows side by side
    extern __shared__ __align__(16) float kept[];            // [array][NV][half][threads][4]
    __shared__ float part[2][8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int t = ONE ? lane % (ONE ? LANES : 1) : threadIdx.x, threads = ONE ? LANES : blockDim.x;
    // A last vector that the row does not fill is the row's last eight elements instead, loaded like the others
    // (30,005 x 2,572 bf16: with loads and stores of its own 1.15 times as long).  `again` of them are the vector's before it as well:
    // no sum has them twice, and they are stored twice only where both results lie apart from x and h.  Else what this
    // thread reads there may be a result that another thread has stored, and enters nothing.  Rows of less than eight
    // elements (`tiny`) are loaded in parts.
    const int C = p.width, vecs = (C + 7) >> 3, rest = REST ? C & 7 : 0;
    const bool tiny = REST && C < 8;
    auto first = [&](int u) { return REST && !tiny ? min(8 * u, C - 8) : 8 * u; };
    auto again = [&](int u) { return REST && !tiny && u == vecs - 1 ? 8 - rest : 0; };
    int turn = 0;
    auto total = [&](float v) {
        if constexpr (ONE) {
            v = dpp_add<0xB1>(v);                             // quad_perm 1 0 3 2
            v = dpp_add<0x4E>(v);                             // quad_perm 2 3 0 1
            if constexpr (LANES >= 8) v = dpp_add<0x141>(v);   // row_half_mirror: the other quad of eight lanes
            if constexpr (LANES >= 16) v = dpp_add<0x140>(v);  // row_mirror: the other eight of sixteen
            if constexpr (LANES >= 32) v = sum_xor16(v);
            if constexpr (LANES >= 64) v = sum_xor32(v);
        } else {   // (two buffers in turn: a wave is at most one sum ahead of another's reads)
            v = wave_sum(v);
            float* s = part[turn++ & 1];
            if (lane == 0) s[wave] = v;
            __syncthreads();
            const f32x4 a = *(const f32x4*)s, b = *(const f32x4*)(s + 4);
            v = a[0];
#pragma unroll
            for (int w = 1; w < 8; w++)
                if (w < waves) v += w < 4 ? a[w] : b[w - 4];
        }
        return v;
    };

    const int walk = ONE ? blockIdx.x * 4 + wave : blockIdx.x;
    const int side = ONE ? lane / (ONE ? LANES : 1) : 0;
    int row = walk * p.per * ROWS + side;
    const int end = min((walk + 1) * p.per * ROWS, p.rows);
    int e = min(row, p.rows - 1) / p.call.n, i = row - e * p.call.n, len = p.call.len(e);
    bool on = row < end && i < len;

    // a row's elements as they are stored
    Raw8<RB> xr[NV];
    Raw8<HB> hr[NV];
    auto load = [&](int e, int i, bool on) {
        const int64_t xa = e * p.x.sb + i * p.x.st, ha = p.h.p ? e * p.h.sb + i * p.h.st : 0;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int u = t + v * threads;
            xr[v] = Raw8<RB>{};
            hr[v] = Raw8<HB>{};
            if (!on | (u >= vecs)) continue;
            if (!tiny) {
                xr[v] = load_raw<RB>(p.x.p, xa + first(u));
                if (p.h.p) hr[v] = load_raw<HB>(p.h.p, ha + first(u));
            } else {
                xr[v] = load_raw_part<RB>(p.x.p, xa, rest);
                if (p.h.p) hr[v] = load_raw_part<HB>(p.h.p, ha, rest);
            }
        }
    };

    // a modulation or gain of vector u's elements, `none` where there is none
    auto vec = [&](const void* m, int64_t at, int bf16, int u, float none, float (&o)[8]) {
#pragma unroll
        for (int j = 0; j < 8; j++) o[j] = none;
        if (!m || u >= vecs) return;
        if (!tiny) {
            const f32x4 a = load4(m, at + first(u), bf16), b = load4(m, at + first(u) + 4, bf16);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                o[j] = a[j];
                o[4 + j] = b[j];
            }
        } else {
            if (bf16) widen<true>(load_raw_part<true>(m, at, rest), o);
            else widen<false>(load_raw_part<false>(m, at, rest), o);
        }
    };
    // the factor or addend `which` of vector u of a row
    auto fold = [&](int which, int e, int i, int u, float (&o)[8]) {
        float a[8];
        const Rows& m = which <= kPostAddend ? p.gate : p.scale;
        const NormSpec& s = which <= kPostAddend ? p.post : p.pre;
        vec(m.p, e * m.sb + i * m.st, m.bf16, u, which <= kPostAddend ? 1.0f : 0.0f, a);
        if (which > kPostAddend) {
#pragma unroll
            for (int j = 0; j < 8; j++) a[j] += 1.0f;
        }
        if (which == kPostFactor || which == kPreFactor) {
            vec(s.gain, 0, 0, u, 1.0f, o);
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] *= a[j];
        } else {
            vec(s.bias, 0, 0, u, 0.0f, o);
            float b[8];
            vec(which == kPreAddend ? p.shift.p : nullptr, e * p.shift.sb + i * p.shift.st, p.shift.bf16, u, 0.0f, b);
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] = fmaf(o[j], a[j], b[j]);
        }
    };
    const bool has[4] = {p.h.p && (p.gate.p || p.post.gain), p.h.p && p.post.bias, p.y.p && (p.scale.p || p.pre.gain),
                         p.y.p && (p.pre.bias || p.shift.p)};
    auto place = [&](int which, int v) {
        const int array = which > 0 ? has[0] + (which > 1 ? has[1] + (which > 2 ? has[2] : 0) : 0) : 0;
        return kept + ((array * NV + v) * 2 * (int)blockDim.x + (int)threadIdx.x) * 4;
    };
    auto keep = [&](int e) {
#pragma unroll
        for (int which = 0; which < 4; which++) {
            if (!has[which]) continue;
#pragma unroll
            for (int v = 0; v < NV; v++) {
                float o[8];
                fold(which, e, 0, t + v * threads, o);
                float* to = place(which, v);
                *(f32x4*)to = f32x4{o[0], o[1], o[2], o[3]};
                *(f32x4*)(to + 4 * blockDim.x) = f32x4{o[4], o[5], o[6], o[7]};
            }
        }
    };
    auto get = [&](int which, int e, int i, int v, float (&o)[8]) {
        if constexpr (KEEP) {
            const float* from = place(which, v);
            const f32x4 a = *(const f32x4*)from, b = *(const f32x4*)(from + 4 * blockDim.x);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                o[j] = a[j];
                o[4 + j] = b[j];
            }
        } else {
            fold(which, e, i, t + v * threads, o);
        }
    };

    // the factor 1 / sqrt(mean square + eps) of x, with DC_NORM_LAYER of x less its mean, which is taken from x here
    const float inv_c = 1.0f / (float)C;
    auto root = [&](const NormSpec& s, float (&x)[NV][8]) {
        // the sum of f(x) over this thread's elements
        auto over = [&](auto f) {
            float sum = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; v++) {
                if constexpr (REST) {
                    const int skip = again(t + v * threads);
#pragma unroll
                    for (int j = 0; j < 8; j++) sum = f(sum, j < skip ? 0.0f : x[v][j]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; j++) sum = f(sum, x[v][j]);
                }
            }
            return sum;
        };
        if (s.kind == DC_NORM_LAYER) {
            const float mean = total(over([](float sum, float x) { return sum + x; })) * inv_c;
#pragma unroll
            for (int v = 0; v < NV; v++)
#pragma unroll
                for (int j = 0; j < 8; j++) x[v][j] -= (t + v * threads < vecs) & (!tiny | (j < rest)) ? mean : 0.0f;
        }
        return __builtin_amdgcn_rsqf(total(over([](float sum, float x) { return fmaf(x, x, sum); })) * inv_c + s.eps);   // 1 ulp
    };
    // Elements that two threads have are stored by both, the same bits, where both have read the inputs.
    const bool twice = REST && !tiny && p.apart;
    auto store = [&](const Rows& o, int64_t at, int v, auto bf16, const float (&x)[8]) {
        const int u = t + v * threads;
        if (u < (!REST || twice ? vecs : C >> 3)) {
            store8<decltype(bf16)::value>(o.p, at + first(u), x);
        } else if (REST && u < vecs) {
            if (tiny) store_part<decltype(bf16)::value, false>(o.p, at, rest, x);
            else store_part<decltype(bf16)::value, true>(o.p, at + 8 * u, rest, x);
        }
    };

    const bool by_entry = (p.gate.p && p.gate.sb) || (p.scale.p && p.scale.sb) || (p.shift.p && p.shift.sb);
    int kept_of = -1;   // the entry whose factors are kept
    load(e, i, on);
    for (int it = 0; it < p.per; it++) {
        // the next row's place; rows behind an entry's last token are passed over
        const int nr = row + ROWS;
        int ne = e, ni = i + ROWS, nlen = len;
        if (ni >= p.call.n) {
            ne = min(nr, p.rows - 1) / p.call.n;
            ni = nr - ne * p.call.n;
            nlen = p.call.len(ne);
        }
        const bool non = (nr < end) & (ni < nlen) & (it + 1 < p.per);

        float x[NV][8], h[NV][8];
#pragma unroll
        for (int v = 0; v < NV; v++) {
            widen<RB>(xr[v], x[v]);
            widen<HB>(hr[v], h[v]);
        }
        if (KEEP && on && (kept_of < 0 || (by_entry && kept_of != e))) {
            keep(e);
            kept_of = e;
        }
        if (ONE || non) load(ne, ni, non);
        if (ONE || on) {   // (a block's row is on for all of its threads)
            const int mi = on ? i : 0;   // whose modulations are read: a lane group without a row may stand past the last token
            float f = 1.0f;
            if (p.h.p && p.post.kind) f = root(p.post, h);
#pragma unroll
            for (int v = 0; v < NV; v++) {
#pragma unroll
                for (int j = 0; j < 8; j++) x[v][j] *= p.x_scale;
                if (p.h.p) {
#pragma unroll
                    for (int j = 0; j < 8; j++) h[v][j] *= f;
                    float o[8];
                    if (has[kPostFactor]) {
                        get(kPostFactor, e, mi, v, o);
#pragma unroll
                        for (int j = 0; j < 8; j++) h[v][j] *= o[j];
                    }
                    if (has[kPostAddend]) {
                        get(kPostAddend, e, mi, v, o);   // (of elements past a tiny row's last: zeros)
#pragma unroll
                        for (int j = 0; j < 8; j++) h[v][j] += o[j];
                    }
#pragma unroll
                    for (int j = 0; j < 8; j++) x[v][j] += h[v][j];
                }
            }
            if (p.r.p && on) {
                const int64_t at = e * p.r.sb + i * p.r.st;
#pragma unroll
                for (int v = 0; v < NV; v++) store(p.r, at, v, std::integral_constant<bool, RB>{}, x[v]);
            }
            if (p.y.p) {
                f = 1.0f;
                if (p.pre.kind) f = root(p.pre, x);
                const int64_t at = e * p.y.sb + i * p.y.st;
#pragma unroll
                for (int v = 0; v < NV; v++) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; j++) x[v][j] *= f;
                    if (has[kPreFactor]) {
                        get(kPreFactor, e, mi, v, o);
#pragma unroll
                        for (int j = 0; j < 8; j++) x[v][j] *= o[j];
                    }
                    if (has[kPreAddend]) {
                        get(kPreAddend, e, mi, v, o);
#pragma unroll
                        for (int j = 0; j < 8; j++) x[v][j] += o[j];
                    }
                    if (on) store(p.y, at, v, std::integral_constant<bool, HB>{}, x[v]);
                }
            }
        }
        row = nr;
        e = ne;
        i = ni;
        len = nlen;
        on = non;
    }
}

template <bool RB, bool HB, bool REST> hipError_t launch_norm_t(NormParams p, hipStream_t st)
{
    const int vecs = (p.width + 7) / 8;
    const bool one = vecs <= 128;
    const int lanes = vecs <= 8 ? 8 : vecs <= 16 ? 16 : vecs <= 32 ? 32 : 64;
    const int nv = one ? (vecs <= 64 ? 1 : 2) : vecs <= 256 ? 1 : vecs <= 1024 ? 2 : 4;
    const int waves = one ? 4 : (vecs + 64 * nv - 1) / (64 * nv);
    const int arrays = (p.h.p && (p.gate.p || p.post.gain)) + (p.h.p && p.post.bias) + (p.y.p && (p.scale.p || p.pre.gain)) +
                       (p.y.p && (p.pre.bias || p.shift.p));
    const int lds = arrays * nv * 32 * 64 * waves;
    const bool by_token = (p.gate.p && p.gate.st) || (p.scale.p && p.scale.st) || (p.shift.p && p.shift.st);
    const bool keep = !by_token && lds <= 64 * 1024;
    // rows of a walk: as few as give every CU 32 walks of a wave, or blocks of 64 waves
    // (21,001 of 30,005 rows of 2,571, walks that end at their entry's last token: 145 us with eight blocks, 133;
    // 16,384 of 4,096 111 and 105; more walks read factors more often); of rows that blocks of 16 waves a CU walk in
    // two to some turns, so many, so that walks load ahead (bf16, us, with 64 and 16 waves: 4,000 rows of 4,096 33.7 and
    // 29.0, of 2,048 17.9 and 16.7, 1,500 of 4,096 15.8 and 14.8; of 8,192, blocks of eight waves, 52.7 and 56.1)
    const int64_t sides = one ? 64 / lanes : 1, units = (p.rows + sides - 1) / sides, few = 256 * 16 / waves;
    const int64_t want = one ? 256 * 32 : waves <= 4 && 3 * units >= 4 * few && units <= 256 * 16 ? few : 256 * 64 / waves;
    p.per = (int)((units + want - 1) / want);
    const int64_t walks = (units + p.per - 1) / p.per, blocks = one ? (walks + 3) / 4 : walks;
#define DCB_NORM(NV, LANES)                                                                          \
    (keep ? launch_with(norm_kernel<RB, HB, NV, LANES, true, REST>, blocks, 64 * waves, lds, st, p)   \
          : launch_with(norm_kernel<RB, HB, NV, LANES, false, REST>, blocks, 64 * waves, 0, st, p))
    if (!one) return nv == 1 ? DCB_NORM(1, 0) : nv == 2 ? DCB_NORM(2, 0) : DCB_NORM(4, 0);
    if (nv == 2) return DCB_NORM(2, 64);
    return lanes == 8 ? DCB_NORM(1, 8) : lanes == 16 ? DCB_NORM(1, 16) : lanes == 32 ? DCB_NORM(1, 32) : DCB_NORM(1, 64);
#undef DCB_NORM
}

hipError_t launch_norm(NormParams p, hipStream_t st)
{
    p.rows = p.call.batch * p.call.n;
    p.apart = results_apart(p.x.p, p.h.p, p.r.p, p.y.p);
    const bool hb = p.y.p ? p.y.bf16 : p.h.p ? p.h.bf16 : p.x.bf16;
#define DCB_NORM(RB, HB) (p.width % 8 ? launch_norm_t<RB, HB, true>(p, st) : launch_norm_t<RB, HB, false>(p, st))
    if (p.x.bf16) return hb ? DCB_NORM(true, true) : DCB_NORM(true, false);
    return hb ? DCB_NORM(false, true) : DCB_NORM(false, false);
#undef DCB_NORM
}

}  // namespace dcb
