// gfx950 kernel of a block's norms: the residual add with the norm after a
// sublayer and its gate, and the modulated norm before the next one.
#include <type_traits>

#include "block_internal.h"
#include "dc_flow.h"

namespace dcb {

// r = x_scale x + gate post(h), y = pre(r) (1 + scale) + shift.
//
// A thread holds NV vectors of eight consecutive elements of a row (vector
// threadIdx + i * threads), so that the row is read once and both norms work on
// registers.  Gains, biases and modulations are folded into two factors and two
// addends per element (gate gain, gate bias, gain (1 + scale), bias (1 + scale) +
// shift) and kept from row to row while they stay the same.  With ONE a wave has
// a row to itself and no barrier; else a block of up to eight waves has.  The mean is
// subtracted before squares are summed (two sums a LayerNorm): no cancellation.
template <bool RB, bool HB, int NV, bool ONE>
__global__ __launch_bounds__(ONE ? 256 : 512) void norm_kernel(const NormParams p)
{
    __shared__ float part[4][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int t = ONE ? lane : threadIdx.x, threads = ONE ? 64 : blockDim.x;
    const int C = p.width, full = C >> 3, rest = C & 7;
    int turn = 0;
    auto total = [&](float v) {
        v = wave_sum(v);
        if constexpr (!ONE) {   // (four buffers in turn: a wave is at most one sum ahead of another's reads)
            float* s = part[turn++ & 3];
            if (lane == 0) s[wave] = v;
            __syncthreads();
            v = s[0];
            for (int w = 1; w < waves; w++) v += s[w];
        }
        return v;
    };

    int row = (ONE ? blockIdx.x * 4 + wave : blockIdx.x) * p.per;
    const int end = min(row + p.per, p.rows);
    if (row >= end) return;
    int e = row / p.call.n, i = row - e * p.call.n, len = p.call.len(e);

    // a row's elements as they are stored
    Raw8<RB> xr[NV];
    Raw8<HB> hr[NV];
    auto load = [&](int e, int i) {
        const int64_t xa = e * p.x.sb + i * p.x.st, ha = e * p.h.sb + i * p.h.st;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int u = t + v * threads;
            if (u < full) {
                xr[v] = load_raw<RB>(p.x.p, xa + 8 * u);
                if (p.h.p) hr[v] = load_raw<HB>(p.h.p, ha + 8 * u);
            } else if (u == full && rest) {
                xr[v] = load_raw_part<RB>(p.x.p, xa + 8 * u, rest);
                if (p.h.p) hr[v] = load_raw_part<HB>(p.h.p, ha + 8 * u, rest);
            } else {
                xr[v] = Raw8<RB>{};
                hr[v] = Raw8<HB>{};
            }
        }
    };

    float A[NV][8], B[NV][8], G[NV][8], T[NV][8];
    // a vector of modulations or gains, `none` where there are none
    auto vec = [&](const Rows& m, int e, int i, int u, float none, float (&o)[8]) {
#pragma unroll
        for (int j = 0; j < 8; j++) o[j] = none;
        if (!m.p || 8 * u >= C) return;
        const int64_t at = e * m.sb + i * m.st + 8 * u;
        if (u < full) {
            const f32x4 a = load4(m.p, at, m.bf16), b = load4(m.p, at + 4, m.bf16);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                o[j] = a[j];
                o[4 + j] = b[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 7; j++)
                if (j < rest) o[j] = load1(m.p, at + j, m.bf16);
        }
    };
    auto factors = [&](int e, int i) {
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int u = t + v * threads;
            float a[8], b[8], c[8];
            if (p.h.p) {
                vec(p.gate, e, i, u, 1.0f, a);
                vec(Rows{(void*)p.post.gain, 0, 0, 0}, 0, 0, u, 1.0f, b);
                vec(Rows{(void*)p.post.bias, 0, 0, 0}, 0, 0, u, 0.0f, c);
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    A[v][j] = a[j] * b[j];
                    B[v][j] = a[j] * c[j];
                }
            }
            if (p.y.p) {
                vec(p.scale, e, i, u, 0.0f, a);
                vec(Rows{(void*)p.pre.gain, 0, 0, 0}, 0, 0, u, 1.0f, b);
                vec(Rows{(void*)p.pre.bias, 0, 0, 0}, 0, 0, u, 0.0f, c);
                float s[8];
                vec(p.shift, e, i, u, 0.0f, s);
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    G[v][j] = b[j] * (1.0f + a[j]);
                    T[v][j] = c[j] * (1.0f + a[j]) + s[j];
                }
            }
        }
    };

    // x less its mean (LayerNorm) times 1 / sqrt(mean square + eps), in place
    const float inv_c = 1.0f / (float)C;
    auto norm = [&](const NormSpec& s, float (&x)[NV][8]) {
        if (s.kind == DC_NORM_LAYER) {
            float sum = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; v++)
#pragma unroll
                for (int j = 0; j < 8; j++) sum += x[v][j];
            const float mean = total(sum) * inv_c;
#pragma unroll
            for (int v = 0; v < NV; v++)
#pragma unroll
                for (int j = 0; j < 8; j++) x[v][j] = 8 * (t + v * threads) + j < C ? x[v][j] - mean : 0.0f;
        }
        float ss = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
            for (int j = 0; j < 8; j++) ss = fmaf(x[v][j], x[v][j], ss);
        const float f = __builtin_amdgcn_rsqf(total(ss) * inv_c + s.eps);   // 1 ulp
#pragma unroll
        for (int v = 0; v < NV; v++)
#pragma unroll
            for (int j = 0; j < 8; j++) x[v][j] *= f;
    };
    auto store = [&](const Rows& o, int e, int i, auto bf16, const float (&x)[NV][8]) {
        const int64_t at = e * o.sb + i * o.st;
#pragma unroll
        for (int v = 0; v < NV; v++) {
            const int u = t + v * threads;
            if (u < full) {
                store8<decltype(bf16)::value>(o.p, at + 8 * u, x[v]);
            } else if (u == full) {
#pragma unroll
                for (int j = 0; j < 7; j++)
                    if (j < rest) store1(o.p, at + 8 * u + j, decltype(bf16)::value, x[v][j]);
            }
        }
    };

    const bool by_token = (p.gate.p && p.gate.st) || (p.scale.p && p.scale.st) || (p.shift.p && p.shift.st);
    const bool by_entry = (p.gate.p && p.gate.sb) || (p.scale.p && p.scale.sb) || (p.shift.p && p.shift.sb);
    bool stale = true;
    if (i < len) load(e, i);
    while (true) {
        // the next row's place; rows behind an entry's last token are passed over
        int nr = row + 1, ne = e, ni = i + 1, nlen = len;
        if (ni >= p.call.n) {
            ne = e + 1;
            ni = 0;
            nlen = nr < end ? p.call.len(ne) : 0;
        }
        if (i < len) {
            float x[NV][8], h[NV][8];
#pragma unroll
            for (int v = 0; v < NV; v++) {
                widen<RB>(xr[v], x[v]);
                widen<HB>(hr[v], h[v]);
            }
            if (stale || by_token) factors(e, i);
            stale = false;
            if (nr < end && ni < nlen) load(ne, ni);
            if (p.h.p && p.post.kind) norm(p.post, h);
#pragma unroll
            for (int v = 0; v < NV; v++)
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    x[v][j] *= p.x_scale;
                    if (p.h.p) x[v][j] = 8 * (t + v * threads) + j < C ? x[v][j] + fmaf(h[v][j], A[v][j], B[v][j]) : 0.0f;
                }
            if (p.r.p) store(p.r, e, i, std::integral_constant<bool, RB>{}, x);
            if (p.y.p) {
                if (p.pre.kind) norm(p.pre, x);
#pragma unroll
                for (int v = 0; v < NV; v++)
#pragma unroll
                    for (int j = 0; j < 8; j++) x[v][j] = fmaf(x[v][j], G[v][j], T[v][j]);
                store(p.y, e, i, std::integral_constant<bool, HB>{}, x);
            }
        } else if (nr < end && ni < nlen) {
            load(ne, ni);
        }
        if (nr >= end) break;
        stale |= ne != e && by_entry;
        row = nr;
        e = ne;
        i = ni;
        len = nlen;
    }
}

template <bool RB, bool HB> hipError_t launch_norm_t(NormParams p, hipStream_t st)
{
    const int vecs = (p.width + 7) / 8;
    const bool one = vecs <= 128;
    const int nv = one ? (vecs <= 64 ? 1 : 2) : vecs <= 256 ? 1 : vecs <= 1024 ? 2 : 4;
    const int waves = one ? 4 : (vecs + 64 * nv - 1) / (64 * nv);
    const int64_t want = 256 * 8;   // blocks that fill the card
    const int64_t units = one ? want * 4 : want;
    p.per = (int)((p.rows + units - 1) / units);
    const int64_t walks = (p.rows + p.per - 1) / p.per, blocks = one ? (walks + 3) / 4 : walks;
#define DCB_NORM(NV, ONE) launch_with(norm_kernel<RB, HB, NV, ONE>, blocks, 64 * waves, 0, st, p)
    if (one) return nv == 1 ? DCB_NORM(1, true) : DCB_NORM(2, true);
    return nv == 1 ? DCB_NORM(1, false) : nv == 2 ? DCB_NORM(2, false) : DCB_NORM(4, false);
#undef DCB_NORM
}

hipError_t launch_norm(NormParams p, hipStream_t st)
{
    p.rows = p.call.batch * p.call.n;
    const bool hb = p.y.p ? p.y.bf16 : p.h.p ? p.h.bf16 : p.x.bf16;
    if (p.x.bf16) return hb ? launch_norm_t<true, true>(p, st) : launch_norm_t<true, false>(p, st);
    return hb ? launch_norm_t<false, true>(p, st) : launch_norm_t<false, false>(p, st);
}

}  // namespace dcb
