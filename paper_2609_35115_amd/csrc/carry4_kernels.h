// gfx950 kernels of the attention operators: per-head norms with the position
// rotation, the store of keys and values into a carry held in 4 bits, and the
// attention over it.  Part of flow_kernels.hip (one code object), whose vector
// types and cross-lane helpers it uses.
#include <algorithm>

#include "carry4_internal.h"
#include "carry4_plan.h"

namespace dcf {

// A launch has fewer than 2^32 threads: more are refused here, since a launch that
// fails leaves its error for the thread's next runtime call.
template <class P> hipError_t launch_with(void (*kernel)(P), int64_t blocks, hipStream_t st, P p)
{
    if (blocks >= (int64_t)1 << 24) return hipErrorInvalidConfiguration;
    void* args[] = {&p};
    return hipLaunchKernel((const void*)kernel, dim3((unsigned)blocks), dim3(256), args, 0, st);
}

// An entry's span of a call.  Values that no caller may pass (a negative
// position, a length or a number of first tokens past the call's or the
// carry's) are taken as none and as the largest, so that no access leaves the
// carry or the rows whatever the device arrays hold.
struct Span {
    int64_t pos, total;   // first position of the call, position after its last token
    int len, sinks;
    __device__ __forceinline__ Span(const Spans& s, const Carry4& c, int e)
    {
        const int b = s.div == 1 ? e : e / s.div;
        pos = s.pos ? s.pos[b] : 0;
        len = s.lens ? min(max(s.lens[b], 0), s.n) : s.n;
        sinks = min(max(s.sinks ? s.sinks[b] : s.sinks_all, 0), c.sinks);
        if (pos < 0 || pos > (int64_t)1 << 60) pos = len = 0;
        total = pos + len;
    }
};

// Token `off` of the `per` that start at token t0 (of entries of n tokens each;
// t0, n uniform): a 64-bit division a lane costs as much as a head's row.  A call
// has at most 2^30 rows, so its tokens' numbers fit 31 bits.
struct Token {
    int e, i;   // of the last token, past the end
    bool on;
    __device__ __forceinline__ Token(int64_t t0, int off, int per, int entries, int n)
    {
        const int64_t tokens = (int64_t)entries * n;
        on = t0 + off < tokens;
        const uint32_t u = (uint32_t)min(t0, tokens - 1), e0 = u / (uint32_t)n, x = u - e0 * (uint32_t)n + off;
        const uint32_t q = n >= per ? (x >= (uint32_t)n ? 1 : 0) : x / (uint32_t)n;
        e = (int)(e0 + q);
        i = (int)(x - q * (uint32_t)n);
        if (!on) {
            e = entries - 1;
            i = n - 1;
        }
    }
};

// Sum and maximum over aligned groups of LANES lanes (4, 8 or 16), in every
// lane, one fixed order.
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int LANES, class F> __device__ __forceinline__ uint32_t lanes_reduce(uint32_t v, F f)
{
    v = f(v, dpp<0xB1>(v));                           // quad_perm 1 0 3 2
    v = f(v, dpp<0x4E>(v));                           // quad_perm 2 3 0 1
    if constexpr (LANES >= 8) v = f(v, dpp<0x141>(v));   // row_half_mirror: the other quad of eight lanes
    if constexpr (LANES >= 16) v = f(v, dpp<0x140>(v));  // row_mirror: the other eight of sixteen
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
    return __uint_as_float(lanes_reduce<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

template <bool BF16> struct Raw8 { u32x4 w[BF16 ? 1 : 2]; };   // eight elements as they are stored

template <bool BF16> __device__ __forceinline__ Raw8<BF16> load_raw(const void* p, int64_t at, int wide)
{
    Raw8<BF16> r;
    if constexpr (BF16) {
        const uint16_t* s = (const uint16_t*)p + at;
        if (wide) {
            r.w[0] = *(const u32x4*)s;
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) r.w[0][j] = s[2 * j] | (uint32_t)s[2 * j + 1] << 16;
        }
    } else {
        const uint32_t* s = (const uint32_t*)p + at;
        if (wide) {
            r.w[0] = *(const u32x4*)s;
            r.w[1] = *(const u32x4*)(s + 4);
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                r.w[0][j] = s[j];
                r.w[1][j] = s[4 + j];
            }
        }
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ void widen(const Raw8<BF16>& r, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if constexpr (BF16) {
            x[2 * j] = bf2f(r.w[0][j] & 0xffffu);
            x[2 * j + 1] = __uint_as_float(r.w[0][j] & 0xffff0000u);
        } else {
            x[j] = __uint_as_float(r.w[0][j]);
            x[4 + j] = __uint_as_float(r.w[1][j]);
        }
    }
}

template <bool BF16> __device__ __forceinline__ void load8(const void* p, int64_t at, int wide, float (&x)[8])
{
    widen<BF16>(load_raw<BF16>(p, at, wide), x);
}
template <bool BF16> __device__ __forceinline__ void store8(void* p, int64_t at, int wide, const float (&x)[8])
{
    if (BF16 && wide) {
        *(u32x4*)((uint16_t*)p + at) = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    } else if (wide) {
        store4<BF16>(p, at, f32x4{x[0], x[1], x[2], x[3]});
        store4<BF16>(p, at + 4, f32x4{x[4], x[5], x[6], x[7]});
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) store1<BF16>(p, at + j, x[j]);
    }
}

// position * freq as a fraction of a turn, in [-1/2, 1/2].  Both products carry
// their rounding error along (fma), so the fraction is right to fp32 for
// positions up to 2^53; a plain fp64 product is off by 10^-5 turns at 10^11.
__device__ __forceinline__ float turn_fraction(int64_t pos, float freq)
{
    const double inv = 0.15915494309189535, inv_lo = -9.839338337591243e-18;   // 1 / (2 pi), and what the first leaves out
    const double a = (double)pos, b = (double)freq;
    const double t = a * b, te = fma(a, b, -t);
    const double u = t * inv, ue = fma(t, inv, -u) + fma(t, inv_lo, te * inv);
    return (float)((u - __builtin_rint(u)) + ue);
}

// ------------------------------- norms, rotation and the store into the carry
//
// D / 8 lanes hold a head's row, eight consecutive elements each, and `waves` of
// a block's four waves the same 64 / (D / 8) tokens, whose heads they share out;
// so the cosines and sines of those tokens' 256 angles are computed once for all
// of the block's heads.
//
// y = x / sqrt(mean(x^2) + eps) gain, sums in fp32.  The angle position *
// freqs[j] is taken in 64 bits (fp32 would be off by half a radian at position
// 10^7 and one radian a position) and reduced to a fraction of a turn there;
// only that fraction is rounded to fp32.
// Pair j is dimensions (j, j + rot / 2), or (2 j, 2 j + 1) interleaved; a
// dimension past rot is only normalised.
//
// The store: a group of 32 values shares the scale 2^e with the least e in
// [-126, 126] for which 6 * 2^e is at least its largest magnitude (so none is
// cut), and an element is the nearest E2M1 value of x 2^-e, ties to even.
// Scaling by a power of two is exact, so the codes do not depend on the
// precision they are computed in.  A group with a NaN or an infinity is NaN, and so
// is one with an element that would be 2^128 (3.5 * 2^126 and more): held as an
// infinity it would turn a masked probability of zero into NaN.
//
// What bounds it: HBM.  Norm and rotation of 32,768 tokens of 40 heads of 128 (671 MB)
// 129 us, 5.2 TB/s; of 14,336 of 16 heads of 64 (59 MB) 13.3 us, 17.6 where the 256 MB
// last-level cache holds neither side.  A load of the next row
// before this one is worked on, partners by DPP instead of LDS and one reciprocal
// root took the first from 315 to 161, the block's shared sines to 139, 32-bit
// divisions to 129.  The store of 16,384 tokens of 8 heads of 128 (85 MB) 22.9 us, 3.7
// TB/s, and 16.9 over buffers that stay in the cache; two thirds of its time are the
// codes' stores (stores past the caches took 8% less, but the attention that follows
// read 3% slower).  Norm, rotation and store in one pass of 16,384 tokens of 32 and
// twice 8 heads (353 MB) 72.7 us, 4.9 TB/s; of 14,336 of three times 8 of 64 (66 MB)
// 23.0 us.
// The value of the lane whose number differs by half a row's lanes (D = 64:
// lane ^ 4; 128: lane ^ 8), without an LDS round trip.
template <int L> __device__ __forceinline__ float half_row(float v)
{
    const uint32_t u = __float_as_uint(v);
    if constexpr (L == 16) return __uint_as_float(dpp<0x128>(u));        // row_ror:8
    return __uint_as_float(dpp<0x1B>(dpp<0x141>(u)));                    // row_half_mirror (^ 7), quad_perm 3 2 1 0 (^ 3)
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void heads_kernel(const HeadsParams p)
{
    constexpr int L = D / 8, TPW = 64 / L;   // lanes of a row, tokens of a wave
    __shared__ __align__(16) float turn[4][2][TPW][D / 2];   // of each group: cosines, sines
    const int lane = threadIdx.x & 63, l = lane % L;
    // `waves` waves work on a group of tokens, wave `wave` of group `group` of the block's
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = p.waves;
    const int wave = all & (waves - 1), group = all >> __builtin_ctz(waves);
    const int64_t g = (int64_t)(blockIdx.x >> p.split_bits) * (4 >> __builtin_ctz(waves)) + group;
    const Token tk(g * TPW, lane / L, TPW, p.entries, p.sp.n);
    const int e = tk.e, i = tk.i;
    const Span sp(p.sp, p.c, e);
    const bool on = tk.on && i < sp.len;
    const int64_t pos = sp.pos + i;

    const int jobs = p.q.heads + p.k.heads + p.v.heads;
    const int part = waves * (int)(blockIdx.x & ((1u << p.split_bits) - 1)) + wave;
    const int j0 = min(part * p.share, jobs), j1 = min(j0 + p.share, jobs);

    // the rotation of this lane's dimensions (identity past rot): a group's 256
    // angles are shared out over its lanes
    float cs[8], sn[8];
    const bool inter = p.interleaved && p.rot;   // (without a rotation there are no cosines and sines)
    const int half = p.rot >> 1;
    const bool first = 8 * l < half;                     // half-split pairs: this lane holds the pairs' first members
    if (p.norm && p.rot) {
        for (int a = wave; a < 4; a += waves) {
            const int u = 64 * a + lane, f = u % (D / 2), of = u / (D / 2);
            const int64_t at = ((int64_t)__shfl((int)(pos >> 32), of * L) << 32) | (uint32_t)__shfl((int)pos, of * L);
            float c = 1.0f, s = 0.0f;
            if (f < half) sincospif(2.0f * turn_fraction(at, p.freqs[f]), &s, &c);
            turn[group][0][of][f] = c;
            turn[group][1][of][f] = s;
        }
        __syncthreads();
        const int f0 = (inter ? 4 * l : first ? 8 * l : 8 * l - half) & (D / 2 - 1), f4 = (f0 + 4) & (D / 2 - 1);
        const float *c = turn[group][0][lane / L], *s = turn[group][1][lane / L];
        const f32x4 ca = *(const f32x4*)(c + f0), cb = *(const f32x4*)(c + f4);
        const f32x4 sa = *(const f32x4*)(s + f0), sb = *(const f32x4*)(s + f4);
        const float sign = !inter && first ? -1.0f : 1.0f;   // that the pair's other member enters with
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const bool on = 8 * l + j < p.rot;
            cs[j] = !on ? 1.0f : inter ? ca[j >> 1] : j < 4 ? ca[j & 3] : cb[j & 3];
            sn[j] = !on ? 0.0f : sign * (inter ? sa[j >> 1] : j < 4 ? sa[j & 3] : sb[j & 3]);
        }
    }
    const int partner = (lane & ~(L - 1)) | ((8 * l < p.rot ? (first ? l + half / 8 : l - half / 8) : l) & (L - 1));

    // where this token's rows go in the carry; a token that a later one of the
    // same call overwrites is left out (ring slots are written once)
    int64_t slot = -1;
    if (p.c.base && on) {
        if (pos < sp.sinks) slot = pos;
        else if (pos + p.c.ring >= sp.total) slot = p.c.sinks + (pos - sp.sinks) % p.c.ring;
    }

    // one kind of rows after the other, the next row loaded while this one is
    // worked on
    int jb = 0;
    auto rows_of = [&](int kind, const HeadRows& in, const HeadRows& out, const float* gains) {
        const int h0 = max(j0 - jb, 0), h1 = min(j1 - jb, in.heads);
        jb += in.heads;
        if (h0 >= h1) return;
        float gain[8];
        const bool norm = p.norm && kind < 2;
#pragma unroll
        for (int k = 0; k < 8; k++) gain[k] = 1.0f;
        if (norm && gains) {
#pragma unroll
            for (int k = 0; k < 8; k++) gain[k] = gains[8 * l + k];
        }
        const int64_t at0 = in.at(p.sp.div, e, i, 0) + 8 * l;
        const int64_t out0 = out.p ? out.at(p.sp.div, e, i, 0) + 8 * l : 0;
        Raw8<BF16> next{};
        if (on) next = load_raw<BF16>(in.p, at0 + h0 * in.sh, p.wide_in);
        for (int h = h0; h < h1; h++) {
            float x[8];
            widen<BF16>(next, x);
            if (on && h + 1 < h1) next = load_raw<BF16>(in.p, at0 + (h + 1) * in.sh, p.wide_in);
            if (norm) {
                float ss = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; k++) ss = fmaf(x[k], x[k], ss);
                ss = lanes_sum<L>(ss);
                const float r = __builtin_amdgcn_rsqf(ss * (1.0f / D) + p.eps);   // 1 ulp
#pragma unroll
                for (int k = 0; k < 8; k++) x[k] = x[k] * r * gain[k];
                if (inter) {
#pragma unroll
                    for (int k = 0; k < 8; k += 2) {
                        const float a = x[k], b = x[k + 1];
                        x[k] = a * cs[k] - b * sn[k];
                        x[k + 1] = b * cs[k] + a * sn[k];
                    }
                } else if (p.rot == D) {
#pragma unroll
                    for (int k = 0; k < 8; k++) x[k] = x[k] * cs[k] + half_row<L>(x[k]) * sn[k];
                } else if (p.rot) {
#pragma unroll
                    for (int k = 0; k < 8; k++) x[k] = x[k] * cs[k] + __shfl(x[k], partner) * sn[k];
                }
            }
            if (out.p) {
                if (on) store8<BF16>(out.p, out0 + h * out.sh, p.wide_out, x);
                continue;
            }
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 8; k++) top = max(top, __float_as_uint(x[k]) & 0x7fffffffu);   // NaN and infinity are the largest
            top = lanes_reduce<4>(top, [](uint32_t a, uint32_t b) { return max(a, b); });
            uint32_t s = (uint32_t)min(max((int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0), 1), 253);
            const float scale = __uint_as_float(s << 23);
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
            if (top >= 0x7f600000u) {   // 3.5 * 2^126
                s = 255;
                w = 0;
            }
            if (slot >= 0) {
                const int N = p.c.slots(), kv = kind == 2;
                uint8_t* reg = p.c.base + ((int64_t)e * p.c.heads + h) * p.c.region;
                *(uint32_t*)(reg + ((int64_t)kv * N + slot) * (D / 2) + 4 * l) = w;
                if ((l & 3) == 0) reg[(int64_t)N * D + ((int64_t)kv * N + slot) * (D / 32) + (l >> 2)] = (uint8_t)s;
            }
        }
    };
    rows_of(0, p.q, p.q_out, p.q_gain);
    rows_of(1, p.k, p.k_out, p.k_gain);
    rows_of(2, p.v, HeadRows{}, nullptr);
}

template <bool BF16, int D> hipError_t launch_heads_d(HeadsParams p, hipStream_t st)
{
    constexpr int TPW = 64 / (D / 8);
    const int64_t tokens = (int64_t)p.entries * p.sp.n, groups = (tokens + TPW - 1) / TPW;
    const int jobs = p.q.heads + p.k.heads + p.v.heads;
    // a block walks all heads of its tokens unless that leaves fewer than two blocks
    // a CU (14,336 rows of 16 heads: 16.3 us, 28.7 with four times the blocks; 4,011
    // of 12: 11.2 and 20.6).  Where the groups alone fill the card, a wave walks
    // three heads or more: what it does once a token (angles, the place in the carry)
    // costs as much as a few rows (us with one, two and four waves a group: 2
    // rows, 74,046 tokens 21, 22 and 28; 6, 13,146 18, 17 and 23; 40, 32,768 -,
    // 146 and 136; but 10 waves or fewer in all, 4.6 with four and 6.6 with one).
    p.waves = groups < 1024 || jobs > 16 ? 4 : jobs > 4 ? 2 : 1;
    p.split_bits = 0;
    while ((4ll << p.split_bits) < jobs && groups << p.split_bits < 512) p.split_bits++;
    const int parts = p.waves << p.split_bits;
    p.share = (jobs + parts - 1) / parts;
    const int64_t per = 4 / p.waves;   // groups of a block
    return launch_with(heads_kernel<BF16, D>, (groups + per - 1) / per << p.split_bits, st, p);
}

hipError_t launch_heads(HeadsParams p, int D, int bf16, hipStream_t st)
{
    if (D == 64) return bf16 ? launch_heads_d<true, 64>(p, st) : launch_heads_d<false, 64>(p, st);
    return bf16 ? launch_heads_d<true, 128>(p, st) : launch_heads_d<false, 128>(p, st);
}

// ---------------------------------------------------------------- carry read

// Eight values of lane l of a carry row: codes of dimensions 8 l .. 8 l + 7.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t s, float (&x)[8])
{
    const float scale = __uint_as_float(s << 23);   // 255: an infinity, for which the conversion gives NaN
#define DCF_PAIR(j)                                                                                                \
    {                                                                                                              \
        const uint32_t v = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, j));   \
        x[2 * j] = bf2f(v & 0xffffu);                                                                              \
        x[2 * j + 1] = __uint_as_float(v & 0xffff0000u);                                                           \
    }
    DCF_PAIR(0) DCF_PAIR(1) DCF_PAIR(2) DCF_PAIR(3)
#undef DCF_PAIR
}

// Block b's token group when consecutive groups go to one XCD (blocks are dealt
// to the eight XCDs in turn): a line of scale bytes holds 32 to 64 tokens', and
// each XCD would fetch it for its part (16,384 tokens of 8 heads: 17.0 -> 15.7 us;
// the store and the norms are slower that way, 23.1 -> 24.6 and 140 -> 147).
__device__ __forceinline__ int64_t xcd_group(unsigned b, unsigned blocks) { return (int64_t)(b & 7) * (blocks >> 3) + (b >> 3); }
inline int64_t xcd_blocks(int64_t groups) { return (groups + 7) / 8 * 8; }   // some past the last group

// Lanes, tokens and waves as in heads_kernel; a wave walks a share of the (kv, head) rows.
template <bool BF16, int D> __global__ __launch_bounds__(256) void read4_kernel(const Read4Params p)
{
    constexpr int L = D / 8, TPW = 64 / L;
    const int lane = threadIdx.x & 63, l = lane % L, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = p.waves;
    const int wave = all & (waves - 1), group = all >> __builtin_ctz(waves), heads = p.c.heads;
    const int64_t g = xcd_group(blockIdx.x, gridDim.x) * (4 >> __builtin_ctz(waves)) + group;
    const Token tk(g * TPW, lane / L, TPW, p.entries, p.sp.n);
    const int e = tk.e, i = tk.i;
    const Span sp(p.sp, p.c, e);
    if (!tk.on || i >= sp.len) return;
    const int64_t pos = sp.pos + i;
    const int64_t slot = pos < sp.sinks ? pos : p.c.sinks + (pos - sp.sinks) % p.c.ring;
    const int N = p.c.slots();
    const int j0 = wave * p.share, j1 = j0 + p.share;
    for (int kv = 0; kv < 2; kv++) {
        const HeadRows& o = kv ? p.v : p.k;
        const int64_t at = o.at(p.sp.div, e, i, 0) + 8 * l;
        const uint8_t* codes = p.c.base + (int64_t)e * heads * p.c.region + ((int64_t)kv * N + slot) * (D / 2) + 4 * l;
        const uint8_t* scale = p.c.base + (int64_t)e * heads * p.c.region + (int64_t)N * D + ((int64_t)kv * N + slot) * (D / 32) + (l >> 2);
        const int h0 = max(j0 - kv * heads, 0), h1 = min(j1 - kv * heads, heads);
#pragma unroll 2
        for (int h = h0; h < h1; h++) {
            float x[8];
            decode8(*(const uint32_t*)(codes + h * p.c.region), scale[h * p.c.region], x);
            store8<BF16>(o.p, at + h * o.sh, p.wide, x);
        }
    }
}

template <bool BF16, int D> hipError_t launch_read4_d(Read4Params p, hipStream_t st)
{
    constexpr int TPW = 64 / (D / 8);
    const int64_t groups = ((int64_t)p.entries * p.sp.n + TPW - 1) / TPW;
    const int jobs = 2 * p.c.heads;
    p.waves = groups < 1024 || jobs > 16 ? 4 : jobs > 4 ? 2 : 1;
    p.share = (jobs + p.waves - 1) / p.waves;
    const int64_t per = 4 / p.waves;
    return launch_with(read4_kernel<BF16, D>, xcd_blocks((groups + per - 1) / per), st, p);
}

hipError_t launch_read4(const Read4Params& p, int bf16, hipStream_t st)
{
    if (p.c.D == 64) return bf16 ? launch_read4_d<true, 64>(p, st) : launch_read4_d<false, 64>(p, st);
    return bf16 ? launch_read4_d<true, 128>(p, st) : launch_read4_d<false, 128>(p, st);
}
// Eq. carry's order of one (entry, kv), for audits (heads of 64, the flow decoder's).
__global__ __launch_bounds__(256) void carry4_gather_kernel(const Carry4 c, const Spans spans, int e, int kv, int f_chunk,
                                                            int nh, int frames, float* out)
{
    constexpr int D = 64, L = D / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / L;   // (frame, head)
    const int l = (int)(u % L), f = (int)(row / c.heads), h = (int)(row % c.heads);
    if (f >= frames) return;
    const Span sp(spans, c, e);
    const int64_t at = f < nh * f_chunk ? sp.pos - (int64_t)(f / f_chunk + 1) * f_chunk + f % f_chunk : f - nh * f_chunk;
    const int64_t slot = at < sp.sinks ? max(at, (int64_t)0) : c.sinks + (at - sp.sinks) % c.ring;
    const int N = c.slots();
    const uint8_t* reg = c.base + ((int64_t)e * c.heads + h) * c.region;
    float x[8];
    decode8(*(const uint32_t*)(reg + ((int64_t)kv * N + slot) * (D / 2) + 4 * l),
            reg[(int64_t)N * D + ((int64_t)kv * N + slot) * (D / 32) + (l >> 2)], x);
    store8<false>(out, row * D + 8 * l, 1, x);
}

hipError_t launch_carry4_gather(const Carry4& c, const Spans& sp, int e, int kv, int f_chunk, int nh, int frames,
                                float* out, hipStream_t st)
{
    if (c.D != 64) return hipErrorInvalidValue;
    const unsigned blocks = (unsigned)(((int64_t)frames * c.heads * 8 + 255) / 256);
    hipLaunchKernelGGL(carry4_gather_kernel, dim3(blocks), dim3(256), 0, st, c, sp, e, kv, f_chunk, nh, frames, out);
    return hipGetLastError();
}

// ------------------------------------------------------------------ attention
//
// O = softmax(scale Q K^T) V over an entry's visible tokens, one (entry, key
// head) region and 16 query rows a block; a row is (token i, query head), the
// `group` query heads of a key head side by side, so shared heads share the
// loads of their keys.
//
// The visible tokens of the block's rows are one list: the first tokens
// [0, ns), then the window's [lo, hi), whose ring slots wrap once at most.
// A tile is 32 consecutive members of that list; the four waves take a tile
// each in turn, with its codes prefetched one tile ahead, and keep their own
// running maximum, sum and output, merged through LDS at the end (or, when the
// list is split over blocks too, by attend4_join).
//
// S^T = K Q^T: lane (r, g) = (lane % 16, lane / 16) holds of key row r the
// dimensions [g D / 4, (g + 1) D / 4), one load of D / 8 bytes and one scale,
// and the queries in the same order, so the codes go to bf16 fragments with one
// conversion per two values (exact: an E2M1 value times a power of two).
// O^T += V^T P^T: a lane's eight probabilities of one query are keys 4 g .. + 3
// of both halves of the tile; its value fragment, eight keys of one dimension,
// comes from LDS by transposing reads of the tile's values as bf16.
// fp32 rows: queries and probabilities as the sum of three bf16 planes, so
// three products give the fp32 one (keys and values are exact in bf16).  bf16
// rows: a probability is rounded to bf16 for the product, half a step of the
// result's own type; its sum is not.
//
// What bounds it: long lists HBM (131,004 keys of 128, 64 regions, 1.14 GB: 215 us,
// 5.3 TB/s, the rate of a large copy; 8% more at three waves a SIMD, the compiler's
// choice without a bound), short ones latency (458 keys of 64: 7.0 us in a graph).
constexpr int kKeyTile = 32;

template <int PL> struct Planes { bf16x8_t f[PL]; };

// The high halves of eight fp32 words.
__device__ __forceinline__ bf16x8_t high8(const uint32_t (&y)[8])
{
    u32x4 r;
#pragma unroll
    for (int j = 0; j < 4; j++) r[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], 0x07060302u);
    return __builtin_bit_cast(bf16x8_t, r);
}

// x rounded to bf16, or whole in three planes: eight of its bits each, cut off
// one after the other (rounded planes take a conversion more: fp32 calls of the wide
// kernel 5 to 9% slower).
template <int PL> __device__ __forceinline__ Planes<PL> split8(const float (&x)[8])
{
    Planes<PL> r;
    if constexpr (PL == 1) {
#pragma unroll
        for (int j = 0; j < 8; j++) r.f[0][j] = (__bf16)x[j];
    } else {
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; j++) y[j] = __float_as_uint(x[j]);
#pragma unroll
        for (int k = 0; k < PL; k++) {
            r.f[k] = high8(y);
#pragma unroll
            for (int j = 0; j < 8; j++)
                y[j] = __float_as_uint(__uint_as_float(y[j]) - __uint_as_float(y[j] & 0xffff0000u));
        }
    }
    return r;
}

// The rows' visible members of the block's list.
struct RowSpan {
    int sink_hi, lo, hi;   // visible: [0, sink_hi) and [lo, hi)
    __device__ __forceinline__ bool sees(int key) const   // (no short circuits: a branch a score)
    {
        return (key < sink_hi) | ((uint32_t)(key - lo) < (uint32_t)max(hi - lo, 0));
    }
};

struct KeyList {
    int ns, nk, ring0;       // first tokens, members, ring index of the first window token
    int64_t first;           // position of the first window token
    int sinks, ring;
    __device__ __forceinline__ KeyList(const Attend4Params& p, const Span& sp, int i0, int i1)
    {
        const int64_t p0 = sp.pos + i0, p1 = sp.pos + i1;
        first = (p.causal ? p0 - p.window + 1 : sp.pos - p.window);
        if (first < sp.sinks) first = sp.sinks;
        const int64_t end = p.causal ? p1 + 1 : sp.total;
        // tokens that the call's own have overwritten are not seen
        const int64_t oldest = sp.total - p.c.ring;
        if (first < oldest) first = oldest;
        ns = (int)(end < sp.sinks ? end : (int64_t)sp.sinks);
        nk = ns + (end > first ? (int)(end - first) : 0);
        sinks = p.c.sinks;
        ring = p.c.ring;
        ring0 = end > first ? (int)((first - sp.sinks) % p.c.ring) : 0;
    }
    // slot of member t; members past the list's end give its last one's
    __device__ __forceinline__ int slot(int t) const
    {
        t = min(t, nk - 1);
        int w = ring0 + (t - ns);
        if (w >= ring) w -= ring;
        return t < ns ? t : sinks + w;
    }
    __device__ __forceinline__ RowSpan row(const Attend4Params& p, const Span& sp, int i) const
    {
        RowSpan r{ns, ns, nk};
        if (p.causal) {
            const int64_t at = sp.pos + i, lo = at - p.window + 1;
            if (at + 1 < ns) r.sink_hi = (int)(at + 1);
            if (lo > first) r.lo = ns + (int)(lo - first);
            r.hi = at + 1 > first ? ns + (int)(at + 1 - first) : ns;
            if (r.hi > nk) r.hi = nk;
        }
        return r;
    }
};

// 1 / l for the result of token i's row.  l = 0: the row sees nothing and its
// result is 0, or every score that it sees is -infinity (an infinite query) and
// there is no softmax: NaN, as for the other infinities.
__device__ __forceinline__ float inverse_sum(const Attend4Params& p, const Span& sp, int i, float l)
{
    if (__builtin_expect(l != 0.0f, 1)) return 1.0f / l;
    const RowSpan r = KeyList(p, sp, i, i).row(p, sp, i);
    return r.sink_hi > 0 || r.hi > r.lo ? NAN : 0.0f;
}

template <int D> struct Tile4 {   // a lane's part of 32 keys' and values' codes and scales
    static constexpr int W = D / 32;   // words
    uint32_t k[2][W], v[2][W], ks[2], vs[2];
    __device__ __forceinline__ void load(const uint8_t* reg, int N, const KeyList& list, int t0, int r, int g)
    {
#pragma unroll
        for (int b = 0; b < 2; b++) {
            const uint32_t s = (uint32_t)list.slot(t0 + 16 * b + r);
            const uint8_t* kp = reg + (s * (uint32_t)(D / 2) + (uint32_t)(g * (D / 8)));
            const uint8_t* vp = kp + (uint32_t)N * (D / 2);
            const uint8_t* sc = reg + (uint32_t)N * D + s * (uint32_t)(D / 32) + (uint32_t)(g * (D / 32) / 4);
            if constexpr (W == 4) {
                const u32x4 a = *(const u32x4*)kp, c = *(const u32x4*)vp;
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    k[b][w] = a[w];
                    v[b][w] = c[w];
                }
            } else {
                const u32x2 a = *(const u32x2*)kp, c = *(const u32x2*)vp;
#pragma unroll
                for (int w = 0; w < 2; w++) {
                    k[b][w] = a[w];
                    v[b][w] = c[w];
                }
            }
            ks[b] = sc[0];
            vs[b] = sc[(uint32_t)N * (D / 32)];
        }
    }
};

// Eight codes -> a bf16 fragment.
__device__ __forceinline__ bf16x8_t decode_frag(uint32_t w, uint32_t s)
{
    const float scale = __uint_as_float(s << 23);
    const u32x4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
    return __builtin_bit_cast(bf16x8_t, v);
}

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ uint32_t or_xor16_32(uint32_t v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const uint32_t a0 = a[0], a1 = a[1], w = a0 | a1;
    const auto c = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    const uint32_t c0 = c[0], c1 = c[1];
    return c0 | c1;
}
__device__ __forceinline__ float sum_xor16_32(float v)
{
    v = sum_xor16(v);
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto c = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t c0 = c[0], c1 = c[1];
    return __uint_as_float(c0) + __uint_as_float(c1);
}

// One wave's running softmax over its tiles for 16 rows: O^T in the MFMA's
// result layout (lane (q, g): query q, dimensions 16 b + 4 g .. + 3).
template <int D> struct Running {
    f32x4 o[D / 16];
    float m, l;
    uint32_t bad;   // groups of 32 dimensions in which a visible value is NaN
};

// The plane that a lane of column group `plane` holds (the fourth is zero).
__device__ __forceinline__ bf16x8_t plane8(const float (&x)[8], int plane)
{
    uint32_t y[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
        float v = x[j];
#pragma unroll
        for (int k = 0; k < 3; k++) v -= __uint_as_float(__float_as_uint(v) & (k < plane ? 0xffff0000u : 0u));
        y[j] = __float_as_uint(v);
    }
    return high8(y);
}
// The sum of a row of 16 lanes' four quads, in every quad.
__device__ __forceinline__ float sum_quads(float v)
{
    v += __uint_as_float(dpp<0x128>(__float_as_uint(v)));          // row_ror:8
    return v + __uint_as_float(dpp<0x124>(__float_as_uint(v)));    // row_ror:4
}

// FOLD: calls of up to four fp32 rows.  The planes of a row are columns of one
// product instead of products of their own (column 4 k + q: plane k of row q), and
// meet after it (one token, 20,000 keys of 128, 144 regions: 120 -> 91 us, bf16
// rows 83; 11,800 of 64, 135 regions 49 -> 43 and 36).
template <bool BF16, int D, bool FOLD>
__global__ __launch_bounds__(256, !BF16 && !FOLD ? 1 : D == 128 ? 4 : 5) void attend4_kernel(const Attend4Params p)
{
    constexpr int PL = BF16 || FOLD ? 1 : 3, KS = D / 32, DB = D / 16, RB = FOLD ? 4 : 16;
    constexpr int VROW = 2 * D + 32;   // bytes of a value row in LDS: eight banks on from row to row
    constexpr int WAVE_LDS = kKeyTile * VROW > 16 * D * 4 + 128 ? kKeyTile * VROW : 16 * D * 4 + 128;
    __shared__ __align__(16) unsigned char smem[4 * WAVE_LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int regions = p.entries * p.c.heads, split = blockIdx.x % p.splits;
    const int eh = blockIdx.x / p.splits % regions, e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p.sp, p.c, e);
    const int rows = sp.len * p.group, row0 = RB * (blockIdx.x / p.splits / regions);
    if (row0 >= rows) return;                       // (uniform: the block's rows are behind the entry's last token)
    const int last = min(row0 + RB - 1, rows - 1), my_row = min(row0 + r % RB, rows - 1);
    const KeyList list(p, sp, row0 / p.group, last / p.group);
    const RowSpan mine = list.row(p, sp, my_row / p.group);
    const RowSpan lead = list.row(p, sp, row0 / p.group), tail = list.row(p, sp, last / p.group);
    const int open_lo = lead.sink_hi == list.ns && tail.lo == list.ns ? 0 : tail.lo;   // members visible to every row
    const int N = p.c.slots();
    const uint8_t* reg = p.c.base + (int64_t)eh * p.c.region;

    // queries as B operand: lane (q, g) holds dimensions g D / 4 + 8 c .. + 7
    Planes<PL> qf[KS];
    {
        const int i = my_row / p.group, hq = h * p.group + my_row % p.group;
        const int64_t at = p.q.at(p.sp.div, e, i, hq) + g * (D / 4);
#pragma unroll
        for (int c = 0; c < KS; c++) {
            float x[8];
            load8<BF16>(p.q.p, at + 8 * c, p.wide_in, x);
            if constexpr (FOLD) qf[c].f[0] = plane8(x, r >> 2);
            else qf[c] = split8<PL>(x);
        }
    }

    const int tiles = (list.nk + kKeyTile - 1) / kKeyTile;
    const int t_lo = (int)((int64_t)tiles * split / p.splits), t_hi = (int)((int64_t)tiles * (split + 1) / p.splits);

    Running<D> acc;
#pragma unroll
    for (int b = 0; b < DB; b++) acc.o[b] = f32x4{0, 0, 0, 0};
    acc.m = -INFINITY;
    acc.l = 0.0f;
    acc.bad = 0;

    unsigned char* vt = smem + wave * WAVE_LDS;
    Tile4<D> cur;
    int t = t_lo + wave;
    if (t < t_hi) cur.load(reg, N, list, t * kKeyTile, r, g);
    for (; t < t_hi; t += 4) {
        Tile4<D> now = cur;
        if (t + 4 < t_hi) cur.load(reg, N, list, (t + 4) * kKeyTile, r, g);
        const int t0 = t * kKeyTile;

        // a NaN group among the values is kept out of the products (a probability
        // of zero would not cancel it) and noted for the rows that see its key
        uint64_t nanv[2];
#pragma unroll
        for (int b = 0; b < 2; b++) {
            nanv[b] = __ballot(now.vs[b] == 255);
            if (nanv[b] && now.vs[b] == 255) {
#pragma unroll
                for (int w = 0; w < Tile4<D>::W; w++) now.v[b][w] = 0;
                now.vs[b] = 127;
            }
        }
        // values to LDS as bf16 rows
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int w = 0; w < Tile4<D>::W; w++)
                *(bf16x8_t*)(vt + (16 * b + r) * VROW + g * (D / 2) + 16 * w) = decode_frag(now.v[b][w], now.vs[b]);

        f32x4 s[2];
#pragma unroll
        for (int b = 0; b < 2; b++) {
            s[b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < KS; c++) {
                const bf16x8_t kf = decode_frag(now.k[b][c], now.ks[b]);
#pragma unroll
                for (int k = PL - 1; k >= 0; k--) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c].f[k], s[b], 0, 0, 0);
            }
        }
        const bool open = (t0 + kKeyTile <= lead.sink_hi) || (t0 >= open_lo && t0 + kKeyTile <= lead.hi);
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (FOLD) s[b][i] = sum_quads(s[b][i]);
                s[b][i] *= p.scale_log2;
                const int key = t0 + 16 * b + 4 * g + i;
                const bool see = open | mine.sees(key);
                if (!see) s[b][i] = -INFINITY;
                if ((nanv[b] != 0) && see) {
                    const uint64_t x = nanv[b] >> (4 * g + i);
#pragma unroll
                    for (int gg = 0; gg < KS; gg++) acc.bad |= (uint32_t)((x >> (16 * (gg * (4 / KS)))) & 1) << gg;
                }
                top = fmaxf(top, s[b][i]);
            }
        top = max_xor16_32(top);
        const float m = fmaxf(acc.m, top);
        const float base = m == -INFINITY ? 0.0f : m;   // nothing visible yet: every probability is 0
        const float alpha = __builtin_amdgcn_exp2f(acc.m - base);
        acc.m = m;
        float pr[8], sum = 0.0f;
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                pr[4 * b + i] = __builtin_amdgcn_exp2f(s[b][i] - base);
                sum += pr[4 * b + i];
            }
        acc.l = acc.l * alpha + sum;   // this lane's keys; the lanes of a query are summed at the end
        Planes<PL> pf;
        if constexpr (FOLD) pf.f[0] = plane8(pr, r >> 2);
        else pf = split8<PL>(pr);
        // (the wave's own region: its LDS operations complete in order)
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < DB; b++) {
            const unsigned char* a = vt + (4 * g + (r >> 2)) * VROW + 32 * b + 8 * (r & 3);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 16 * VROW));
            struct Two { s16x4 a, b; } two = {lo, hi};
            const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, two);
#pragma unroll
            for (int i = 0; i < 4; i++) acc.o[b][i] *= alpha;
#pragma unroll
            for (int k = PL - 1; k >= 0; k--) acc.o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf.f[k], acc.o[b], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    }
    if constexpr (FOLD) {
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) acc.o[b][i] = sum_quads(acc.o[b][i]);
    }
    acc.l = sum_xor16_32(acc.l);
    acc.bad = or_xor16_32(acc.bad);
    if (acc.bad) {
#pragma unroll
        for (int b = 0; b < DB; b++)
            if ((acc.bad >> (b / 2)) & 1) acc.o[b] = f32x4{NAN, NAN, NAN, NAN};
    }

    // merge the four waves: every wave's rows and statistics through LDS
    __syncthreads();
    float* mine_o = (float*)vt;                       // [16 queries][D], then m, l [16]
#pragma unroll
    for (int b = 0; b < DB; b++) *(f32x4*)(mine_o + r * D + 16 * b + 4 * g) = acc.o[b];
    if (g == 0) {
        mine_o[16 * D + r] = acc.m;
        mine_o[16 * D + 16 + r] = acc.l;
    }
    __syncthreads();
    constexpr int CH = D / 4;                         // four dimensions a thread
    for (int u = threadIdx.x; u < RB * CH; u += 256) {
        const int q = u / CH, d = 4 * (u % CH);
        if (row0 + q > last) continue;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; w++) m = fmaxf(m, ((const float*)(smem + w * WAVE_LDS))[16 * D + q]);
        const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float* src = (const float*)(smem + w * WAVE_LDS);
            const float f = __builtin_amdgcn_exp2f(src[16 * D + q] - base);
            l += src[16 * D + 16 + q] * f;
            const f32x4 x = *(const f32x4*)(src + q * D + d);
#pragma unroll
            for (int i = 0; i < 4; i++) o[i] += x[i] * f;
        }
        const int row = row0 + q;
        if (p.splits == 1) {
            const int i = row / p.group, hq = h * p.group + row % p.group;
            const float inv = inverse_sum(p, sp, i, l);
            const int64_t at = p.o.at(p.sp.div, e, i, hq) + d;
            if (p.wide_out) {
                store4<BF16>(p.o.p, at, f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++) store1<BF16>(p.o.p, at + k, o[k] * inv);
            }
        } else {
            const int64_t part = ((int64_t)eh * p.sp.n * p.group + row) * p.splits + split;
            const int64_t parts = (int64_t)regions * p.sp.n * p.group * p.splits;
            *(f32x4*)(p.ws + part * D + d) = o;
            if (d == 0) {
                p.ws[parts * D + 2 * part] = m;
                p.ws[parts * D + 2 * part + 1] = l;
            }
        }
    }
}

// Calls of many query rows: a block of NW waves works on 16 QG NW rows, each wave
// on its own 16 QG; 64-key tiles are decoded once for the block, into LDS as bf16
// rows (keys for 16-byte operand reads, values for transposing ones), with the
// next tile's codes loaded into registers meanwhile.  The running maximum is
// only moved when a score passes it by more than 2^8 (a probability's rounding
// to bf16 is relative, and 2^8 times more fits fp32 with room), so the output
// is rarely rescaled; in bf16 the probabilities' sum is one more row of the
// second product (ones, so the sum is of the rounded ones), not vector work.
//
// What bounds it: the vector unit.  56 queries over 458 keys of 64, 2,048 regions: 33 us
// (65% of the cycles issue vector work, an exponential taking four; the matrix unit
// 24%, LDS 52%); 80 where every 16 rows decoded the keys.  A causal prompt of 8,192
// queries, 4 to a key head of 128, window 4,096: 290 us, 963 TFLOP/s; two waves a
// SIMD whose vector (46%) and matrix work (42%) overlap only in part.
// Queries scaled in two bf16 planes, so that scores come ready for the exponential,
// were slower (38 us); so were waves of 32 rows for the short lists (44), and two
// tiles in LDS, one decoded while the other is worked on (42: fewer waves a SIMD).
constexpr int kWideTile = 64;
constexpr float kSlack = 8.0f;

template <bool BF16, int D, int QG, int NW> struct Wide4 {
    static constexpr int KROW = 2 * D + 16, VROW = 2 * D + 32;   // bytes: an LDS row's banks shift from row to row
    static constexpr int G = D / 32;
    // 16-byte code chunks (32 values, one scale) a thread: wave w's are sets w + NW c
    // of 2 G sets of 64, the keys' first
    static constexpr int CH = 2 * G / NW;
    static_assert(kWideTile == 64 && CH * NW == 2 * G);
    static constexpr int LDS = kWideTile * (KROW + VROW) + kWideTile * G + 16;
};

template <bool BF16, int D, int QG, int NW>
__global__ __launch_bounds__(64 * NW, QG == 2 ? (D == 64 ? 3 : 2) : BF16 ? (D == 64 ? 5 : 3) : 2) void attend4_wide(const Attend4Params p)
{
    using W = Wide4<BF16, D, QG, NW>;
    constexpr int PL = BF16 ? 1 : 3, KS = D / 32, DB = D / 16, VB = 4, RB = 16 * QG * NW;
    __shared__ __align__(16) unsigned char smem[W::LDS];
    unsigned char *kt = smem, *vt = smem + kWideTile * W::KROW;
    uint8_t* nanb = vt + kWideTile * W::VROW;          // [key][group of 32 values]: the values are NaN
    uint8_t* nany = nanb + kWideTile * W::G;           // [wave]: some of its chunks are, and it has set nanb for them

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int regions = p.entries * p.c.heads, split = blockIdx.x % p.splits;
    const int eh = blockIdx.x / p.splits % regions, e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p.sp, p.c, e);
    const int rows = sp.len * p.group, row0 = RB * (blockIdx.x / p.splits / regions);
    if (row0 >= rows) return;
    const int last = min(row0 + RB - 1, rows - 1);
    const KeyList list(p, sp, row0 / p.group, last / p.group);
    const RowSpan lead = list.row(p, sp, row0 / p.group), tail = list.row(p, sp, last / p.group);
    const int open_lo = lead.sink_hi == list.ns && tail.lo == list.ns ? 0 : tail.lo;
    const int N = p.c.slots();
    const uint8_t* reg = p.c.base + (int64_t)eh * p.c.region;

    RowSpan mine[QG];
    Planes<PL> qf[QG][KS];
#pragma unroll
    for (int u = 0; u < QG; u++) {
        const int row = min(row0 + 16 * (QG * wave + u) + r, rows - 1), i = row / p.group, hq = h * p.group + row % p.group;
        mine[u] = list.row(p, sp, i);
        const int64_t at = p.q.at(p.sp.div, e, i, hq) + 8 * g;
#pragma unroll
        for (int c = 0; c < KS; c++) {
            float x[8];
            load8<BF16>(p.q.p, at + 32 * c, p.wide_in, x);
            qf[u][c] = split8<PL>(x);
        }
    }

    const int tiles = (list.nk + kWideTile - 1) / kWideTile;
    const int t_lo = (int)((int64_t)tiles * split / p.splits), t_hi = (int)((int64_t)tiles * (split + 1) / p.splits);

    struct Chunks {
        u32x4 w[W::CH];
        uint32_t s[W::CH];
    } cur;
    auto load = [&](int t) {
#pragma unroll
        for (int c = 0; c < W::CH; c++) {
            const int kv = (wave + NW * c) / W::G, u = (wave + NW * c) % W::G * 64 + lane;
            const uint32_t slot = (uint32_t)list.slot(t * kWideTile + u / W::G) + (uint32_t)(kv * N), grp = (uint32_t)(u % W::G);
            cur.w[c] = *(const u32x4*)(reg + (slot * (uint32_t)(D / 2) + 16 * grp));
            cur.s[c] = reg[(uint32_t)N * D + slot * (uint32_t)W::G + grp];
        }
    };
    auto store = [&]() {
        bool any = false;   // NaN values are kept out of the products and noted
#pragma unroll
        for (int c = 0; c < W::CH; c++)
            if ((wave + NW * c) / W::G) any |= __any(cur.s[c] == 255);
        nany[wave] = any;
        if (__builtin_expect(any, 0)) {
#pragma unroll
            for (int c = 0; c < W::CH; c++)
                if ((wave + NW * c) / W::G) {
                    const bool nan = cur.s[c] == 255;
                    nanb[(wave + NW * c) % W::G * 64 + lane] = nan;
                    if (nan) {
                        cur.w[c] = u32x4{0, 0, 0, 0};
                        cur.s[c] = 127;
                    }
                }
        }
#pragma unroll
        for (int c = 0; c < W::CH; c++) {
            const int kv = (wave + NW * c) / W::G, u = (wave + NW * c) % W::G * 64 + lane;
            const int key = u / W::G, grp = u % W::G;
            unsigned char* to = (kv ? vt + key * W::VROW : kt + key * W::KROW) + 64 * grp;
#pragma unroll
            for (int k = 0; k < 4; k++) *(bf16x8_t*)(to + 16 * k) = decode_frag(cur.w[c][k], cur.s[c]);
        }
    };

    f32x4 o[QG][DB], ls[QG];   // ls: the probabilities' sums (bf16: every row the whole sum; fp32: [0], this lane's keys)
    float base[QG], limit[QG];   // of a row: what its scores are taken from (0 before any), and what moves it
    uint32_t nan_seen[QG];
#pragma unroll
    for (int u = 0; u < QG; u++) {
#pragma unroll
        for (int b = 0; b < DB; b++) o[u][b] = f32x4{0, 0, 0, 0};
        ls[u] = f32x4{0, 0, 0, 0};
        base[u] = 0.0f;
        limit[u] = -INFINITY;
        nan_seen[u] = 0;
    }
    bf16x8_t ones;
#pragma unroll
    for (int j = 0; j < 8; j++) ones[j] = (__bf16)1.0f;

    const bool rows_left = row0 + 16 * QG * wave <= last;
    if (t_lo < t_hi) load(t_lo);
    for (int t = t_lo; t < t_hi; t++) {
        if (t > t_lo) __syncthreads();   // the previous tile has been read
        store();
        if (t + 1 < t_hi) load(t + 1);
        __syncthreads();
        if (!rows_left) continue;   // the wave only decodes
        const int t0 = t * kWideTile;
        // a scale that turns the scores' order around takes the masking path too
        const bool open = ((t0 + kWideTile <= lead.sink_hi) | ((t0 >= open_lo) & (t0 + kWideTile <= lead.hi))) & (p.scale_log2 > 0.0f);

        // scores: the next score block's key fragments are read while this one's
        // are multiplied
        f32x4 s[QG][4];
        bf16x8_t kf[2][KS];
        auto read_k = [&](int b) {
#pragma unroll
            for (int c = 0; c < KS; c++) kf[b & 1][c] = *(const bf16x8_t*)(kt + (16 * b + r) * W::KROW + 64 * c + 16 * g);
        };
        read_k(0);
#pragma unroll
        for (int b = 0; b < 4; b++) {
            if (b + 1 < 4) read_k(b + 1);
#pragma unroll
            for (int u = 0; u < QG; u++) s[u][b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < KS; c++)
#pragma unroll
                for (int u = 0; u < QG; u++)
#pragma unroll
                    for (int k = PL - 1; k >= 0; k--)
                        s[u][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[b & 1][c], qf[u][c].f[k], s[u][b], 0, 0, 0);
        }
        // the first values' fragments, read while the probabilities are computed
        bf16x8_t vf[2][VB];
        auto read_v = [&](int half, int b0) {
#pragma unroll
            for (int b = 0; b < VB; b++) {
                const unsigned char* a = vt + (32 * half + 4 * g + (r >> 2)) * W::VROW + 32 * (b0 + b) + 8 * (r & 3);
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 16 * W::VROW));
                struct Two { s16x4 a, b; } two = {lo, hi};
                vf[(half * DB + b0) / VB & 1][b] = __builtin_bit_cast(bf16x8_t, two);
            }
        };
        read_v(0, 0);
        const float mul = open ? p.scale_log2 : 1.0f;
        uint32_t nan_waves = 0;
#pragma unroll
        for (int w = 0; w < NW; w++) nan_waves |= nany[w];

#pragma unroll
        for (int u = 0; u < QG; u++) {
            // (masked scores are scaled before their mask: 0 times an infinity is NaN)
            if (!open) {
#pragma unroll
                for (int b = 0; b < 4; b++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        s[u][b][i] = mine[u].sees(t0 + 16 * b + 4 * g + i) ? s[u][b][i] * p.scale_log2 : -INFINITY;
            }
            if (__builtin_expect(nan_waves != 0, 0)) {
#pragma unroll 1
                for (int k = 0; k < 16; k++) {
                    const int at = 16 * (k >> 2) + 4 * g + (k & 3);
                    for (int gg = 0; gg < W::G; gg++)
                        if (mine[u].sees(t0 + at) && nany[(W::G + (at * W::G + gg) / 64) % NW] && nanb[at * W::G + gg])
                            nan_seen[u] |= 1u << gg;
                }
            }
            // (the lanes of a row compare their own keys; they meet only to move its base)
            float top = s[u][0][0];
#pragma unroll
            for (int k = 1; k < 16; k++) top = fmaxf(top, s[u][k >> 2][k & 3]);
            if (__any(top * mul > limit[u])) {
                top = max_xor16_32(top) * mul;
                const bool move = top > limit[u];
                // (from base itself: limit - kSlack is off by up to 2^-21 of a power of two)
                const float f = move ? __builtin_amdgcn_exp2f((limit[u] == -INFINITY ? -INFINITY : base[u]) - top) : 1.0f;
                if (move) {
                    limit[u] = top + kSlack;
                    base[u] = top;
                }
#pragma unroll
                for (int b = 0; b < DB; b++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[u][b][i] *= f;
#pragma unroll
                for (int i = 0; i < 4; i++) ls[u][i] *= f;
            }
        }
        // each half tile's probabilities and products (a list that ends in the
        // first half has no second)
#pragma unroll
        for (int half = 0; half < 2; half++) {
            if (D == 64 && half && t0 + 32 >= list.nk) break;
            Planes<PL> pf[QG];
#pragma unroll
            for (int u = 0; u < QG; u++) {
                float pr[8];
#pragma unroll
                for (int j = 0; j < 8; j++)
                    pr[j] = __builtin_amdgcn_exp2f(fmaf(s[u][2 * half + (j >> 2)][j & 3], mul, -base[u]));
                if constexpr (!BF16) {
#pragma unroll
                    for (int j = 0; j < 8; j++) ls[u][0] += pr[j];
                }
                pf[u] = split8<PL>(pr);
            }
#pragma unroll
            for (int b0 = 0; b0 < DB; b0 += VB) {
                if (b0 + VB < DB) read_v(half, b0 + VB);
                else if (half == 0) read_v(1, 0);
#pragma unroll
                for (int b = 0; b < VB; b++)
#pragma unroll
                    for (int u = 0; u < QG; u++)
#pragma unroll
                        for (int k = PL - 1; k >= 0; k--)
                            o[u][b0 + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[(half * DB + b0) / VB & 1][b], pf[u].f[k], o[u][b0 + b], 0, 0, 0);
            }
            if constexpr (BF16) {
#pragma unroll
                for (int u = 0; u < QG; u++) ls[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[u].f[0], ls[u], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < QG; u++) {
        const float l = BF16 ? ls[u][0] : sum_xor16_32(ls[u][0]);
        const uint32_t nan = or_xor16_32(nan_seen[u]);
        const int row = row0 + 16 * (QG * wave + u) + r;
        if (row > last) continue;
        const int i = row / p.group, hq = h * p.group + row % p.group;
        const int64_t at = p.o.at(p.sp.div, e, i, hq);
        const int64_t part = ((int64_t)eh * p.sp.n * p.group + row) * p.splits + split;
        const int64_t parts = (int64_t)regions * p.sp.n * p.group * p.splits;
        const float inv = p.splits > 1 ? 0.0f : inverse_sum(p, sp, i, l);
#pragma unroll
        for (int b = 0; b < DB; b++) {
            f32x4 x = o[u][b];
            if ((nan >> (b / 2)) & 1) x = f32x4{NAN, NAN, NAN, NAN};
            const int d = 16 * b + 4 * g;
            if (p.splits > 1) {
                *(f32x4*)(p.ws + part * D + d) = x;
            } else if (p.wide_out) {
                store4<BF16>(p.o.p, at + d, f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv});
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++) store1<BF16>(p.o.p, at + d + k, x[k] * inv);
            }
        }
        if (p.splits > 1 && g == 0) {
            p.ws[parts * D + 2 * part] = limit[u] == -INFINITY ? -INFINITY : base[u];
            p.ws[parts * D + 2 * part + 1] = l;
        }
    }
}

// Joins the splits of a row: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// NG groups of D / 4 threads share a row's splits, each with its own running
// maximum, and meet in LDS (512 splits of 60 rows: 130 -> 8 us against one thread
// for all of them).
template <bool BF16, int D, int NG> __global__ __launch_bounds__(256) void attend4_join(const Attend4Params p)
{
    constexpr int CH = D / 4, ROWS = 256 / (CH * NG);   // rows of a block
    __shared__ __align__(16) float sm[NG > 1 ? ROWS * NG * (D + 2) : 1];
    const int rows = p.sp.n * p.group;
    const int64_t regions = (int64_t)p.entries * p.c.heads;
    const int ch = threadIdx.x % CH, grp = threadIdx.x / CH % NG, local = threadIdx.x / (CH * NG), d = 4 * ch;
    const int64_t id = (int64_t)blockIdx.x * ROWS + local;
    const bool in = id < regions * rows;
    const int64_t at_id = in ? id : 0;
    const int eh = (int)(at_id / rows), row = (int)(at_id % rows), e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p.sp, p.c, e);
    const bool on = in && row < sp.len * p.group;
    const int64_t parts = regions * rows * p.splits;
    const float* ml = p.ws + parts * D + 2 * at_id * p.splits;
    const float* po = p.ws + at_id * p.splits * D + d;
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (on) {
        for (int s = grp; s < p.splits; s += NG) {
            const float ms = ml[2 * s], top = fmaxf(m, ms), base = top == -INFINITY ? 0.0f : top;
            const float a = __builtin_amdgcn_exp2f(m - base), b = __builtin_amdgcn_exp2f(ms - base);
            const f32x4 x = *(const f32x4*)(po + (int64_t)s * D);
            m = top;
            l = l * a + ml[2 * s + 1] * b;
#pragma unroll
            for (int k = 0; k < 4; k++) o[k] = o[k] * a + x[k] * b;
        }
    }
    if constexpr (NG > 1) {
        *(f32x4*)(sm + (local * NG + grp) * D + d) = o;
        float* stat = sm + ROWS * NG * D + 2 * (local * NG + grp);
        if (ch == 0) {
            stat[0] = m;
            stat[1] = l;
        }
        __syncthreads();
        if (grp) return;
        const float* all = sm + ROWS * NG * D + 2 * local * NG;
        for (int g = 0; g < NG; g++) m = fmaxf(m, all[2 * g]);
        const float base = m == -INFINITY ? 0.0f : m;
        l = 0.0f;
        o = f32x4{0, 0, 0, 0};
        for (int g = 0; g < NG; g++) {
            const float f = __builtin_amdgcn_exp2f(all[2 * g] - base);
            const f32x4 x = *(const f32x4*)(sm + (local * NG + g) * D + d);
            l += all[2 * g + 1] * f;
#pragma unroll
            for (int k = 0; k < 4; k++) o[k] += x[k] * f;
        }
    }
    if (!on) return;
    const int i = row / p.group, hq = h * p.group + row % p.group;
    const float inv = inverse_sum(p, sp, i, l);
    const int64_t at = p.o.at(p.sp.div, e, i, hq) + d;
    if (p.wide_out) {
        store4<BF16>(p.o.p, at, f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
    } else {
#pragma unroll
        for (int k = 0; k < 4; k++) store1<BF16>(p.o.p, at + k, o[k] * inv);
    }
}

static Plan4 plan4(const Carry4& c, int entries, int n, int group, int window, bool bf16)
{
    return plan4(c.D, c.sinks, c.ring, (int64_t)entries * c.heads, n, group, window, bf16);
}

int attend4_splits(const Carry4& c, int entries, int n, int group, int window, int bf16, int64_t* ws_bytes)
{
    const Plan4 pl = plan4(c, entries, n, group, window, bf16 != 0);
    if (ws_bytes)
        *ws_bytes = pl.splits > 1 ? (int64_t)entries * c.heads * n * group * pl.splits * (c.D + 2) * 4 : 0;
    return pl.splits;
}

template <bool BF16, int D> hipError_t launch_attend4_d(const Attend4Params& p, hipStream_t st)
{
    const int64_t rows = (int64_t)p.sp.n * p.group;
    const int rb = plan4(p.c, p.entries, p.sp.n, p.group, p.window, BF16).rows;
    const int64_t blocks = (int64_t)p.splits * p.entries * p.c.heads * ((rows + rb - 1) / rb);
    hipError_t e = hipErrorInvalidValue;
    if (rb == 16 && !BF16 && rows <= 4) e = launch_with(attend4_kernel<BF16, D, !BF16>, blocks, st, p);
    else if (rb == 16) e = launch_with(attend4_kernel<BF16, D, false>, blocks, st, p);
    else if (rb == 64 || !BF16) e = launch_with(attend4_wide<BF16, D, 1, 4>, blocks, st, p);
    else if constexpr (BF16) e = launch_with(attend4_wide<BF16, D, 2, 4>, blocks, st, p);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t all = (int64_t)p.entries * p.c.heads * rows;
    // (of many rows a group takes one each: 8,000 rows in five splits 31 us with a
    // block a row, 21 with 16)
    constexpr int per = 256 / (D / 4);   // rows of a block, or groups of one row
    if (p.splits <= 4 || all >= 2048) return launch_with(attend4_join<BF16, D, 1>, (all + per - 1) / per, st, p);
    return launch_with(attend4_join<BF16, D, per>, all, st, p);
}

hipError_t launch_attend4(const Attend4Params& p, int bf16, hipStream_t st)
{
    if (p.c.D == 64) return bf16 ? launch_attend4_d<true, 64>(p, st) : launch_attend4_d<false, 64>(p, st);
    return bf16 ? launch_attend4_d<true, 128>(p, st) : launch_attend4_d<false, 128>(p, st);
}

}  // namespace dcf
