// gfx950 kernels of the attention operators: per-head norms with the position
// rotation, the store of keys and values into a carry held in 4 bits, and the
// attention over it.  Part of flow_kernels.hip (one code object), whose vector
// types and cross-lane helpers it uses.

namespace dcf {

template <class P> hipError_t launch_with(void (*kernel)(P), dim3 grid, dim3 block, hipStream_t st, P p)
{
    void* args[] = {&p};
    return hipLaunchKernel((const void*)kernel, grid, block, args, 0, st);
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
        const int b = e / s.div;
        pos = s.pos ? s.pos[b] : 0;
        len = s.lens ? min(max(s.lens[b], 0), s.n) : s.n;
        sinks = min(max(s.sinks ? s.sinks[b] : s.sinks_all, 0), c.sinks);
        if (pos < 0 || pos > (int64_t)1 << 60) pos = len = 0;
        total = pos + len;
    }
};

// Sum and maximum over aligned groups of LANES lanes (4, 8, 16 or 32), in
// every lane, one fixed order.
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
    if constexpr (LANES >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        const uint32_t a0 = a[0], a1 = a[1];
        v = f(a0, a1);
    }
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
    return __uint_as_float(lanes_reduce<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}

// Eight consecutive elements of a row.
template <bool BF16> __device__ __forceinline__ void load8(const void* p, int64_t at, int wide, float (&x)[8])
{
    if constexpr (BF16) {
        const uint16_t* s = (const uint16_t*)p + at;
        if (wide) {
            const u32x4 w = *(const u32x4*)s;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                x[2 * j] = bf2f(w[j] & 0xffffu);
                x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] = bf2f(s[j]);
        }
    } else {
        const float* s = (const float*)p + at;
        if (wide) {
            const f32x4 a = *(const f32x4*)s, b = *(const f32x4*)(s + 4);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                x[j] = a[j];
                x[4 + j] = b[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] = s[j];
        }
    }
}
template <bool BF16> __device__ __forceinline__ void store8(void* p, int64_t at, int wide, const float (&x)[8])
{
    if (wide) {
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
// D / 8 lanes hold a head's row, eight consecutive elements each, and a wave
// 64 / (D / 8) tokens, whose heads it walks; so the cosines and sines of a
// lane's token and dimensions are computed once for all its heads.
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
// precision they are computed in.  A group with a NaN or an infinity is NaN.
template <bool BF16, bool OUT16, int D>
__global__ __launch_bounds__(256) void heads_kernel(const HeadsParams p)
{
    constexpr int L = D / 8, TPW = 64 / L;   // lanes of a row, tokens of a wave
    const int lane = threadIdx.x & 63, l = lane % L;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int n = p.sp.n;
    const int64_t tokens = (int64_t)p.entries * n;
    const int64_t t = (int64_t)(wave / p.splits) * TPW + lane / L;
    const int e = (int)(min(t, tokens - 1) / n), i = (int)(min(t, tokens - 1) % n);
    const Span sp(p.sp, p.c, e);
    const bool on = t < tokens && i < sp.len;
    const int64_t pos = sp.pos + i;

    const int jobs = p.q.heads + p.k.heads + p.v.heads;
    const int part = wave % p.splits;
    const int j0 = (int)((int64_t)jobs * part / p.splits), j1 = (int)((int64_t)jobs * (part + 1) / p.splits);

    // the rotation of this lane's dimensions; identity past rot
    float cs[8], sn[8];
    const bool inter = p.interleaved != 0;
    const int half = p.rot >> 1;
    const bool first = 8 * l < half;                     // half-split pairs: this lane holds the pairs' first members
    if (p.norm) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int d = 8 * l + j, f = inter ? d >> 1 : first ? d : d - half;
            cs[j] = 1.0f;
            sn[j] = 0.0f;
            if (d < p.rot && !(inter && (j & 1))) {
                sincospif(2.0f * turn_fraction(pos, p.freqs[f]), &sn[j], &cs[j]);
            }
            if (inter && (j & 1)) {
                cs[j] = cs[j - 1];
                sn[j] = sn[j - 1];
            }
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

    for (int j = j0; j < j1; j++) {
        const int kind = j < p.q.heads ? 0 : j < p.q.heads + p.k.heads ? 1 : 2;
        const int h = kind == 0 ? j : kind == 1 ? j - p.q.heads : j - p.q.heads - p.k.heads;
        const HeadRows& in = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
        float x[8] = {};
        if (on) load8<BF16>(in.p, in.at(p.sp.div, e, i, h) + 8 * l, p.wide_in, x);
        if (p.norm && kind < 2) {
            float ss = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; k++) ss = fmaf(x[k], x[k], ss);
            ss = lanes_sum<L>(ss);
            const float r = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
            const float* gain = kind == 0 ? p.q_gain : p.k_gain;
#pragma unroll
            for (int k = 0; k < 8; k++) x[k] = x[k] * r * (gain ? gain[8 * l + k] : 1.0f);
            if (inter) {
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const float a = x[k], b = x[k + 1];
                    x[k] = a * cs[k] - b * sn[k];
                    x[k + 1] = b * cs[k] + a * sn[k];
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const float y = __shfl(x[k], partner);
                    x[k] = x[k] * cs[k] + (first ? -y : y) * sn[k];
                }
            }
        }
        if (kind == 0 || (kind == 1 && p.k_out.p)) {
            const HeadRows& o = kind == 0 ? p.q_out : p.k_out;
            if (on) store8<OUT16>(o.p, o.at(p.sp.div, e, i, h) + 8 * l, p.wide_out, x);
        } else {
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
            if (top >= 0x7f800000u) {
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
    }
}

template <bool BF16, bool OUT16, int D> hipError_t launch_heads_d(HeadsParams p, hipStream_t st)
{
    constexpr int TPW = 64 / (D / 8);
    const int64_t tokens = (int64_t)p.entries * p.sp.n, groups = (tokens + TPW - 1) / TPW;
    const int jobs = p.q.heads + p.k.heads + p.v.heads;
    // a wave walks all heads of its tokens unless that leaves few waves
    int64_t splits = 1;
    while (splits < jobs && groups * splits < 4096) splits *= 2;
    p.splits = (int)(splits < jobs ? splits : jobs);
    return launch_with(heads_kernel<BF16, OUT16, D>, dim3((unsigned)((groups * p.splits + 3) / 4)), dim3(256), st, p);
}

hipError_t launch_heads(HeadsParams p, int D, int bf16, hipStream_t st)
{
    if (D == 64)
        return bf16 ? launch_heads_d<true, true, 64>(p, st)
                    : p.out_bf16 ? launch_heads_d<false, true, 64>(p, st) : launch_heads_d<false, false, 64>(p, st);
    return bf16 ? launch_heads_d<true, true, 128>(p, st)
                : p.out_bf16 ? launch_heads_d<false, true, 128>(p, st) : launch_heads_d<false, false, 128>(p, st);
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

template <bool BF16, int D> __global__ __launch_bounds__(256) void read4_kernel(const Read4Params p)
{
    constexpr int L = D / 8;
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;   // (entry, token, head)
    const int l = threadIdx.x % L, kv = blockIdx.y;
    if (row >= (int64_t)p.entries * p.sp.n * p.c.heads) return;
    const int h = (int)(row % p.c.heads), i = (int)(row / p.c.heads % p.sp.n), e = (int)(row / p.c.heads / p.sp.n);
    const Span sp(p.sp, p.c, e);
    if (i >= sp.len) return;
    const int64_t pos = sp.pos + i;
    const int64_t slot = pos < sp.sinks ? pos : p.c.sinks + (p.c.ring ? (pos - sp.sinks) % p.c.ring : 0);
    if (slot >= p.c.slots()) return;
    const int N = p.c.slots();
    const uint8_t* reg = p.c.base + ((int64_t)e * p.c.heads + h) * p.c.region;
    const uint32_t w = *(const uint32_t*)(reg + ((int64_t)kv * N + slot) * (D / 2) + 4 * l);
    const uint32_t s = reg[(int64_t)N * D + ((int64_t)kv * N + slot) * (D / 32) + (l >> 2)];
    float x[8];
    decode8(w, s, x);
    const HeadRows& o = kv ? p.v : p.k;
    store8<BF16>(o.p, o.at(p.sp.div, e, i, h) + 8 * l, p.wide, x);
}

hipError_t launch_read4(const Read4Params& p, int bf16, hipStream_t st)
{
    const int64_t threads = (int64_t)p.entries * p.sp.n * p.c.heads * (p.c.D / 8);
    const dim3 grid((unsigned)((threads + 255) / 256), 2), block(256);
    if (p.c.D == 64)
        return bf16 ? launch_with(read4_kernel<true, 64>, grid, block, st, p) : launch_with(read4_kernel<false, 64>, grid, block, st, p);
    return bf16 ? launch_with(read4_kernel<true, 128>, grid, block, st, p) : launch_with(read4_kernel<false, 128>, grid, block, st, p);
}

template <int D>
__global__ __launch_bounds__(256) void carry4_gather_kernel(const Carry4 c, const Spans spans, int e, int kv, int f_chunk,
                                                            int nh, int frames, float* out)
{
    constexpr int L = D / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / L;   // (frame, head)
    const int l = (int)(u % L), f = (int)(row / c.heads), h = (int)(row % c.heads);
    if (f >= frames) return;
    const Span sp(spans, c, e);
    const int64_t at = f < nh * f_chunk ? sp.pos - (int64_t)(f / f_chunk + 1) * f_chunk + f % f_chunk : f - nh * f_chunk;
    int64_t slot = at < sp.sinks ? at : c.sinks + (at - sp.sinks) % c.ring;
    slot = slot < 0 ? 0 : slot;
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
    const unsigned blocks = (unsigned)(((int64_t)frames * c.heads * (c.D / 8) + 255) / 256);
    if (c.D == 64) hipLaunchKernelGGL(carry4_gather_kernel<64>, dim3(blocks), dim3(256), 0, st, c, sp, e, kv, f_chunk, nh, frames, out);
    else hipLaunchKernelGGL(carry4_gather_kernel<128>, dim3(blocks), dim3(256), 0, st, c, sp, e, kv, f_chunk, nh, frames, out);
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
// three products give the fp32 one (keys and values are exact in bf16).
constexpr int kKeyTile = 32;

template <int PL> struct Planes { bf16x8_t f[PL]; };

template <int PL> __device__ __forceinline__ Planes<PL> split8(const float (&x)[8])
{
    Planes<PL> r;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; j++) y[j] = x[j];
#pragma unroll
    for (int k = 0; k < PL; k++) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const __bf16 b = (__bf16)y[j];
            r.f[k][j] = b;
            if (k + 1 < PL) y[j] -= (float)b;
        }
    }
    return r;
}

// The rows' visible members of the block's list.
struct RowSpan {
    int sink_hi, lo, hi;   // visible: [0, sink_hi) and [lo, hi)
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

template <bool BF16, int D>
__global__ __launch_bounds__(256) void attend4_kernel(const Attend4Params p)
{
    constexpr int PL = BF16 ? 1 : 3, KS = D / 32, DB = D / 16;
    constexpr int VROW = 2 * D + 32;   // bytes of a value row in LDS: eight banks on from row to row
    constexpr int WAVE_LDS = kKeyTile * VROW > 16 * D * 4 + 128 ? kKeyTile * VROW : 16 * D * 4 + 128;
    __shared__ __align__(16) unsigned char smem[4 * WAVE_LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int regions = p.entries * p.c.heads, split = blockIdx.x % p.splits;
    const int eh = blockIdx.x / p.splits % regions, e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p.sp, p.c, e);
    const int rows = sp.len * p.group, row0 = 16 * (blockIdx.x / p.splits / regions);
    if (row0 >= rows) return;                       // (uniform: the block's rows are behind the entry's last token)
    const int last = min(row0 + 15, rows - 1);
    const KeyList list(p, sp, row0 / p.group, last / p.group);
    const RowSpan mine = list.row(p, sp, min(row0 + r, rows - 1) / p.group);
    const RowSpan lead = list.row(p, sp, row0 / p.group), tail = list.row(p, sp, last / p.group);
    const int open_lo = lead.sink_hi == list.ns && tail.lo == list.ns ? 0 : tail.lo;   // members visible to every row
    const int N = p.c.slots();
    const uint8_t* reg = p.c.base + (int64_t)eh * p.c.region;

    // queries as B operand: lane (q, g) holds dimensions g D / 4 + 8 c .. + 7
    Planes<PL> qf[KS];
    {
        const int row = min(row0 + r, rows - 1), i = row / p.group, hq = h * p.group + row % p.group;
        const int64_t at = p.q.at(p.sp.div, e, i, hq) + g * (D / 4);
#pragma unroll
        for (int c = 0; c < KS; c++) {
            float x[8];
            load8<BF16>(p.q.p, at + 8 * c, p.wide_in, x);
            qf[c] = split8<PL>(x);
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
                s[b][i] *= p.scale_log2;
                const int key = t0 + 16 * b + 4 * g + i;
                const bool see = open || (key < mine.sink_hi || (key >= mine.lo && key < mine.hi));
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
        const Planes<PL> pf = split8<PL>(pr);
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
    for (int u = threadIdx.x; u < 16 * CH; u += 256) {
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
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
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

// Joins the splits of a row: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
template <bool BF16, int D> __global__ __launch_bounds__(256) void attend4_join(const Attend4Params p)
{
    constexpr int CH = D / 4;
    const int rows = p.sp.n * p.group;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, regions = (int64_t)p.entries * p.c.heads;
    const int64_t id = u / CH;
    const int d = 4 * (int)(u % CH);
    if (id >= regions * rows) return;
    const int eh = (int)(id / rows), row = (int)(id % rows), e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p.sp, p.c, e);
    if (row >= sp.len * p.group) return;
    const int64_t parts = regions * rows * p.splits;
    const float* ml = p.ws + parts * D + 2 * id * p.splits;
    float m = -INFINITY, l = 0.0f;
    for (int s = 0; s < p.splits; s++) m = fmaxf(m, ml[2 * s]);
    const float base = m == -INFINITY ? 0.0f : m;
    f32x4 o = {0, 0, 0, 0};
    for (int s = 0; s < p.splits; s++) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * s] - base);
        l += ml[2 * s + 1] * f;
        const f32x4 x = *(const f32x4*)(p.ws + (id * p.splits + s) * D + d);
#pragma unroll
        for (int k = 0; k < 4; k++) o[k] += x[k] * f;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int i = row / p.group, hq = h * p.group + row % p.group;
    const int64_t at = p.o.at(p.sp.div, e, i, hq) + d;
    if (p.wide_out) {
        store4<BF16>(p.o.p, at, f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv});
    } else {
#pragma unroll
        for (int k = 0; k < 4; k++) store1<BF16>(p.o.p, at + k, o[k] * inv);
    }
}

int attend4_splits(const Carry4& c, int entries, int n, int group, int window, int64_t* ws_bytes)
{
    const int64_t rows = (int64_t)n * group, blocks = (int64_t)entries * c.heads * ((rows + 15) / 16);
    const int64_t most = (int64_t)c.sinks + (window < c.ring ? window : c.ring) + n;
    int64_t s = 1024 / (blocks > 0 ? blocks : 1), per = (most + 8 * kKeyTile - 1) / (8 * kKeyTile);
    if (s > per) s = per;
    if (s < 1) s = 1;
    if (ws_bytes) *ws_bytes = s > 1 ? (int64_t)entries * c.heads * rows * s * (c.D + 2) * 4 : 0;
    return (int)s;
}

template <bool BF16, int D> hipError_t launch_attend4_d(const Attend4Params& p, hipStream_t st)
{
    const int rows = p.sp.n * p.group;
    const unsigned blocks = (unsigned)((int64_t)p.splits * p.entries * p.c.heads * ((rows + 15) / 16));
    hipError_t e = launch_with(attend4_kernel<BF16, D>, dim3(blocks), dim3(256), st, p);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t threads = (int64_t)p.entries * p.c.heads * rows * (D / 4);
    return launch_with(attend4_join<BF16, D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), st, p);
}

hipError_t launch_attend4(const Attend4Params& p, int bf16, hipStream_t st)
{
    if (p.c.D == 64) return bf16 ? launch_attend4_d<true, 64>(p, st) : launch_attend4_d<false, 64>(p, st);
    return bf16 ? launch_attend4_d<true, 128>(p, st) : launch_attend4_d<false, 128>(p, st);
}

}  // namespace dcf
