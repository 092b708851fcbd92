// gfx950 kernels of the paged cache: the store of new keys and values, and the
// attention of a call's tokens over the cache.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "block_internal.h"
#include "paged_plan.h"

namespace dcb {

// An entry's span of a call.  Values that no caller may pass (a negative
// position, a length past the call's) are taken as none and as the largest.
struct Span {
    int64_t pos, total;   // first position of the call, position after its last token
    int len;
    __device__ __forceinline__ Span(const PagedParams& p, int e)
    {
        pos = p.pos[e];
        len = p.lens ? min(max(p.lens[e], 0), p.n) : p.n;
        if (pos < 0 || pos > (int64_t)1 << 60) pos = len = 0;
        total = pos + len;
    }
};

// The page of position x of entry e (unsigned: a number outside the pool is
// `pages` or more).
__device__ __forceinline__ uint32_t page_of(const Paged& c, int e, int x) { return (uint32_t)c.table[e * c.table_stride + (x >> c.shift)]; }

// Bytes from a pool's start to row `off` of a page.
__device__ __forceinline__ uint64_t row_offset(uint32_t page, uint32_t sp, uint32_t off, uint32_t st)
{
    return ((uint64_t)page * sp + (uint64_t)off * st) << 4;
}

// ------------------------------------------------------------------- store
//
// A thread copies 16 bytes of a key and of its value.  What bounds it: HBM (16,384
// tokens of eight bf16 heads of 128, 134 MB, past the caches: 28.6 us, 4.7 TB/s), or the launch.
template <int ES> __global__ __launch_bounds__(256) void append_kernel(const PagedParams p)
{
    constexpr int CE = 16 / ES;
    const int cpr = p.c.D / CE, per = p.c.heads * cpr;   // chunks of a row, of a token
    const uint64_t u = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t token = (uint32_t)(u / per), in = (uint32_t)(u - (uint64_t)token * per);
    const int e = token / p.n, i = token - e * p.n, h = in / cpr, ch = in - h * cpr;
    if (e >= p.c.batch) return;
    const Span sp(p, e);
    const int64_t x = sp.pos + i;
    if (i >= sp.len || x >= p.c.limit) return;
    const uint32_t page = page_of(p.c, e, (int)x);
    if (page >= (uint32_t)p.c.pages) return;
    const int off = (int)x & ((1 << p.c.shift) - 1);
    const u32x4 a = *(const u32x4_any*)((const char*)p.k.p + (p.k.at(e, i, h) + ch * CE) * ES);
    const u32x4 b = *(const u32x4_any*)((const char*)p.v.p + (p.v.at(e, i, h) + ch * CE) * ES);
    *(u32x4*)(p.c.k + row_offset(page, p.c.kp, off, p.c.kt) + 16 * ((uint64_t)h * p.c.kh + ch)) = a;
    *(u32x4*)(p.c.v + row_offset(page, p.c.vp, off, p.c.vt) + 16 * ((uint64_t)h * p.c.vh + ch)) = b;
}

hipError_t launch_append(const PagedParams& p, hipStream_t st)
{
    const int64_t threads = (int64_t)p.c.batch * p.n * p.c.heads * (p.c.D / (p.c.bf16 ? 8 : 4));
    return p.c.bf16 ? launch_with(append_kernel<2>, (threads + 255) / 256, 256, 0, st, p)
                    : launch_with(append_kernel<4>, (threads + 255) / 256, 256, 0, st, p);
}

// --------------------------------------------------------------- attention
//
// O = softmax(scale Q K^T) V.  A row is (token i, query head), the `group` query
// heads of a key head side by side, so shared heads share the loads of their keys.
// A block walks tiles of KT keys, which begin at multiples of KT: those of the first
// tokens, then those from its first row's window on.
//
// S^T = K Q^T and O^T += V^T P^T, so that a lane (r, g) = (lane % 16, lane / 16)
// holds of query r the scores of keys 4 g .. 4 g + 3 of every sixteen, and of its
// result the dimensions 16 b + 4 g .. + 3.  bf16: the product with the values takes a
// probability in two bf16 parts in blocks of 16 rows (the loads bound them: of one token
// over 65,000 keys of 8 entries 386 us, one part 384), and rounded to bf16, half a step
// of the result's own type, in blocks of more (the products bound them: of 4,096 tokens
// of 2 entries over 6,000 others 533 us, two parts 711; all normally distributed).
// Errors are 1.00 and 1.41 times those of the result's own rounding.  fp32: four 16x16x4 products of a
// 16-byte chunk's elements, in fp32 throughout.
struct RowSpan {
    int hi, lo, sinks;   // a row sees the positions below hi, of those the ones from lo on and the first `sinks`
    RowSpan() = default;
    __device__ __forceinline__ RowSpan(const PagedParams& p, const Span& sp, int i)
    {
        const int64_t at = sp.pos + i, limit = p.c.limit;
        hi = (int)min(p.causal ? at + 1 : sp.total, limit);
        lo = p.window ? (int)min(max(p.causal ? at + 1 - p.window : sp.pos - p.window, (int64_t)0), limit) : 0;
        sinks = p.sinks;
    }
    __device__ __forceinline__ bool sees(int x) const { return (x < hi) & ((x >= lo) | (x < sinks)); }
};

// The tiles of a block whose rows lie between `lead` and `tail`.
template <int KT> struct Tiles {
    int of_sinks, skip, n;   // tiles of the first tokens, tiles left out behind them, tiles in all
    int all_hi, all_lo;      // every row sees [all_lo, all_hi)
    __device__ __forceinline__ Tiles(const RowSpan& lead, const RowSpan& tail)
    {
        of_sinks = (min(tail.sinks, tail.hi) + KT - 1) / KT;
        const int from = max(lead.lo / KT, of_sinks), end = (tail.hi + KT - 1) / KT;
        skip = from - of_sinks;
        n = of_sinks + max(end - from, 0);
        all_hi = lead.hi;
        all_lo = tail.lo <= tail.sinks ? 0 : tail.lo;
    }
    __device__ __forceinline__ int first(int t) const { return KT * (t < of_sinks ? t : t + skip); }   // position
    __device__ __forceinline__ bool open(int x, int sinks) const { return (x + KT <= all_hi) & ((x >= all_lo) | (x + KT <= sinks)); }
};

template <bool BF16> __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 acc)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int t = 0; t < 4; t++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[t]), __uint_as_float(b[t]), acc, 0, 0, 0);
        return acc;
    }
}

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ u32x4 read_tr(const unsigned char* lo, const unsigned char* hi)
{
    struct Two {
        s16x4 a, b;
    } two = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lo), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)hi)};
    return __builtin_bit_cast(u32x4, two);
}

// A loaded value is waited for here (or the compiler waits where a loop uses it, in
// every turn, and for that turn's loads as well).
__device__ __forceinline__ void arrived(u32x4& x) { asm volatile("" : "+v"(x)); }

// Bits of a chunk's elements that are an infinity or a NaN.
template <bool BF16> __device__ __forceinline__ uint32_t special_of(u32x4 w)
{
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const uint32_t hi = (w[k] & 0x7f800000u) == 0x7f800000u, lo = (w[k] & 0x7f80u) == 0x7f80u;
        bits |= BF16 ? (lo | hi << 1) << (2 * k) : hi << k;
    }
    return bits;
}

// Values that are no numbers reach the rows that see them only, and 0 times them is
// not 0: they are added to the rows' results one by one here, and the caller sets
// them to zero before the product.  `where(c)` is the lane's c-th chunk of a tile's
// `chunks`: its address, key and first dimension; s holds the probabilities.
struct ChunkAt {
    unsigned char* p;
    int key, d;
};
template <bool BF16, int QG, int NB, int DB, class Where, class Sees>
__device__ __forceinline__ void add_special(int chunks, Where where, Sees sees, const f32x4 (&s)[QG][NB], f32x4 (&o)[QG][DB])
{
    const int r = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
#pragma unroll 1
    for (int c = 0; c < chunks; c++) {
        const ChunkAt at = where(c);
        uint32_t bits = special_of<BF16>(*(const u32x4*)at.p);
#pragma unroll 1
        for (uint64_t lanes = __ballot(bits != 0); lanes; lanes = __ballot(bits != 0)) {
            const int from = __builtin_ctzll(lanes), el = __builtin_ctz(__builtin_amdgcn_readlane(bits, from));
            const int key = __builtin_amdgcn_readlane(at.key, from), d = __builtin_amdgcn_readlane(at.d, from) + el;
            float v = load1(at.p, el, BF16);
            v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), from));
            if ((int)(threadIdx.x & 63) == from) bits &= bits - 1;
            const int j = 4 * (key >> 4) + (key & 3);
#pragma unroll
            for (int u = 0; u < QG; u++) {
                float pk = s[u][0][0];
#pragma unroll
                for (int x = 1; x < 4 * NB; x++) pk = j == x ? s[u][x >> 2][x & 3] : pk;
                pk = __shfl(pk, 16 * ((key >> 2) & 3) + r);
                const bool mine = sees(u, key) & (g == ((d >> 2) & 3));
#pragma unroll
                for (int b = 0; b < DB; b++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (mine & (16 * b + i == (d & ~12))) o[u][b][i] = fmaf(pk, v, o[u][b][i]);
            }
        }
    }
}
// A chunk without them.
template <bool BF16> __device__ __forceinline__ u32x4 clear_special(u32x4 w)
{
    const uint32_t bits = special_of<BF16>(w);
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if constexpr (BF16) w[k] &= ((bits >> (2 * k)) & 1 ? 0xffff0000u : 0xffffffffu) & ((bits >> (2 * k)) & 2 ? 0x0000ffffu : 0xffffffffu);
        else w[k] = (bits >> k) & 1 ? 0 : w[k];
    }
    return w;
}

// The base of a row's exponentials where it saw keys, all of whose scores are
// -infinity: its result is NaN (there is no softmax), but not if a key of another
// part has a finite score.  -infinity: it saw nothing.
constexpr float kSawNothingFinite = -FLT_MAX;

// A row's base is moved only when a score passes it by more than this (a
// probability's rounding to bf16 is relative, and 2^8 times more fits fp32 with
// room), so its sums are rarely rescaled.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ float inverse(float l, float m) { return l != 0.0f ? 1.0f / l : m == -INFINITY ? 0.0f : NAN; }

__device__ __forceinline__ bool any_lane_of_row(bool b)
{
    const uint64_t x = __ballot(b), y = x | x >> 32, z = y | y >> 16;
    return (z >> (threadIdx.x & 15)) & 1;
}

__device__ __forceinline__ void store_result(const PagedParams& p, int e, int h, int row, int d, float inv, f32x4 x)
{
    const int i = row / p.group, hq = h * p.group + row % p.group;
    store4(p.o.p, p.o.at(e, i, hq) + d, p.c.bf16, f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv});
}
// Partial results: the rows' sums [part][D], then base and sum of each.
__device__ __forceinline__ void store_part(const PagedParams& p, int64_t eh, int row, int split, int d, f32x4 x, float m, float l)
{
    const int64_t rows = (int64_t)p.n * p.group, part = (eh * rows + row) * p.splits + split;
    const int64_t parts = (int64_t)p.c.batch * p.c.heads * rows * p.splits;
    *(f32x4*)(p.ws + part * p.c.D + d) = x;
    if (d == 0) {
        p.ws[parts * p.c.D + 2 * part] = m;
        p.ws[parts * p.c.D + 2 * part + 1] = l;
    }
}

// Eight probabilities as the sum of two bf16 parts.  The high one is cut from (1 - 2^-8)
// of a probability, so that the low one, the exact difference, is not 0 either, and an
// infinite value stays an infinity in both products.  It is below 2^-6 of the
// probability, and rounded by 2^-15 of it at most.
struct Parts {
    u32x4 high, low;
};
__device__ __forceinline__ Parts two_parts(f32x4 a, f32x4 b)
{
    Parts p;
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const uint32_t u = __float_as_uint(x[2 * k] * 0.99609375f), v = __float_as_uint(x[2 * k + 1] * 0.99609375f);
        p.high[k] = __builtin_amdgcn_perm(v, u, 0x07060302u);
        p.low[k] = pack2(x[2 * k] - __uint_as_float(u & 0xffff0000u), x[2 * k + 1] - __uint_as_float(v & 0xffff0000u));
    }
    return p;
}

// Up to 16 rows a block.  Each of its four waves takes a tile of keys in turn,
// straight from memory to registers, one tile ahead (the pages two ahead), with its
// own base and sums; the waves meet in LDS at the end.  Values go
// through LDS, for transposed reads.
//
// What bounds it: HBM (one token of eight entries over 65,000 keys of eight bf16
// heads of 128, 2.1 GB: 391 us, 5.5 TB/s; over 30,000 in fp32 358 us, 5.5), with few
// keys the launch and a tile's latency (13 fp32 tokens of three entries over 281 keys
// 10 us), a second launch where keys are split.
template <bool BF16, int D> constexpr int few_blocks() { return D == 64 ? 4 : BF16 ? 3 : 2; }   // on a CU, by registers
template <bool BF16, int D> __global__ __launch_bounds__(256, (few_blocks<BF16, D>())) void attend_few(const PagedParams p)
{
    constexpr int ES = BF16 ? 2 : 4, CE = 16 / ES, NB = BF16 ? 2 : 1, KT = 16 * NB;   // sixteens and keys of a tile
    constexpr int KS = D * ES / 64, DB = D / 16;
    constexpr int VROW = D * ES + (BF16 ? 32 : 16);   // bytes of a value row in LDS: its banks shift from row to row
    constexpr int WAVE_LDS = KT * VROW > 16 * D * 4 + 128 ? KT * VROW : 16 * D * 4 + 128;
    __shared__ __align__(16) unsigned char smem[4 * WAVE_LDS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int regions = p.c.batch * p.c.heads, split = blockIdx.x % p.splits;
    const int eh = blockIdx.x / p.splits % regions, e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p, e);
    const int rows = sp.len * p.group, row0 = 16 * (blockIdx.x / p.splits / regions);
    if (row0 >= rows) return;
    const int last = min(row0 + 15, rows - 1), my_row = min(row0 + r, last);
    const RowSpan mine(p, sp, my_row / p.group), lead(p, sp, row0 / p.group), tail(p, sp, last / p.group);
    const Tiles<KT> tiles(lead, tail);

    u32x4 qf[KS];
    {
        const char* q = (const char*)p.q.p + p.q.at(e, my_row / p.group, h * p.group + my_row % p.group) * ES;
#pragma unroll
        for (int c = 0; c < KS; c++) qf[c] = *(const u32x4_any*)(q + 64 * c + 16 * g);
#pragma unroll
        for (int c = 0; c < KS; c++) arrived(qf[c]);
    }
    const int t_lo = (int)((int64_t)tiles.n * split / p.splits), t_hi = (int)((int64_t)tiles.n * (split + 1) / p.splits);

    f32x4 o[1][DB];
#pragma unroll
    for (int b = 0; b < DB; b++) o[0][b] = f32x4{0, 0, 0, 0};
    float base = 0.0f, limit = -INFINITY, l = 0.0f;   // what a row's scores are taken from (0 before any), and what moves it
    bool saw = false;

    unsigned char* vt = smem + wave * WAVE_LDS;
    u32x4 kn[NB][KS], vn[NB][KS];
    uint32_t page[NB], hole_n = 0;
    const int in_page = (1 << p.c.shift) - 1;
    const bool wide_pages = p.c.shift >= 4;   // sixteen rows lie in one page
    const char *kh = p.c.k + 16 * (uint64_t)h * p.c.kh, *vh = p.c.v + 16 * (uint64_t)h * p.c.vh;
    const uint64_t kl = row_offset(0, 0, r, p.c.kt) + 16 * g, vl = row_offset(0, 0, r, p.c.vt) + 16 * g;
    auto find = [&](int t) {
        const int x = tiles.first(t) + r;
#pragma unroll
        for (int b = 0; b < NB; b++) page[b] = page_of(p.c, e, min(x + 16 * b, tail.hi - 1));
    };
    auto load = [&](int t) {
        hole_n = 0;
#pragma unroll
        for (int b = 0; b < NB; b++) {
            const int x0 = tiles.first(t) + 16 * b;
            const uint32_t one = __builtin_amdgcn_readfirstlane(page[b]);
            if (wide_pages & (one < (uint32_t)p.c.pages) & (x0 + 16 <= tail.hi)) {
                const uint32_t off = x0 & in_page;
                const char *ka = kh + row_offset(one, p.c.kp, off, p.c.kt) + kl, *va = vh + row_offset(one, p.c.vp, off, p.c.vt) + vl;
#pragma unroll
                for (int c = 0; c < KS; c++) {
                    kn[b][c] = *(const u32x4*)(ka + 64 * c);
                    vn[b][c] = *(const u32x4*)(va + 64 * c);
                }
                continue;
            }
            // rows past the last key and holes are zeros
            const bool in = x0 + r < tail.hi, hole = page[b] >= (uint32_t)p.c.pages;
            const uint32_t off = (x0 + r) & in_page;
            hole_n |= (uint32_t)(__ballot(in & hole) & 0xffff) << (16 * b);
            const char *ka = kh + row_offset(page[b], p.c.kp, off, p.c.kt) + 16 * g, *va = vh + row_offset(page[b], p.c.vp, off, p.c.vt) + 16 * g;
#pragma unroll
            for (int c = 0; c < KS; c++) kn[b][c] = vn[b][c] = u32x4{0, 0, 0, 0};
            if (in & !hole) {
#pragma unroll
                for (int c = 0; c < KS; c++) {
                    kn[b][c] = *(const u32x4*)(ka + 64 * c);
                    vn[b][c] = *(const u32x4*)(va + 64 * c);
                }
            }
        }
    };
    int t = t_lo + wave;
    if (t < t_hi) {
        find(t);
        load(t);
        if (t + 4 < t_hi) find(t + 4);
    }
    for (; t < t_hi; t += 4) {
        const int x0 = tiles.first(t);
        const uint32_t hole = hole_n;
        f32x4 s[1][NB];
#pragma unroll
        for (int b = 0; b < NB; b++) {
            s[0][b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < KS; c++) s[0][b] = mma<BF16>(kn[b][c], qf[c], s[0][b]);
#pragma unroll
            for (int c = 0; c < KS; c++) *(u32x4*)(vt + (16 * b + r) * VROW + 64 * c + 16 * g) = vn[b][c];
        }
        if (t + 4 < t_hi) {
            load(t + 4);
            if (t + 8 < t_hi) find(t + 8);
        }
        const bool open = tiles.open(x0, p.sinks) & (hole == 0);
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) s[0][b][i] *= p.scale_log2;
        if (open) {
            saw = true;
        } else {
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int k = 16 * b + 4 * g + i;
                    const bool see = mine.sees(x0 + k) & !((hole >> k) & 1);
                    saw |= see;
                    s[0][b][i] = see ? s[0][b][i] : -INFINITY;
                }
        }
        // (the lanes of a row compare their own keys; they meet only to move its base)
        float top = s[0][0][0];
#pragma unroll
        for (int k = 1; k < 4 * NB; k++) top = fmaxf(top, s[0][k >> 2][k & 3]);
        if (__any(top > limit)) {
            top = max_xor16_32(top);
            const bool move = top > limit;
            const float f = move ? __builtin_amdgcn_exp2f((limit == -INFINITY ? -INFINITY : base) - top) : 1.0f;
            if (move) {
                limit = top + kSlack;
                base = top;
            }
            l *= f;
#pragma unroll
            for (int b = 0; b < DB; b++)
#pragma unroll
                for (int i = 0; i < 4; i++) o[0][b][i] *= f;
        }
#pragma unroll
        for (int b = 0; b < NB; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                s[0][b][i] = __builtin_amdgcn_exp2f(s[0][b][i] - base);
                l += s[0][b][i];   // this lane's keys; the lanes of a query are summed at the end
            }
        // (the wave's own region: its LDS operations complete in order)
        __builtin_amdgcn_wave_barrier();
        if (!open) {
            bool special = false;
            auto where = [&](int c) {
                const int key = 16 * (c / KS) + r, at = 64 * (c % KS) + 16 * g;
                return ChunkAt{vt + key * VROW + at, key, at / ES};
            };
#pragma unroll
            for (int c = 0; c < NB * KS; c++) special |= special_of<BF16>(*(const u32x4*)where(c).p) != 0;
            if (__builtin_expect(__any(special), 0)) {
                add_special<BF16>(NB * KS, where, [&](int, int k) { return mine.sees(x0 + k) & !((hole >> k) & 1); }, s, o);
#pragma unroll
                for (int c = 0; c < NB * KS; c++) *(u32x4*)where(c).p = clear_special<BF16>(*(const u32x4*)where(c).p);
                __builtin_amdgcn_wave_barrier();
            }
        }
        if constexpr (BF16) {
            const Parts pf = two_parts(s[0][0], s[0][1]);
#pragma unroll
            for (int b = 0; b < DB; b++) {
                const unsigned char* a = vt + (4 * g + (r >> 2)) * VROW + 32 * b + 8 * (r & 3);
                const u32x4 v = read_tr(a, a + 16 * VROW);
                o[0][b] = mma<true>(v, pf.low, o[0][b]);
                o[0][b] = mma<true>(v, pf.high, o[0][b]);
            }
        } else {
#pragma unroll
            for (int b = 0; b < DB; b++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    o[0][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(*(const float*)(vt + (4 * g + i) * VROW + 64 * b + 4 * r), s[0][0][i], o[0][b], 0, 0, 0);
        }
        __builtin_amdgcn_wave_barrier();
    }
    l = sum_xor32(sum_xor16(l));
    const float m = limit != -INFINITY ? base : any_lane_of_row(saw) ? kSawNothingFinite : -INFINITY;

    __syncthreads();
    float* mine_o = (float*)vt;                       // [16 queries][D], then m, l [16]
#pragma unroll
    for (int b = 0; b < DB; b++) *(f32x4*)(mine_o + r * D + 16 * b + 4 * g) = o[0][b];
    if (g == 0) {
        mine_o[16 * D + r] = m;
        mine_o[16 * D + 16 + r] = l;
    }
    __syncthreads();
    constexpr int CH = D / 4;                         // four dimensions a thread
    for (int u = threadIdx.x; u < 16 * CH; u += 256) {
        const int q = u / CH, d = 4 * (u % CH);
        if (row0 + q > last) continue;
        float mx = -INFINITY, sum = 0.0f;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; w++) mx = fmaxf(mx, ((const float*)(smem + w * WAVE_LDS))[16 * D + q]);
        const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float* src = (const float*)(smem + w * WAVE_LDS);
            const float f = __builtin_amdgcn_exp2f(src[16 * D + q] - base);
            sum += src[16 * D + 16 + q] * f;
            const f32x4 y = *(const f32x4*)(src + q * D + d);
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] += y[i] * f;
        }
        if (p.splits == 1) store_result(p, e, h, row0 + q, d, inverse(sum, mx), x);
        else store_part(p, eh, row0 + q, split, d, x, mx, sum);
    }
}

// Many rows: a block of four waves works on 64 QG rows, each wave on its own 16 QG.
// Tiles of keys and values go from memory to LDS directly, through two buffers, the
// next one on its way while this one is worked on (the pages two ahead); 16-byte
// chunks are stored with their index XORed with bits of the row, so that the rows
// of an operand read lie in different banks.  In bf16 the probabilities' sum is one
// more row of the second product.
//
// What bounds it: the products, the exponentials and the maxima between them, about
// equal (4,096 tokens of two entries over 6,000 others, 16 heads of 128 and four key
// heads: 527 and 557 us on two cards, 1,025 and 970 TFLOP/s; 8,192 tokens of 16 heads of
// 64 169 and 176, 815 and 780, with twice the exponentials a product and the sums' row a
// fifth of the second product); in fp32 its own products (two entries of 1,024 tokens
// over 2,000 others 384 us, 110 TFLOP/s of 157).
template <bool BF16, int D, int QG> __global__ __launch_bounds__(256, 2) void attend_many(const PagedParams p)
{
    constexpr int ES = BF16 ? 2 : 4, NB = BF16 ? 4 : 2, KT = 16 * NB, KS = D * ES / 64, DB = D / 16, RB = 64 * QG;
    constexpr int ROW = D * ES, CPR = ROW / 16, LOADS = KT * CPR / 256;   // bytes, chunks of a row; a thread's of a tile
    constexpr int TILE = KT * ROW;
    __shared__ __align__(16) unsigned char smem[4 * TILE];                // [buffer][keys, values]
    __shared__ __align__(4) uint8_t holes[2][KT];
    __shared__ int hole_any[2][4], special_any[4];
    __device__ static const u32x4 zeros = {0, 0, 0, 0};

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int regions = p.c.batch * p.c.heads, split = blockIdx.x % p.splits;
    const int eh = blockIdx.x / p.splits % regions, e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p, e);
    // (the last rows, which see the most keys, first)
    const int blocks = (p.n * p.group + RB - 1) / RB;
    const int rows = sp.len * p.group, row0 = RB * (blocks - 1 - (int)(blockIdx.x / p.splits / regions));
    if (row0 >= rows) return;
    const int last = min(row0 + RB - 1, rows - 1);
    const RowSpan lead(p, sp, row0 / p.group), tail(p, sp, last / p.group);
    const Tiles<KT> tiles(lead, tail);

    RowSpan mine[QG];
    u32x4 qf[QG][KS];
#pragma unroll
    for (int u = 0; u < QG; u++) {
        const int row = min(row0 + 16 * (QG * wave + u) + r, last), i = row / p.group;
        mine[u] = RowSpan(p, sp, i);
        const char* q = (const char*)p.q.p + p.q.at(e, i, h * p.group + row % p.group) * ES;
#pragma unroll
        for (int c = 0; c < KS; c++) qf[u][c] = *(const u32x4_any*)(q + 64 * c + 16 * g);
    }
#pragma unroll
    for (int u = 0; u < QG; u++)
#pragma unroll
        for (int c = 0; c < KS; c++) arrived(qf[u][c]);
    const int t_lo = (int)((int64_t)tiles.n * split / p.splits), t_hi = (int)((int64_t)tiles.n * (split + 1) / p.splits);

    // which chunk of a row lies in place c of it (and the other way round)
    auto swz_k = [](int row) { return CPR == 8 ? (row >> 1) & 7 : row & 15; };
    auto swz_v = [](int row) { return !BF16 ? ((row >> 2) & 3) << 2 : D == 64 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; };
    // an instruction of a wave loads WR consecutive rows; their place, if they lie in one page, is uniform
    constexpr int WR = 64 / CPR;
    const bool wide_pages = ((1 << p.c.shift) >= WR) & (p.c.kt < 1u << 24) & (p.c.vt < 1u << 24);
    const bool one_page = wide_pages & ((1 << p.c.shift) >= KT);
    const int in_page = (1 << p.c.shift) - 1;
    const char *kh = p.c.k + 16 * (uint64_t)h * p.c.kh, *vh = p.c.v + 16 * (uint64_t)h * p.c.vh;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem) + wave * 1024);
    uint32_t page[LOADS];
    auto find = [&](int t) {
        const int x = tiles.first(t) + tid / CPR;
#pragma unroll
        for (int c = 0; c < LOADS; c++) page[c] = page_of(p.c, e, min(x + c * (256 / CPR), tail.hi - 1));
    };
    // tile t into buffer `buf`
    auto load = [&](int t, int buf) {
        const int x0 = tiles.first(t);
        const uint32_t to = lds0 + buf * 2 * TILE;
        const uint32_t page0 = __builtin_amdgcn_readfirstlane(page[0]);
        if (one_page & (page0 < (uint32_t)p.c.pages) & (x0 + KT <= tail.hi)) {   // the usual tile: whole, of one page
            const int w0 = wave * WR, in = lane / CPR;
            const uint32_t off = (x0 & in_page) + w0;
            const char *kb = kh + row_offset(page0, p.c.kp, off, p.c.kt), *vb = vh + row_offset(page0, p.c.vp, off, p.c.vt);
#pragma unroll
            for (int c = 0; c < LOADS; c++) {
                const int row = tid / CPR + c * (256 / CPR);
                dma16(kb, 16 * in * p.c.kt + 16 * (tid % CPR ^ swz_k(row)), to + c * 4096);
                dma16(vb, 16 * in * p.c.vt + 16 * (tid % CPR ^ swz_v(row)), to + TILE + c * 4096);
                kb += (uint64_t)p.c.kt * (16 * (256 / CPR));
                vb += (uint64_t)p.c.vt * (16 * (256 / CPR));
            }
            if (tid < 4) hole_any[buf][tid] = 0;
            return;
        }
        bool any = false;
#pragma unroll
        for (int c = 0; c < LOADS; c++) {
            const int row = tid / CPR + c * (256 / CPR), w0 = wave * WR + c * (256 / CPR), in = lane / CPR;
            const uint32_t ck = 16 * (tid % CPR ^ swz_k(row)), cv = 16 * (tid % CPR ^ swz_v(row));
            const uint32_t one = __builtin_amdgcn_readfirstlane(page[c]);
            if (wide_pages & (one < (uint32_t)p.c.pages) & (x0 + w0 + WR <= tail.hi)) {
                const uint32_t off = (x0 + w0) & in_page;
                dma16(kh + row_offset(one, p.c.kp, off, p.c.kt), 16 * in * p.c.kt + ck, to + c * 4096);
                dma16(vh + row_offset(one, p.c.vp, off, p.c.vt), 16 * in * p.c.vt + cv, to + TILE + c * 4096);
                if (lane < WR) holes[buf][w0 + lane] = 0;
            } else {   // rows past the last key and holes are zeros
                const bool on = x0 + row < tail.hi, hole = page[c] >= (uint32_t)p.c.pages;
                const uint32_t off = (x0 + row) & in_page;
                any |= on & hole;
                if (lane % CPR == 0) holes[buf][row] = on & hole;
                const bool there = on & !hole;
                dma16(there ? kh + row_offset(page[c], p.c.kp, off, p.c.kt) + ck : (const char*)&zeros, to + c * 4096);
                dma16(there ? vh + row_offset(page[c], p.c.vp, off, p.c.vt) + cv : (const char*)&zeros, to + TILE + c * 4096);
            }
        }
        hole_any[buf][wave] = __any(any);
    };

    f32x4 o[QG][DB], ls[QG];   // ls: the probabilities' sums (bf16: every row the whole sum; fp32: [0], this lane's keys)
    float base[QG], limit[QG];   // of a row: what its scores are taken from (0 before any), and what moves it
    bool saw[QG];
#pragma unroll
    for (int u = 0; u < QG; u++) {
#pragma unroll
        for (int b = 0; b < DB; b++) o[u][b] = f32x4{0, 0, 0, 0};
        ls[u] = f32x4{0, 0, 0, 0};
        base[u] = 0.0f;
        limit[u] = -INFINITY;
        saw[u] = false;
    }
    const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};

    const bool rows_left = row0 + 16 * QG * wave <= last;
    // where this lane's operands lie in a buffer
    uint32_t ka[KS], va[DB];
#pragma unroll
    for (int c = 0; c < KS; c++) ka[c] = r * ROW + 16 * ((4 * c + g) ^ swz_k(r));
#pragma unroll
    for (int b = 0; b < DB; b++) {
        const int row = 4 * g + (r >> 2);   // (bf16; fp32: of the first of four rows that have the same places)
        va[b] = BF16 ? row * ROW + 16 * ((2 * b) ^ swz_v(row)) + 8 * (r & 3) : 4 * g * ROW + 16 * ((4 * b) ^ swz_v(4 * g)) + 4 * r;
    }
    auto step = [&](int t, auto which) {
        constexpr int buf = decltype(which)::value;
        dma_wait();        // this tile is in LDS
        __syncthreads();   // for every wave, and the one before has been read
        if (t + 1 < t_hi) {
            load(t + 1, 1 - buf);
            if (t + 2 < t_hi) find(t + 2);
        }
        unsigned char *kt = smem + buf * 2 * TILE, *vt = kt + TILE;
        const int x0 = tiles.first(t);
        const bool any_hole = hole_any[buf][0] | hole_any[buf][1] | hole_any[buf][2] | hole_any[buf][3];
        // (a scale that turns the scores' order around takes the masking path too)
        const bool open = tiles.open(x0, p.sinks) & !any_hole & (p.scale_log2 > 0.0f);

        // scores: the next keys' operands are read while these are multiplied
        bool special = false;
        auto where = [&](int c) {
            const int at = 1024 * c + 16 * lane, key = at / ROW;
            return ChunkAt{vt + at, key, ((at % ROW / 16) ^ swz_v(key)) * (16 / ES)};
        };
        if (!open) {
            for (int c = wave; c < TILE / 1024; c += 4) special |= special_of<BF16>(*(const u32x4*)where(c).p) != 0;
            special_any[wave] = __any(special);
            __syncthreads();
            special = special_any[0] | special_any[1] | special_any[2] | special_any[3];
        }
        if (!rows_left & !special) return;
        f32x4 s[QG][NB];
        u32x4 kf[2][KS];
        auto read_k = [&](int b) {
#pragma unroll
            for (int c = 0; c < KS; c++) kf[b & 1][c] = *(const u32x4*)(kt + 16 * b * ROW + ka[c]);
        };
        read_k(0);
#pragma unroll
        for (int b = 0; b < NB; b++) {
            if (b + 1 < NB) read_k(b + 1);
#pragma unroll
            for (int u = 0; u < QG; u++) s[u][b] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < KS; c++)
#pragma unroll
                for (int u = 0; u < QG; u++) s[u][b] = mma<BF16>(kf[b & 1][c], qf[u][c], s[u][b]);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the first values' operands, read while the probabilities are computed
        constexpr int VB = 4;
        u32x4 vf[2][VB];
        auto read_v = [&](int half, int b0) {
#pragma unroll
            for (int b = 0; b < VB; b++) {
                const unsigned char* a = vt + 32 * half * ROW + va[b0 + b];
                vf[(half * DB + b0) / VB & 1][b] = read_tr(a, a + 16 * ROW);
            }
        };
        if constexpr (BF16) read_v(0, 0);
        const float mul = open ? p.scale_log2 : 1.0f;
#pragma unroll
        for (int u = 0; u < QG; u++) {
            // (masked scores are scaled before their mask: 0 times an infinity is NaN)
            if (!open) {
#pragma unroll
                for (int b = 0; b < NB; b++) {
                    const uint32_t hole = any_hole ? *(const uint32_t*)(holes[buf] + 16 * b + 4 * g) : 0;   // of four keys, a byte each
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const bool see = mine[u].sees(x0 + 16 * b + 4 * g + i) & !((hole >> (8 * i)) & 1);
                        saw[u] |= see;
                        s[u][b][i] = see ? s[u][b][i] * p.scale_log2 : -INFINITY;
                    }
                }
            } else {
                saw[u] = true;
            }
            // (the lanes of a row compare their own keys; they meet only to move its base)
            float top = s[u][0][0];
#pragma unroll
            for (int k = 1; k < 4 * NB; k++) top = fmaxf(top, s[u][k >> 2][k & 3]);
            if (__any(top * mul > limit[u])) {
                top = max_xor16_32(top) * mul;
                const bool move = top > limit[u];
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
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int i = 0; i < 4; i++) s[u][b][i] = __builtin_amdgcn_exp2f(fmaf(s[u][b][i], mul, -base[u]));
        }
        if (__builtin_expect(special, 0)) {   // (a rule on the tile: the block's waves meet here)
            if (rows_left)
                add_special<BF16>(TILE / 1024, where, [&](int u, int k) { return mine[u].sees(x0 + k) & !(any_hole && holes[buf][k]); }, s, o);
            __syncthreads();
            for (int c = wave; c < TILE / 1024; c += 4) *(u32x4*)where(c).p = clear_special<BF16>(*(const u32x4*)where(c).p);
            __syncthreads();
            if constexpr (BF16) read_v(0, 0);
        }
        if (!rows_left) return;
        if constexpr (BF16) {
#pragma unroll
            for (int half = 0; half < 2; half++) {
                u32x4 pf[QG];
#pragma unroll
                for (int u = 0; u < QG; u++) {
                    const f32x4 a = s[u][2 * half], b = s[u][2 * half + 1];
                    pf[u] = u32x4{pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]), pack2(b[2], b[3])};
                }
#pragma unroll
                for (int b0 = 0; b0 < DB; b0 += VB) {
                    if (b0 + VB < DB) read_v(half, b0 + VB);
                    else if (half == 0) read_v(1, 0);
#pragma unroll
                    for (int b = 0; b < VB; b++)
#pragma unroll
                        for (int u = 0; u < QG; u++) o[u][b0 + b] = mma<true>(vf[(half * DB + b0) / VB & 1][b], pf[u], o[u][b0 + b]);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int u = 0; u < QG; u++) ls[u] = mma<true>(ones, pf[u], ls[u]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < QG; u++)
#pragma unroll
                for (int k = 0; k < 4 * NB; k++) ls[u][0] += s[u][k >> 2][k & 3];
#pragma unroll
            for (int k = 0; k < NB; k++)
#pragma unroll
                for (int b = 0; b < DB; b++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float x = *(const float*)(vt + (16 * k + i) * ROW + va[b]);
#pragma unroll
                        for (int u = 0; u < QG; u++) o[u][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s[u][k][i], o[u][b], 0, 0, 0);
                    }
        }
    };
    if (t_lo < t_hi) {
        find(t_lo);
        load(t_lo, 0);
        if (t_lo + 1 < t_hi) find(t_lo + 1);
    }
    for (int t = t_lo; t < t_hi; t += 2) {   // (the buffers' places are constants of the code)
        step(t, std::integral_constant<int, 0>{});
        if (t + 1 < t_hi) step(t + 1, std::integral_constant<int, 1>{});
    }
#pragma unroll
    for (int u = 0; u < QG; u++) {
        const float l = BF16 ? ls[u][0] : sum_xor32(sum_xor16(ls[u][0]));
        const float m = limit[u] != -INFINITY ? base[u] : any_lane_of_row(saw[u]) ? kSawNothingFinite : -INFINITY;
        const int row = row0 + 16 * (QG * wave + u) + r;
        if (row > last) continue;
        const float inv = inverse(l, m);
#pragma unroll
        for (int b = 0; b < DB; b++) {
            const int d = 16 * b + 4 * g;
            if (p.splits > 1) store_part(p, eh, row, split, d, o[u][b], m, l);
            else store_result(p, e, h, row, d, inv, o[u][b]);
        }
    }
}

// Joins the splits of a row: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// NG groups of D / 4 threads share a row's splits, each with its own running
// maximum, and meet in LDS.  Its parts come from L2 as a rule: the launch bounds it (3 us).
template <int D, int NG> __global__ __launch_bounds__(256) void join_kernel(const PagedParams p)
{
    constexpr int CH = D / 4, ROWS = 256 / (CH * NG);   // rows of a block
    __shared__ __align__(16) float sm[NG > 1 ? ROWS * NG * (D + 2) : 1];
    const int rows = p.n * p.group;
    const int64_t regions = (int64_t)p.c.batch * p.c.heads;
    const int ch = threadIdx.x % CH, grp = threadIdx.x / CH % NG, local = threadIdx.x / (CH * NG), d = 4 * ch;
    const int64_t id = (int64_t)blockIdx.x * ROWS + local;
    const bool in = id < regions * rows;
    const int64_t at_id = in ? id : 0;
    const int eh = (int)(at_id / rows), row = (int)(at_id % rows), e = eh / p.c.heads, h = eh % p.c.heads;
    const Span sp(p, e);
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
    if (on) store_result(p, e, h, row, d, inverse(l, m), o);
}

// ------------------------------------------------------------------ launch

template <bool BF16, int D> hipError_t launch_attend_d(const PagedParams& p, const PagedPlan& plan, hipStream_t st)
{
    const int64_t rows = (int64_t)p.n * p.group, regions = (int64_t)p.c.batch * p.c.heads;
    const int64_t blocks = p.splits * regions * ((rows + plan.rows - 1) / plan.rows);
    hipError_t e = hipErrorInvalidValue;
    if (plan.rows == 16) e = launch_with(attend_few<BF16, D>, blocks, 256, 0, st, p);
    else if (plan.rows == 64) e = launch_with(attend_many<BF16, D, 1>, blocks, 256, 0, st, p);
    else if constexpr (BF16) e = launch_with(attend_many<BF16, D, 2>, blocks, 256, 0, st, p);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t all = regions * rows;
    constexpr int per = 256 / (D / 4);   // rows of a block, or groups of one row
    if (p.splits <= 4 || all >= 2048) return launch_with(join_kernel<D, 1>, (all + per - 1) / per, 256, 0, st, p);
    return launch_with(join_kernel<D, per>, all, 256, 0, st, p);
}

hipError_t launch_attend(const PagedParams& p, const PagedPlan& plan, hipStream_t st)
{
    if (p.c.D == 64) return p.c.bf16 ? launch_attend_d<true, 64>(p, plan, st) : launch_attend_d<false, 64>(p, plan, st);
    return p.c.bf16 ? launch_attend_d<true, 128>(p, plan, st) : launch_attend_d<false, 128>(p, plan, st);
}

}  // namespace dcb
