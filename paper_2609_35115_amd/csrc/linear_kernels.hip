// gfx950 kernels of the matrix product with an epilogue:
//   out = residual_scale residual + gate act(x W^T + bias).
#include <algorithm>
#include <type_traits>

#include "block_internal.h"
#include "dc_flow.h"
#include "linear_plan.h"

namespace dcb {

// Both operands' rows run along K, and both go to the matrix cores in chunks of
// 16 bytes: a group of four consecutive chunks of a row (64 bytes) is what the
// four lane groups of an operand hold, one each.  In bf16 that is one
// 16x16x32 product, in fp32 four 16x16x4 ones, the t-th of element t of every
// lane's chunk (a sum's terms in another order).  The weight is the first
// operand: a lane's four results are four consecutive columns of one row.
constexpr int kChunks = 8;   // chunks of a row that one K step takes (128 bytes)

template <bool BF16> constexpr int chunk_elems() { return BF16 ? 8 : 4; }

template <bool BF16> __device__ __forceinline__ f32x4 mma(u32x4 w, u32x4 x, f32x4 acc)
{
    if constexpr (BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int t = 0; t < 4; t++) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[t]), __uint_as_float(x[t]), acc, 0, 0, 0);
        return acc;
    }
}

// A chunk at element k of a row of K, zeros past the row's end.
template <bool BF16> __device__ __forceinline__ u32x4 load_chunk(const void* row, int k, int K)
{
    constexpr int CE = chunk_elems<BF16>();
    if (k + CE <= K) return *(const u32x4_any*)((const char*)row + (int64_t)k * (16 / CE));
    u32x4 c = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < CE - 1; j++) {
        if (k + j >= K) break;
        if constexpr (BF16) c[j >> 1] |= (uint32_t)((const uint16_t*)row)[k + j] << (16 * (j & 1));
        else c[j] = ((const uint32_t*)row)[k + j];
    }
    return c;
}

// Chunks at element k of several rows, `whole` (uniform) where none passes its row's end.
template <bool BF16, int N> __device__ __forceinline__ void load_chunks(const char* const (&row)[N], int k, int K, bool whole, u32x4 (&to)[N])
{
    if (whole) {
#pragma unroll
        for (int c = 0; c < N; c++) to[c] = *(const u32x4_any*)(row[c] + (int64_t)k * (BF16 ? 2 : 4));
    } else {
#pragma unroll
        for (int c = 0; c < N; c++) to[c] = load_chunk<BF16>(row[c], k, K);
    }
}

// GELU in its tanh form, 0.5 v (1 + tanh z) = v / (1 + e^-2z): no cancellation for
// negative v.
template <bool EXACT> __device__ __forceinline__ float activate(float v, int act)
{
    if (act == DC_ACT_NONE) return v;
    const float k2 = -2.0f * 0.7978845608028654f * 1.4426950408889634f;   // -2 sqrt(2 / pi) log2(e)
    const float z = act == DC_ACT_GELU ? v * (k2 + k2 * 0.044715f * (v * v)) : v * -1.4426950408889634f;
    const float d = 1.0f + __builtin_amdgcn_exp2f(z);
    return EXACT ? v / d : v * __builtin_amdgcn_rcpf(d);   // 1 ulp, of a result that is rounded to bf16 next
}

// Token i of entry e that row m of the call is; i < 0 where the call does not have it.
struct Place {
    int e, i;
    __device__ __forceinline__ bool on() const { return i >= 0; }
};
__device__ __forceinline__ Place place_of(const LinearParams& p, int m)
{
    const int e = min(m, p.M - 1) / p.call.n, i = m - e * p.call.n;
    return Place{e, m < p.M && i < p.call.len(e) ? i : -1};
}

// Columns n .. n + 7 of a row, from the sums a (and b, the factor's, with glu),
// biases ba, bb.
struct Eight {
    float v[8];
};
__device__ __forceinline__ Eight load8(const void* p, int64_t at, int bf16)
{
    const f32x4 a = load4(p, at, bf16), b = load4(p, at + 4, bf16);
    return Eight{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ Eight load_bias(const LinearParams& p, int n, int part)
{
    Eight x{};
    if (p.bias && n + 8 <= p.N) {
        x = load8(p.bias, (int64_t)part * p.N + n, 0);
    } else if (p.bias) {
#pragma unroll
        for (int k = 0; k < 7; k++)
            if (n + k < p.N) x.v[k] = p.bias[(int64_t)part * p.N + n + k];
    }
    return x;
}
__device__ __forceinline__ void epilogue(const LinearParams& p, const Place& at, int n, Eight a, Eight b, const Eight& ba, const Eight& bb)
{
    if (!at.on() || n >= p.N) return;
    auto row = [&](const Rows& x) { return at.e * x.sb + at.i * x.st + n; };
    const int64_t o = row(p.out);
    const bool full = n + 8 <= p.N;
#pragma unroll
    for (int k = 0; k < 8; k++) a.v[k] += ba.v[k];
    if (p.act) {
        if (p.out.bf16) {
#pragma unroll
            for (int k = 0; k < 8; k++) a.v[k] = activate<false>(a.v[k], p.act);
        } else {
#pragma unroll
            for (int k = 0; k < 8; k++) a.v[k] = activate<true>(a.v[k], p.act);
        }
    }
    if (p.glu) {
#pragma unroll
        for (int k = 0; k < 8; k++) a.v[k] *= b.v[k] + bb.v[k];
    }
    if (full) {
        if (p.gate.p) {
            const Eight x = load8(p.gate.p, row(p.gate), p.gate.bf16);
#pragma unroll
            for (int k = 0; k < 8; k++) a.v[k] *= x.v[k];
        }
        if (p.res.p) {
            const Eight x = load8(p.res.p, row(p.res), p.res.bf16);
#pragma unroll
            for (int k = 0; k < 8; k++) a.v[k] = fmaf(p.res_scale, x.v[k], a.v[k]);
        }
        if (p.out.bf16) store8<true>(p.out.p, o, a.v);
        else store8<false>(p.out.p, o, a.v);
        return;
    }
#pragma unroll
    for (int k = 0; k < 7; k++) {
        if (n + k >= p.N) break;
        float v = a.v[k];
        if (p.gate.p) v *= load1(p.gate.p, row(p.gate) + k, p.gate.bf16);
        if (p.res.p) v = fmaf(p.res_scale, load1(p.res.p, row(p.res) + k, p.res.bf16), v);
        store1(p.out.p, o + k, p.out.bf16, v);
    }
}

// What a wave does with its `rows` rows of sums in LDS (`pitch` floats apart, with
// glu the factors COLS / 2 floats behind; `places` are the rows', m0 on): the
// epilogue, or a split's partial sums ([split][M][part_row]), eight columns a lane
// and whole rows side by side.
template <int COLS>
__device__ __forceinline__ void finish(const LinearParams& p, const Place* places, const float* sums, int rows, int pitch, int m0, int n0, int split)
{
    const int lane = threadIdx.x & 63;
    const int per = p.glu ? COLS / 16 : COLS / 8;             // lanes of a row
    const int q = lane & (per - 1), n = n0 + 8 * q;
    const Eight ba = load_bias(p, n, 0), bb = p.glu ? load_bias(p, n, 1) : Eight{};
#pragma unroll 2
    for (int r = lane / per; r < rows; r += 64 / per) {
        const float* s = sums + r * pitch + 8 * q;
        auto eight = [](const float* s) {
            const f32x4 x = *(const f32x4*)s, y = *(const f32x4*)(s + 4);
            return Eight{{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]}};
        };
        const Eight a = eight(s), b = eight(s + (p.glu ? COLS / 2 : 0));
        if (p.splits > 1) {
            if (m0 + r >= p.M || n >= p.N) continue;
            float* to = p.ws + ((int64_t)split * p.M + m0 + r) * part_row(p.N, p.glu) + n;
            *(f32x4*)to = f32x4{a.v[0], a.v[1], a.v[2], a.v[3]};
            *(f32x4*)(to + 4) = f32x4{a.v[4], a.v[5], a.v[6], a.v[7]};
            if (p.glu) {
                to += part_half(p.N);
                *(f32x4*)to = f32x4{b.v[0], b.v[1], b.v[2], b.v[3]};
                *(f32x4*)(to + 4) = f32x4{b.v[4], b.v[5], b.v[6], b.v[7]};
            }
        } else {
            epilogue(p, places[r], n, a, b, ba, bb);
        }
    }
}

// ----------------------------------------------------------- tiles of rows
//
// A block computes BM rows by BN columns (with glu BN / 2 columns and their
// factors), its WM x WN waves a part each.

// Which tile and split a block has.  Blocks are dealt to the eight XCDs in turn: each
// takes a run of the tiles, in strips of eight row tiles, whose operands its L2
// holds.
template <int BM, int BN> struct TileAt {
    int m0, n0, split;
    __device__ __forceinline__ TileAt(const LinearParams& p)
    {
        const int BC = p.glu ? BN / 2 : BN;   // columns of a block
        const int mt = (p.M + BM - 1) / BM, nt = (p.N + BC - 1) / BC;
        const int64_t eighth = (int64_t)mt * nt * p.splits / 8;
        int64_t id = blockIdx.x;
        if (id < eighth * 8) id = id % 8 * eighth + id / 8;
        split = (int)(id % p.splits);
        const int tile = (int)(id / p.splits), strip = tile / (8 * nt), in = tile - strip * 8 * nt;
        const int high = min(8, mt - 8 * strip);
        m0 = (8 * strip + in % high) * BM;
        n0 = in / high * BC;
    }
};

// The weight's row that is row r of a block's BN, columns past N from its last row.
template <int BN, int WN, int ES> __device__ __forceinline__ const char* weight_row(const LinearParams& p, int n0, int r)
{
    constexpr int NI = BN / WN / 16;
    int col, part = 0;
    if (p.glu) {   // a wave's first half of 16-column groups, and the same columns' factors
        const int w = r / (BN / WN), f = r / 16 % NI;
        part = f >= NI / 2;
        col = n0 + w * (BN / WN / 2) + (f - part * (NI / 2)) * 16 + r % 16;
    } else {
        col = n0 + r;
    }
    return (const char*)p.w + ((int64_t)part * p.N + min(col, p.N - 1)) * p.wstride * ES;
}

// The operands' rows that a thread loads: its chunk of rows tid / 8 + c T / 8, first
// the BM rows of x, then those of the weight.  Rows that the call does not have are
// read from the weight instead and columns past N from its last row: their results
// are not stored.  `places` becomes the rows' places (every thread calls).  Whether
// any of this thread's is a row of x that the call has.
template <int BM, int BN, int WN, int T, int ES, int LOADS>
__device__ __forceinline__ bool operand_rows(const LinearParams& p, const TileAt<BM, BN>& at, Place (&places)[BM], const char* (&row)[LOADS])
{
    for (int m = threadIdx.x; m < BM; m += T) places[m] = place_of(p, at.m0 + m);
    __syncthreads();
    bool any = false;
#pragma unroll
    for (int c = 0; c < LOADS; c++) {
        const int rr = threadIdx.x / kChunks + c * (T / kChunks);
        if (rr < BM) {
            const Place x = places[rr];
            any |= x.on();
            row[c] = x.on() ? (const char*)p.x.p + (x.e * p.x.sb + x.i * p.x.st) * ES : (const char*)p.w;
        } else {
            row[c] = weight_row<BN, WN, ES>(p, at.n0, rr - BM);
        }
    }
    return any;
}

// The sums of a wave's rows (m0 on) and columns (n0 on) go through LDS, up to 64 rows
// at a time, so that a row's columns are stored side by side.
template <int MI, int NI> constexpr int out_rows() { return MI < 4 ? 16 * MI : 64; }
template <int MI, int NI> constexpr int out_bytes() { return out_rows<MI, NI>() * (16 * NI + 4) * 4; }
template <int MI, int NI>
__device__ __forceinline__ void write_out(const LinearParams& p, const Place* places, float* mine, const f32x4 (&acc)[MI][NI], int m0, int n0, int split)
{
    constexpr int SR = out_rows<MI, NI>(), PITCH = 16 * NI + 4;
    const int l16 = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
#pragma unroll
    for (int c = 0; c < MI; c += SR / 16) {
#pragma unroll
        for (int i = 0; i < SR / 16; i++)
#pragma unroll
            for (int j = 0; j < NI; j++) *(f32x4*)(mine + (16 * i + l16) * PITCH + 16 * j + 4 * g) = acc[c + i][j];
        // (the wave's own region: its LDS operations complete in order)
        __builtin_amdgcn_wave_barrier();
        finish<16 * NI>(p, places + 16 * c, mine, SR, PITCH, m0 + 16 * c, n0, split);
        __builtin_amdgcn_wave_barrier();
    }
}

template <int N> __device__ __forceinline__ void dma_wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Both operands' K steps go through a ring of ST LDS buffers, the next ones on
// their way while one is multiplied; a row's eight chunks are stored with their index
// XORed with the row's low bits, so that the sixteen rows of an operand read lie in
// different banks.  With WIDE the loads go from memory to LDS directly, else (rows
// or K not of whole chunks) through registers, by eight waves (14,336 x 514 -> 2,047 65 us,
// four 74; 3,000 x 3,001 -> 3,000 120 and 127).
//
// What bounds it, in bf16: large products, the matrix cores and the loads' way from L2
// to LDS together (256 x 256: 8,192^3 812 and 866 us on two cards, 1,350 and 1,270
// TFLOP/s; 4,096^3 106 and 114, of which 0.81 are left without the loads and 0.99
// without the products); smaller tiles, that way alone (64 x 64 tiles of
// 4,096^3 ask for 19 TB/s, and take as long without the products); one block a CU, the
// loads' latency, so that four waves and two steps took 64 us for 512 x 4,096 -> 8,192,
// eight and four 44 (28 without the loads).
template <bool BF16, int BM, int BN, int WM, int WN, bool WIDE, int ST>
__global__ __launch_bounds__(64 * WM * WN, 2) void tile_kernel(const LinearParams p)
{
    constexpr int T = 64 * WM * WN, MI = BM / WM / 16, NI = BN / WN / 16, CE = chunk_elems<BF16>(), ES = 16 / CE;
    constexpr int KT = kChunks * CE, ROWS = BM + BN, LOADS = ROWS * kChunks / T;
    constexpr int BUF = ROWS * kChunks * 16;
    constexpr int OUT = WM * WN * out_bytes<MI, NI>(), LDS = ST * BUF > OUT ? ST * BUF : OUT;
    static_assert(ROWS * kChunks % T == 0 && T / kChunks % 8 == 0 && (WIDE || ST == 2) && NI % 2 == 0);   // (pairs: glu)
    __shared__ __align__(16) unsigned char smem[LDS];
    __shared__ int some;
    __shared__ Place places[BM];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4, wm = wave % WM, wn = wave / WM;
    const TileAt<BM, BN> at(p);
    if (tid == 0) some = 0;
    const char* row[LOADS];
    if (operand_rows<BM, BN, WN, T, ES>(p, at, places, row)) some = 1;
    __syncthreads();
    if (!some) return;   // all rows are behind their entries' last tokens

    const int kc = ((tid % kChunks) ^ (tid / kChunks & 7)) * CE;   // where in the K step this thread's chunk lies
    const int steps = (p.K + KT - 1) / KT;
    const int s0 = (int)((int64_t)steps * at.split / p.splits), s1 = (int)((int64_t)steps * (at.split + 1) / p.splits);

    u32x4 stage[LOADS];   // (not WIDE)
    __device__ static const u32x4 zeros = {0, 0, 0, 0};
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem) + wave * 1024);
    auto fetch = [&](int s, int slot) {
        const int k = s * KT + kc;
        if constexpr (WIDE) {
#pragma unroll
            for (int c = 0; c < LOADS; c++)
                dma16(k < p.K ? row[c] + (int64_t)k * ES : (const char*)&zeros, lds0 + slot * BUF + c * (T * 16));
        } else {
            load_chunks<BF16>(row, k, p.K, (s + 1) * KT <= p.K, stage);
        }
    };
    auto keep = [&](int slot) {
        if constexpr (!WIDE) {
#pragma unroll
            for (int c = 0; c < LOADS; c++) *(u32x4*)(smem + slot * BUF + (c * T + tid) * 16) = stage[c];
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = f32x4{0, 0, 0, 0};

    // operands of a half step (four chunks)
    struct Half {
        u32x4 x[MI], w[NI];
    } even, odd;
    const unsigned char *xl = smem + (wm * (BM / WM) + l16) * 128, *wl = smem + (BM + wn * (BN / WN) + l16) * 128;
    auto read = [&](Half& o, int slot, int h) {
        const int ch = slot * BUF + ((4 * h + g) ^ (l16 & 7)) * 16;
#pragma unroll
        for (int j = 0; j < NI; j++) o.w[j] = *(const u32x4*)(wl + j * 2048 + ch);
#pragma unroll
        for (int i = 0; i < MI; i++) o.x[i] = *(const u32x4*)(xl + i * 2048 + ch);
    };
    auto multiply = [&](const Half& o) {
#pragma unroll
        for (int i = 0; i < MI; i++)
#pragma unroll
            for (int j = 0; j < NI; j++) acc[i][j] = mma<BF16>(o.w[j], o.x[i], acc[i][j]);
    };
    // one read for every few products
    auto mix = [&]() {
#pragma unroll
        for (int k = 0; k < MI + NI; k++) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, MI * NI * (BF16 ? 1 : 4) / (MI + NI), 0);
        }
    };

    // Step s: its second half is read while the first is multiplied; then every
    // wave is done with its buffer and the next step's has arrived, so that the
    // loads of step s + ST begin and the next first half is read while the second is
    // multiplied.
    if (s0 < s1) {
        if constexpr (WIDE) {
#pragma unroll
            for (int q = 0; q < ST; q++)
                if (s0 + q < s1) fetch(s0 + q, q);
            if (s0 + ST <= s1) dma_wait_but<(ST - 1) * LOADS>();
            else dma_wait();
        } else {
            fetch(s0, 0);
            keep(0);
            if (s0 + 1 < s1) fetch(s0 + 1, 1);
        }
        __syncthreads();
        read(even, 0, 0);
        int slot = 0, next = 1;
        for (int s = s0; s < s1; s++) {
            read(odd, slot, 1);
            multiply(even);
            mix();
            if constexpr (!WIDE) {
                if (s + 1 < s1) keep(next);
            } else {
                if (s + ST <= s1) dma_wait_but<(ST - 2) * LOADS>();   // (the last steps' waits are for all that is left)
                else dma_wait();
            }
            __syncthreads();
            if (s + ST < s1) fetch(s + ST, slot);
            slot = next;
            next = next + 1 == ST ? 0 : next + 1;
            read(even, slot, 0);   // (past the last step: what lies there, unused)
            multiply(odd);
            mix();
        }
    }
    __syncthreads();
    write_out<MI, NI>(p, places + wm * (BM / WM), (float*)(smem + wave * out_bytes<MI, NI>()), acc, at.m0 + wm * (BM / WM),
                      at.n0 + wn * (p.glu ? BN / WN / 2 : BN / WN), at.split);
}

// fp32 on the bf16 matrix cores, which are sixteen times as fast: every value is
// the sum of three bf16 planes of eight of its bits each (cut off one after the
// other, exactly; below 2^-110 the last bits are lost), and six of the nine products
// of planes are added, the smallest first.  What is left out is below 2^-21 of a
// product's magnitude (a second plane is below 2^-7 of its value, a third below 2^-15,
// and two products of both are left out), 2^-24 on average.  An infinity has planes
// that are NaN: sums that come out as NaN are computed again by fp32's own products
// (only those, so that a row's bits do not depend on other rows).  The planes are made
// on the way to LDS: K steps of 32 values through registers and two buffers.
//
// What bounds it: the products, and in smaller tiles the planes (5.5 operations a value:
// 64 x 64 tiles spend as long on them).  4,096^3 563 and 597 us on two cards,
// 244 and 230 TFLOP/s of fp32 (by fp32's own products 1.7 times as long); 4,011 x 1,001
// -> 777 45 and 47.
template <int BM, int BN, int WM, int WN> __global__ __launch_bounds__(64 * WM * WN, 2) void plane_kernel(const LinearParams p)
{
    constexpr int T = 64 * WM * WN, MI = BM / WM / 16, NI = BN / WN / 16, KT = 32;
    constexpr int ROWS = BM + BN, LOADS = ROWS * kChunks / T, PLANE = ROWS * 64, BUF = 3 * PLANE;
    constexpr int OUT = WM * WN * out_bytes<MI, NI>(), LDS = 2 * BUF > OUT ? 2 * BUF : OUT;
    static_assert(ROWS * kChunks % T == 0);
    __shared__ __align__(16) unsigned char smem[LDS];
    __shared__ int some;
    __shared__ Place places[BM];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4, wm = wave % WM, wn = wave / WM;
    const TileAt<BM, BN> at(p);
    if (tid == 0) some = 0;
    const char* row[LOADS];
    if (operand_rows<BM, BN, WN, T, 4>(p, at, places, row)) some = 1;
    __syncthreads();
    if (!some) return;

    const int steps = (p.K + KT - 1) / KT;
    const int s0 = (int)((int64_t)steps * at.split / p.splits), s1 = (int)((int64_t)steps * (at.split + 1) / p.splits);
    // loads of step s, and their way into a buffer
    u32x4 stage[LOADS];
    auto fetch = [&](int s, u32x4 (&to)[LOADS]) {
        load_chunks<false>(row, s * KT + 4 * (tid % kChunks), p.K, (s + 1) * KT <= p.K, to);
    };
    // (chunks of eight values, their index XORed with bits of the row: the eight rows that are read at once lie in
    // different banks)
    auto keep = [&](const u32x4 (&from)[LOADS], int buf) {
#pragma unroll
        for (int c = 0; c < LOADS; c++) {
            const int r = tid / kChunks + c * (T / kChunks);
            unsigned char* to = smem + buf * BUF + r * 64 + ((tid % kChunks / 2) ^ ((r >> 1) & 3)) * 16 + tid % 2 * 8;
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; j++) y[j] = from[c][j];
#pragma unroll
            for (int q = 0; q < 3; q++) {
                *(u32x2*)(to + q * PLANE) = u32x2{__builtin_amdgcn_perm(y[1], y[0], 0x07060302u), __builtin_amdgcn_perm(y[3], y[2], 0x07060302u)};
#pragma unroll
                for (int j = 0; j < 4; j++) y[j] = __float_as_uint(__uint_as_float(y[j]) - __uint_as_float(y[j] & 0xffff0000u));
            }
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    const int ch = l16 * 64 + (g ^ ((l16 >> 1) & 3)) * 16;
    const unsigned char *xl = smem + wm * (BM / WM) * 64 + ch, *wl = smem + (BM + wn * (BN / WN)) * 64 + ch;

    // Of the two waves on a SIMD one makes the next step's planes before its products,
    // the other after them: vector and matrix work side by side.
    const bool ahead = T == 512 && wave >= 4;
    if (s0 < s1) {
        fetch(s0, stage);
        keep(stage, 0);
        if (s0 + 1 < s1) fetch(s0 + 1, stage);
        __syncthreads();
        for (int s = s0, buf = 0; s < s1; s++, buf ^= 1) {
            auto next = [&]() {
                if (s + 1 < s1) keep(stage, buf ^ 1);
                if (s + 2 < s1) fetch(s + 2, stage);
            };
            if (ahead) next();
            u32x4 w[3][NI];
#pragma unroll
            for (int q = 0; q < 3; q++)
#pragma unroll
                for (int j = 0; j < NI; j++) w[q][j] = *(const u32x4*)(wl + buf * BUF + q * PLANE + j * 1024);
#pragma unroll
            for (int i = 0; i < MI; i++) {
                u32x4 x[3];
#pragma unroll
                for (int q = 0; q < 3; q++) x[q] = *(const u32x4*)(xl + buf * BUF + q * PLANE + i * 1024);
#pragma unroll
                for (int t = 0; t < 6; t++) {
                    constexpr int kw[6] = {2, 0, 1, 1, 0, 0}, kx[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
                    for (int j = 0; j < NI; j++) acc[i][j] = mma<true>(w[kw[t]][j], x[kx[t]], acc[i][j]);
                }
            }
            if (!ahead) next();
            __syncthreads();
        }
    }
    float nan = 0.0f;   // 0 times a sum: NaN for one that is no number
#pragma unroll
    for (int i = 0; i < MI; i++)
#pragma unroll
        for (int j = 0; j < NI; j++)
#pragma unroll
            for (int k = 0; k < 4; k++) nan = fmaf(0.0f, acc[i][j][k], nan);
    if (__builtin_expect(__any(nan != nan), 0)) {
#pragma unroll
        for (int i = 0; i < MI; i++) {
            const Place x = places[wm * (BM / WM) + 16 * i + l16];
            const char* xr = x.on() ? (const char*)p.x.p + (x.e * p.x.sb + x.i * p.x.st) * 4 : (const char*)p.w;
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const char* wr = weight_row<BN, WN, 4>(p, at.n0, wn * (BN / WN) + 16 * j + l16);
                f32x4 own = {0, 0, 0, 0};
#pragma unroll 1
                for (int k = s0 * KT; k < min(s1 * KT, p.K); k += 16)
                    own = mma<false>(load_chunk<false>(wr, k + 4 * g, p.K), load_chunk<false>(xr, k + 4 * g, p.K), own);
#pragma unroll
                for (int k = 0; k < 4; k++) acc[i][j][k] = acc[i][j][k] != acc[i][j][k] ? own[k] : acc[i][j][k];
            }
        }
    }
    __syncthreads();
    write_out<MI, NI>(p, places + wm * (BM / WM), (float*)(smem + wave * out_bytes<MI, NI>()), acc, at.m0 + wm * (BM / WM),
                      at.n0 + wn * (p.glu ? BN / WN / 2 : BN / WN), at.split);
}

// ------------------------------------------------------------- few rows
//
// Calls of up to 16 MB rows: what counts is the weight's way from memory.  A block's
// four waves share the K of sixteen columns (NT = 2, with glu: and their factors)
// and all rows; weights and rows go from memory straight to the
// operand registers, U groups of four chunks at a time, and the waves' sums meet
// in LDS.
//
// What bounds it: HBM where the weight is large (4 x 4,096 -> 8,192, weights past the caches,
// in a graph: bf16 15.3 us, 4.4 TB/s; gated halves, twice the weight, 28.4, 4.7; fp32
// 33.7, 4.0; 16 rows 19.6, gated 32.5, since every block reads all of them; the same
// weight again, from the memory-side cache, 13.8, 24.2, 25.1, 17.5 and 25.6), else the
// launch and a load's latency for every U groups (4 x 512 -> 1,536 in a graph 3.6 us).
template <bool BF16, int MB, int NT, bool WIDE>
__global__ __launch_bounds__(256) void few_kernel(const LinearParams p)
{
    constexpr int CE = chunk_elems<BF16>(), ES = 16 / CE, U = 4, KG = 4 * CE;   // elements of a group of chunks
    __shared__ __align__(16) float sums[4][16 * MB * (16 * NT + 4)];
    __shared__ Place places[16 * MB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    constexpr int BC = 16;   // (NT = 2: with glu, their factors)
    const int split = blockIdx.x % p.splits, n0 = blockIdx.x / p.splits * BC;

    const char *xrow[MB], *wrow[NT];
#pragma unroll
    for (int i = 0; i < MB; i++) {
        const Place at = place_of(p, 16 * i + l16);
        if (wave == 0 && g == 0) places[16 * i + l16] = at;
        xrow[i] = at.on() ? (const char*)p.x.p + (at.e * p.x.sb + at.i * p.x.st) * ES : (const char*)p.w;
    }
#pragma unroll
    for (int j = 0; j < NT; j++) {
        wrow[j] = (const char*)p.w + ((int64_t)j * p.N + min(n0 + l16, p.N - 1)) * p.wstride * ES;
    }
    const int groups = (p.K + KG - 1) / KG, parts = 4 * p.splits, part = 4 * split + wave;
    const int g0 = (int)((int64_t)groups * part / parts), g1 = (int)((int64_t)groups * (part + 1) / parts);

    const bool dwords = !(((uintptr_t)p.x.p | (uintptr_t)p.w | 2 * (p.x.sb | p.x.st | p.wstride)) & 2);   // all rows at dwords
    // (`whole`, uniform: no lane's chunk passes the row's end)
    auto chunk = [&](const char* r, int k, bool whole) {
        if constexpr (WIDE) return k < p.K ? *(const u32x4*)(r + (int64_t)k * ES) : u32x4{0, 0, 0, 0};
        if (whole) {
            const char* a = r + (int64_t)k * ES;
            if (BF16 && !dwords) a -= (uintptr_t)a & 2;   // (see shift)
            return (u32x4) * (const u32x4_any*)a;
        }
        return k < p.K ? load_chunk<BF16>(r, k, p.K) : u32x4{0, 0, 0, 0};
    };
    // Loads at two bytes past a dword go at a third of the rate.  Instead the dwords from two bytes before are loaded
    // and shifted with the first one of the row's next chunk: the next lane group's, or (of the last group) the next
    // of the U's, or `end`, the dword at the last chunk's last element.
    auto last = [&](const char* r, int k) { return *(const uint32_t*)(r + 2 * (int64_t)k - ((uintptr_t)r & 2 ? 0 : 2)); };
    auto shift = [&](const char* r, u32x4 (&c)[U], uint32_t end) {
        const uint32_t sh = 8 * ((uintptr_t)r & 2);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const uint32_t next = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * ((lane + 16) & 63), (int)(g ? c[u][0] : u + 1 < U ? c[u + 1][0] : end));
#pragma unroll
            for (int t = 0; t < 4; t++) c[u][t] = __builtin_amdgcn_alignbit(t < 3 ? c[u][t + 1] : next, c[u][t], sh);
        }
    };
    f32x4 acc[MB][NT];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) acc[i][j] = f32x4{0, 0, 0, 0};
    for (int q = g0; q < g1; q += U) {
        u32x4 w[NT][U], x[MB][U];
        const bool whole = q + U <= g1 && (q + U) * KG <= p.K;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int k = q + u < g1 ? (q + u) * KG + g * CE : p.K;   // (past this wave's part: zeros)
#pragma unroll
            for (int j = 0; j < NT; j++) w[j][u] = chunk(wrow[j], k, whole);
#pragma unroll
            for (int i = 0; i < MB; i++) x[i][u] = chunk(xrow[i], k, whole);
        }
        if constexpr (BF16 && !WIDE) {
            if (whole && !dwords) {   // (uniform)
                uint32_t we[NT], xe[MB];
#pragma unroll
                for (int j = 0; j < NT; j++) we[j] = last(wrow[j], (q + U) * KG - 1);
#pragma unroll
                for (int i = 0; i < MB; i++) xe[i] = last(xrow[i], (q + U) * KG - 1);
#pragma unroll
                for (int j = 0; j < NT; j++) shift(wrow[j], w[j], we[j]);
#pragma unroll
                for (int i = 0; i < MB; i++) shift(xrow[i], x[i], xe[i]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < MB; i++)
#pragma unroll
                for (int j = 0; j < NT; j++) acc[i][j] = mma<BF16>(w[j][u], x[i][u], acc[i][j]);
    }
    constexpr int COLS = 16 * NT, PITCH = COLS + 4;
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) *(f32x4*)(sums[wave] + (16 * i + l16) * PITCH + 16 * j + 4 * g) = acc[i][j];
    __syncthreads();
    for (int u = tid; u < 16 * MB * COLS / 4; u += 256) {
        const int at = u / (COLS / 4) * PITCH + 4 * (u % (COLS / 4));
        f32x4 v = *(const f32x4*)(sums[0] + at);
#pragma unroll
        for (int w = 1; w < 4; w++) v += *(const f32x4*)(sums[w] + at);
        *(f32x4*)(sums[0] + at) = v;
    }
    __syncthreads();
    if (wave < MB) finish<COLS>(p, places + 16 * wave, sums[0] + 16 * wave * PITCH, 16, PITCH, 16 * wave, n0, split);
}

// The splits' partial sums and the epilogue, eight columns a thread.
__global__ __launch_bounds__(256) void join_kernel(const LinearParams p)
{
    const int64_t eights = part_half(p.N) / 8, u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (u >= eights * p.M) return;
    const int m = (int)(u / eights), n = 8 * (int)(u % eights);
    const Place at = place_of(p, m);
    if (!at.on()) return;
    const int64_t row = part_row(p.N, p.glu);
    const float* s = p.ws + m * row + n;
    Eight a{}, b{};
    for (int k = 0; k < p.splits; k++, s += (int64_t)p.M * row) {
        const Eight x = load8(s, 0, 0);
#pragma unroll
        for (int j = 0; j < 8; j++) a.v[j] += x.v[j];
        if (p.glu) {
            const Eight y = load8(s, part_half(p.N), 0);
#pragma unroll
            for (int j = 0; j < 8; j++) b.v[j] += y.v[j];
        }
    }
    epilogue(p, at, n, a, b, load_bias(p, n, 0), p.glu ? load_bias(p, n, 1) : Eight{});
}

// ------------------------------------------------------------------ launch

template <bool BF16> hipError_t launch_few(const LinearParams& p, int kind, int64_t blocks, hipStream_t st)
{
#define DCB_FEW(MB, NT) (p.wide ? launch_with(few_kernel<BF16, MB, NT, true>, blocks, 256, 0, st, p) : launch_with(few_kernel<BF16, MB, NT, false>, blocks, 256, 0, st, p))
    if (p.glu) return kind == kFew16 ? DCB_FEW(1, 2) : DCB_FEW(2, 2);
    return kind == kFew16 ? DCB_FEW(1, 1) : DCB_FEW(2, 1);
#undef DCB_FEW
}

static hipError_t launch_kind(const LinearParams& p, int kind, hipStream_t st)
{
    // (these have no variant for rows that are not of whole chunks)
    if ((kind == kTile256 || kind == kRing128) && !p.wide) kind = kTile128;
    const LinearCost& c = kLinearCost[p.bf16 ? 1 : 0][kind];
    const int bc = linear_columns(kind, c.bn, p.glu);
    const int64_t blocks = (int64_t)((p.M + c.bm - 1) / c.bm) * ((p.N + bc - 1) / bc) * p.splits;
    switch (kind) {
    case kFew16:
    case kFew32: return p.bf16 ? launch_few<true>(p, kind, blocks, st) : launch_few<false>(p, kind, blocks, st);
    case kTile64:
        return p.wide ? launch_with(tile_kernel<true, 64, 64, 2, 2, true, 4>, blocks, 256, 0, st, p)
                      : launch_with(tile_kernel<true, 64, 64, 4, 2, false, 2>, blocks, 512, 0, st, p);
    case kTile128:
        return p.wide ? launch_with(tile_kernel<true, 128, 128, 2, 2, true, 2>, blocks, 256, 0, st, p)
                      : launch_with(tile_kernel<true, 128, 128, 2, 4, false, 2>, blocks, 512, 0, st, p);
    case kRing128: return launch_with(tile_kernel<true, 128, 128, 2, 4, true, 4>, blocks, 512, 0, st, p);
    case kTile256: return launch_with(tile_kernel<true, 256, 256, 2, 4, true, 2>, blocks, 512, 0, st, p);
    case kPlane64: return launch_with(plane_kernel<64, 64, 2, 2>, blocks, 256, 0, st, p);
    case kPlane128: return launch_with(plane_kernel<128, 128, 2, 4>, blocks, 512, 0, st, p);
    case kPlane256: return launch_with(plane_kernel<256, 128, 4, 2>, blocks, 512, 0, st, p);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_linear(const LinearParams& p, const LinearPlan& plan, hipStream_t st)
{
    const hipError_t e = launch_kind(p, plan.kind, st);
    if (e != hipSuccess || p.splits == 1) return e;
    return launch_with(join_kernel, ((int64_t)(part_half(p.N) / 8) * p.M + 255) / 256, 256, 0, st, p);
}

}  // namespace dcb
