// Internal interface between the C entries of a block's operators
// (block_runtime.hip) and their kernels (norm_kernels.hip, linear_kernels.hip,
// paged_kernels.hip), and what the kernels share.  Not part of the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dcb {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
// (global memory takes vectors at any element's alignment)
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef u32x4 __attribute__((aligned(4))) u32x4_dwords;
typedef u32x2 __attribute__((aligned(2))) u32x2_any;
typedef uint32_t __attribute__((aligned(2))) u32_any;

// Rows of tokens: token i of entry e at p + e sb + i st, in elements (p null: none).
struct Rows {
    void* p;
    int64_t sb, st;
    int bf16;
};

struct Call {
    const int* lens;   // null: n each
    int batch, n;
    __device__ __forceinline__ int len(int e) const { return lens ? min(max(lens[e], 0), n) : n; }
};

struct NormSpec {
    int kind;          // 0: none, DC_NORM_RMS, DC_NORM_LAYER
    float eps;
    const float *gain, *bias;
};

struct NormParams {
    Rows x, h, gate, r, scale, shift, y;
    NormSpec post, pre;
    Call call;
    int width;
    float x_scale;
    int rows, per;     // set at the launch: rows in all, rows of a block's (or wave's) walk
    int apart;         // set at the launch: results_apart (norm_plan.h)
};
hipError_t launch_norm(NormParams p, hipStream_t st);

struct LinearParams {
    const void* w;
    const float* bias;
    int64_t wstride;
    int K, N, bf16, act, glu;
    Rows x, gate, res, out;
    float res_scale;
    Call call;
    int M;             // batch * n
    int wide;          // every 16-byte chunk of x's and the weight's rows is aligned
    int splits;
    float* ws;         // splits > 1: [split][M][N or 2 N] partial sums
};
struct LinearPlan;   // linear_plan.h
hipError_t launch_linear(const LinearParams& p, const LinearPlan& plan, hipStream_t st);

// Rows of heads, as dc_head_rows.
struct HeadsOf {
    void* p;
    int64_t sb, st, sh;
    int heads;
    __device__ __forceinline__ int64_t at(int e, int i, int h) const { return e * sb + (int64_t)i * st + h * sh; }
};

struct Paged {
    const int* table;
    int64_t table_stride;
    char *k, *v;
    uint32_t kp, kt, kh, vp, vt, vh;  // strides in units of 16 bytes
    int batch, heads, D, bf16;
    int shift, pages, limit;          // log2 of the page size; pages of the pool; positions of an entry
};

struct PagedParams {
    Paged c;
    HeadsOf q, o, k, v;               // attend: q, o; append: k, v
    const int64_t* pos;
    const int* lens;
    int n, group, window, sinks, causal;
    float scale_log2;                 // score scale * log2(e)
    int splits;
    float* ws;
};
struct PagedPlan;   // paged_plan.h
hipError_t launch_append(const PagedParams& p, hipStream_t st);
hipError_t launch_attend(const PagedParams& p, const PagedPlan& plan, hipStream_t st);

#ifdef __HIPCC__

// A launch has fewer than 2^32 threads: more are refused here, since a launch that
// fails leaves its error for the thread's next runtime call.
template <class P> hipError_t launch_with(void (*kernel)(P), int64_t blocks, int threads, int lds, hipStream_t st, P p)
{
    if (blocks * threads >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
    void* args[] = {&p};
    return hipLaunchKernel((const void*)kernel, dim3((unsigned)blocks), dim3((unsigned)threads), args, lds, st);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const bf16x2_t v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }

// Element `at` of p, and its store.
__device__ __forceinline__ float load1(const void* p, int64_t at, int bf16)
{
    return bf16 ? bf2f(((const uint16_t*)p)[at]) : ((const float*)p)[at];
}
__device__ __forceinline__ void store1(void* p, int64_t at, int bf16, float v)
{
    if (bf16) ((uint16_t*)p)[at] = (uint16_t)(pack2(v, 0.0f) & 0xffffu);
    else ((float*)p)[at] = v;
}

// Four consecutive elements, of any alignment.
__device__ __forceinline__ f32x4 load4(const void* p, int64_t at, int bf16)
{
    if (bf16) {
        const u32x2 w = *(const u32x2_any*)((const uint16_t*)p + at);
        return f32x4{bf2f(w[0] & 0xffffu), __uint_as_float(w[0] & 0xffff0000u), bf2f(w[1] & 0xffffu), __uint_as_float(w[1] & 0xffff0000u)};
    }
    return __builtin_bit_cast(f32x4, *(const u32x4_any*)((const float*)p + at));
}
__device__ __forceinline__ void store4(void* p, int64_t at, int bf16, f32x4 v)
{
    if (bf16) *(u32x2_any*)((uint16_t*)p + at) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
    else *(u32x4_any*)((float*)p + at) = __builtin_bit_cast(u32x4, v);
}

// Eight consecutive elements as they are stored, of any alignment.
template <bool BF16> struct Raw8 { u32x4 w[BF16 ? 1 : 2]; };
template <bool BF16> __device__ __forceinline__ Raw8<BF16> load_raw(const void* p, int64_t at)
{
    Raw8<BF16> r;
    if constexpr (BF16) {
        r.w[0] = *(const u32x4_any*)((const uint16_t*)p + at);
    } else {
        r.w[0] = *(const u32x4_any*)((const float*)p + at);
        r.w[1] = *(const u32x4_any*)((const float*)p + at + 4);
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
// The first m (1 to 7, uniform) of eight elements, zeros behind them: four, two and
// one at a time, straight to where they belong.
template <bool BF16, int M> __device__ __forceinline__ Raw8<BF16> load_raw_m(const void* p, int64_t at)
{
    constexpr int two = M & 4, one = M & 6;   // where the pair and the last one begin
    Raw8<BF16> r{};
    if constexpr (BF16) {
        const uint16_t* s = (const uint16_t*)p + at;
        if constexpr (M & 4) {
            const u32x2 x = *(const u32x2_any*)s;
            r.w[0][0] = x[0];
            r.w[0][1] = x[1];
        }
        if constexpr (M & 2) r.w[0][two / 2] = *(const u32_any*)(s + two);
        if constexpr (M & 1) r.w[0][one / 2] = s[one];
    } else {
        const uint32_t* s = (const uint32_t*)p + at;
        if constexpr (M & 4) r.w[0] = *(const u32x4_any*)s;
        if constexpr (M & 2) {
            const u32x2 x = *(const u32x2_any*)(s + two);
            r.w[two / 4][0] = x[0];
            r.w[two / 4][1] = x[1];
        }
        if constexpr (M & 1) r.w[one / 4][one % 4] = s[one];
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ Raw8<BF16> load_raw_part(const void* p, int64_t at, int m)
{
    switch (m) {
    case 1: return load_raw_m<BF16, 1>(p, at);
    case 2: return load_raw_m<BF16, 2>(p, at);
    case 3: return load_raw_m<BF16, 3>(p, at);
    case 4: return load_raw_m<BF16, 4>(p, at);
    case 5: return load_raw_m<BF16, 5>(p, at);
    case 6: return load_raw_m<BF16, 6>(p, at);
    default: return load_raw_m<BF16, 7>(p, at);
    }
}
// Stores m (1 to 7, uniform) of eight elements: the first ones, or (LAST) the last ones.
template <bool BF16, int M, bool LAST> __device__ __forceinline__ void store_m(void* p, int64_t at, const float (&x)[8])
{
    constexpr int two = M & 4, one = M & 6, from = LAST ? 8 - M : 0;
    if constexpr (M & 4) store4(p, at, BF16, f32x4{x[from], x[from + 1], x[from + 2], x[from + 3]});
    if constexpr (M & 2) {
        if constexpr (BF16) *(u32_any*)((uint16_t*)p + at + two) = pack2(x[from + two], x[from + two + 1]);
        else *(u32x2_any*)((float*)p + at + two) = u32x2{__float_as_uint(x[from + two]), __float_as_uint(x[from + two + 1])};
    }
    if constexpr (M & 1) store1(p, at + one, BF16, x[from + one]);
}
template <bool BF16, bool LAST> __device__ __forceinline__ void store_part(void* p, int64_t at, int m, const float (&x)[8])
{
    switch (m) {
    case 1: return store_m<BF16, 1, LAST>(p, at, x);
    case 2: return store_m<BF16, 2, LAST>(p, at, x);
    case 3: return store_m<BF16, 3, LAST>(p, at, x);
    case 4: return store_m<BF16, 4, LAST>(p, at, x);
    case 5: return store_m<BF16, 5, LAST>(p, at, x);
    case 6: return store_m<BF16, 6, LAST>(p, at, x);
    default: return store_m<BF16, 7, LAST>(p, at, x);
    }
}
template <bool BF16> __device__ __forceinline__ void store8(void* p, int64_t at, const float (&x)[8])
{
    if constexpr (BF16) {
        *(u32x4_any*)((uint16_t*)p + at) = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    } else {
        store4(p, at, 0, f32x4{x[0], x[1], x[2], x[3]});
        store4(p, at + 4, 0, f32x4{x[4], x[5], x[6], x[7]});
    }
}

// 16 bytes a lane from memory to LDS, lane i's to `lds` + 16 i (an LDS byte address,
// uniform).  As an instruction of its own: the compiler waits for a load of the
// builtin before any LDS read, since the two might meet.  (M0 is a register that the
// compiler keeps nothing in.)  The caller waits (dma_wait) before the barrier
// behind which the bytes are read.
__device__ __forceinline__ void dma16(const void* from, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(lds));
}
// The same from base + off, base uniform.
__device__ __forceinline__ void dma16(const char* base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds));
}
__device__ __forceinline__ void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ __forceinline__ float dpp_add(float v) { return v + __uint_as_float(dpp<CTRL>(__float_as_uint(v))); }
// v and the value of the lane 16, or 32, lanes apart.
__device__ __forceinline__ float sum_xor16(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];   // (scalars: a bit cast straight from element 1 reads element 0)
    return __uint_as_float(a0) + __uint_as_float(a1);
}
__device__ __forceinline__ float sum_xor32(float v)
{
    const uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    return __uint_as_float(a0) + __uint_as_float(a1);
}
__device__ __forceinline__ float max_xor16_32(float v)
{
    uint32_t u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    u = __float_as_uint(fmaxf(__uint_as_float(a0), __uint_as_float(a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return fmaxf(__uint_as_float(b0), __uint_as_float(b1));
}
// The sum over a wave, in every lane, in one fixed order.
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0xB1>(v);    // quad_perm 1 0 3 2
    v = dpp_add<0x4E>(v);    // quad_perm 2 3 0 1
    v = dpp_add<0x141>(v);   // row_half_mirror: the other quad of eight lanes
    v = dpp_add<0x140>(v);   // row_mirror: the other eight of sixteen
    return sum_xor32(sum_xor16(v));
}

#endif

}  // namespace dcb
