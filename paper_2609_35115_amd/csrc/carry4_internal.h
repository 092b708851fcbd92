// Internal interface between the runtimes (carry4_runtime.hip, flow_runtime.hip)
// and the kernels of the attention operators (carry4_kernels.h).  Not part of
// the ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dcf {

// Entry e of a call (a stream, or a stream's guidance branch) and key head h
// own one region of `region` bytes: the key codes [slots][D / 2], the value
// codes, the key scales [slots][D / 32], the value scales.  Slots [0, sinks)
// hold an entry's first tokens, slot sinks + (p - s) % ring the token at
// position p >= s, s being the entry's number of first tokens.  A code is E2M1
// (sign, two exponent bits, one of mantissa; dimension d in bits 4 (d % 2) of
// byte d / 2), a scale byte x stands for 2^(x - 127) and 255 for NaN.
struct Carry4 {
    uint8_t* base;
    int64_t region;
    int heads, D, sinks, ring;
    __host__ __device__ int slots() const { return sinks + ring; }
};
inline int64_t carry4_region(int slots, int D) { return ((int64_t)slots * (D + D / 16) + 255) / 256 * 256; }

// Where the entries' calls stand: entry e reads pos[e / div] (the position of
// its first token of this call), lens[e / div] tokens of it (n where null) and
// keeps sinks[e / div] first tokens (sinks_all where null).
struct Spans {
    const int64_t* pos;   // null: 0
    const int* lens;
    const int* sinks;
    int div, n, sinks_all;
};

// Rows of heads: head h of token i of entry e = b div + c at p + b sb + c sc +
// (i + row0 + slot[b] row_step) st + h sh, in elements (no slot term where slot
// is null); a row's D elements are consecutive.
struct HeadRows {
    void* p;
    int64_t sb, st, sh;
    int heads;
    int64_t sc;
    const int* slot;
    int row0, row_step;
    __device__ __forceinline__ int64_t at(int div, int e, int i, int h) const
    {
        const int b = div == 1 ? e : e / div;
        const int64_t row = (int64_t)i + row0 + (slot ? (int64_t)slot[b] * row_step : 0);
        return b * sb + (e - b * div) * sc + row * st + h * sh;
    }
};

// Per-head norm and position rotation, the store into the carry, or both:
// q (and, without a carry, k) is written to q_out (k_out), k and v into the
// carry.  A null row set is left out.
struct HeadsParams {
    HeadRows q, k, v, q_out, k_out;
    const float *q_gain, *k_gain;   // [D] or null (ones)
    const float* freqs;             // [rot / 2] radians per position
    int rot, interleaved, norm;
    float eps;
    int wide_in, wide_out;          // every row of the inputs / outputs is 16-byte aligned
    Carry4 c;                       // base null: no carry
    Spans sp;
    int entries;
    int waves, split_bits, share;   // set at the launch: waves of a token group, blocks (a power of two), rows of a wave
};

struct Attend4Params {
    HeadRows q, o;
    Carry4 c;
    Spans sp;
    int entries, group;      // query heads to a key head
    int window, causal;
    float scale_log2;        // score scale * log2(e)
    int wide_in, wide_out;   // 16-byte aligned rows
    int splits;
    float* ws;               // splits > 1: partial results
};

// Positions pos .. pos + len of every entry, as the values that the carry holds.
struct Read4Params {
    Carry4 c;
    Spans sp;
    HeadRows k, v;           // outputs
    int entries, wide;       // wide: every row is 16-byte aligned
    int waves, share;   // set at the launch, as in HeadsParams
};

// The carry of (entry e, kv) in Eq. carry's logical order, widened to fp32: the
// nh newest chunks of f_chunk tokens before pos, newest first, then the first
// tokens; out [frames][heads * D].
hipError_t launch_carry4_gather(const Carry4& c, const Spans& sp, int e, int kv, int f_chunk, int nh, int frames,
                                float* out, hipStream_t st);
hipError_t launch_heads(HeadsParams p, int D, int bf16, hipStream_t st);
// Key splits of an attention call, and the bytes of workspace they take.
int attend4_splits(const Carry4& c, int entries, int n, int group, int window, int bf16, int64_t* ws_bytes);
hipError_t launch_attend4(const Attend4Params& p, int bf16, hipStream_t st);
hipError_t launch_read4(const Read4Params& p, int bf16, hipStream_t st);

}  // namespace dcf
