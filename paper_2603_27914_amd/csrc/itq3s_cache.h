// The 4-bit cache of keys and values: its layout, and what the kernels that write, read and attend over it share.
//
// Blocks of 32 tokens of one kv head, 32 D + 128 bytes, in the order the attention kernel's matrix operands want:
//   keys    token after token, D/2 bytes each; digit of channel 8 w + j is nibble (j >> 1) + 4 (j & 1) of word w, so that
//           three shifts and masks of a word are four pairs of neighbouring channels
//   values  token t = 16 jh + 4 g + jl, channel 64 h + 32 p + 16 n + c: nibble n of byte
//           1024 h + 16 (16 g + c) + 8 p + 4 jh + 2 (jl & 1) + (jl >> 1): eight tokens of a channel beside each other,
//           the eight that the accumulator layout of the scores leaves in one lane; a token owns its bytes, so
//           tokens are written without reading their neighbours
//   steps   32 words, fp16 step of the key | fp16 step of the value << 16
// Stored nibbles are digit + 8.
#pragma once
#include "itq3s_dev.h"
#include "itq3s_kernels.h"

namespace itq3s {

constexpr int kCacheBlock = 32;  // tokens

template <int D>
constexpr int kBlockBytes = 32 * D + 128;

// Byte offset of (block of 32 tokens, head): pages of `blocks` blocks a head, head after head.
template <int D>
__device__ __forceinline__ int64_t block_offset(int64_t page, int head, int heads, int blocks, int block) {
    return ((page * heads + head) * blocks + block) * (int64_t)kBlockBytes<D>;
}

// Where token t of a block keeps the value byte of channels (32-group p, c) and (p, c + 16).
__device__ __forceinline__ int value_byte(int t, int p, int c) {
    const int g = (t >> 2) & 3, jl = t & 3;
    return (p >> 1) * 1024 + (16 * g + c) * 16 + (p & 1) * 8 + (t >> 4) * 4 + (jl & 1) * 2 + (jl >> 1);
}

// Digits of a word, as pairs of fp16: nibbles 0 and 4, 1 and 5, 2 and 6, 3 and 7.  A nibble v is put into the mantissa of
// 1024 (where it stands in the lowest bits) or of 64 (in bits 4..7), exactly; the digit is what is left without 1032 or 72.
__device__ __forceinline__ half2v low_pair(uint32_t w) {
    return __builtin_bit_cast(half2v, (w & 0x000f000fu) | 0x64006400u) + half2v{(_Float16)-1032.f, (_Float16)-1032.f};
}
__device__ __forceinline__ half2v high_pair(uint32_t w) {
    return __builtin_bit_cast(half2v, (w & 0x00f000f0u) | 0x54005400u) + half2v{(_Float16)-72.f, (_Float16)-72.f};
}

template <int D>
constexpr double kRootD = D == 64 ? 8.0 : D == 128 ? 11.313708498984760390 : 16.0;

template <int MASK>
__device__ __forceinline__ double row_xor(double v) { return row_xor_f64<MASK>(v); }
template <int MASK>
__device__ __forceinline__ float row_xor(float v) { return __builtin_bit_cast(float, row_xor_i32<MASK>(__builtin_bit_cast(int, v))); }

template <int D, int MASK, typename R>
__device__ __forceinline__ void hadamard_across(R (&v)[8], int lane) {
    if constexpr (MASK < D / 8) {
        const R sign = (lane & MASK) != 0 ? (R)-1 : (R)1;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_elementwise_fma(sign, v[j], row_xor<MASK>(v[j]));
    }
}

// Sum and maximum over the D / 8 lanes of a row.
template <int D, int MASK = 1, typename R>
__device__ __forceinline__ R row_sum(R v) {
    if constexpr (MASK < D / 8) return row_sum<D, 2 * MASK>(v + row_xor<MASK>(v));
    else return v;
}
template <int D, int MASK = 1, typename R>
__device__ __forceinline__ R row_max(R v) {
    if constexpr (MASK < D / 8) return row_max<D, 2 * MASK>(__builtin_elementwise_max(v, row_xor<MASK>(v)));
    else return v;
}

// The transform of a row, eight neighbouring channels a lane, without the factor 1 / sqrt(D).
template <int D, typename R>
__device__ __forceinline__ void hadamard(R (&v)[8], int lane = lane_id()) {
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((j & h) == 0) {
                const R a = v[j], b = v[j + h];
                v[j] = a + b;
                v[j + h] = a - b;
            }
    hadamard_across<D, 1>(v, lane);
    hadamard_across<D, 2>(v, lane);
    hadamard_across<D, 4>(v, lane);
    hadamard_across<D, 8>(v, lane);
    hadamard_across<D, 16>(v, lane);
}

}  // namespace itq3s
