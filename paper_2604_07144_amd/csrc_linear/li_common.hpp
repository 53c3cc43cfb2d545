// Types, parameter blocks and small device helpers shared by the kernels of weights in 4 bits.
#ifndef LI_COMMON_HPP
#define LI_COMMON_HPP

#include "../csrc_attn/at_codes.hpp"
#include "autopoiesis_linear.h"

namespace {

constexpr uint32_t kBlock = 128;                    // columns of a block: 64 bytes of codes

struct Weights {
    char *codes, *pairs;
    int64_t code_stride, pair_stride;
    uint32_t n_out, n_in, blocks;
};

struct LinearParams {
    Weights w[2];                                   // a matrix; or gate and up
    const char *x, *add;
    char* y;
    int64_t x_stride, add_stride, y_stride;
    uint32_t n_tokens, act;
    float* parts;                                   // [part][token][output, of both matrices] where inputs are cut into parts
    uint32_t part_blocks, n_parts;
};

// Eight codes of a word as 16 + code in the 16-bit type: a code's bits beside the exponent of 16 are that value exactly, so a
// pair of them costs a shift and an and-or.
template <typename E> __device__ __forceinline__ u32x4 codes16(uint32_t w) {
    u32x4 r;
    if constexpr (std::is_same_v<E, bf16>) {
        r[0] = (w << 3 & 0x00780078u) | 0x41804180u, r[1] = (w >> 1 & 0x00780078u) | 0x41804180u;
        r[2] = (w >> 5 & 0x00780078u) | 0x41804180u, r[3] = (w >> 9 & 0x00780078u) | 0x41804180u;
    } else {
        r[0] = (w << 6 & 0x03C003C0u) | 0x4C004C00u, r[1] = (w << 2 & 0x03C003C0u) | 0x4C004C00u;
        r[2] = (w >> 2 & 0x03C003C0u) | 0x4C004C00u, r[3] = (w >> 6 & 0x03C003C0u) | 0x4C004C00u;
    }
    return r;
}

template <typename E> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec8<bf16>, a), __builtin_bit_cast(Vec8<bf16>, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec8<fp16>, a), __builtin_bit_cast(Vec8<fp16>, b), c, 0, 0, 0);
}

// The bytes of a block's pairs, as words (one for each group).
template <uint32_t G> using PairWords = uint32_t __attribute__((ext_vector_type(kBlock / G)));

__device__ __forceinline__ float activated(float g, uint32_t act) {
    if (act == AP_SILU) return g / (1.0f + __expf(-g));
    return 0.5f * g * (1.0f + tanhf(0.79788456080286536f * fmaf(0.044715f * g * g, g, g)));
}

template <typename E> __device__ __forceinline__ float load16(const char* p) { return (float)*reinterpret_cast<const E*>(p); }
template <typename E> __device__ __forceinline__ void store16(char* p, float x) { *reinterpret_cast<E*>(p) = (E)x; }

// Sums of a token and output with everything that is left to do to them.
template <typename E, bool kGated> __device__ __forceinline__ void finish(const LinearParams& p, uint32_t t, uint32_t n, float a, float b) {
    if constexpr (kGated) a = activated(a, p.act) * b;
    else if (p.add) a += load16<E>(p.add + (int64_t)t * p.add_stride + 2ull * n);
    store16<E>(p.y + (int64_t)t * p.y_stride + 2ull * n, a);
}

}  // namespace

#endif  // LI_COMMON_HPP
