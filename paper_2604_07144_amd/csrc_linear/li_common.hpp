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

// 16 bytes (4 bytes) of each lane from memory to LDS, from `from` + kOffset to the LDS address `to` + kOffset + 16 (4) * lane.  The data
// passes no register, so that nothing here is in flight that the compiler could take for there; a wait for it has to come between it
// and the barrier after which it is read.  (m0 says where in LDS: a reserved register, in which the compiler keeps nothing and which
// it takes in no list of what a statement changes.)
template <uint32_t kOffset> __device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off offset:%2" : : "s"(to), "v"(from), "n"(kOffset) : "memory");
}
__device__ __forceinline__ void load4_to_lds(const char* from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(to), "v"(from) : "memory");
}
// Until no more than n loads are on their way; until all reads of LDS have come.  (The compiler knows of the builtin.)
template <uint32_t n> __device__ __forceinline__ void wait_loads() {
    static_assert(n < 64);
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4) << 14);
    asm volatile("" : : : "memory");
}
__device__ __forceinline__ void wait_lds() {
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" : : : "memory");
}

// In LDS a row of an operand is 64 bytes, four pieces, which are turned by a number that goes by the row: the 16 lanes that a read takes
// at once (lanes 0 to 3, 12 to 15 and 20 to 27; and so on) find theirs in 16 different places of 256 bytes.
__device__ __forceinline__ uint32_t turned(uint32_t row, uint32_t piece) { return piece ^ (0x78u >> row / 4 * 2 & 3u); }
// Likewise rows of 128 bytes, eight pieces.
__device__ __forceinline__ uint32_t wide_turned(uint32_t row, uint32_t piece) { return piece ^ (row / 2 & 7u); }

__device__ const u32x4 kZeros = {};                 // stands in for columns that are not there

// Eight codes of a word as 16 + code in the 16-bit type: a code's bits beside the exponent of 16 are that value exactly, so a
// pair of them costs a shift and an and-or.  That one takes no literals, and the compiler would split it in two: so the mask is
// held in a scalar register and the exponents in a vector register.
template <typename E> struct Unpack {
    static constexpr bool kBf16 = std::is_same_v<E, bf16>;
    uint32_t mask = kBf16 ? 0x00780078u : 0x03C003C0u, sixteen = kBf16 ? 0x41804180u : 0x4C004C00u;
    __device__ __forceinline__ Unpack() {
        asm volatile("" : "+s"(mask));
        asm volatile("" : "+v"(sixteen));
    }
    __device__ __forceinline__ u32x4 operator()(uint32_t w) const {
        u32x4 r;
        if constexpr (kBf16) r[0] = w << 3, r[1] = w >> 1, r[2] = w >> 5, r[3] = w >> 9;
        else r[0] = w << 6, r[1] = w << 2, r[2] = w >> 2, r[3] = w >> 6;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) r[i] = (r[i] & mask) | sixteen;
        return r;
    }
};

template <typename E> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec8<bf16>, a), __builtin_bit_cast(Vec8<bf16>, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec8<fp16>, a), __builtin_bit_cast(Vec8<fp16>, b), c, 0, 0, 0);
}

// c += a b of 16 x 4 and 4 x 16 numbers in 32 bits: a lane has row (column) lane % 16 and place lane / 16 of the sum.
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// The number of lane ^ M.
template <uint32_t M> __device__ __forceinline__ uint32_t across(uint32_t x) {
    if constexpr (M == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true);              // quads 1 0 3 2
    else if constexpr (M == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true);         // quads 2 3 0 1
    else if constexpr (M == 4) return (uint32_t)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);   // 8 turned round, quads turned round
    else if constexpr (M == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xF, 0xF, true);        // 16 moved on by 8
    else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <uint32_t M> __device__ __forceinline__ float across(float x) { return __uint_as_float(across<M>(__float_as_uint(x))); }
template <uint32_t M> __device__ __forceinline__ uint64_t across(uint64_t x) { return (uint64_t)across<M>((uint32_t)(x >> 32)) << 32 | across<M>((uint32_t)x); }

// The bytes of a block's pairs, as words (one for each group).
template <uint32_t G> using PairWords = uint32_t __attribute__((ext_vector_type(kBlock / G)));

// Both are g / (1 + e^-z), with z = g, and with 2 sqrt(2 / pi) (g + 0.044715 g^3): (1 + tanh u) / 2 is 1 / (1 + e^-2u), which does not cancel.  e^-z is a
// square and everything 2^-40 as large until it has been inverted: nothing overflows before the factor of g, a number down to 2^-149, is
// lost for the result's type too.  (Gated 14336 of 4096, 4999 tokens 1106 us, with tanh and whole divisions 1119.)
__device__ __forceinline__ float activated(float g, uint32_t act) {
    const float z = act == AP_SILU ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g), root = __builtin_amdgcn_exp2f(-0.72134752044448170f * z);
    return g * (__builtin_amdgcn_rcpf(fmaf(root * 0x1p-40f, root, 0x1p-40f)) * 0x1p-40f);
}

template <typename E> __device__ __forceinline__ float load16(const char* p) { return (float)*reinterpret_cast<const E*>(p); }
template <typename E> __device__ __forceinline__ void store16(char* p, float x) { *reinterpret_cast<E*>(p) = (E)x; }

// Sums of a token and output with everything that is left to do to them.
template <typename E, bool kGated> __device__ __forceinline__ void finish(const LinearParams& p, uint32_t t, uint32_t n, float a, float b) {
    if constexpr (kGated) a = activated(a, p.act) * b;
    else if (p.add) a += load16<E>(p.add + (int64_t)t * p.add_stride + 2ull * n);
    store16<E>(p.y + (int64_t)t * p.y_stride + 2ull * n, a);
}

// The sums of a token and output: finished, or of a part as they are.
template <typename E, bool kGated> __device__ __forceinline__ void put(const LinearParams& p, uint32_t part, uint32_t n, uint32_t t, float a, float b) {
    if (p.n_parts == 1) return finish<E, kGated>(p, t, n, a, b);
    float* row = p.parts + ((uint64_t)part * p.n_tokens + t) * ((kGated ? 2 : 1) * (uint64_t)p.w[0].n_out) + n;
    row[0] = a;
    if (kGated) row[p.w[0].n_out] = b;
}

// Whether four neighbouring outputs, from a multiple of four on, can be written at once: results; sums of parts.
__device__ __forceinline__ bool four_results(const LinearParams& p) {
    uintptr_t all = reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)p.y_stride;
    if (p.add) all |= reinterpret_cast<uintptr_t>(p.add) | (uintptr_t)p.add_stride;
    return all % 8 == 0;
}
__device__ __forceinline__ bool four_sums(const LinearParams& p) { return p.w[0].n_out % 4 == 0; }

// finish and put of the four outputs from n on, a multiple of four; those that there are.
template <typename E, bool kGated> __device__ __forceinline__ void finish4(const LinearParams& p, bool at_once, uint32_t t, uint32_t n, f32x4 a, f32x4 b) {
    if (!at_once || n + 4 > p.w[0].n_out) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (n + j < p.w[0].n_out) finish<E, kGated>(p, t, n + j, a[j], b[j]);
        return;
    }
    if constexpr (kGated) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) a[j] = activated(a[j], p.act) * b[j];
    } else if (p.add) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(p.add + (int64_t)t * p.add_stride + 2ull * n);
        a += f32x4{low16<E>(x[0]), high16<E>(x[0]), low16<E>(x[1]), high16<E>(x[1])};
    }
    *reinterpret_cast<u32x2*>(p.y + (int64_t)t * p.y_stride + 2ull * n) = u32x2{pack2<E>(a[0], a[1]), pack2<E>(a[2], a[3])};
}
template <typename E, bool kGated> __device__ __forceinline__ void put4(const LinearParams& p, bool at_once, uint32_t part, uint32_t n, uint32_t t, f32x4 a, f32x4 b) {
    if (p.n_parts == 1) return finish4<E, kGated>(p, at_once, t, n, a, b);
    if (!at_once) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (n + j < p.w[0].n_out) put<E, kGated>(p, part, n + j, t, a[j], b[j]);
        return;
    }
    float* row = p.parts + ((uint64_t)part * p.n_tokens + t) * ((kGated ? 2 : 1) * (uint64_t)p.w[0].n_out) + n;
    *reinterpret_cast<f32x4*>(row) = a;
    if (kGated) *reinterpret_cast<f32x4*>(row + p.w[0].n_out) = b;
}

}  // namespace

#endif  // LI_COMMON_HPP
