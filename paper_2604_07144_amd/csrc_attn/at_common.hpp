// Types, parameter blocks and small device helpers shared by the cache and attention kernels.
#ifndef AT_COMMON_HPP
#define AT_COMMON_HPP

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "autopoiesis_attn.h"

namespace {

constexpr uint32_t kLanes = 64;

using bf16 = __bf16;
using fp16 = _Float16;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename E> using Vec2 = E __attribute__((ext_vector_type(2)));
template <typename E> using Vec8 = E __attribute__((ext_vector_type(8)));

// The cache as the kernels take it.  Page of position p = p / page_size by a product: with l = ceil(log2(page_size)) and
// magic = ceil(2^(31 + l) / page_size), p * magic >> (31 + l) is exact for p < 2^31.
struct Cache {
    char *k, *v;
    char *k_pairs, *v_pairs;
    int64_t page_stride, head_stride, slot_stride;
    int64_t pair_page_stride, pair_head_stride, pair_slot_stride;
    uint32_t n_pages, page_size, magic, shift;
};

struct Batch {
    const int32_t *first, *kv_len, *table;
    int64_t table_stride;
    uint32_t n_seqs, n_tokens, max_new, max_kv;
};

struct Rows {
    char* data;
    int64_t token_stride, head_stride;
};

// Where a position lies in the cache; `there` is false where the table names no page.
struct Place {
    uint32_t page, slot;
    bool there;
};

__device__ __forceinline__ Place place_of(const Cache& c, const int32_t* __restrict__ row, uint32_t p, uint32_t limit) {
    Place r;
    const bool in = p < limit;
    const uint32_t at = in ? p : 0u;
    const uint32_t n = __umulhi(at * 2u, c.magic) >> c.shift;
    r.slot = at - n * c.page_size;
    r.page = in ? (uint32_t)row[n] : 0xFFFFFFFFu;
    r.there = r.page < c.n_pages;
    return r;
}

// How many i of 1 .. n have f(i) <= t, for an f that does not decrease; the wavefront looks at 64 of them at a time.  Whatever
// f is, only 1 .. n are asked for and the answer is in 0 .. n.
template <typename F> __device__ __forceinline__ uint32_t count_to(uint32_t n, uint32_t t, F f) {
    const uint32_t lane = threadIdx.x & (kLanes - 1), end = n;
    uint32_t lo = 0;
    while (n > kLanes) {
        const uint32_t step = (n + kLanes - 1) / kLanes, at = lo + (lane + 1) * step;
        const bool below = at < lo + n && f(at) <= t;
        lo += (uint32_t)__popcll(__ballot(below)) * step;
        n = min(step, end - lo);
    }
    const bool below = lane < n && f(lo + lane + 1) <= t;
    return lo + (uint32_t)__popcll(__ballot(below));
}

// The sequence that holds new token t; n_seqs where none does.
__device__ __forceinline__ uint32_t seq_of(const Batch& b, uint32_t t) {
    return count_to(b.n_seqs, t, [&](uint32_t i) { return (uint32_t)b.first[i]; });
}

// A sequence of the batch: its first new row, how many it has, the tokens it holds (all clamped to what was described).
struct Seq {
    int32_t first, n_new, kv_len;
    int32_t pos0;          // position of the first new token; may be negative
};

__device__ __forceinline__ Seq seq_at(const Batch& b, uint32_t s) {
    Seq r;
    const int32_t lo = b.first[s], hi = b.first[s + 1], held = b.kv_len[s];
    r.first = min(max(lo, 0), (int32_t)b.n_tokens);
    r.n_new = min(max(hi, r.first), (int32_t)b.n_tokens) - r.first;
    r.kv_len = min(max(held, 0), (int32_t)b.max_kv);
    r.pos0 = (int32_t)max((int64_t)held - r.n_new, (int64_t)INT32_MIN);
    return r;
}

// The same number, but computed here: keeps what depends on it from being moved out of a loop and held in registers.
__device__ __forceinline__ uint32_t here(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A number that is the same in all lanes, in a scalar register.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename E> __device__ __forceinline__ uint16_t bits16(E x) { return __builtin_bit_cast(uint16_t, x); }
template <typename E> __device__ __forceinline__ E from_bits16(uint32_t x) { return __builtin_bit_cast(E, (uint16_t)x); }

template <typename E> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    const f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, Vec2<E>));
}

// Value of one half of a dword of the 16-bit type.
template <typename E> __device__ __forceinline__ float low16(uint32_t x) {
    if constexpr (std::is_same_v<E, bf16>) return __uint_as_float(x << 16);
    else return (float)from_bits16<fp16>(x & 0xFFFFu);
}
template <typename E> __device__ __forceinline__ float high16(uint32_t x) {
    if constexpr (std::is_same_v<E, bf16>) return __uint_as_float(x & 0xFFFF0000u);
    else return (float)from_bits16<fp16>(x >> 16);
}

// Eight codes of a dword as values of the 16-bit type, rounded once from 32 bits: (lo + step * code).
template <typename E> __device__ __forceinline__ u32x4 decode8(uint32_t codes, float step, float lo) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = (float)((codes >> (8 * i)) & 15u), b = (float)((codes >> (8 * i + 4)) & 15u);
        r[i] = pack2<E>(fmaf(step, a, lo), fmaf(step, b, lo));
    }
    return r;
}

}  // namespace

#endif  // AT_COMMON_HPP
