// Packing rows of weights in 4 bits, and reading them back.
//
// One pass over the memory, which bounds both.  A lane has eight columns, 16 bytes of values and a word of codes; sixteen
// lanes a block, so a wavefront four of them, which may be of different rows.  The range of a group is taken over 4, 8 or 16 lanes.
//
// Measured, 28672 rows of 8192, groups of 64: packing 174 us (3.5 TB/s: memory and vector unit in turn; with a division for each value
// 196), reading back 119 (5.1 TB/s, what a copy moves); 4096 of 4096 14 to 16 and 8.
#ifndef LI_PACK_HPP
#define LI_PACK_HPP

#include "li_common.hpp"

namespace {

constexpr uint32_t kPackThreads = 256, kPackUnits = 4;      // blocks of lanes that a workgroup takes one after another

struct PackParams {
    Weights w;
    char* values;
    int64_t stride;
    uint32_t magic, shift;                          // of a division by w.blocks
};

struct PackPlace {
    uint32_t row, block, lane;                      // lane of the block's sixteen
    bool there, inside;                             // of the matrix; the lane's columns are not what fills the block up
};
__device__ __forceinline__ PackPlace pack_place(const PackParams& p, uint32_t unit) {
    PackPlace r;
    const uint64_t at = ((uint64_t)blockIdx.x * kPackUnits + unit) * (kPackThreads / 16) + threadIdx.x / 16;
    r.lane = threadIdx.x % 16;
    r.there = at < (uint64_t)p.w.n_out * p.w.blocks;
    const uint32_t n = r.there ? (uint32_t)at : 0u;
    r.row = __umulhi(n * 2u, p.magic) >> p.shift;
    r.block = n - r.row * p.w.blocks;
    r.inside = r.there && r.block * kBlock + r.lane * 8 < p.w.n_in;
    return r;
}
// Columns 8 l .. 8 l + 7 of a block (m = l / 4, q = l % 4) are word 4 q + m.
__device__ __forceinline__ uint32_t word_of(uint32_t lane) { return lane % 4 * 4 + lane / 4; }

template <typename E, uint32_t G> __global__ __launch_bounds__(kPackThreads) void k_pack(const PackParams p) {
    PackPlace at[kPackUnits];
    u32x4 x[kPackUnits];
#pragma unroll
    for (uint32_t u = 0; u < kPackUnits; ++u) {
        at[u] = pack_place(p, u);
        x[u] = u32x4{};
        if (at[u].inside) x[u] = *reinterpret_cast<const u32x4*>(p.values + (int64_t)at[u].row * p.stride + 2ull * (at[u].block * kBlock + at[u].lane * 8));
    }
#pragma unroll
    for (uint32_t u = 0; u < kPackUnits; ++u) {
        float lo = INFINITY, hi = -INFINITY, numbers = 0.0f;
        if (at[u].inside) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = low16<E>(x[u][i]), b = high16<E>(x[u][i]);
                lo = fminf(fminf(lo, a), b), hi = fmaxf(fmaxf(hi, a), b);
                numbers = fmaf(a, 0.0f, fmaf(b, 0.0f, numbers));       // NaN as soon as one is not a number
            }
        }
        uint32_t odd = numbers != numbers;
        odd |= at[u].inside ? 2u : 0u;                      // bit 0: not all are numbers; bit 1: there are some
        auto widen = [&](auto m) {
            lo = fminf(lo, across<m()>(lo)), hi = fmaxf(hi, across<m()>(hi));
            odd |= across<m()>(odd);
        };
        widen(std::integral_constant<uint32_t, 1>{}), widen(std::integral_constant<uint32_t, 2>{});
        if constexpr (G >= 64) widen(std::integral_constant<uint32_t, 4>{});
        if constexpr (G >= 128) widen(std::integral_constant<uint32_t, 8>{});
        const uint32_t pair = odd & 2 ? group_pair<E>(lo, hi, !(odd & 1)) : 0u;
        const float step = low16<E>(pair), low = high16<E>(pair);
        // As code_of, without a division for each value: with the inverse of the step rounded to the nearest, one step of correction makes
        // a product the quotient rounded to the nearest.  Steps near the ends of the range are left to code_of.
        uint32_t word = 0;
        if (at[u].inside) {
            const float d = step * 0.0625f, from = low * -0.0625f, near = __builtin_amdgcn_rcpf(d), inverse = fmaf(fmaf(-d, near, 1.0f), near, near);
            if (d > 0x1p-90f && d < 0x1p90f) {
                float even = 0.0f, odds = 0.0f;                        // codes as digits: whole numbers below 2^16
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    auto code = [&](float v) {
                        const float n = fmaf(v, 0.0625f, from), q = n * inverse;
                        return fminf(fmaxf(rintf(fmaf(fmaf(-d, q, n), inverse, q)), 0.0f), 15.0f);
                    };
                    even = fmaf(code(low16<E>(x[u][i])), (float)(1 << 4 * i), even), odds = fmaf(code(high16<E>(x[u][i])), (float)(1 << 4 * i), odds);
                }
                word = (uint32_t)even | (uint32_t)odds << 16;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    word |= code_of(low16<E>(x[u][i]), low, step) << (4 * i) | code_of(high16<E>(x[u][i]), low, step) << (4 * i + 16);
            }
        }
        if (at[u].there) {
            reinterpret_cast<uint32_t*>(p.w.codes + (int64_t)at[u].row * p.w.code_stride + (int64_t)at[u].block * (kBlock / 2))[word_of(at[u].lane)] = word;
            if (at[u].lane % (G / 8) == 0)
                reinterpret_cast<uint32_t*>(p.w.pairs + (int64_t)at[u].row * p.w.pair_stride)[at[u].block * (kBlock / G) + at[u].lane / (G / 8)] = pair;
        }
    }
}

template <typename E, uint32_t G> __global__ __launch_bounds__(kPackThreads) void k_unpack(const PackParams p) {
    PackPlace at[kPackUnits];
    uint32_t word[kPackUnits], pair[kPackUnits];
#pragma unroll
    for (uint32_t u = 0; u < kPackUnits; ++u) {
        at[u] = pack_place(p, u);
        word[u] = pair[u] = 0;
        if (at[u].inside) {
            word[u] = reinterpret_cast<const uint32_t*>(p.w.codes + (int64_t)at[u].row * p.w.code_stride + (int64_t)at[u].block * (kBlock / 2))[word_of(at[u].lane)];
            pair[u] = reinterpret_cast<const uint32_t*>(p.w.pairs + (int64_t)at[u].row * p.w.pair_stride)[at[u].block * (kBlock / G) + at[u].lane / (G / 8)];
        }
    }
#pragma unroll
    for (uint32_t u = 0; u < kPackUnits; ++u) {
        const float step = low16<E>(pair[u]), low = high16<E>(pair[u]);
        u32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = pack2<E>(fmaf(step, (float)(word[u] >> (4 * i) & 15u), low), fmaf(step, (float)(word[u] >> (4 * i + 16) & 15u), low));
        if (at[u].inside) *reinterpret_cast<u32x4*>(p.values + (int64_t)at[u].row * p.stride + 2ull * (at[u].block * kBlock + at[u].lane * 8)) = x;
    }
}

}  // namespace

#endif  // LI_PACK_HPP
