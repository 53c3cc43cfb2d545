// Products of few rows with weights in 4 bits: the steps of a replica's slots.  The weights are read once and the memory
// bounds it, so everything else has to stay below that.
//
// y[t][n] = sum over groups g of  step[n][g] S[t][n] + (lo[n][g] - 16 step[n][g]) X[t],   S = sum x (16 + code),  X = sum x
// over the group's columns.  S and X come from the matrix units, with tokens as rows and outputs as columns of 16x16x32 tiles: the
// factors 16 + code are exact in the 16-bit type and so no weight is rounded; X is the product with a column of ones.  A
// lane then has four tokens of one output, whose pair is the lane's own.
//
// A lane's 16 bytes of codes are what it multiplies in a block of 128 columns, so a wavefront reads 64 neighbouring bytes of 16 rows.
// The wavefronts of a workgroup have the same outputs and take the blocks in turns, and their sums meet in LDS.
#ifndef LI_FEW_HPP
#define LI_FEW_HPP

#include "li_common.hpp"

namespace {

constexpr uint32_t kFewWaves = 8;

template <typename E> constexpr uint32_t kOnes = std::is_same_v<E, bf16> ? 0x3F803F80u : 0x3C003C00u;

// R tiles of 16 outputs (gated: half of them of gate, half of up), TT tiles of 16 tokens.
template <typename E, uint32_t G, uint32_t R, uint32_t TT, bool kGated>
__global__ __launch_bounds__(kFewWaves * kLanes) void k_linear_few(const LinearParams p) {
    constexpr uint32_t kGroups = kBlock / G, kSteps = G / 32, kOuts = kGated ? R / 2 : R;
    __shared__ f32x4 sums[kFewWaves][R * TT][kLanes];
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes), col = lane % 16, q = lane / 16;
    const uint32_t n0 = blockIdx.x * (kOuts * 16), t0 = blockIdx.y * (TT * 16);

    const char *codes[R], *pairs[R];
#pragma unroll
    for (uint32_t r = 0; r < R; ++r) {
        const Weights& w = p.w[kGated ? r / kOuts : 0];
        const uint32_t n = min(n0 + (kGated ? r % kOuts : r) * 16 + col, w.n_out - 1);     // beyond the last: computed twice, not kept
        codes[r] = w.codes + (int64_t)n * w.code_stride + q * 16;
        pairs[r] = w.pairs + (int64_t)n * w.pair_stride;
    }
    const char* x[TT];
    bool there[TT];
#pragma unroll
    for (uint32_t i = 0; i < TT; ++i) {
        const uint32_t t = t0 + i * 16 + col;
        there[i] = t < p.n_tokens;
        x[i] = p.x + (int64_t)(there[i] ? t : 0u) * p.x_stride + q * 16;
    }

    f32x4 acc[R][TT] = {};
    for (uint32_t b = wave; b < p.w[0].blocks; b += kFewWaves) {
        u32x4 c[R], a[TT][4];
        PairWords<G> pr[R];
#pragma unroll
        for (uint32_t r = 0; r < R; ++r) {
            c[r] = *reinterpret_cast<const u32x4*>(codes[r] + (int64_t)b * 64);
            pr[r] = *reinterpret_cast<const PairWords<G>*>(pairs[r] + (int64_t)b * (4 * kGroups));
        }
#pragma unroll
        for (uint32_t i = 0; i < TT; ++i)
#pragma unroll
            for (uint32_t m = 0; m < 4; ++m) {
                a[i][m] = u32x4{};
                if (there[i] && b * kBlock + m * 32 + q * 8 < p.w[0].n_in) a[i][m] = *reinterpret_cast<const u32x4*>(x[i] + (int64_t)b * 256 + m * 64);
            }
#pragma unroll
        for (uint32_t g = 0; g < kGroups; ++g) {
            f32x4 ones[TT];
#pragma unroll
            for (uint32_t i = 0; i < TT; ++i) {
                ones[i] = f32x4{};
#pragma unroll
                for (uint32_t m = 0; m < kSteps; ++m) {
                    const uint32_t one = kOnes<E>;
                    ones[i] = mfma16<E>(a[i][g * kSteps + m], u32x4{one, one, one, one}, ones[i]);
                }
            }
#pragma unroll
            for (uint32_t r = 0; r < R; ++r) {
                f32x4 s[TT] = {};
#pragma unroll
                for (uint32_t m = 0; m < kSteps; ++m) {
                    const u32x4 w = codes16<E>(c[r][g * kSteps + m]);
#pragma unroll
                    for (uint32_t i = 0; i < TT; ++i) s[i] = mfma16<E>(a[i][g * kSteps + m], w, s[i]);
                }
                const float step = low16<E>(pr[r][g]), low = fmaf(-16.0f, step, high16<E>(pr[r][g]));
#pragma unroll
                for (uint32_t i = 0; i < TT; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) acc[r][i][j] = fmaf(step, s[i][j], fmaf(low, ones[i][j], acc[r][i][j]));
            }
        }
    }
#pragma unroll
    for (uint32_t r = 0; r < R; ++r)
#pragma unroll
        for (uint32_t i = 0; i < TT; ++i) sums[wave][r * TT + i][lane] = acc[r][i];
    __syncthreads();
    for (uint32_t u = wave; u < kOuts * TT; u += kFewWaves) {
        f32x4 a{}, b{};
#pragma unroll
        for (uint32_t w = 0; w < kFewWaves; ++w) {
            a += sums[w][u][lane];
            if (kGated) b += sums[w][u + kOuts * TT][lane];
        }
        const uint32_t n = n0 + u / TT * 16 + col, t = t0 + u % TT * 16 + q * 4;
        if (n < p.w[0].n_out)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (t + j < p.n_tokens) finish<E, kGated>(p, t + j, n, a[j], b[j]);
    }
}

}  // namespace

#endif  // LI_FEW_HPP
