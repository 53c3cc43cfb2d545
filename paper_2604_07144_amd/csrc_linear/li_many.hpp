// Products of many rows with weights in 4 bits: whole prompts, and chunks of them.  The matrix units bound this.
//
// Mathematics as in the kernel of few rows.  A workgroup has TT tiles of 16 tokens and eight wavefronts side by side over the
// outputs, four tiles of 16 each, so an operand of x that is read from LDS meets four of weights, and codes are unpacked once for
// all tokens.  Blocks of 128 columns follow one another; the next one is on its way to the other half of LDS while the present
// one is worked on.  The sums X of x, which all outputs share, are taken by a wavefront for each tile of tokens.
//
// A tile of 16 tokens and 64 outputs is 16 products (256 cycles) and 32 multiply-adds that scale them, which the compiler puts between the
// next tile's products.  Measured, gated 14336 outputs of 4096 inputs, bf16, TFLOP/s (a large product of the library 1130 to 1160): 4999 tokens
// 1000 to 1060 from card to card with groups of 128 (under a kernel trace 956); 2048 tokens 924 with groups of 128, 758 of 64, 597 of 32,
// which scale two and four times as often.  Without the loads 20 % less time, without the scaling 4 %; weights two blocks ahead in a ring of
// three changed nothing.  Results leave four outputs a thread: one at a time 300 tokens, 2048 outputs of 1024 inputs, took 20.1 us for 16.4 (14.7
// since the parts are joined four at a time too).
#ifndef LI_MANY_HPP
#define LI_MANY_HPP

#include "li_few.hpp"

namespace {

constexpr uint32_t kManyWaves = 8, kManyTiles = 4;           // tiles of outputs of a wavefront

template <uint32_t G, uint32_t TT> struct ManyShape {
    static constexpr uint32_t kWords = kBlock / G, kPairLoads = kWords;                     // 64 rows of so many words
    static constexpr uint32_t kX = TT * 4096, kCodes = kManyWaves * kManyTiles * 1024, kPairs = kManyWaves * kPairLoads * 256;
    static constexpr uint32_t kStage = kX + kCodes + kPairs, kLds = 2 * kStage + kWords * TT * 64;
    // (lo - 16 step) X by a product in 32 bits, as in the kernel of few rows.  Gated 14336 of 4096, 2048 tokens, off / on: groups of 32 866 / 828 us,
    // of 64 645 / 698.
    static constexpr bool kLowByMatrix = G == 32;
    static constexpr uint32_t kXLoads = (TT + 1) / 2;                                       // of a wavefront; the last may have fewer
};

template <typename E, uint32_t G, uint32_t TT, bool kGated, bool kWhole>
__global__ __launch_bounds__(kManyWaves * kLanes) void k_linear_many(const LinearParams p, const uint32_t out_tiles, const uint32_t token_tiles) {
    using Shape = ManyShape<G, TT>;
    constexpr uint32_t R = kManyTiles, kOuts = kGated ? R / 2 : R, kWords = Shape::kWords, kSteps = G / 32;
    __shared__ __attribute__((aligned(16))) char lds[Shape::kLds];
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes), col = lane % 16, q = lane / 16;
    // Workgroups that run next to each other on an XCD (every eighth) have the same outputs, eight tiles of tokens of them.
    const uint32_t n_ids = out_tiles * token_tiles, all = n_ids * p.n_parts, xcd = blockIdx.x % 8, flat = xcd * (all / 8) + min(xcd, all % 8) + blockIdx.x / 8;
    const uint32_t part = flat / n_ids, at = flat % n_ids;
    constexpr uint32_t kBand = 8;
    const uint32_t band = at / (kBand * out_tiles), in_band = at - band * kBand * out_tiles, height = min(kBand, token_tiles - band * kBand);
    const uint32_t t0 = (band * kBand + in_band % height) * (TT * 16), n0 = (in_band / height * kManyWaves + wave) * (kOuts * 16);
    const uint32_t begin = part * p.part_blocks, end = min(begin + p.part_blocks, p.w[0].blocks);

    const uint32_t lrow = lane / 4, lpiece = turned(lrow, lane % 4), slot = (col * 4 + turned(col, q)) * 16;
    const char *codes[R], *pairs[Shape::kPairLoads], *x[Shape::kXLoads];
#pragma unroll
    for (uint32_t r = 0; r < R; ++r) {
        const Weights& w = p.w[kGated ? r / kOuts : 0];
        codes[r] = w.codes + (int64_t)min(n0 + (kGated ? r % kOuts : r) * 16 + lrow, w.n_out - 1) * w.code_stride + (int64_t)begin * 64 + lpiece * 16;
    }
#pragma unroll
    for (uint32_t i = 0; i < Shape::kPairLoads; ++i) {
        const uint32_t e = i * kLanes + lane, r = e / (16 * kWords), row = e / kWords % 16;
        const Weights& w = p.w[kGated ? r / kOuts : 0];
        pairs[i] = w.pairs + (int64_t)min(n0 + (kGated ? r % kOuts : r) * 16 + row, w.n_out - 1) * w.pair_stride + (int64_t)begin * (4 * kWords) + e % kWords * 4;
    }
    // pieces of x, 32 columns of a tile, in order over the wavefronts
#pragma unroll
    for (uint32_t j = 0; j < Shape::kXLoads; ++j) {
        const uint32_t f = wave * Shape::kXLoads + j;
        x[j] = p.x + (int64_t)min(t0 + f / 4 * 16 + lrow, p.n_tokens - 1) * p.x_stride + (int64_t)begin * 256 + f % 4 * 64 + lpiece * 16;
    }
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds;
    auto load = [&](uint32_t b, uint32_t half) {
        const uint32_t to = base + half * Shape::kStage;
#pragma unroll
        for (uint32_t r = 0; r < R; ++r) {
            load_to_lds<0>(codes[r], to + Shape::kX + (wave * R + r) * 1024);
            codes[r] += 64;
        }
#pragma unroll
        for (uint32_t i = 0; i < Shape::kPairLoads; ++i) {
            load4_to_lds(pairs[i], to + Shape::kX + Shape::kCodes + (wave * Shape::kPairLoads + i) * 256);
            pairs[i] += 4 * kWords;
        }
#pragma unroll
        for (uint32_t j = 0; j < Shape::kXLoads; ++j) {
            const uint32_t f = wave * Shape::kXLoads + j;
            if (TT % 2 && f >= TT * 4) break;
            const bool in = kWhole || b * kBlock + f % 4 * 32 + lpiece * 8 < p.w[0].n_in;
            load_to_lds<0>(in ? x[j] : (const char*)&kZeros, to + f * 1024);
            x[j] += 256;
        }
    };
    const Unpack<E> unpack;
    f32x4 acc[R][TT] = {};
    float* const sums = reinterpret_cast<float*>(lds + 2 * Shape::kStage);                  // X: [group][token], or [tile][lane]
    load(begin, 0);
    for (uint32_t b = begin; b < end; ++b) {
        const uint32_t half = (b - begin) % 2;
        const char* const in = lds + half * Shape::kStage;
        wait_loads<0>();
        __syncthreads();
        if (b + 1 < end) load(b + 1, half ^ 1);
        if constexpr (Shape::kLowByMatrix) {
            if (wave < TT) {
                f32x4 s = {};
#pragma unroll
                for (uint32_t m = 0; m < 4; ++m) s = sum_of_group<E>(m, *reinterpret_cast<const u32x4*>(in + (wave * 4 + m) * 1024 + slot), col, s);
                sums[wave * kLanes + lane] = s[0];
            }
        } else if (wave < TT) {
#pragma unroll
            for (uint32_t g = 0; g < kWords; ++g) {
                const uint32_t one = kOnes<E>;
                f32x4 s = {};
#pragma unroll
                for (uint32_t m = g * kSteps; m < (g + 1) * kSteps; ++m)
                    s = mfma16<E>(*reinterpret_cast<const u32x4*>(in + (wave * 4 + m) * 1024 + slot), u32x4{one, one, one, one}, s);
                if (col == 0) *reinterpret_cast<f32x4*>(sums + g * (TT * 16) + wave * 16 + q * 4) = s;
            }
        }
        u32x4 w[R][4];
        float step[R][kWords], low[R][kWords], low4[R];
#pragma unroll
        for (uint32_t r = 0; r < R; ++r) {
            const u32x4 c = *reinterpret_cast<const u32x4*>(in + Shape::kX + (wave * R + r) * 1024 + slot);
            const PairWords<G> pr = *reinterpret_cast<const PairWords<G>*>(in + Shape::kX + Shape::kCodes + wave * Shape::kPairLoads * 256 + (r * 16 + col) * kWords * 4);
#pragma unroll
            for (uint32_t m = 0; m < 4; ++m) w[r][m] = unpack(c[m]);
#pragma unroll
            for (uint32_t g = 0; g < kWords; ++g) step[r][g] = low16<E>(pr[g]), low[r][g] = fmaf(-16.0f, step[r][g], high16<E>(pr[g]));
            if constexpr (Shape::kLowByMatrix) {
                const uint32_t word = *reinterpret_cast<const uint32_t*>(in + Shape::kX + Shape::kCodes + wave * Shape::kPairLoads * 256 + ((r * 16 + col) * kWords + q) * 4);
                low4[r] = fmaf(-16.0f, low16<E>(word), high16<E>(word));
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < TT; ++i) {
            u32x4 a[4];
#pragma unroll
            for (uint32_t m = 0; m < 4; ++m) a[m] = *reinterpret_cast<const u32x4*>(in + (i * 4 + m) * 1024 + slot);
#pragma unroll
            for (uint32_t g = 0; g < kWords; ++g) {
                f32x4 s[R] = {};
#pragma unroll
                for (uint32_t m = g * kSteps; m < (g + 1) * kSteps; ++m)
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) s[r] = mfma16<E>(a[m], w[r][m], s[r]);
                if (i == 0 && g == 0) __syncthreads();                                      // X is there; codes are unpacked beside the first products
                if constexpr (Shape::kLowByMatrix) {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r)
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) acc[r][i][j] = fmaf(step[r][g], s[r][j], acc[r][i][j]);
                    if (g + 1 == kWords) {
                        const float xs = sums[i * kLanes + lane];
#pragma unroll
                        for (uint32_t r = 0; r < R; ++r) acc[r][i] = mfma4(xs, low4[r], acc[r][i]);
                    }
                    continue;
                }
                const f32x4 xs = *reinterpret_cast<const f32x4*>(sums + g * (TT * 16) + i * 16 + q * 4);
#pragma unroll
                for (uint32_t r = 0; r < R; ++r)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) acc[r][i][j] = fmaf(step[r][g], s[r][j], fmaf(low[r][g], xs[j], acc[r][i][j]));
            }
        }
    }
    // Results go through LDS, a tile of tokens at a time, so that a thread has four neighbouring outputs, and neighbouring threads the next.
    constexpr uint32_t kWide = kManyWaves * kOuts * 16, kRow = kWide * (kGated ? 2 : 1) + 4;
    const bool at_once = p.n_parts == 1 ? four_results(p) : four_sums(p);
    float* const out = reinterpret_cast<float*>(lds);                                       // [16 tokens][output, of both matrices]
#pragma unroll
    for (uint32_t i = 0; i < TT; ++i) {
        __syncthreads();
#pragma unroll
        for (uint32_t r = 0; r < R; ++r)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) out[(q * 4 + j) * kRow + (kGated && r >= kOuts ? kWide : 0) + wave * kOuts * 16 + r % kOuts * 16 + col] = acc[r][i][j];
        __syncthreads();
#pragma unroll 1
        for (uint32_t e = threadIdx.x * 4; e < 16 * kWide; e += kManyWaves * kLanes * 4) {
            const uint32_t t = t0 + i * 16 + e / kWide, n = n0 - wave * kOuts * 16 + e % kWide;
            const float* from = out + e / kWide * kRow + e % kWide;
            const f32x4 a = *reinterpret_cast<const f32x4*>(from), b = *reinterpret_cast<const f32x4*>(from + (kGated ? kWide : 0));
            if (t < p.n_tokens && n < p.w[0].n_out) put4<E, kGated>(p, at_once, part, n, t, a, b);
        }
    }
}

}  // namespace

#endif  // LI_MANY_HPP
