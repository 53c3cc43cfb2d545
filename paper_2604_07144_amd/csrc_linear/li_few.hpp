// Products of few rows with weights in 4 bits: the steps of a replica's slots.  The weights are read once and the memory
// bounds it, so everything else has to stay below that.
//
// y[t][n] = sum over groups g of  step[n][g] S[t][n] + (lo[n][g] - 16 step[n][g]) X[t],   S = sum x (16 + code),  X = sum x
// over the group's columns.  S and X come from the matrix units, with tokens as rows and outputs as columns of 16x16x32 tiles: the
// factors 16 + code are exact in the 16-bit type and so no weight is rounded; X is the product with a column of ones.  A
// lane then has four tokens of one output, whose pair is the lane's own.
//
// The lanes of an operand that lie next to each other are 16 different rows, and a load takes as many turns as it has such
// places.  So codes, pairs and x come straight to LDS, lanes next to each other to a row's bytes next to each other, and from there to the
// operands.  Several steps are on their way at once, in a ring.
//
// A workgroup's wavefronts are kAside that lie side by side over the outputs and share x (gated: half of them over gate, half over
// up), times kDeep that take the blocks of 128 columns in turns; these meet in LDS at the end.  With few outputs the inputs are cut
// into parts besides, whose sums k_join_parts adds up.
//
// What bounds it: up to 16 tokens what a CU brings to LDS, codes from memory and x and pairs from the L2 (about 9 TB/s over the chip, where
// loads that go to registers row by row reach a third); from 32 tokens on that and the vector unit in turn, as the wavefronts that share
// x keep step.  Measured, groups of 128, bf16, us of a graph's steps with weights that come from memory (in brackets the bytes
// at the 5.1 TB/s of a copy): one token, 4096 outputs of 4096 inputs 4.9 (1.7); 8 tokens, gated 14336 of 4096 20 (12.2), 128256 of 4096 74 (55); 64
// tokens, 10240 of 8192 in fp16 32 (9.1).  With weights that the chip's caches hold: the gated product 15.7, the last one 26.7.
#ifndef LI_FEW_HPP
#define LI_FEW_HPP

#include "li_common.hpp"

namespace {

template <typename E> constexpr uint32_t kOnes = std::is_same_v<E, bf16> ? 0x3F803F80u : 0x3C003C00u;

// c with the sums over 32 columns of x added, in the lanes that have group g: c[0] is of group lane / 16 and token lane % 16.  (Ones in the rows of
// those lanes only; x is the other operand here.)
template <typename E> __device__ __forceinline__ f32x4 sum_of_group(uint32_t g, u32x4 x, uint32_t col, f32x4 c) {
    const uint32_t one = col / 4 == g ? kOnes<E> : 0;
    return mfma16<E>(u32x4{one, one, one, one}, x, c);
}

// Of a kernel for up to T tokens.  kHeld: all of x is brought to LDS first, and stays; there is room for kHeldBytes of it.
constexpr uint32_t kHeldBytes = 64 * 1024;
template <uint32_t G, uint32_t T, bool kGated, bool kHeld> struct FewShape {
    static constexpr uint32_t kWaves = !kHeld && (T == 8 || T == 16) ? 8 : 16, kTiles = T <= 16 ? 1 : T / 16, kAside = T <= 16 ? (kGated ? 2 : 1) : T / 8;
    static constexpr uint32_t kDeep = kWaves / kAside, kOuts = kGated ? kAside / 2 : kAside;     // kOuts: tiles of 16 outputs side by side
    static constexpr uint32_t kWords = kBlock / G, kPairLoads = (16 * kWords + kLanes - 1) / kLanes;
    // x of a step and deep index: kTiles times 4 KiB, or of fewer than 16 tokens as many rows of 256 bytes; in loads of 1 KiB
    static constexpr uint32_t kRows = T < 16 ? T : 16, kXBytes = kTiles * kRows * 256, kXLoads = kHeld ? 0 : (kXBytes / 1024 + kAside - 1) / kAside;
    static constexpr uint32_t kLoads = 1 + kPairLoads + kXLoads;                                    // of a wavefront and step
    static constexpr uint32_t kX = kHeld ? 0 : kDeep * kXBytes, kCodes = kWaves * 1024, kPairs = kWaves * kPairLoads * 256, kStage = kX + kCodes + kPairs;
    static constexpr uint32_t kSumLanes = T < 16 ? T * 4 : kLanes;                                  // that have tokens
    static constexpr bool kOneTile = T > 16;                                                        // a workgroup has one tile of outputs, not several
    static constexpr uint32_t kSums = kWaves * kTiles * kSumLanes * 16, kApart = (kOneTile ? 0 : kSums) + (kHeld ? kHeldBytes : 0);   // in the ring, or beside it
    // X of a tile of tokens is taken by one of the wavefronts that share x, where that spares more than the barrier it needs: [deep][group][token].
    // Gated, 14336 outputs of 4096 inputs, groups of 128, each its own / shared: 64 tokens 38 / 35 us, 32 tokens 29 / 30.  Groups of 32 and 64
    // have (lo - 16 step) X on the matrix units too, in 32 bits and four groups at once, which spares half of the multiply-adds; X is then
    // [deep][tile][lane], of group lane / 16 and token lane % 16.  64 tokens, gated 14336 of 8192, groups of 32: 86 / 77 us; 14336 of 4096,
    // groups of 64 40.4 / 38.3, of 128 35.7 / 38.6.
    static constexpr bool kShareX = kTiles == 4, kLowByMatrix = kShareX && G <= 64;
    static constexpr uint32_t kXSums = !kShareX ? 0 : kDeep * kTiles * (kLowByMatrix ? kLanes * 4 : kWords * 64);
    static constexpr uint32_t kFit = (160 * 1024 - kApart - kXSums) / kStage, kRing = kFit < 8 ? kFit : 8;
    static constexpr uint32_t kLds = kApart + kXSums + (kRing * kStage > kSums ? kRing * kStage : kSums);
};

// The wait for all but the `keep` newest steps of loads of `kLoads` each.
template <uint32_t kLoads, uint32_t kMost> __device__ __forceinline__ void wait_steps(uint32_t keep) {
    if constexpr (kMost > 0) {
        if (keep < kMost) return wait_steps<kLoads, kMost - 1>(keep);
    }
    wait_loads<kLoads * kMost>();
}

template <typename E, uint32_t G, uint32_t T, bool kGated, bool kHeld, bool kWhole>
__global__ __launch_bounds__((FewShape<G, T, kGated, kHeld>::kWaves * kLanes)) void k_linear_few(const LinearParams p) {
    using Shape = FewShape<G, T, kGated, kHeld>;
    constexpr uint32_t TT = Shape::kTiles, kAside = Shape::kAside, kDeep = Shape::kDeep, kOuts = Shape::kOuts, kGroups = kBlock / G, kSteps = G / 32;
    constexpr uint32_t kRing = Shape::kRing, kWords = Shape::kWords, kRows = Shape::kRows;
    __shared__ __attribute__((aligned(16))) char lds[Shape::kLds];
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes), col = lane % 16, q = lane / 16;
    const uint32_t aside = wave % kAside, deep = wave / kAside;
    const uint32_t begin = blockIdx.z * p.part_blocks, end = min(begin + p.part_blocks, p.w[0].blocks), steps = (end - begin + kDeep - 1) / kDeep;
    const Weights& w = p.w[kGated ? aside / kOuts : 0];

    // An even share of the outputs for each workgroup, and of those for each tile and wavefront: `rows` of them, which need not be the
    // 16 that there is room for.
    const uint32_t n_begin = (uint32_t)((uint64_t)w.n_out * blockIdx.x / gridDim.x), n_end = (uint32_t)((uint64_t)w.n_out * (blockIdx.x + 1) / gridDim.x);
    const uint32_t tiles = Shape::kOneTile ? 1 : (n_end - n_begin + kOuts * 16 - 1) / (kOuts * 16);
    const uint32_t rows = (n_end - n_begin + tiles * kOuts - 1) / (tiles * kOuts);

    // A workgroup's steps begin at one of their own: rows are often some power of two apart, and all workgroups would come to the same
    // memory channels at once.
    const uint32_t first_step = blockIdx.x / 8 % steps;
    uint32_t fill = 0, use = 0, load_step = first_step, load_left = steps, load_tile = 0;

    // Codes: a lane has 16 bytes of row lane / 4.
    const uint32_t slot = (col * 4 + turned(col, q)) * 16;
    const char *codes, *pairs[Shape::kPairLoads];
    auto enter = [&] {                                     // the rows of tile load_tile; beyond the wavefront's its last one again, not kept
        const uint32_t n0 = n_begin + (load_tile * kOuts + aside % kOuts) * rows, n1 = min(min(n0 + rows, n_end), w.n_out) - 1;
        codes = w.codes + (int64_t)min(n0 + lane / 4, n1) * w.code_stride + turned(lane / 4, lane % 4) * 16;
#pragma unroll
        for (uint32_t i = 0; i < Shape::kPairLoads; ++i) {
            const uint32_t e = min(i * kLanes + lane, 16 * kWords - 1);
            pairs[i] = w.pairs + (int64_t)min(n0 + e / kWords, n1) * w.pair_stride + e % kWords * 4;
        }
    };
    enter();
    // x: rows of 64 (fewer than 16 tokens) or 128 bytes, kRows of them for each 32 or 64 columns of a tile
    constexpr uint32_t kRowLanes = T < 16 ? 4 : 8;
    const char* x[Shape::kXLoads + 1];
    uint32_t x_col[Shape::kXLoads + 1];                    // first column of a lane's piece in the block
    uint32_t x_slot[2];                                    // where the lane's operand of 32 columns lies, in those, of even and odd ones
#pragma unroll
    for (uint32_t j = 0; j < Shape::kXLoads; ++j) {
        const uint32_t e = (aside * Shape::kXLoads + j) * kLanes + lane;                    // piece of 16 bytes of all of the step's
        const uint32_t in = e % (TT * kRows * 16), row = in / kRowLanes % kRows, part = in / kRowLanes / kRows;
        if constexpr (T < 16) {
            x_col[j] = part * 32 + turned(row, in % 4) * 8;
            x[j] = p.x + (int64_t)min(row, p.n_tokens - 1) * p.x_stride + x_col[j] * 2;
        } else {                                           // [tile][half of the columns][row]
            const uint32_t at = part / 2 * 16 + row;
            x_col[j] = part % 2 * 64 + wide_turned(row, in % 8) * 8;
            x[j] = p.x + (int64_t)min(at, p.n_tokens - 1) * p.x_stride + x_col[j] * 2;
        }
    }
    if constexpr (T < 16) x_slot[0] = x_slot[1] = (col % T * 4 + turned(col % T, q)) * 16;
    else x_slot[0] = col * 128 + wide_turned(col, q) * 16, x_slot[1] = col * 128 + wide_turned(col, 4 + q) * 16;

    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)lds;
    const uint32_t base_x = base + deep * Shape::kXBytes + aside * Shape::kXLoads * 1024 % Shape::kXBytes, base_codes = base + Shape::kX + wave * 1024,
                   base_pairs = base + Shape::kX + Shape::kCodes + wave * Shape::kPairLoads * 256;
    const uint32_t held = base + Shape::kLds - kHeldBytes;
    if constexpr (kHeld) {                                 // [block] as a step's
        static_assert(T < 16);
        const uint32_t pieces = (end - begin) * kRows * 16;
        for (uint32_t e0 = wave * kLanes; e0 < pieces; e0 += Shape::kWaves * kLanes) {
            const uint32_t e = min(e0 + lane, pieces - 1), b = begin + e / (kRows * 16), in = e % (kRows * 16), row = in / 4 % kRows;
            const uint32_t c = b * kBlock + in / 4 / kRows * 32 + turned(row, in % 4) * 8;
            const bool there = kWhole || c < p.w[0].n_in;
            load_to_lds<0>(there ? p.x + (int64_t)min(row, p.n_tokens - 1) * p.x_stride + 2ull * c : (const char*)&kZeros, held + e0 * 16);
        }
    }
    auto load = [&] {
        const uint32_t b = min(begin + load_step * kDeep + deep, end - 1);                  // behind the last block: the last one, not added
        load_to_lds<0>(codes + (uint64_t)b * 64, base_codes + fill);
#pragma unroll
        for (uint32_t i = 0; i < Shape::kPairLoads; ++i) load4_to_lds(pairs[i] + (uint64_t)b * (4 * kWords), base_pairs + fill + i * 256);
#pragma unroll
        for (uint32_t j = 0; j < Shape::kXLoads; ++j) {
            const bool in = kWhole || b * kBlock + x_col[j] < p.w[0].n_in;
            load_to_lds<0>(in ? x[j] + (uint64_t)b * 256 : (const char*)&kZeros, base_x + fill + j * 1024);
        }
        fill = fill == (kRing - 1) * Shape::kStage ? 0 : fill + Shape::kStage;
        load_step = load_step + 1 == steps ? 0 : load_step + 1;
        if (--load_left == 0) {
            load_left = steps;
            if (++load_tile < tiles) enter();
        }
    };
    uint32_t use_step = first_step;
    const Unpack<E> unpack;
    f32x4 acc[TT] = {};
    float* const x_sums = reinterpret_cast<float*>(lds + Shape::kLds - Shape::kXSums - (kHeld ? kHeldBytes : 0));
    auto add = [&] {
        const char* const at = lds + use;
        const char* const at_x = kHeld ? lds + (Shape::kLds - kHeldBytes) + (use_step * kDeep + deep) * Shape::kXBytes : at + deep * Shape::kXBytes;
        const u32x4 c = *reinterpret_cast<const u32x4*>(at + Shape::kX + wave * 1024 + slot);
        const PairWords<G> pr = *reinterpret_cast<const PairWords<G>*>(at + Shape::kX + Shape::kCodes + wave * Shape::kPairLoads * 256 + col * kWords * 4);
        float* const sums = x_sums + deep * (kGroups * TT * 16) + q * 4;
        if constexpr (Shape::kLowByMatrix) {
            float* const xs = x_sums + deep * (TT * kLanes) + lane;
            if (aside < TT) {
                f32x4 mine = {};
#pragma unroll
                for (uint32_t m = 0; m < 4; ++m) mine = sum_of_group<E>(m / kSteps, *reinterpret_cast<const u32x4*>(at_x + aside * 4096 + m / 2 * 2048 + x_slot[m % 2]), col, mine);
                xs[aside * kLanes] = mine[0];
            }
#pragma unroll
            for (uint32_t g = 0; g < kGroups; ++g) {
                f32x4 s[TT] = {};
#pragma unroll
                for (uint32_t m = g * kSteps; m < (g + 1) * kSteps; ++m) {
                    const u32x4 v = unpack(c[m]);
#pragma unroll
                    for (uint32_t i = 0; i < TT; ++i) s[i] = mfma16<E>(*reinterpret_cast<const u32x4*>(at_x + i * 4096 + m / 2 * 2048 + x_slot[m % 2]), v, s[i]);
                }
                const float step = low16<E>(pr[g]);
#pragma unroll
                for (uint32_t i = 0; i < TT; ++i)
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) acc[i][j] = fmaf(step, s[i][j], acc[i][j]);
            }
            __syncthreads();
            const uint32_t word = *reinterpret_cast<const uint32_t*>(at + Shape::kX + Shape::kCodes + wave * Shape::kPairLoads * 256 + (col * kWords + q % kWords) * 4);
            const float low = fmaf(-16.0f, low16<E>(word), high16<E>(word));
#pragma unroll
            for (uint32_t i = 0; i < TT; ++i) acc[i] = mfma4(xs[i * kLanes], low, acc[i]);
            return;
        }
        const uint32_t one = kOnes<E>;
        const u32x4 all_ones = {one, one, one, one};
        if constexpr (Shape::kShareX) {
            if (aside < TT) {
#pragma unroll
                for (uint32_t g = 0; g < kGroups; ++g) {
                    f32x4 ones = {};
#pragma unroll
                    for (uint32_t m = g * kSteps; m < (g + 1) * kSteps; ++m)
                        ones = mfma16<E>(*reinterpret_cast<const u32x4*>(at_x + aside * 4096 + m / 2 * 2048 + x_slot[m % 2]), all_ones, ones);
                    if (col == 0) *reinterpret_cast<f32x4*>(sums + (g * TT + aside) * 16) = ones;
                }
            }
        }
#pragma unroll
        for (uint32_t g = 0; g < kGroups; ++g) {
            f32x4 ones[TT] = {}, s[TT] = {};
#pragma unroll
            for (uint32_t m = g * kSteps; m < (g + 1) * kSteps; ++m) {
                u32x4 a[TT];
#pragma unroll
                for (uint32_t i = 0; i < TT; ++i) a[i] = *reinterpret_cast<const u32x4*>(at_x + (T < 16 ? m * (kRows * 64) : i * 4096 + m / 2 * 2048) + x_slot[m % 2]);
                if constexpr (!Shape::kShareX)
#pragma unroll
                    for (uint32_t i = 0; i < TT; ++i) ones[i] = mfma16<E>(a[i], all_ones, ones[i]);
                const u32x4 v = unpack(c[m]);
#pragma unroll
                for (uint32_t i = 0; i < TT; ++i) s[i] = mfma16<E>(a[i], v, s[i]);
            }
            if constexpr (Shape::kShareX) {
                if (g == 0) __syncthreads();
#pragma unroll
                for (uint32_t i = 0; i < TT; ++i) ones[i] = *reinterpret_cast<const f32x4*>(sums + (g * TT + i) * 16);
            }
            const float step = low16<E>(pr[g]), low = fmaf(-16.0f, step, high16<E>(pr[g]));
#pragma unroll
            for (uint32_t i = 0; i < TT; ++i)
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) acc[i][j] = fmaf(step, s[i][j], fmaf(low, ones[i][j], acc[i][j]));
        }
    };
    uint32_t use_left = steps, use_tile = 0;
    auto leave = [&] {                                     // a tile is done: its sums meet, and each thread finishes single outputs
        constexpr uint32_t kWide = Shape::kSumLanes, kTile = kWide * 4;
        float* const sums = reinterpret_cast<float*>(lds + (Shape::kOneTile ? 0 : kRing * Shape::kStage));          // [wavefront][tile][lane][4]
        __syncthreads();
        if (lane < kWide)
#pragma unroll
            for (uint32_t i = 0; i < TT; ++i) *reinterpret_cast<f32x4*>(sums + (wave * TT + i) * kTile + lane * 4) = acc[i];
#pragma unroll
        for (uint32_t i = 0; i < TT; ++i) acc[i] = f32x4{};
        __syncthreads();
#pragma unroll 1
        for (uint32_t e = threadIdx.x; e < kOuts * TT * kTile; e += Shape::kWaves * kLanes) {
            const uint32_t u = e / kTile, w0 = u / TT, i = u % TT, l = e % kTile / 4;
            const float* from = sums + (w0 * TT + i) * kTile + e % kTile;
            float s = 0.0f, s2 = 0.0f;
#pragma unroll
            for (uint32_t d = 0; d < kDeep; ++d) {
                s += from[d * kAside * TT * kTile];
                if (kGated) s2 += from[(d * kAside + kOuts) * TT * kTile];
            }
            const uint32_t n0 = n_begin + (use_tile * kOuts + w0) * rows, n1 = min(min(n0 + rows, n0 + 16), n_end), n = n0 + l % 16, t = i * 16 + l / 16 * 4 + e % 4;
            if (n < n1 && t < p.n_tokens) put<E, kGated>(p, blockIdx.z, n, t, s, s2);
        }
        use_left = steps, ++use_tile;
    };
    auto arrived = [&] {
        if constexpr (kAside > 1 && !kHeld) __syncthreads();
        else wait_lds();                                   // what is loaded next comes to where the last step was read
    };
    const uint32_t all = tiles * steps;
    for (uint32_t i = 0; i < min(all, kRing - 1); ++i) load();
    if constexpr (kHeld) {                                 // x was first: what came after it may still be on its way
        wait_steps<Shape::kLoads, kRing - 1>(min(all, kRing - 1));
        __syncthreads();
    }
    for (uint32_t i = 0; i < all; ++i) {
        wait_steps<Shape::kLoads, kRing - 2>(min(all - 1 - i, kRing - 2));
        arrived();
        if (i + kRing - 1 < all) load();
        if (begin + use_step * kDeep + deep < end) add();
        else if constexpr (Shape::kShareX) __syncthreads();                                  // the one in add
        use = use == (kRing - 1) * Shape::kStage ? 0 : use + Shape::kStage;
        use_step = use_step + 1 == steps ? 0 : use_step + 1;
        if (--use_left == 0) leave();
    }
}

// Sums of the parts, in order; four outputs a thread.  (Parts are asked for only where all sums of one are fewer than 2^32.)
template <typename E, bool kGated> __global__ __launch_bounds__(256) void k_join_parts(const LinearParams p) {
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, n_out = p.w[0].n_out, fours = (n_out + 3) / 4, t = at / fours, n = at % fours * 4;
    if (t >= p.n_tokens) return;
    const uint64_t width = (kGated ? 2 : 1) * (uint64_t)n_out;
    const float* from = p.parts + (uint64_t)t * width + n;
    const bool at_once = four_sums(p);
    auto four = [&](const float* x) {
        if (at_once) return *reinterpret_cast<const f32x4*>(x);
        f32x4 r = {};
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (n + j < n_out) r[j] = x[j];
        return r;
    };
    f32x4 a = {}, b = {};
    for (uint32_t z = 0; z < p.n_parts; ++z, from += (uint64_t)p.n_tokens * width) {
        a += four(from);
        if (kGated) b += four(from + n_out);
    }
    finish4<E, kGated>(p, four_results(p), t, n, a, b);
}

}  // namespace

#endif  // LI_FEW_HPP
