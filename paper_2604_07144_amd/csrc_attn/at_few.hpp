// Attention of few rows over a long cache: a sequence's new tokens times the query heads of one key/value head make at
// most 32 rows (one new token: the A / K heads that share a key/value head).
//
// Mathematics: one pass over the keys with the running maximum m and sum l of a softmax, o = sum_j e^{s_j - m} v_j
// scaled down whenever m grows; parts of the key axis are joined by their (m, l, o).
//
// Every key and value is read once, for all rows that share it, so memory bounds this: per position and key/value head
// 4 * D bytes (16 bits) against 4 * D * rows operations.  What follows from it:
//  - Work is dealt out evenly whatever the lengths: the tiles (32 keys) of all sequences and heads are one line, and each
//    of a fixed number of wavefronts takes an equal piece of it, which may begin and end inside a sequence.  Every
//    workgroup works the line out from the lengths on the device; a second kernel joins what was cut.
//    Few and short sequences are not cut: eight wavefronts share each (sequence, head) and join their parts in LDS.
//  - Wavefronts go their own way, without a barrier, and have the next 32 keys and values on their way to registers while
//    they work on the present ones.  Loads take whole rows, 16 bytes a lane; the exchange into the operand layouts of the
//    matrix units is LDS's, which has bandwidth to spare here.
//  - Products run as S^T = K Q^T and O^T = V^T P^T: rows of queries are columns there, so the running maximum of a row
//    lives in the lanes of one column, and the weights leave the first product in exactly the registers from which the
//    second takes them.  Values come out of LDS transposed.
//  - In 4 bits nothing is decoded: codes enter the matrix units as they are.  A 16-bit floating-point number whose bits are
//    a small whole number n has the value n * 2^-133 (bf16) or n * 2^-24 (fp16), which the matrix units honour, so masking
//    the two halves of bytes is all the conversion there is.  Scores are step * (codes . q) + lo * (sum of q), per group of
//    64 channels; for values each weight is multiplied by the key's step before its one rounding, and lo is summed apart
//    in 32 bits.  So neither keys nor values are rounded at all.
//
// Measured, one token, 128 channels, bf16: 64 sequences of 4096 to 8192, 32 heads of their own 6.0 TB/s in 16 bits and 5.2 in 4;
// with 32 heads on 8 5.6 and 4.7.  Shorter batches pay 5 us for the launch that joins, and 4 bits are bound by instructions
// there: about 380 a tile of 32 keys, 45 % of what the SIMDs give out, so 64 slots with bimodal lengths take 39 us
// (2.9 TB/s) where 16 bits take 88 (4.6).
#ifndef AT_FEW_HPP
#define AT_FEW_HPP

#include "at_parts.hpp"

namespace {

constexpr uint32_t kLineWaves = 4, kLineThreads = kLineWaves * kLanes;   // of a workgroup that works on the line
constexpr uint32_t kFewRows = 32;        // most rows (new tokens times shared heads) of the kernel
constexpr uint32_t kFewSeqs = 256;       // most sequences of a launch (a thread each): the line of their tiles stands in LDS
constexpr uint32_t kFewEnter = 3;        // what beginning with a sequence costs a wavefront, in tiles

__device__ __forceinline__ u32x2 lds_transposed8(const char* at) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2* Ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((Ptr)(at)));
}

template <typename E> constexpr int kCodeExponent = std::is_same_v<E, bf16> ? 133 : 24;      // a code n as bits: n * 2^-this
template <typename E> constexpr int kOperandExponent = std::is_same_v<E, bf16> ? 125 : 14;   // the other operand is brought below 2^this
// Steps of values from here on stay out of the products, so that no such step, which perhaps few rows see, takes the others'
// weights out of the operand's range.
template <typename E> constexpr float kStepMost = std::is_same_v<E, bf16> ? 65536.0f : 8.0f;

// 16 codes of 8 bytes' halves as two operands: per dword bytes 0 and 2, low and high halves (times 16), then bytes 1 and 3
__device__ __forceinline__ u32x4 spread(uint32_t x) {
    const uint32_t y = x >> 8;
    return u32x4{x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u};
}

// max over the lanes of a column (lanes 16 apart)
__device__ __forceinline__ float max_column(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_column(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A sequence as the workers look it up: its first new row, how many it has, the first one's position, what they see.
struct FewSeq {
    int32_t first, n_new, pos0;
    Span span;
};

// Wavefronts of a workgroup: a team, which shares a (sequence, head), has 8 where registers allow two on a SIMD.
template <uint32_t D, uint32_t kBits, uint32_t kTiles, bool kTeam>
constexpr uint32_t kFewWaves = kTeam && !(D == 128 && kBits == 16 && kTiles == 2) ? 8 : 4;

// Variants of the line (4 bits) that run with twice the wavefronts on a SIMD where each still has a good share of the line.  (128
// channels have 15 of their 256 registers in scratch memory then.)
template <uint32_t D, uint32_t kBits, uint32_t kTiles, bool kTeam>
constexpr bool kFewDoubles = kBits == 4 && !kTeam && (D == 64 ? kTiles == 1 : kTiles == 2);
// Wavefronts that registers leave room for on a SIMD.
template <uint32_t D, uint32_t kBits, uint32_t kTiles, bool kTeam>
constexpr uint32_t kFewPerSimd = D == 128 && kBits == 16 && kTiles == 2 ? 1 : D == 64 && kFewDoubles<D, kBits, kTiles, kTeam> ? 4 : 2;

// kTiles: tiles of 16 rows.  kTeam: a workgroup takes a (sequence, head) and joins its wavefronts' parts itself.
template <typename E, uint32_t D, uint32_t kBits, uint32_t kTiles, bool kTeam>
__global__ __launch_bounds__((kFewWaves<D, kBits, kTiles, kTeam> * kLanes), (kFewPerSimd<D, kBits, kTiles, kTeam>)) void k_attend_few(const AttnParams p) {
    constexpr uint32_t kWaves = kFewWaves<D, kBits, kTiles, kTeam>;
    constexpr bool kCodes = kBits == 4;
    constexpr uint32_t kGroups = D / 64;
    constexpr uint32_t kSteps = D / 32, kOut = D / 16;      // products over channels; tiles of 16 channels of the result
    constexpr uint32_t kRowBytes = kCodes ? D / 2 : 2 * D, kSideBytes = kFewKeys * kRowBytes;
    constexpr uint32_t kLaneRows = kRowBytes / 16;          // lanes that read a row
    constexpr uint32_t kRowsAtOnce = kLanes / kLaneRows, kLoads = kFewKeys / kRowsAtOnce;
    constexpr uint32_t kPairFloats = 2 * kGroups;           // (step, lo) of a key
    // A maximum is only raised when a score, in powers of two, passes it by this; in 4 bits and fp16 that comes off the weights' range.
    constexpr float kFewHeadroom = kCodes && std::is_same_v<E, fp16> ? 4.0f : 8.0f;
    constexpr float kUp = kCodes ? 0.0f : kWeightUp<E>;     // (codes have their own, with the step)
    constexpr int kWeightExponent = std::is_same_v<E, fp16> ? 10 : 100;
    constexpr uint32_t kWaveBytes = 2 * kSideBytes + (kCodes ? 2 * kFewKeys * kPairFloats * 4 : 0);
    constexpr uint32_t kOutStride = D + 4;                  // floats between rows where a team's results meet
    constexpr uint32_t kJoinBytes = kTeam ? 16 * kOutStride * 4 : 0;
    __shared__ __attribute__((aligned(16))) char lds[kWaves * (kWaveBytes > kJoinBytes ? kWaveBytes : kJoinBytes)];
    __shared__ int64_t lds_rows[kWaves][kFewKeys];
    __shared__ uint32_t lds_line[kTeam ? 1 : kFewSeqs + 1], lds_sum[kWaves];
    __shared__ FewSeq lds_seq[kTeam ? 1 : kFewSeqs];
    __shared__ float lds_m[kTeam ? kWaves : 1][16], lds_l[kTeam ? kWaves : 1][16];
    static_assert(kFewSeqs == kLineThreads);

    const uint32_t lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), col = lane % 16, quad = lane / 16;

    const uint32_t worker = blockIdx.x * kWaves + wave;
    uint32_t unit = 0, unit_end = 1;
    if constexpr (!kTeam) {
        // The line: a sequence has, for each head, kFewEnter places for beginning with it and one for each tile; none where it
        // is not this kernel's.  lds_line[s]: places of the sequences before s, for one head.
        uint32_t mine = 0;
        if (threadIdx.x < p.batch.n_seqs) {
            const Seq seq = seq_at(p.batch, threadIdx.x);
            const int32_t n_new = min(seq.n_new, (int32_t)p.batch.max_new);
            const uint32_t rows = (uint32_t)n_new * p.group;
            if (rows != 0 && rows <= p.few_rows) {
                const Span sp = span_of<kFewKeys>(p, seq, 0, n_new - 1);
                mine = sp.tiles + kFewEnter;
                lds_seq[threadIdx.x] = FewSeq{seq.first, n_new, seq.pos0, sp};
            }
        }
        uint32_t upto = mine;
#pragma unroll
        for (uint32_t m = 1; m < kLanes; m *= 2) {
            const uint32_t other = __shfl_up(upto, m);
            if (lane >= m) upto += other;
        }
        if (lane == kLanes - 1) lds_sum[wave] = upto;
        __syncthreads();
        uint32_t total = 0;
        for (uint32_t w = 0; w < kWaves; ++w) {
            if (w < wave) upto += lds_sum[w];
            total += lds_sum[w];
        }
        lds_line[threadIdx.x + 1] = upto;
        if (threadIdx.x == 0) lds_line[0] = 0;
        __syncthreads();
        const uint32_t units = total * p.kv_heads, per = max(p.few_least, (units + p.few_waves - 1) / p.few_waves);
        if (p.few_plan && blockIdx.x == 0) {                                  // for the kernel that joins
            if (threadIdx.x < p.batch.n_seqs) p.few_plan[2 + threadIdx.x] = upto;
            if (threadIdx.x == 0) p.few_plan[0] = per, p.few_plan[1] = 0;
        }
        if (p.few_plan) {
            unit = min(worker * per, units), unit_end = min(unit + per, units);
        } else {                                                // no split: each worker has a (sequence, head)
            const uint32_t s = worker / p.kv_heads;
            if (s >= p.batch.n_seqs) return;
            const uint32_t of_head = lds_line[s + 1] - lds_line[s];
            unit = lds_line[s] * p.kv_heads + (worker - s * p.kv_heads) * of_head, unit_end = unit + of_head;
        }
        unit = __builtin_amdgcn_readfirstlane(unit), unit_end = __builtin_amdgcn_readfirstlane(unit_end);
    }

    // where the lane's 16 bytes of load i lie: row i * kRowsAtOnce + lane / kLaneRows, piece lane % kLaneRows
    const uint32_t load_row = lane / kLaneRows, load_piece = lane % kLaneRows;
    char* const k_lds = lds + wave * kWaveBytes;
    char* const v_lds = k_lds + kSideBytes;
    float* const k_par = reinterpret_cast<float*>(k_lds + 2 * kSideBytes);
    float* const v_par = k_par + kFewKeys * kPairFloats;
    // Pieces of 16 bytes of a row change places by the key, so that what one read takes at once lies in different banks.
    auto k_at = [](uint32_t key, uint32_t piece) {
        if constexpr (kCodes) return key * kRowBytes + (piece ^ (D == 128 ? (key >> 2) & 3u : (key >> 3) & 1u)) * 16;
        else return key * kRowBytes + (piece ^ (D == 128 ? key & 15u : (key >> 1) & 7u)) * 16;
    };
    auto v_at = [](uint32_t key, uint32_t piece) {
        if constexpr (kCodes) return key * kRowBytes + (piece ^ (D == 128 ? ((key >> 2) & 1u) | ((key >> 3) & 2u) : (key >> 4) & 1u)) * 16;
        else return key * kRowBytes + (piece ^ (D == 128 ? (key & 7u) << 1 : ((key >> 1) & 3u) << 1)) * 16;
    };

    while (unit < unit_end) {
        // the piece of the line: the last sequence whose tiles begin at or before the unit, its head, tiles; a team's wavefronts
        // take every kWaves-th tile of theirs
        uint32_t s, head, first_tile, last_tile, tiles;
        FewSeq its;
        if constexpr (kTeam) {
            s = blockIdx.x / p.kv_heads, head = blockIdx.x - s * p.kv_heads;
            const Seq seq = seq_at(p.batch, s);
            its.first = seq.first, its.n_new = min(seq.n_new, (int32_t)p.batch.max_new), its.pos0 = seq.pos0;
            if (its.n_new == 0 || (uint32_t)its.n_new * p.group > p.few_rows) return;
            its.span = span_of<kFewKeys>(p, seq, 0, its.n_new - 1);
            tiles = uniform(its.span.tiles), first_tile = wave, last_tile = tiles;
            unit = unit_end;
        } else {
            s = 0;
            for (uint32_t s_end = p.batch.n_seqs; s_end - s > 1;) {
                const uint32_t mid = (s + s_end) / 2;
                if (uniform(lds_line[mid]) * p.kv_heads <= unit) s = mid;
                else s_end = mid;
            }
            const uint32_t line = uniform(lds_line[s]), of_head = uniform(lds_line[s + 1]) - line, at_line = unit - line * p.kv_heads;
            head = at_line / of_head;
            const uint32_t place = at_line - head * of_head, n_units = min(of_head - place, unit_end - unit);
            tiles = of_head - kFewEnter, first_tile = max(place, kFewEnter) - kFewEnter, last_tile = max(place + n_units, kFewEnter) - kFewEnter;
            unit += n_units;
            if (first_tile == last_tile && (tiles || place)) continue;   // the beginning alone, which the next worker has too
            its = lds_seq[s];
        }
        const int32_t seq_first = uniform(its.first), n_new = uniform(its.n_new), pos_first = uniform(its.pos0), pos_last = pos_first + n_new - 1;
        const uint32_t rows = (uint32_t)n_new * p.group;
        Span sp;
        sp.sink_end = uniform(its.span.sink_end), sp.begin = uniform(its.span.begin), sp.end = uniform(its.span.end), sp.sink_tiles = uniform(its.span.sink_tiles);
        constexpr uint32_t kStep = kTeam ? kWaves : 1;

        // ---- what is fetched: places of a tile's keys (lane % 32 has a key), then its rows
        const int32_t* table = p.batch.table + (int64_t)s * p.batch.table_stride;
        const int64_t head_at = (int64_t)head * p.cache.head_stride, pair_head_at = (int64_t)head * p.cache.pair_head_stride;
        Place ahead;
        struct {
            u32x4 k[kLoads], v[kLoads];
            u32x2 pair;                             // of the keys (lanes below 32) or the values
            uint32_t seen;                          // one bit a key of the tile: it is there
        } raw;
        auto places = [&](uint32_t tile) {
            int32_t base, end;
            tile_at<kFewKeys>(sp, tile, base, end);
            ahead = place_of(p.cache, table, tile < last_tile ? (uint32_t)(base + (int32_t)(lane % kFewKeys)) : 0xFFFFFFFFu, (uint32_t)end);
        };
        // The places of the tile after are asked for before the rows, so that waiting for them does not wait for the rows too.
        auto fetch = [&](uint32_t next) {         // where nothing is, the cache's first row stands in
            raw.seen = (uint32_t)__ballot(ahead.there);
            const int64_t page = ahead.there ? ahead.page : 0, slot = ahead.there ? ahead.slot : 0;
            if (lane < kFewKeys) lds_rows[wave][lane] = page * p.cache.page_stride + slot * p.cache.slot_stride + head_at;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            places(next);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const int64_t at = lds_rows[wave][i * kRowsAtOnce + load_row] + 16 * load_piece;
                raw.k[i] = *reinterpret_cast<const u32x4*>(p.cache.k + at);
                raw.v[i] = *reinterpret_cast<const u32x4*>(p.cache.v + at);
            }
            if constexpr (kCodes) {
                const char* pairs = (lane < kFewKeys ? p.cache.k_pairs : p.cache.v_pairs) + page * p.cache.pair_page_stride + slot * p.cache.pair_slot_stride + pair_head_at;
                if constexpr (kGroups == 2) raw.pair = *reinterpret_cast<const u32x2*>(pairs);
                else raw.pair[0] = *reinterpret_cast<const uint32_t*>(pairs);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        };
        places(first_tile);
        fetch(first_tile + kStep);

        // ---- queries as the second operand: column = row of the result.  Product i takes channels 32 i + 8 quad + 0..7; in
        // 4 bits, of each 64, first the codes of 8 bytes' first dwords, then of the second: byte 8 quad + 4 (i % 2), with the
        // channels in spread()'s order and those that come times 16 divided by it.
        u32x4 q[kTiles][kSteps];
        int32_t pos[kTiles];                            // position of the column's token
        float q_sum[kTiles][kGroups], q_scale[kTiles], unit_of[kTiles];   // scores are in units of unit_of (1 in 16 bits), which is in powers of two
#pragma unroll
        for (uint32_t n = 0; n < kTiles; ++n) {
            const uint32_t r = min(n * 16 + here(col), rows - 1), quad = here(lane) / 16, token = over_group(p, r);
            pos[n] = pos_first + (int32_t)token;
            const char* row = p.q.data + (int64_t)(seq_first + (int32_t)token) * p.q.token_stride + (int64_t)(head * p.group + r - token * p.group) * p.q.head_stride;
            unit_of[n] = 1.0f;
            if constexpr (!kCodes) {
#pragma unroll
                for (uint32_t i = 0; i < kSteps; ++i) q[n][i] = *reinterpret_cast<const u32x4*>(row + 64 * i + 16 * quad);
            } else {
                float most = 0.0f, x[kSteps][8];
#pragma unroll
                for (uint32_t i = 0; i < kSteps; ++i) {
                    const u32x4 y = *reinterpret_cast<const u32x4*>(row + 128 * (i / 2) + 32 * quad + 16 * (i % 2));
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][2 * j] = low16<E>(y[j]), x[i][2 * j + 1] = high16<E>(y[j]);
                }
#pragma unroll
                for (uint32_t i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[i][j]));
                most = max_column(most);
                // The row is brought below 1 (the largest numbers below 4) by a power of two, so nothing is rounded that counts, and that
                // goes into the unit of its scores together with the scale; what would take the unit out of range stays with the row.
                const int e = most < INFINITY ? min(exponent_above(most), 126) : 0, e_scale = exponent_above(p.scale_log2);
                const int e_unit = min(max(e, -100 - e_scale), 100 - e_scale), e_row = min(max(e - e_unit, -100), 100);
                unit_of[n] = p.scale_log2 * power2(e_unit / 2) * power2(e_unit - e_unit / 2);
                q_scale[n] = power2(kCodeExponent<E> - kOperandExponent<E> + e_row);
#pragma unroll
                for (uint32_t g = 0; g < kGroups; ++g) {
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float& y = x[2 * g + j / 8][j % 8];
                        y *= power2(-e);
                        sum += y;
                    }
                    q_sum[n][g] = sum_column(sum) * power2(e_row);
                }
#pragma unroll
                for (uint32_t i = 0; i < kSteps; ++i) {
                    constexpr int kOrder[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float f = power2(kOperandExponent<E> - (j % 2 ? 4 : 0));
                        q[n][i][j] = pack2<E>(x[i][kOrder[2 * j]] * f, x[i][kOrder[2 * j + 1]] * f);
                    }
                }
            }
        }

        // In 4 bits o[.][2 b] holds the even, o[.][2 b + 1] the odd channels (times 16) of the 16 bytes b, all times 2^-133
        // (-24) and the scale of the weights; eights: the sum of 8 times the weights alike; lows: what the middle codes add.
        f32x4 o[kTiles][kOut], eights[kTiles][kGroups];
        float m[kTiles], l[kTiles], lows[kTiles][kGroups];
        int step_exp = -20;                             // weights are taken times step / 2^step_exp
#pragma unroll
        for (uint32_t n = 0; n < kTiles; ++n) {
            m[n] = -INFINITY, l[n] = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < kOut; ++i) o[n][i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (uint32_t g = 0; g < kGroups; ++g) eights[n][g] = f32x4{0, 0, 0, 0}, lows[n][g] = 0.0f;
        }

        for (uint32_t tile = first_tile; tile < last_tile; tile += kStep) {
            const uint32_t seen = raw.seen;
            uint32_t apart = 0;                         // one bit a key: one of its values' steps is above kStepMost
            float apart_step[kGroups];                  // lanes from 32 on: these steps, others 0
            // rows to LDS; values (in 4 bits: pairs) that are not there as zeros
            if (!kCodes && seen != ~0u) {
#pragma unroll
                for (uint32_t i = 0; i < kLoads; ++i)
                    if (!((seen >> (i * kRowsAtOnce + load_row)) & 1u)) raw.v[i] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t key = i * kRowsAtOnce + load_row;
                *reinterpret_cast<u32x4*>(k_lds + k_at(key, load_piece)) = raw.k[i];
                *reinterpret_cast<u32x4*>(v_lds + v_at(key, load_piece)) = raw.v[i];
            }
            if constexpr (kCodes) {
                const bool there = (seen >> (lane % kFewKeys)) & 1u;
                float par[kPairFloats];
                bool larger = false;
#pragma unroll
                for (uint32_t g = 0; g < kGroups; ++g) {
                    par[2 * g] = there ? low16<E>(raw.pair[g]) : 0.0f, par[2 * g + 1] = there ? high16<E>(raw.pair[g]) : 0.0f;
                    larger |= lane >= kFewKeys && fabsf(par[2 * g]) >= power2(step_exp);
                    apart_step[g] = 0.0f;
                }
                if (__any(larger)) {                    // a larger step than any so far (the first steps do this, seldom others)
                    float most = 0.0f;
#pragma unroll
                    for (uint32_t g = 0; g < kGroups; ++g) {
                        const float size = fabsf(par[2 * g]);
                        if (lane < kFewKeys) continue;
                        if (size < kStepMost<E>) most = fmaxf(most, size);
                        else if (size < INFINITY) apart_step[g] = par[2 * g], par[2 * g] = 0.0f;
                    }
                    bool out = apart_step[0] != 0.0f;
                    if constexpr (kGroups == 2) out |= apart_step[kGroups - 1] != 0.0f;
                    apart = (uint32_t)(__ballot(out) >> kFewKeys);
#pragma unroll
                    for (uint32_t x = 1; x < kLanes; x *= 2) most = fmaxf(most, __shfl_xor(most, x));
                    const int e = max(__builtin_amdgcn_readfirstlane(exponent_above(most)), step_exp);
                    const float down = power2(max(step_exp - e, -126));
                    step_exp = e;
#pragma unroll
                    for (uint32_t n = 0; n < kTiles; ++n) {
#pragma unroll
                        for (uint32_t i = 0; i < kOut; ++i) o[n][i] *= down;
#pragma unroll
                        for (uint32_t g = 0; g < kGroups; ++g) eights[n][g] *= down;
                    }
                }
                if (lane >= kFewKeys) {                 // values: step in the weights' scale, and what the middle code stands for
                    const float f = power2(kWeightExponent - step_exp);
#pragma unroll
                    for (uint32_t g = 0; g < kGroups; ++g) par[2 * g + 1] = fmaf(8.0f, par[2 * g], par[2 * g + 1]), par[2 * g] *= f;
                }
                float* to = (lane < kFewKeys ? k_par : v_par) + (lane % kFewKeys) * kPairFloats;
                if constexpr (kGroups == 2) *reinterpret_cast<f32x4*>(to) = f32x4{par[0], par[1], par[2], par[3]};
                else *reinterpret_cast<f32x2*>(to) = f32x2{par[0], par[1]};
            }
            fetch(tile + 2 * kStep);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            int32_t base, end;
            tile_at<kFewKeys>(sp, tile, base, end);

            // scores (S^T = K Q^T), in units of unit_of; the lane has keys 4 quad + 0..3 of both halves for its column
            float x[kTiles][8];
#pragma unroll
            for (uint32_t r = 0; r < 2; ++r) {
                if constexpr (!kCodes) {
                    f32x4 sc[kTiles];
#pragma unroll
                    for (uint32_t n = 0; n < kTiles; ++n) sc[n] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (uint32_t i = 0; i < kSteps; ++i) {
                        const u32x4 a = *reinterpret_cast<const u32x4*>(k_lds + k_at(16 * r + col, 4 * i + quad));
#pragma unroll
                        for (uint32_t n = 0; n < kTiles; ++n) sc[n] = mfma16<E>(a, q[n][i], sc[n]);
                    }
#pragma unroll
                    for (uint32_t n = 0; n < kTiles; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[n][4 * r + j] = sc[n][j] * p.scale_log2;
                } else {
                    f32x4 sc[kTiles][kGroups];
#pragma unroll
                    for (uint32_t g = 0; g < kGroups; ++g) {
                        const u32x2 a = *reinterpret_cast<const u32x2*>(k_lds + k_at(16 * r + col, 2 * g + quad / 2) + 8 * (quad % 2));
#pragma unroll
                        for (uint32_t n = 0; n < kTiles; ++n) {
                            sc[n][g] = mfma16<E>(spread(a[0]), q[n][2 * g], f32x4{0, 0, 0, 0});
                            sc[n][g] = mfma16<E>(spread(a[1]), q[n][2 * g + 1], sc[n][g]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float* par = k_par + (16 * r + 4 * quad + j) * kPairFloats;
#pragma unroll
                        for (uint32_t n = 0; n < kTiles; ++n) {
                            if constexpr (kGroups == 2)
                                x[n][4 * r + j] = fmaf(fmaf(par[2], sc[n][1][j], par[0] * sc[n][0][j]), q_scale[n], fmaf(par[3], q_sum[n][1], par[1] * q_sum[n][0]));
                            else
                                x[n][4 * r + j] = fmaf(par[0] * sc[n][0][j], q_scale[n], par[1] * q_sum[n][0]);
                        }
                    }
                }
            }

            // does every row see every key of the tile?
            const bool sink_part = tile < sp.sink_tiles;
            const bool each = n_new > 1 && (base + (int32_t)kFewKeys - 1 > pos_first || (p.window && !sink_part && (int64_t)base <= (int64_t)pos_last - p.window));
            u32x4 w[kCodes ? 1 : kTiles];               // weights as the second product takes them
            u32x4 wg[kCodes ? kTiles : 1][kGroups];
            uint32_t shows[kTiles];                     // one bit a key of the lane: the column's row sees it
#pragma unroll
            for (uint32_t n = 0; n < kTiles; ++n) {
                uint32_t sees = 0xFFu;
                if (each || seen != ~0u) {
                    sees = (seen >> (4 * quad) & 15u) | (seen >> (16 + 4 * quad) & 15u) << 4;
                    if (each) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int32_t key = base + (j / 4) * 16 + (int32_t)(4 * quad) + j % 4;
                            const bool sight = key <= pos[n] && (!p.window || (int64_t)key > (int64_t)pos[n] - p.window || (uint32_t)key < p.sinks);
                            if (!sight) sees &= ~(1u << j);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!((sees >> j) & 1u)) x[n][j] = -INFINITY;
                }
                shows[n] = sees;
                float top = x[n][0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, x[n][j]);
                top = max_column(top) * unit_of[n];
                const bool raise = top > m[n] + kFewHeadroom || (m[n] == -INFINITY && top > m[n]);
                if (__any(raise)) {
                    const float grown = raise ? top : m[n], keep = raise && m[n] != -INFINITY ? exp2_of(m[n] - grown) : 1.0f;
                    m[n] = grown;
                    l[n] *= keep;
#pragma unroll
                    for (uint32_t i = 0; i < kOut; ++i) o[n][i] *= keep;
                    if constexpr (kCodes) {
#pragma unroll
                        for (uint32_t g = 0; g < kGroups; ++g) eights[n][g] *= keep, lows[n][g] *= keep;
                    }
                }
                const float from = m[n] == -INFINITY ? 0.0f : m[n] - kUp;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[n][j] = exp2_of(fmaf(x[n][j], unit_of[n], -from));
                    if constexpr (kCodes) l[n] += x[n][j];
                }
                if constexpr (!kCodes) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[n][j] = pack2<E>(x[n][2 * j], x[n][2 * j + 1]), l[n] = add2<E>(w[n][j], l[n]);
                }
            }
            if constexpr (kCodes) {
                auto weigh = [&](auto masked) {
#pragma unroll
                    for (uint32_t h = 0; h < 2; ++h) {      // keys 4 quad + 0..3 of the first 16, then of the second
                        float par[4][kPairFloats];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (uint32_t c = 0; c < kPairFloats; ++c) par[j][c] = v_par[(16 * h + 4 * quad + j) * kPairFloats + c];
#pragma unroll
                        for (uint32_t n = 0; n < kTiles; ++n)
#pragma unroll
                            for (uint32_t g = 0; g < kGroups; ++g) {
                                float y[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    y[j] = x[n][4 * h + j] * par[j][2 * g];
                                    float low = par[j][2 * g + 1];
                                    if (masked() && !((shows[n] >> (4 * h + j)) & 1u)) y[j] = 0.0f, low = 0.0f;
                                    lows[n][g] = fmaf(x[n][4 * h + j], low, lows[n][g]);
                                }
                                wg[n][g][2 * h] = pack2<E>(y[0], y[2]);          // keys in spread()'s order: bytes 0 and 2, then 1 and 3
                                wg[n][g][2 * h + 1] = pack2<E>(y[1], y[3]);
                            }
                    }
                };
                for (uint32_t left = apart; left; left &= left - 1) {       // key by key, in 32 bits
                    const uint32_t k = (uint32_t)__builtin_ctz(left), j = (k / 16) * 4 + k % 4;
                    const float scale = power2(kWeightExponent - kCodeExponent<E> - step_exp);
#pragma unroll
                    for (uint32_t n = 0; n < kTiles; ++n) {
                        float weight = x[n][0];
#pragma unroll
                        for (uint32_t i = 1; i < 8; ++i) weight = i == j ? x[n][i] : weight;
                        weight = __shfl(weight, (int)(k % 16 / 4 * 16 + col));
#pragma unroll
                        for (uint32_t b = 0; b < kOut / 2; ++b) {
                            const float step = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(apart_step[b / 2]), kFewKeys + k)) * scale * weight;
                            const uint32_t codes = *reinterpret_cast<const uint32_t*>(v_lds + v_at(k, b) + 4 * quad);
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                o[n][2 * b][c] += step * (float)(codes >> (8 * c) & 15u);
                                o[n][2 * b + 1][c] += step * (float)(codes >> (8 * c) & 0xF0u);
                            }
                        }
                    }
                }
                if (each) weigh(std::true_type{});          // a pair that is NaN reaches nobody who does not see it
                else weigh(std::false_type{});
            }

            // O^T += V^T P^T: the transposing read gives the lane its 8 keys of one channel (of one byte's two channels)
            if constexpr (kCodes) {
                const uint32_t j = col / 2, key = (j / 4) * 16 + 4 * quad + j % 4;
                constexpr uint32_t kEight = 0x00080008u;
#pragma unroll
                for (uint32_t n = 0; n < kTiles; ++n)
#pragma unroll
                    for (uint32_t g = 0; g < kGroups; ++g) eights[n][g] = mfma16<E>(u32x4{kEight, kEight, kEight, kEight}, wg[n][g], eights[n][g]);
#pragma unroll
                for (uint32_t b = 0; b < kOut / 2; ++b) {
                    const u32x2 a = lds_transposed8(v_lds + v_at(key, b) + 8 * (col % 2));
                    const u32x4 x0 = spread(a[0]), x1 = spread(a[1]);
                    const u32x4 even = {x0[0], x0[2], x1[0], x1[2]}, odd = {x0[1], x0[3], x1[1], x1[3]};
#pragma unroll
                    for (uint32_t n = 0; n < kTiles; ++n) {
                        o[n][2 * b] = mfma16<E>(even, wg[n][b / 2], o[n][2 * b]);
                        o[n][2 * b + 1] = mfma16<E>(odd, wg[n][b / 2], o[n][2 * b + 1]);
                    }
                }
            } else {
                const uint32_t key = 4 * quad + col / 4, part = (col % 4) / 2, byte = (col % 2) * 8;
                auto operand = [&](uint32_t i) {
                    const u32x2 lo = lds_transposed(v_lds + v_at(key, 2 * i + part) + byte), hi = lds_transposed(v_lds + v_at(16 + key, 2 * i + part) + byte);
                    return u32x4{lo[0], lo[1], hi[0], hi[1]};
                };
                if (!each) {
#pragma unroll
                    for (uint32_t i = 0; i < kOut; ++i) {
                        const u32x4 a = operand(i);
#pragma unroll
                        for (uint32_t n = 0; n < kTiles; ++n) o[n][i] = mfma16<E>(a, w[n], o[n][i]);
                    }
                } else {                                    // a NaN or infinity that only some rows see must not reach the others as 0 * NaN
#pragma unroll
                    for (uint32_t i = 0; i < kOut; ++i) {
                        const u32x4 a = operand(i);
                        bool bad = false;
#pragma unroll
                        for (int j = 0; j < 4; ++j) bad |= not_finite16(a[j], kExponent<E>);
                        if (!__any(bad)) {
#pragma unroll
                            for (uint32_t n = 0; n < kTiles; ++n) o[n][i] = mfma16<E>(a, w[n], o[n][i]);
                            continue;
                        }
#pragma unroll 1
                        for (uint32_t k = 0; k < kFewKeys; ++k) {        // key by key, and only the columns whose row sees it take the sum
                            const uint32_t j = (k / 16) * 4 + k % 4, in_quad = (k % 16) / 4;
                            u32x4 only;                     // the key's place in both operands
#pragma unroll
                            for (uint32_t d = 0; d < 4; ++d) only[d] = quad == in_quad && d == j / 2 ? (j % 2 ? 0xFFFF0000u : 0xFFFFu) : 0u;
#pragma unroll
                            for (uint32_t n = 0; n < kTiles; ++n) {
                                const f32x4 one = mfma16<E>(a & only, w[n] & only, f32x4{0, 0, 0, 0});
                                if ((__shfl(shows[n], 16 * in_quad + col) >> j) & 1u) o[n][i] += one;
                            }
                        }
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }

        // ---- the piece's rows: a team's wavefronts meet in LDS; otherwise finished where all of the sequence's tiles are here,
        // and to the workspace where not
        const bool whole = kTeam || last_tile - first_tile == tiles;
        const uint32_t slot = 2 * worker + (first_tile ? 0u : 1u);
#pragma unroll
        for (uint32_t n = 0; n < kTiles; ++n) {
            const uint32_t row = n * 16 + here(col), quad = here(lane) / 16;
            const float sum = sum_column(l[n]);
            float f = !kTeam && whole ? (sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f) : 1.0f, low[kGroups];
            if constexpr (kCodes) {
#pragma unroll
                for (uint32_t g = 0; g < kGroups; ++g) low[g] = sum_column(lows[n][g]) * f;
                f *= power2(kCodeExponent<E> - kWeightExponent + step_exp);
            }
            auto results = [&](auto write) {                // write(c, x): channels c .. c + 3 of the column's row
                if constexpr (!kCodes) {
#pragma unroll
                    for (uint32_t i = 0; i < kOut; ++i) write(16 * i + 4 * quad, o[n][i] * f);
                } else {
#pragma unroll
                    for (uint32_t b = 0; b < kOut / 2; ++b) {
                        f32x4 even, odd;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            even[j] = fmaf(o[n][2 * b][j] - eights[n][b / 2][0], f, low[b / 2]);
                            odd[j] = fmaf(o[n][2 * b + 1][j] * 0.0625f - eights[n][b / 2][0], f, low[b / 2]);
                        }
                        write(32 * b + 8 * quad, f32x4{even[0], odd[0], even[1], odd[1]});
                        write(32 * b + 8 * quad + 4, f32x4{even[2], odd[2], even[3], odd[3]});
                    }
                }
            };
            auto out_row = [&](uint32_t r) {
                const uint32_t token = over_group(p, r);
                return p.out.data + (int64_t)(seq_first + (int32_t)token) * p.out.token_stride + (int64_t)(head * p.group + r - token * p.group) * p.out.head_stride;
            };
            if constexpr (kTeam) {
                __syncthreads();
                float* const meet = reinterpret_cast<float*>(lds);
                results([&](uint32_t c, f32x4 x) { *reinterpret_cast<f32x4*>(meet + (wave * 16 + col) * kOutStride + c) = x; });
                if (quad == 0) lds_m[wave][col] = m[n], lds_l[wave][col] = sum;
                __syncthreads();
                constexpr uint32_t kRowThreads = kWaves * kLanes / 16, kPer = D / kRowThreads;   // threads of a row, channels of a thread
                const uint32_t r = threadIdx.x / kRowThreads, c0 = threadIdx.x % kRowThreads * kPer;
                if (n * 16 + r < rows) {
                    float top = -INFINITY, total = 0.0f, acc[kPer];
#pragma unroll
                    for (uint32_t v = 0; v < kWaves; ++v) top = fmaxf(top, lds_m[v][r]);
                    const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
                    for (uint32_t c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
                    for (uint32_t v = 0; v < kWaves; ++v) {
                        const float weight = exp2_of(lds_m[v][r] - from);
                        total += weight * lds_l[v][r];
#pragma unroll
                        for (uint32_t c = 0; c < kPer; ++c) acc[c] += lds_m[v][r] == -INFINITY ? 0.0f : weight * meet[(v * 16 + r) * kOutStride + c0 + c];
                    }
                    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
                    uint32_t* const dst = reinterpret_cast<uint32_t*>(out_row(n * 16 + r) + 2 * c0);
#pragma unroll
                    for (uint32_t c = 0; c < kPer; c += 2) dst[c / 2] = pack2<E>(acc[c] * inv, acc[c + 1] * inv);
                }
            } else if (row < rows) {
                const uint64_t at = (uint64_t)slot * p.few_stride + row;
                char* const dst = out_row(row);
                float* const part = p.few_o + at * D;
                results([&](uint32_t c, f32x4 x) {
                    if (whole) *reinterpret_cast<u32x2*>(dst + 2 * c) = u32x2{pack2<E>(x[0], x[1]), pack2<E>(x[2], x[3])};
                    else *reinterpret_cast<f32x4*>(part + c) = x;
                });
                if (!whole && quad == 0) p.few_ml[at] = f32x2{m[n] - kUp, sum};
            }
        }
    }
}

// Joins the pieces of a sequence and head that the line was cut into: a wavefront takes one row, a lane D / 64 channels.
// A piece that begins inside the sequence lies in its worker's slot 0, one that only ends inside it in slot 1.
template <typename E, uint32_t D>
__global__ __launch_bounds__(256) void k_join_few(const AttnParams p) {
    const uint32_t row_of = blockIdx.x * 4 + threadIdx.x / kLanes;
    const uint32_t sh = row_of / p.few_stride, row = row_of - sh * p.few_stride, s = sh / p.kv_heads, head = sh - s * p.kv_heads;
    if (s >= p.batch.n_seqs) return;
    const uint32_t per = p.few_plan[0], begin = p.few_plan[1 + s], places = p.few_plan[2 + s] - begin;
    const Seq seq = seq_at(p.batch, s);
    if (places <= kFewEnter || row >= (uint32_t)min(seq.n_new, (int32_t)p.batch.max_new) * p.group) return;
    const uint32_t unit = begin * p.kv_heads + head * places, first = (unit + kFewEnter) / per, last = (unit + places - 1) / per;
    if (first == last) return;                              // written already
    const uint32_t token = over_group(p, row);
    join_row<E, D>(p.few_o, p.few_ml, [&](uint32_t z) { return (uint64_t)(2 * (first + z) + (z == 0 ? 1u : 0u)) * p.few_stride + row; }, last - first + 1,
                   p.out.data + (int64_t)(seq.first + (int32_t)token) * p.out.token_stride + (int64_t)(head * p.group + row - token * p.group) * p.out.head_stride);
}

}  // namespace

#endif  // AT_FEW_HPP
