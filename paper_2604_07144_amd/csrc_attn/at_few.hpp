// Attention of few rows over a long cache: a sequence's new tokens times the query heads of one key/value head make at
// most 64 rows (one new token: the A / K heads that share a key/value head).
//
// Mathematics: one pass over the keys with the running maximum m and sum l of a softmax, o = sum_j e^{s_j - m} v_j
// scaled down whenever m grows; parts of the key axis are joined by their (m, l, o).
//
// Every key and value is read once, for all rows that share it, so memory bounds this: per position and key/value head
// 2 * D * 2 bytes against 4 * D * rows operations.  Therefore: the key axis is split over workgroups (chunks) and over
// the four wavefronts of each, which go their own way without a barrier until the end; a wavefront has the next 32 keys
// and values in registers while it works on the present ones.  Products run on the matrix units as S^T = K Q^T and
// O^T = V^T P^T: rows of queries are columns there, so the running maximum of a row lives in the lanes of one column, and
// the weights leave the first product in exactly the registers from which the second takes them.  Keys go from memory
// straight into the operand registers; values pass through LDS, which hands them back transposed.
#ifndef AT_FEW_HPP
#define AT_FEW_HPP

#include "at_parts.hpp"

namespace {

constexpr uint32_t kFewWaves = 4, kFewThreads = kFewWaves * kLanes;
constexpr uint32_t kFewRows = 64;        // most rows (new tokens times shared heads) of the kernel

// The lane's part of 32 keys or values: rows lane % 16 and 16 + lane % 16, of each the pieces that the matrix units ask of
// this lane.  In 16 bits piece i is 16 bytes at channel 32 i + 8 (lane / 16), so that 4 lanes read 64 bytes of a row at a
// time; in 4 bits the lane's codes lie together, at channel (D / 4) (lane / 16) + 8 i.
template <typename E, uint32_t D, uint32_t kBits> struct Piece {
    static constexpr uint32_t kN = D / 32;
    u32x4 raw[2][kBits == 16 ? kN : (D == 128 ? 1 : 1)];
    uint32_t pair[2];

    __device__ __forceinline__ static uint32_t channel(uint32_t lane, uint32_t i) {
        return kBits == 16 ? 32 * i + 8 * (lane / 16) : (D / 4) * (lane / 16) + 8 * i;
    }
    __device__ __forceinline__ void load(const char* row, const char* pairs, int r, uint32_t lane) {
        if constexpr (kBits == 16) {
#pragma unroll
            for (uint32_t i = 0; i < kN; ++i) raw[r][i] = *reinterpret_cast<const u32x4*>(row + 64 * i + 16 * (lane / 16));
        } else {
            const char* at = row + (D / 8) * (lane / 16);
            if constexpr (D == 128) raw[r][0] = *reinterpret_cast<const u32x4*>(at);
            else {
                const u32x2 x = *reinterpret_cast<const u32x2*>(at);
                raw[r][0] = u32x4{x[0], x[1], 0, 0};
            }
            pair[r] = reinterpret_cast<const uint32_t*>(pairs)[D == 128 ? lane / 32 : 0];
        }
    }
    __device__ __forceinline__ u32x4 get(int r, uint32_t i) const {
        if constexpr (kBits == 16) return raw[r][i];
        else return decode8<E>(raw[r][0][i], low16<E>(pair[r]), high16<E>(pair[r]));
    }
};

// kTiles: tiles of 16 rows.  Workgroups: [chunk][sequence][kv head], so that first chunks, which every sequence has, come first.
template <typename E, uint32_t D, uint32_t kBits, uint32_t kTiles>
__global__ __launch_bounds__(kFewThreads, kTiles <= 2 ? 2 : 1) void k_attend_few(const AttnParams p) {
    constexpr uint32_t kSteps = D / 32, kOut = D / 16;      // products over channels; tiles of 16 channels of the result
    constexpr uint32_t kRowBytes = 2 * D, kWaveBytes = kFewKeys * kRowBytes;
    constexpr uint32_t kOutStride = D + 4;                  // floats between rows where the wavefronts' results meet
    __shared__ __attribute__((aligned(16))) char lds[kFewWaves * (kWaveBytes > 16 * kOutStride * 4 ? kWaveBytes : 16 * kOutStride * 4)];
    __shared__ float lds_m[kFewWaves][16], lds_l[kFewWaves][16];

    const uint32_t head = blockIdx.x % p.kv_heads, zs = blockIdx.x / p.kv_heads, s = zs % p.batch.n_seqs, z = zs / p.batch.n_seqs;
    const uint32_t lane = threadIdx.x & (kLanes - 1), wave = threadIdx.x / kLanes, col = lane % 16, quad = lane / 16;
    const Seq seq = seq_at(p.batch, s);
    const int32_t n_new = min(seq.n_new, (int32_t)p.batch.max_new);
    const uint32_t rows = (uint32_t)n_new * p.group;
    if (rows == 0 || rows > p.few_rows) return;
    const Span sp = span_of<kFewKeys>(p, seq, 0, n_new - 1);
    const uint32_t first_tile = z * p.few_chunk, last_tile = min(first_tile + p.few_chunk, sp.tiles);
    if (z > 0 && first_tile >= sp.tiles) return;
    const bool alone = sp.tiles <= p.few_chunk;             // no other chunk: this one writes the result itself

    // queries as the second operand: column = row of the result
    u32x4 q[kTiles][kSteps];
    int32_t pos[kTiles];                                    // position of the column's token
#pragma unroll
    for (uint32_t n = 0; n < kTiles; ++n) {
        const uint32_t r = min(n * 16 + col, rows - 1), token = over_group(p, r);
        pos[n] = seq.pos0 + (int32_t)token;
        const char* row = p.q.data + (int64_t)(seq.first + (int32_t)token) * p.q.token_stride + (int64_t)(head * p.group + r - token * p.group) * p.q.head_stride;
#pragma unroll
        for (uint32_t i = 0; i < kSteps; ++i) q[n][i] = *reinterpret_cast<const u32x4*>(row + 2 * Piece<E, D, kBits>::channel(lane, i));
    }
    // keys below `all` are seen by every row of the tile's part, keys from `some` on need a look at each row
    const int32_t pos_first = seq.pos0, pos_last = seq.pos0 + n_new - 1;

    f32x4 o[kTiles][kOut];
    float m[kTiles], l[kTiles];
#pragma unroll
    for (uint32_t n = 0; n < kTiles; ++n) {
        m[n] = -INFINITY, l[n] = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i) o[n][i] = f32x4{0, 0, 0, 0};
    }

    const int32_t* table = p.batch.table + (int64_t)s * p.batch.table_stride;
    const int64_t head_at = (int64_t)head * p.cache.head_stride, pair_head_at = (int64_t)head * p.cache.pair_head_stride;
    using Part = Piece<E, D, kBits>;
    Part k_next, v_next;
    uint32_t seen_next = 0;                                 // one bit a key of the tile: it is there

    auto places = [&](uint32_t tile, Place (&at)[2]) {
        int32_t base, end;
        tile_at<kFewKeys>(sp, tile, base, end);
        const bool in = tile < last_tile;
#pragma unroll
        for (int r = 0; r < 2; ++r) at[r] = place_of(p.cache, table, in ? (uint32_t)(base + 16 * r + (int32_t)col) : 0xFFFFFFFFu, (uint32_t)end);
    };
    auto fetch = [&](const Place (&at)[2]) {
        seen_next = ((uint32_t)__ballot(at[0].there) & 0xFFFFu) | (uint32_t)__ballot(at[1].there) << 16;
#pragma unroll
        for (int r = 0; r < 2; ++r) {                       // where nothing is, the cache's first row stands in
            const int64_t page = at[r].there ? at[r].page : 0, slot = at[r].there ? at[r].slot : 0;
            const int64_t row = page * p.cache.page_stride + slot * p.cache.slot_stride + head_at;
            const int64_t pr = kBits == 4 ? page * p.cache.pair_page_stride + slot * p.cache.pair_slot_stride + pair_head_at : 0;
            k_next.load(p.cache.k + row, p.cache.k_pairs + pr, r, lane);
            v_next.load(p.cache.v + row, p.cache.v_pairs + pr, r, lane);
        }
    };

    char* const mine = lds + wave * kWaveBytes;
    // units of 32 bytes of a row of values change places by the key, so that the 8 rows that a transposing read takes at
    // once lie in different banks
    auto swizzle = [](uint32_t key, uint32_t unit) { return D == 128 ? unit ^ (key & 7u) : unit ^ ((key >> 1) & 3u); };

    Place ahead[2];
    uint32_t tile = first_tile + wave;
    places(tile, ahead);
    fetch(ahead);
    places(tile + kFewWaves, ahead);
    for (; tile < last_tile; tile += kFewWaves) {
        const Part k = k_next, v = v_next;
        const uint32_t seen = seen_next;
        if (tile + kFewWaves < last_tile) {
            fetch(ahead);
            places(tile + 2 * kFewWaves, ahead);
        }
        int32_t base, end;
        tile_at<kFewKeys>(sp, tile, base, end);

        // values to LDS, those that are not there as zeros
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const bool there = (seen >> (16 * r + col)) & 1u;
            const uint32_t key = 16 * r + col;
#pragma unroll
            for (uint32_t i = 0; i < kSteps; ++i) {
                u32x4 x = v.get(r, i);
                if (!there) x = u32x4{0, 0, 0, 0};
                const uint32_t at = 2 * Part::channel(lane, i);
                *reinterpret_cast<u32x4*>(mine + key * kRowBytes + swizzle(key, at / 32) * 32 + at % 32) = x;
            }
        }

        // scores: S^T = K Q^T; the lane has keys 4 quad + 0..3 of both halves for its column
        f32x4 sc[kTiles][2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (uint32_t n = 0; n < kTiles; ++n) sc[n][r] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (uint32_t i = 0; i < kSteps; ++i) {
                const u32x4 a = k.get(r, i);
#pragma unroll
                for (uint32_t n = 0; n < kTiles; ++n) sc[n][r] = mfma16<E>(a, q[n][i], sc[n][r]);
            }
        }

        // does every row see every key of the tile?
        const bool sink_part = tile < sp.sink_tiles;
        const bool each = base + (int32_t)kFewKeys - 1 > pos_first ||
                          (p.window && !sink_part && base + (int32_t)kFewKeys > 0 && (int64_t)base <= (int64_t)pos_last - p.window);
        const bool mixed = each && n_new > 1;
        u32x4 w[kTiles];                                    // weights as the second product takes them
        uint32_t shows[kTiles];                             // one bit a key of the lane: the column's row sees it
#pragma unroll
        for (uint32_t n = 0; n < kTiles; ++n) {
            uint32_t sees = (seen >> (4 * quad) & 15u) | (seen >> (16 + 4 * quad) & 15u) << 4;
            if (each) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int32_t key = base + (j / 4) * 16 + (int32_t)(4 * quad) + j % 4;
                    const bool sight = key <= pos[n] && (!p.window || (int64_t)key > (int64_t)pos[n] - p.window || (uint32_t)key < p.sinks);
                    if (!sight) sees &= ~(1u << j);
                }
            }
            shows[n] = sees;
            float x[8], top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = (sees >> j) & 1u ? sc[n][j / 4][j % 4] * p.scale_log2 : -INFINITY;
                top = fmaxf(top, x[j]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float grown = fmaxf(m[n], top), from = grown == -INFINITY ? 0.0f : grown;
            const float keep = exp2_of(m[n] - from);
            m[n] = grown;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = (sees >> j) & 1u ? exp2_of(x[j] - from) : 0.0f;
                sum += x[j];
            }
            l[n] = l[n] * keep + sum;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[n][j] = pack2<E>(x[2 * j], x[2 * j + 1]);
            if (__any(keep != 1.0f)) {
#pragma unroll
                for (uint32_t i = 0; i < kOut; ++i) o[n][i] *= keep;
            }
        }

        // O^T += V^T P^T: the transposing read gives the lane 4 keys of one channel
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const uint32_t key_a = 4 * quad + col / 4, key_b = key_a + 16, part = (col % 4) * 8;
        uint32_t strange = 0;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i) {
            const u32x2 lo = lds_transposed(mine + key_a * kRowBytes + swizzle(key_a, i) * 32 + part);
            const u32x2 hi = lds_transposed(mine + key_b * kRowBytes + swizzle(key_b, i) * 32 + part);
            u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
            if (mixed) {                                    // a NaN or infinity that only some rows see must not reach the others as 0 * NaN
                uint32_t bad = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) bad |= not_finite16(a[j], kExponent<E>);
                strange |= bad;
                if (__any(bad)) continue;
            }
#pragma unroll
            for (uint32_t n = 0; n < kTiles; ++n) o[n][i] = mfma16<E>(a, w[n], o[n][i]);
        }
        if (mixed && __any(strange)) {                      // rare: these 16 channels key by key, each row with the keys that it sees
            for (uint32_t i = 0; i < kOut; ++i) {
                const u32x2 lo = lds_transposed(mine + key_a * kRowBytes + swizzle(key_a, i) * 32 + part);
                const u32x2 hi = lds_transposed(mine + key_b * kRowBytes + swizzle(key_b, i) * 32 + part);
                const u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
                uint32_t bad = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) bad |= not_finite16(a[j], kExponent<E>);
                if (!__any(bad)) continue;
#pragma unroll
                for (uint32_t n = 0; n < kTiles; ++n) {
                    f32x4 add = {0, 0, 0, 0};
                    for (uint32_t key = 0; key < kFewKeys; ++key) {
                        const uint32_t j = (key / 16) * 4 + key % 4, from = (key % 16) / 4 * 16 + col;
                        const uint32_t pairw = __shfl(j / 2 == 0 ? w[n][0] : j / 2 == 1 ? w[n][1] : j / 2 == 2 ? w[n][2] : w[n][3], from);
                        const bool sees = (__shfl(shows[n], from) >> j) & 1u;
                        const float weight = j % 2 ? high16<E>(pairw) : low16<E>(pairw);
#pragma unroll
                        for (uint32_t c = 0; c < 4; ++c) {
                            const uint32_t at = 2 * (16 * i + 4 * quad + c);
                            const uint32_t x = *reinterpret_cast<const uint16_t*>(mine + key * kRowBytes + swizzle(key, at / 32) * 32 + at % 32);
                            if (sees) add[c] += weight * low16<E>(x);
                        }
                    }
#pragma unroll
                    for (uint32_t ii = 0; ii < kOut; ++ii)
                        if (ii == i) o[n][ii] += add;
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    // the wavefronts' parts join: tile of rows by tile of rows, through LDS
#pragma unroll
    for (uint32_t n = 0; n < kTiles; ++n) {
        float sum = l[n];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        __syncthreads();
        float* const mine_o = reinterpret_cast<float*>(lds) + wave * 16 * kOutStride;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i) *reinterpret_cast<f32x4*>(mine_o + col * kOutStride + 16 * i + 4 * quad) = o[n][i];
        if (quad == 0) lds_m[wave][col] = m[n], lds_l[wave][col] = sum;
        __syncthreads();
        constexpr uint32_t kPer = D / 16;                   // channels a thread joins
        const uint32_t r = threadIdx.x / 16, row = n * 16 + r, c0 = (threadIdx.x % 16) * kPer;
        if (row < rows) {
            float top = -INFINITY;
#pragma unroll
            for (uint32_t w = 0; w < kFewWaves; ++w) top = fmaxf(top, lds_m[w][r]);
            const float from = top == -INFINITY ? 0.0f : top;
            float total = 0.0f, acc[kPer];
#pragma unroll
            for (uint32_t c = 0; c < kPer; ++c) acc[c] = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < kFewWaves; ++w) {
                const float f = exp2_of(lds_m[w][r] - from);
                total += f * lds_l[w][r];
                const float* src = reinterpret_cast<const float*>(lds) + (w * 16 + r) * kOutStride + c0;
                if (lds_m[w][r] != -INFINITY) {
#pragma unroll
                    for (uint32_t c = 0; c < kPer; ++c) acc[c] += f * src[c];
                }
            }
            const uint32_t token = over_group(p, row);
            if (alone) {
                const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
                uint32_t* dst = reinterpret_cast<uint32_t*>(p.out.data + (int64_t)(seq.first + (int32_t)token) * p.out.token_stride +
                                                            (int64_t)(head * p.group + row - token * p.group) * p.out.head_stride + 2 * c0);
#pragma unroll
                for (uint32_t c = 0; c < kPer; c += 2) dst[c / 2] = pack2<E>(acc[c] * inv, acc[c + 1] * inv);
            } else {
                const uint64_t at = (((uint64_t)z * p.batch.n_seqs + s) * p.kv_heads + head) * p.few_stride + row;
                float* dst = p.few_o + at * D + c0;
#pragma unroll
                for (uint32_t c = 0; c < kPer; ++c) dst[c] = acc[c];
                if (c0 == 0) p.few_ml[at] = f32x2{top, total};
            }
        }
    }
}

}  // namespace

#endif  // AT_FEW_HPP
