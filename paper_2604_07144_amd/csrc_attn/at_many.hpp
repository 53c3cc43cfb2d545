// Attention of many rows: whole prompts and chunks of them.  A workgroup takes 128 rows of one sequence and key/value
// head (a row is a new token and one of the query heads that share the key/value head, so keys and values are read once
// for all of them) and goes over the keys that they see, 64 at a time.
//
// Mathematics as in the kernel of few rows.  Matrix products bound this: 4 * D operations per row and key, against
// 4 * D bytes per key that serve 128 rows.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 tiles: a wavefront has 32 rows as
// columns, its queries and results stay in registers, the weights go from the first product's result registers to the
// second's operands without moving, and the maximum of a row is over one lane's registers and one exchange between the
// halves of the wavefront.  The maximum that weights are taken against is only raised when a score passes it by 2^8,
// which 32-bit sums and 16-bit weights both have room for.  Keys and values of the next 64 positions are on their way
// to registers while the present ones, in one of two LDS buffers, are worked on.
#ifndef AT_MANY_HPP
#define AT_MANY_HPP

#include "at_parts.hpp"

namespace {

constexpr uint32_t kManyWaves = 4, kManyThreads = kManyWaves * kLanes;
constexpr float kHeadroom = 8.0f;

template <typename E> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec8<bf16>, a), __builtin_bit_cast(Vec8<bf16>, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec8<fp16>, a), __builtin_bit_cast(Vec8<fp16>, b), c, 0, 0, 0);
}

// max over the two halves of the wavefront
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Where 16-byte piece `c` of a key's (value's) row lies in LDS.  Keys: the 16 rows that a read takes at once hold the
// same piece in 16 different places.  Values: the 64 bytes of 4 rows that a transposing read takes at once likewise.
template <uint32_t D> __device__ __forceinline__ uint32_t key_piece(uint32_t key, uint32_t c) {
    return key * (D / 8) + (D == 128 ? c ^ (key & 15u) : c ^ ((key >> 1) & 7u));
}
template <uint32_t D> __device__ __forceinline__ uint32_t value_piece(uint32_t key, uint32_t c) {
    return key * (D / 8) + (D == 128 ? c ^ ((key & 3u) << 2) : c ^ (((key >> 1) & 1u) << 2));
}

// Workgroups: [tile of rows, last first][chunk][kv head]: late rows see most keys, and the heads of a tile, whose keys
// are other memory, spread over the XCDs while all tiles of a head stay on one.
template <typename E, uint32_t D, uint32_t kBits>
__global__ __launch_bounds__(kManyThreads, 2) void k_attend_many(const AttnParams p, const uint32_t n_row_tiles, const uint32_t n_chunks) {
    constexpr uint32_t kSteps = D / 16, kOut = D / 32, kPieces = D / 8, kRowsAtOnce = kManyThreads / kPieces, kLoads = kManyKeys / kRowsAtOnce;
    __shared__ u32x4 lds_k[2][kManyKeys * kPieces], lds_v[2][kManyKeys * kPieces];
    __shared__ uint32_t lds_seen[2][kManyKeys];

    const uint32_t head = blockIdx.x % p.kv_heads, tz = blockIdx.x / p.kv_heads, z = tz % n_chunks, slot = n_row_tiles - 1 - tz / n_chunks;
    const uint32_t lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), col = lane % 32, half = lane / 32;

    // Sequence s has the row tiles from first[s] * group / 128 + s on up to the next one's, which is never too few.
    auto begins = [&](uint32_t i) { return (uint32_t)((uint64_t)(uint32_t)p.batch.first[i] * p.group / kManyRows) + i; };
    const uint32_t s = count_to(p.batch.n_seqs - 1, slot, begins), slot0 = begins(s);
    const Seq seq = seq_at(p.batch, s);
    const int32_t n_new = min(seq.n_new, (int32_t)p.batch.max_new);
    const uint32_t rows = (uint32_t)n_new * p.group;
    if (slot < slot0 || (uint64_t)(slot - slot0) * kManyRows >= rows || rows <= p.few_rows) return;
    const uint32_t row0 = (slot - slot0) * kManyRows, row1 = min(row0 + kManyRows, rows) - 1;
    const Span sp = span_of<kManyKeys>(p, seq, (int32_t)over_group(p, row0), (int32_t)over_group(p, row1));
    const uint32_t first_tile = z * p.many_chunk, last_tile = min(first_tile + p.many_chunk, sp.tiles);
    if (z > 0 && first_tile >= sp.tiles) return;
    const bool alone = sp.tiles <= p.many_chunk;

    const uint32_t r = min(row0 + wave * 32 + col, rows - 1), token = over_group(p, r);
    const int32_t pos = seq.pos0 + (int32_t)token;
    const uint32_t q_head = head * p.group + r - token * p.group;
    // positions of the wavefront's first and last row
    const int32_t pos_first = seq.pos0 + (int32_t)over_group(p, min(row0 + wave * 32, rows - 1));
    const int32_t pos_last = seq.pos0 + (int32_t)over_group(p, min(row0 + wave * 32 + 31, rows - 1));

    u32x4 q[kSteps];
    {
        const char* row = p.q.data + (int64_t)(seq.first + (int32_t)token) * p.q.token_stride + (int64_t)q_head * p.q.head_stride;
#pragma unroll
        for (uint32_t i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const u32x4*>(row + 32 * i + 16 * half);
    }
    f32x16 o[kOut];
#pragma unroll
    for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = -INFINITY, l = 0.0f;                          // m: scaled to powers of two

    const int32_t* table = p.batch.table + (int64_t)s * p.batch.table_stride;
    const int64_t head_at = (int64_t)head * p.cache.head_stride, pair_head_at = (int64_t)head * p.cache.pair_head_stride;
    const uint32_t my_piece = threadIdx.x % kPieces, my_key = threadIdx.x / kPieces;
    u32x4 next_k[kLoads], next_v[kLoads];
    uint32_t pair_k[kLoads], pair_v[kLoads];
    bool next_there[kLoads];
    Place ahead[kLoads];

    auto places = [&](uint32_t tile) {
        int32_t base, end;
        tile_at<kManyKeys>(sp, tile, base, end);
        const bool in = tile < last_tile;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
            ahead[i] = place_of(p.cache, table, in ? (uint32_t)(base + (int32_t)(my_key + i * kRowsAtOnce)) : 0xFFFFFFFFu, (uint32_t)end);
    };
    auto fetch = [&]() {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) {
            next_there[i] = ahead[i].there;
            const int64_t page = ahead[i].there ? ahead[i].page : 0, at = ahead[i].there ? ahead[i].slot : 0;
            const int64_t row = page * p.cache.page_stride + at * p.cache.slot_stride + head_at;
            if constexpr (kBits == 16) {
                next_k[i] = *reinterpret_cast<const u32x4*>(p.cache.k + row + 16 * my_piece);
                next_v[i] = *reinterpret_cast<const u32x4*>(p.cache.v + row + 16 * my_piece);
            } else {
                const int64_t pr = page * p.cache.pair_page_stride + at * p.cache.pair_slot_stride + pair_head_at + 4 * (my_piece / 8);
                next_k[i][0] = *reinterpret_cast<const uint32_t*>(p.cache.k + row + 4 * my_piece);
                next_v[i][0] = *reinterpret_cast<const uint32_t*>(p.cache.v + row + 4 * my_piece);
                pair_k[i] = *reinterpret_cast<const uint32_t*>(p.cache.k_pairs + pr);
                pair_v[i] = *reinterpret_cast<const uint32_t*>(p.cache.v_pairs + pr);
            }
        }
    };
    auto put = [&](uint32_t buf) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) {
            const uint32_t key = my_key + i * kRowsAtOnce;
            u32x4 k, v;
            if constexpr (kBits == 16) {
                k = next_k[i], v = next_v[i];
            } else {
                k = decode8<E>(next_k[i][0], low16<E>(pair_k[i]), high16<E>(pair_k[i]));
                v = decode8<E>(next_v[i][0], low16<E>(pair_v[i]), high16<E>(pair_v[i]));
            }
            if (!next_there[i]) v = u32x4{0, 0, 0, 0};
            lds_k[buf][key_piece<D>(key, my_piece)] = k;
            lds_v[buf][value_piece<D>(key, my_piece)] = v;
            if (my_piece == 0) lds_seen[buf][key] = next_there[i];
        }
    };

    places(first_tile);
    fetch();
    places(first_tile + 1);
    put(0);
    __syncthreads();
    for (uint32_t tile = first_tile; tile < last_tile; ++tile) {
        const uint32_t buf = (tile - first_tile) & 1u;
        if (tile + 1 < last_tile) {
            fetch();
            places(tile + 2);
        }
        int32_t base, end;
        tile_at<kManyKeys>(sp, tile, base, end);
        if (base <= pos_last) {                             // otherwise all of it lies after the wavefront's rows
            f32x16 sc[2];
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t) {
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[t][j] = 0.0f;
#pragma unroll
                for (uint32_t i = 0; i < kSteps; ++i) sc[t] = mfma32<E>(lds_k[buf][key_piece<D>(32 * t + col, 2 * i + half)], q[i], sc[t]);
            }
            // what is not seen: keys that are not there (any row), keys after a row or before its window
            const uint64_t seen = __ballot(lds_seen[buf][lane] != 0);
            const bool sink_part = tile < sp.sink_tiles;
            const bool each = base + (int32_t)kManyKeys - 1 > pos_first || (p.window && !sink_part && (int64_t)base <= (int64_t)pos_last - p.window);
            uint32_t shows = 0xFFFFFFFFu;                   // one bit a register: the row sees the key
            if (each || seen != ~0ull) {
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t at = 32 * t + (j / 4) * 8 + 4 * half + j % 4;
                        const int32_t key = base + (int32_t)at;
                        const bool sight = ((seen >> at) & 1u) && key <= pos &&
                                           (!p.window || (int64_t)key > (int64_t)pos - p.window || (uint32_t)key < p.sinks);
                        if (!sight) shows &= ~(1u << (16 * t + j)), sc[t][j] = -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = fmaxf(top, sc[t][j]);
            top = max_halves(top) * p.scale_log2;
            const bool raise = top > m + kHeadroom || (m == -INFINITY && top > m);
            if (__any(raise)) {
                const float grown = raise ? top : m, keep = raise ? exp2_of(m - grown) : 1.0f;
                m = grown;
                l *= keep;
#pragma unroll
                for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= keep;
            }
            const float from = m == -INFINITY ? 0.0f : m;
            u32x4 w[4];                                     // weights of 16 keys each, as the second product takes them
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float a = exp2_of(fmaf(sc[t][j], p.scale_log2, -from)), b = exp2_of(fmaf(sc[t][j + 1], p.scale_log2, -from));
                    l += a + b;
                    w[2 * t + j / 8][j % 8 / 2] = pack2<E>(a, b);
                }
            const uint32_t key_in = 4 * half + (lane % 16) / 4, piece_in = ((lane / 16) % 2) * 2 + (lane % 4) / 2, byte_in = (lane % 2) * 8;
            uint32_t strange = 0;                           // one bit an operand that holds a NaN or an infinity
#pragma unroll
            for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
                for (uint32_t t = 0; t < 4; ++t) {
                    const char* at = reinterpret_cast<const char*>(lds_v[buf]);
                    const u32x2 lo = lds_transposed(at + value_piece<D>(16 * t + key_in, 4 * i + piece_in) * 16 + byte_in);
                    const u32x2 hi = lds_transposed(at + value_piece<D>(16 * t + 8 + key_in, 4 * i + piece_in) * 16 + byte_in);
                    const u32x4 a = {lo[0], lo[1], hi[0], hi[1]};
                    if (each) {                             // one that not all rows see must not reach the others as 0 * NaN
                        bool bad = false;
#pragma unroll
                        for (int j = 0; j < 4; ++j) bad |= not_finite16(a[j], kExponent<E>);
                        if (__any(bad)) {
                            strange |= 1u << (4 * i + t);
                            continue;
                        }
                    }
                    o[i] = mfma32<E>(a, w[t], o[i]);
                }
            if (strange) {                                  // rare: those 32 channels of those 16 keys, each row with the keys that it sees
#pragma unroll
                for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll 1
                    for (uint32_t t = 0; t < 4; ++t) {
                        if (!((strange >> (4 * i + t)) & 1u)) continue;
#pragma unroll 1
                        for (uint32_t k = 0; k < 16; ++k) {
                            // key 16 t + k is in the lanes of half (k / 4) % 2, in register 8 (t % 2) + 4 (k / 8) + k % 4 of tile t / 2
                            const uint32_t reg = 16 * (t / 2) + 8 * (t % 2) + 4 * (k / 8) + k % 4, from_lane = (k / 4) % 2 * 32 + col;
                            const u32x4 ws = t == 0 ? w[0] : t == 1 ? w[1] : t == 2 ? w[2] : w[3];
                            const uint32_t two = reg % 8 / 2 == 0 ? ws[0] : reg % 8 / 2 == 1 ? ws[1] : reg % 8 / 2 == 2 ? ws[2] : ws[3];
                            const uint32_t two_in = __shfl(two, from_lane);
                            const bool sees = (__shfl(shows, from_lane) >> reg) & 1u;
                            const float weight = reg % 2 ? high16<E>(two_in) : low16<E>(two_in);
                            const uint32_t key = 16 * t + k;
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const uint32_t ch = 32 * i + (j / 4) * 8 + 4 * half + j % 4;
                                const uint16_t x = reinterpret_cast<const uint16_t*>(lds_v[buf])[value_piece<D>(key, ch / 8) * 8 + ch % 8];
                                if (sees) o[i][j] += weight * low16<E>(x);
                            }
                        }
                    }
            }
        }
        if (tile + 1 < last_tile) put(buf ^ 1u);
        __syncthreads();
    }

    const float total = sum_halves(l);
    if (row0 + wave * 32 + col >= rows) return;
    if (alone) {
        const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
        char* dst = p.out.data + (int64_t)(seq.first + (int32_t)token) * p.out.token_stride + (int64_t)q_head * p.out.head_stride;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const u32x2 x = {pack2<E>(o[i][j] * inv, o[i][j + 1] * inv), pack2<E>(o[i][j + 2] * inv, o[i][j + 3] * inv)};
                *reinterpret_cast<u32x2*>(dst + 2 * (32 * i + 2 * j + 4 * half)) = x;
            }
    } else {
        const uint64_t at = ((uint64_t)z * p.batch.n_tokens + (uint32_t)(seq.first + (int32_t)token)) * p.q_heads + q_head;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const f32x4 x = {o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]};
                *reinterpret_cast<f32x4*>(p.many_o + at * D + 32 * i + 2 * j + 4 * half) = x;
            }
        if (half == 0) p.many_ml[at] = f32x2{m, total};
    }
}

// Joins the chunks of a row: a wavefront takes one row (token, head).
template <typename E, uint32_t D>
__global__ __launch_bounds__(256) void k_join_many(const AttnParams p) {
    const uint32_t per_token = (p.q_heads + 3) / 4;
    const uint32_t t = blockIdx.x / per_token, h = blockIdx.x % per_token * 4 + threadIdx.x / kLanes;
    if (h >= p.q_heads) return;
    const uint32_t s = seq_of(p.batch, t);
    if (s >= p.batch.n_seqs) return;
    const Seq seq = seq_at(p.batch, s);
    const int32_t n_new = min(seq.n_new, (int32_t)p.batch.max_new), i = (int32_t)t - seq.first;
    const uint32_t rows = (uint32_t)n_new * p.group;
    if (i < 0 || i >= n_new || rows <= p.few_rows) return;
    const uint32_t head = h / p.group, row = (uint32_t)i * p.group + h - head * p.group;
    const uint32_t r0 = row / kManyRows * kManyRows, r1 = min(r0 + kManyRows, rows) - 1;
    const uint32_t n = (span_of<kManyKeys>(p, seq, (int32_t)over_group(p, r0), (int32_t)over_group(p, r1)).tiles + p.many_chunk - 1) / p.many_chunk;
    if (n <= 1) return;                                     // written already
    join_row<E, D>(p.many_o, p.many_ml, [&](uint32_t z) { return ((uint64_t)z * p.batch.n_tokens + t) * p.q_heads + h; }, n,
                   p.out.data + (int64_t)t * p.out.token_stride + (int64_t)h * p.out.head_stride);
}

}  // namespace

#endif  // AT_MANY_HPP
