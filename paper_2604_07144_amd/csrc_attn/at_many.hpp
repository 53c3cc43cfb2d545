// Attention of many rows: whole prompts and chunks of them.  A workgroup takes some rows of one sequence and key/value
// head (a row is a new token and one of the query heads that share the key/value head, so keys and values are read once
// for all of them) and goes over the keys that they see, 64 at a time.
//
// Mathematics as in the kernel of few rows.  The matrix units and the exponentials bound this together: 64 keys cost a
// wavefront's 32 rows about 1000 cycles of either (128 channels).  S^T = K Q^T and O^T = V^T P^T on 32x32x16 tiles: a
// wavefront has 32 rows as columns, its queries and results stay in registers, the weights go from the first product's
// result registers to the second's operands without moving, and the maximum of a row is over one lane's registers and one
// exchange between the halves of the wavefront.  The maximum that weights are taken against is only raised when a score
// passes it by 8 (a weight would by 2^8), which 32-bit sums and 16-bit weights both have room for.  Two wavefronts of a SIMD take turns at the
// matrix units and the exponentials.  The next 64 keys and values are on their way to the other of two LDS buffers while
// the present ones are worked on: in 16 bits without passing through registers, in 4 bits decoded on the way.
//
// Measured, 32 heads on 8, 128 channels, bf16: the last 2048 tokens of 32768 at 935 to 960 TFLOP/s (a large matrix product of the
// library 1200), whole prompts of 8192 840, of 1024 550, of 512 380: a workgroup's first tile waits for four trips to memory.
// In 4 bits 150 instructions a tile and wavefront of decoding are added, and 740 TFLOP/s are reached.
#ifndef AT_MANY_HPP
#define AT_MANY_HPP

#include "at_parts.hpp"

namespace {

constexpr float kHeadroom = 8.0f;

// A cache in 4 bits is decoded to fp16, whose 11 bits keep codes of 4 on a lowest value and step of 8 where bf16 would round
// them away (a chunk's results were off by 0.0039 of themselves, and are by 0.0017, which is the final rounding).  With bf16 pairs that
// holds a tile whose groups all lie, by their largest magnitude, from 2^-12 up to 2^14 (keys) and 2^8 (values), or are zero.
// By its range fp16 loses at most half of 2^-24 with the lowest value, the rounding and each of 15 steps, 17 * 2^-25: 2^-11.9 of a group
// of 2^-9, and 2^-8.9, which is what bf16 rounds away of its largest, of the smallest group taken.  Any other tile is decoded
// to bf16 and multiplied as that, which takes 1.2 to 1.5 times as long (all tiles of 3 chunks of 1024 tokens over up to 8192 703 us
// against 477, of a prompt of 8192 568 against 415).
constexpr float kGroupLeast = 0.000244140625f, kKeyMost = 16384.0f, kValueMost = 256.0f;
template <typename E> __device__ __forceinline__ bool ordinary(uint32_t key_pair, uint32_t value_pair) {
    auto most = [](uint32_t pr) { return fmaxf(fabsf(high16<E>(pr)), fabsf(fmaf(15.0f, low16<E>(pr), high16<E>(pr)))) + 0.0f * low16<E>(pr); };
    const float k = most(key_pair), v = most(value_pair);
    if constexpr (std::is_same_v<E, fp16>) return v < 65504.0f;              // decoded alike; the values are finite
    else return ((k >= kGroupLeast && k < kKeyMost) || k == 0.0f) && ((v >= kGroupLeast && v < kValueMost) || v == 0.0f);
}

// Eight codes of a dword as fp16: 1024 + code, whose bits are the code's beside an exponent, gives the code exactly, and one
// multiply-add the value, rounded once.  `pair` is (step, lo) in fp16.
__device__ __forceinline__ u32x4 decode8_fp16(uint32_t codes, Vec2<fp16> pair) {
    const Vec2<fp16> unit = {(fp16)1.0f, (fp16)0.0625f}, bias = {(fp16)-1024.0f, (fp16)-64.0f}, step = {pair[0], pair[0]}, lo = {pair[1], pair[1]};
    u32x4 r;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {                      // a byte's low code in the low half, its high code, times 16, in the high half
        const uint32_t x = __builtin_amdgcn_perm(0x64646464u, codes, 0x04000400u + i * 0x00010001u) & 0x64F0640Fu;
        r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_elementwise_fma(__builtin_bit_cast(Vec2<fp16>, x), unit, bias), step, lo));
    }
    return r;
}
template <typename E> __device__ __forceinline__ Vec2<fp16> pair_fp16(uint32_t pr) { return Vec2<fp16>{(fp16)low16<E>(pr), (fp16)high16<E>(pr)}; }

__device__ const u32x4 kZeroRow[16] = {};                   // stands in for keys and values that are not there

template <typename E> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec8<bf16>, a), __builtin_bit_cast(Vec8<bf16>, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec8<fp16>, a), __builtin_bit_cast(Vec8<fp16>, b), c, 0, 0, 0);
}

// max and sum over the two halves of the wavefront
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes of each lane from memory to LDS, to `to` + 16 * lane.  The data passes no register, so that nothing here is in
// flight that the compiler could take for there; wait_loads() has to come between it and the barrier after which it is read.
// (m0 says where in LDS: a reserved register, in which the compiler keeps nothing and which it takes in no list of what a statement
// changes.)
__device__ __forceinline__ void load_to_lds(const char* from, const void* to) {
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(at), "v"(from) : "memory");
}
// 16 bytes at an address that came through LDS, from which the compiler cannot tell that it lies in memory: a load that may be
// either holds up the waits for LDS until it is there.
__device__ __forceinline__ u32x4 load_global(const char* from) {
    return *(__attribute__((address_space(1))) const u32x4*)(uintptr_t)from;
}
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70);                     // vmcnt(0); the compiler knows of it, and waits for none of its own loads again
    asm volatile("" : : : "memory");
}

// Where 16-byte piece `c` of a key's (value's) row lies in LDS, in its row.  Keys: the 16 rows that a read takes at once
// hold the same piece in 16 different places.  Values: the 64 bytes of 4 rows that a transposing read takes at once likewise,
// and so do neighbouring rows of which decoded pieces of one number are written at once.
template <uint32_t D> __device__ __forceinline__ uint32_t key_piece(uint32_t key, uint32_t c) { return D == 128 ? c ^ (key & 15u) : c ^ ((key >> 1) & 7u); }
template <uint32_t D> __device__ __forceinline__ uint32_t value_piece(uint32_t key, uint32_t c) { return D == 128 ? c ^ (key & 3u) * 5u : c ^ ((key >> 1) & 1u) * 5u; }

// Workgroups that registers leave room for on a CU.
template <uint32_t D, uint32_t kBits> constexpr uint32_t kManyPerCu = D == 128 ? 2 : kBits == 16 ? 4 : 3;

// Workgroups: [tile of rows, last first][chunk][kv head]: late rows see most keys, and the heads of a tile, whose keys
// are other memory, spread over the XCDs while all tiles of a head stay on one.
template <typename E, uint32_t D, uint32_t kBits>
__global__ __launch_bounds__(kManyThreads, (kManyPerCu<D, kBits>)) void k_attend_many(const AttnParams p, const uint32_t n_row_tiles, const uint32_t n_chunks) {
    constexpr uint32_t kSteps = D / 16, kOut = D / 32, kPieces = D / 8;
    constexpr bool kCodes = kBits == 4;
    using P = std::conditional_t<kCodes, fp16, E>;          // what ordinary tiles are multiplied in
    constexpr bool kMixed = !std::is_same_v<P, E>;
    __shared__ u32x4 lds_k[2][kManyKeys * kPieces], lds_v[2][kManyKeys * kPieces];
    __shared__ const char *lds_at_k[2][kManyKeys], *lds_at_v[2][kManyKeys];                // where the rows of a tile lie
    __shared__ u32x4 lds_pairs[kCodes ? 2 : 1][kManyKeys];  // of a key's groups, then of a value's
    __shared__ uint32_t lds_odd[4];                         // as lds_seen: a key is not ordinary()
    __shared__ uint32_t lds_strange;                        // the last tile, counted from 1, whose values hold a NaN or an infinity
    __shared__ uint64_t lds_seen[4];                        // one bit a key: it is there; written two tiles ahead, while the present one's is read

    const uint32_t head = blockIdx.x % p.kv_heads, tz = blockIdx.x / p.kv_heads, z = tz % n_chunks, slot = n_row_tiles - 1 - tz / n_chunks;
    const uint32_t lane = threadIdx.x & (kLanes - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), col = lane % 32, half = lane / 32;

    // Sequence s has the row tiles from first[s] * group / kManyRows + s on up to the next one's, which is never too few.
    auto begins = [&](uint32_t i) { return (uint32_t)((uint64_t)(uint32_t)p.batch.first[i] * p.group / kManyRows) + i; };
    uint32_t s, slot0;
    Seq seq;
    if (p.batch.n_seqs <= kLanes) {                         // a lane each, lengths and all in one trip to memory
        const uint32_t i = min(lane, p.batch.n_seqs - 1), first = begins(i);
        const Seq mine = seq_at(p.batch, i);
        s = uniform((uint32_t)__popcll(__ballot(lane > 0 && lane < p.batch.n_seqs && first <= slot)));
        slot0 = __builtin_amdgcn_readlane(first, s);
        seq = Seq{(int32_t)__builtin_amdgcn_readlane(mine.first, s), (int32_t)__builtin_amdgcn_readlane(mine.n_new, s),
                  (int32_t)__builtin_amdgcn_readlane(mine.kv_len, s), (int32_t)__builtin_amdgcn_readlane(mine.pos0, s)};
    } else {
        s = uniform(count_to(p.batch.n_seqs - 1, slot, begins)), slot0 = uniform(begins(s));
        seq = seq_at(p.batch, s);
    }
    seq = Seq{uniform(seq.first), uniform(seq.n_new), uniform(seq.kv_len), uniform(seq.pos0)};
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
    const int32_t behind = p.window ? (int32_t)max((int64_t)pos - p.window, (int64_t)INT32_MIN) : INT32_MIN;   // a key is seen from behind + 1 on
    // positions of the wavefront's first and last row
    const int32_t pos_first = seq.pos0 + (int32_t)over_group(p, min(row0 + wave * 32, rows - 1));
    const int32_t pos_last = seq.pos0 + (int32_t)over_group(p, min(row0 + wave * 32 + 31, rows - 1));

    const char* const q_row = p.q.data + (int64_t)(seq.first + (int32_t)token) * p.q.token_stride + (int64_t)(head * p.group + r - token * p.group) * p.q.head_stride + 16 * half;
    u32x4 q[kSteps];
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const u32x4*>(q_row + 32 * i);
    float q_unit = p.scale_log2;                            // of the scores, in powers of two
    if constexpr (kMixed) {                                 // to fp16: the row's largest is brought just below 2^14 by a power of two
        float most = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kSteps; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = fabsf(low16<E>(q[i][j])), b = fabsf(high16<E>(q[i][j]));
                most = fmaxf(most, fmaxf(a < INFINITY ? a : 0.0f, b < INFINITY ? b : 0.0f));
            }
        const int e = max(exponent_above(max_halves(most)), -100);
        const float up = power2(14 - e);
        q_unit = fmaxf(q_unit * power2(e - 14), 1.17549435e-38f);      // not 0, which would make NaN of what is hidden by minus infinity; scores are as good as 0 there
#pragma unroll
        for (uint32_t i = 0; i < kSteps; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) q[i][j] = pack2<P>(low16<E>(q[i][j]) * up, high16<E>(q[i][j]) * up);
    }
    f32x16 o[kOut];
#pragma unroll
    for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;
    float m = -INFINITY, l = 0.0f;                          // m: scaled to powers of two

    const int32_t* table = p.batch.table + (int64_t)s * p.batch.table_stride;
    const int64_t head_at = (int64_t)head * p.cache.head_stride, pair_head_at = (int64_t)head * p.cache.pair_head_stride;

    // ---- where a tile's keys lie: one wavefront looks them up, a lane a key, two tiles ahead; in 4 bits three, and reads their
    // pairs one tile later
    Place ahead;
    u32x4 ahead_pairs = {0, 0, 0, 0};
    auto fetch_pairs = [&]() {
        ahead_pairs = u32x4{0, 0, 0, 0};
        if (!ahead.there) return;
        const int64_t at = ahead.page * p.cache.pair_page_stride + ahead.slot * p.cache.pair_slot_stride + pair_head_at;
        if constexpr (D == 128) {
            const u32x2 k = *reinterpret_cast<const u32x2*>(p.cache.k_pairs + at), v = *reinterpret_cast<const u32x2*>(p.cache.v_pairs + at);
            ahead_pairs = u32x4{k[0], k[1], v[0], v[1]};
        } else {
            ahead_pairs[0] = *reinterpret_cast<const uint32_t*>(p.cache.k_pairs + at), ahead_pairs[2] = *reinterpret_cast<const uint32_t*>(p.cache.v_pairs + at);
        }
    };
    auto places = [&](uint32_t tile) {
        int32_t base, end;
        tile_at<kManyKeys>(sp, tile, base, end);
        ahead = place_of(p.cache, table, tile < last_tile ? (uint32_t)(base + (int32_t)lane) : 0xFFFFFFFFu, (uint32_t)end);
    };
    auto put_places = [&](uint32_t tile) {                  // counted from the first
        const uint32_t buf = tile & 1u;
        const uint64_t seen = __ballot(ahead.there);
        const int64_t row = ahead.page * p.cache.page_stride + ahead.slot * p.cache.slot_stride + head_at;
        const char* zero = kBits == 16 ? reinterpret_cast<const char*>(kZeroRow) : nullptr;
        lds_at_k[buf][lane] = ahead.there ? p.cache.k + row : zero;
        lds_at_v[buf][lane] = ahead.there ? p.cache.v + row : zero;
        if constexpr (kCodes) {
            lds_pairs[buf][lane] = ahead_pairs;
            const bool odd = __any(!ordinary<E>(ahead_pairs[0], ahead_pairs[2]) || (D == 128 && !ordinary<E>(ahead_pairs[1], ahead_pairs[3])));
            if (lane == 0) lds_odd[tile & 3u] = odd;
        }
        if (lane == 0) lds_seen[tile & 3u] = seen;
    };

    // ---- how a tile comes to LDS.  16 bits: an instruction takes kRows whole rows; lanes ask for the pieces in the order in
    // which they shall lie.  4 bits: a thread takes 16 bytes of codes, 32 channels, of a key and a value.
    constexpr uint32_t kRows = kLanes / kPieces, kLoads = kManyKeys / kRows / kManyWaves;
    constexpr uint32_t kCodePieces = D / 32, kCodeThreads = kManyKeys * kCodePieces;
    u32x4 raw_k = {0, 0, 0, 0}, raw_v = {0, 0, 0, 0};
    const uint32_t code_key = threadIdx.x / kCodePieces, code_piece = threadIdx.x % kCodePieces;
    auto fetch = [&](uint32_t buf) {
        if constexpr (kBits == 16) {
#pragma unroll
            for (uint32_t i = 0; i < kLoads; ++i) {
                const uint32_t at = (i * kManyWaves + wave) * kRows, key = at + lane / kPieces, c = lane % kPieces;
                load_to_lds(lds_at_k[buf][key] + 16 * key_piece<D>(key, c), &lds_k[buf][at * kPieces]);
                load_to_lds(lds_at_v[buf][key] + 16 * value_piece<D>(key, c), &lds_v[buf][at * kPieces]);
            }
        } else if (kCodeThreads >= kManyThreads || threadIdx.x < kCodeThreads) {
            const char *at_k = lds_at_k[buf][code_key], *at_v = lds_at_v[buf][code_key];
            raw_k = raw_v = u32x4{0, 0, 0, 0};
            if (at_k) {
                raw_k = load_global(at_k + 16 * code_piece);
                raw_v = load_global(at_v + 16 * code_piece);
            }
        }
    };
    auto put = [&](uint32_t tile) {                         // counted from the first
        if constexpr (kCodes) {
            if (kCodeThreads >= kManyThreads || threadIdx.x < kCodeThreads) {
                const uint32_t buf = tile & 1u;
                const uint32_t* const pairs = reinterpret_cast<const uint32_t*>(&lds_pairs[buf][code_key]) + code_piece / 2;
                const uint32_t pair_k = pairs[0], pair_v = pairs[2];
                if (!kMixed || !uniform(lds_odd[tile & 3u])) {
                    const Vec2<fp16> half_k = pair_fp16<E>(pair_k), half_v = pair_fp16<E>(pair_v);
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        lds_k[buf][code_key * kPieces + key_piece<D>(code_key, 4 * code_piece + i)] = decode8_fp16(raw_k[i], half_k);
                        lds_v[buf][code_key * kPieces + value_piece<D>(code_key, 4 * code_piece + i)] = decode8_fp16(raw_v[i], half_v);
                    }
                } else {
#pragma unroll 1
                    for (uint32_t i = 0; i < 4; ++i) {
                        lds_k[buf][code_key * kPieces + key_piece<D>(code_key, 4 * code_piece + i)] = decode8<E>(raw_k[i], low16<E>(pair_k), high16<E>(pair_k));
                        lds_v[buf][code_key * kPieces + value_piece<D>(code_key, 4 * code_piece + i)] = decode8<E>(raw_v[i], low16<E>(pair_v), high16<E>(pair_v));
                    }
                }
            }
        }
    };

    // positions of the workgroup's first and last row
    const int32_t all_first = seq.pos0 + (int32_t)uniform(over_group(p, row0)), all_last = seq.pos0 + (int32_t)uniform(over_group(p, row1));

    if (threadIdx.x == 0) lds_strange = 0;
    auto begin_with = [&](uint32_t tile) {                  // counted from the first
        places(first_tile + tile);
        if constexpr (kCodes) fetch_pairs();
        put_places(tile);
    };
    constexpr uint32_t kLookAhead = kCodes ? 3 : 2;
    if (wave == 0) begin_with(0);
    __syncthreads();
    fetch(0);
    if (wave == 0) begin_with(1);
    if (kCodes && wave == kManyWaves - 1) places(first_tile + 2);
    put(0);
    wait_loads();
    __syncthreads();
    auto odd_at = [&](uint32_t tile) { return uniform(lds_odd[(tile - first_tile) & 3u]); };
    auto step = [&](auto type, uint32_t tile) {
        using T = decltype(type);                           // what the tile is multiplied in; other than P only with queries as they were given
        constexpr bool kGiven = !std::is_same_v<T, P>;
        const uint32_t buf = (tile - first_tile) & 1u;
        const uint64_t seen_all = lds_seen[(tile - first_tile) & 3u];
        const uint32_t seen_lo = __builtin_amdgcn_readfirstlane((uint32_t)seen_all), seen_hi = __builtin_amdgcn_readfirstlane((uint32_t)(seen_all >> 32));
        const bool odd = kMixed ? kGiven : !kCodes || odd_at(tile) != 0;
        if (tile + 1 < last_tile) fetch(buf ^ 1u);
        const uint32_t turn = tile - first_tile;
        const bool puts = ((turn + kManyWaves - (kLookAhead - 2)) & (kManyWaves - 1)) == wave;
        if (kCodes && puts) fetch_pairs();
        if ((turn & (kManyWaves - 1)) == wave) places(tile + kLookAhead);
        int32_t base, end;
        tile_at<kManyKeys>(sp, tile, base, end);
        const bool sink_part = tile < sp.sink_tiles;
        // Where not all rows see all keys, a NaN or infinity among the values must not reach the others as 0 * NaN: the rows
        // that see it take it as it is (a weight does not change it), and zero stands in for it.
        if (odd && (base + (int32_t)kManyKeys - 1 > all_first || (p.window && !sink_part && (int64_t)base <= (int64_t)all_last - p.window))) {
            constexpr uint32_t kMine = kManyKeys * kPieces / kManyThreads;
            uint32_t bad = 0;                               // the exponent, all ones, carries into the sign's place
#pragma unroll
            for (uint32_t i = 0; i < kMine; ++i) {
                const u32x4 x = lds_v[buf][i * kManyThreads + threadIdx.x];
#pragma unroll
                for (int j = 0; j < 4; ++j) bad |= (x[j] & 0x7FFF7FFFu) + kExponentStep<E>;
            }
            if (bad & 0x80008000u) lds_strange = tile + 1;
            __syncthreads();
            if (uniform(lds_strange) == tile + 1) {
#pragma unroll 1
                for (uint32_t k = 0; k < kManyKeys; ++k) {
                    const int32_t key = base + (int32_t)k;
                    const bool there = ((k < 32 ? seen_lo >> k : seen_hi >> (k - 32)) & 1u) != 0;
                    const bool sight = there && key <= pos && (key > behind || (uint32_t)key < p.sinks);
#pragma unroll
                    for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const uint32_t c = 32 * i + (j / 4) * 8 + 4 * half + j % 4;
                            const uint32_t x = reinterpret_cast<const uint16_t*>(lds_v[buf])[(k * kPieces + value_piece<D>(k, c / 8)) * 8 + c % 8];
                            if (sight && (x & kExponent<E>) == kExponent<E>) o[i][j] += low16<E>(x);
                        }
                }
                __syncthreads();
#pragma unroll 1
                for (uint32_t i = 0; i < kMine; ++i) {
                    u32x4 x = lds_v[buf][i * kManyThreads + threadIdx.x];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if ((x[j] & kExponent<E>) == kExponent<E>) x[j] &= 0xFFFF0000u;
                        if ((x[j] >> 16 & kExponent<E>) == kExponent<E>) x[j] &= 0xFFFFu;
                    }
                    lds_v[buf][i * kManyThreads + threadIdx.x] = x;
                }
                __syncthreads();
            }
        }
        // work, unless all of the tile lies after the wavefront's rows or before their windows
        if (base <= pos_last && !(p.window && !sink_part && (uint32_t)base >= p.sinks && (int64_t)base + kManyKeys - 1 <= (int64_t)pos_first - p.window)) {
            const float unit = kGiven ? p.scale_log2 : q_unit;
            auto query = [&](uint32_t i) {
                if constexpr (!kGiven) return q[i];
                asm volatile("" : : : "memory");
                return *reinterpret_cast<const u32x4*>(q_row + 32 * i);
            };
            const char* const keys = reinterpret_cast<const char*>(lds_k[buf]);
            const char* const values = reinterpret_cast<const char*>(lds_v[buf]);
            f32x16 sc[2];
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) sc[t][j] = 0.0f;
            // Which wavefront of a SIMD goes first matters where one has products to give out: with 128 channels the first product's
            // (0.99 of the time over calls of many kinds, 0.94 to 1.02), with 64 the second's with its exponentials (0.97, 0.95 to 0.99);
            // the other way round 0.985 (0.88 to 1.10) and 0.995.
            // pieces are told apart by exclusive or, so one number and the product's give the place
            if constexpr (D == 128) __builtin_amdgcn_s_setprio(1);
            const uint32_t key_at = here(col * (2 * D) + key_piece<D>(col, half) * 16);
#pragma unroll
            for (uint32_t i = 0; i < kSteps; ++i) {
                const u32x4 x = query(i);
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t)
                    sc[t] = mfma32<T>(*reinterpret_cast<const u32x4*>(keys + 32 * t * (2 * D) + (key_at ^ (32 * i))), x, sc[t]);
            }
            // six operands are read ahead of the products
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (uint32_t i = 0; i < 2 * kSteps - 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);

            if constexpr (D == 128) __builtin_amdgcn_s_setprio(0);
            // what is not seen: keys that are not there (any row), keys after a row or before its window
            const bool each = base + (int32_t)kManyKeys - 1 > pos_first || (p.window && !sink_part && (int64_t)base <= (int64_t)pos_last - p.window);
            if (each || (seen_lo & seen_hi) != ~0u) {
#pragma unroll
                for (uint32_t t = 0; t < 2; ++t) {
                    // register j has key 8 (j / 4) + j % 4 from here on; bit j of each number says so of it
                    const int32_t key0 = base + (int32_t)(32 * t + 4 * half);
                    const uint32_t there = (t ? seen_hi : seen_lo) >> (4 * half);
                    uint32_t shows = (there & 15u) | (there >> 4 & 0xF0u) | (there >> 8 & 0xF00u) | (there >> 12 & 0xF000u);
                    auto below = [&](int64_t n) {           // registers whose key is below key0 + n
                        const uint32_t x = (uint32_t)min(max(n, (int64_t)0), (int64_t)32);
                        return (1u << (4 * (x / 8) + min(x % 8, 4u))) - 1u;
                    };
                    shows &= below((int64_t)pos - key0 + 1);
                    shows &= ~below((int64_t)behind - key0 + 1) | below((int64_t)p.sinks - key0);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sc[t][j] = (shows >> j) & 1u ? sc[t][j] : -INFINITY;
                }
            }
            float top = sc[0][0];
#pragma unroll
            for (int j = 1; j < 32; ++j) top = fmaxf(top, sc[j / 16][j % 16]);
            top = max_halves(top) * unit;
            const bool raise = top > m + kHeadroom || (m == -INFINITY && top > m);
            if (__any(raise)) {
                const float grown = raise ? top : m, keep = raise && m != -INFINITY ? exp2_of(m - grown) : 1.0f;
                m = grown;
                l *= keep;
#pragma unroll
                for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[i][j] *= keep;
            }
            const float from = m == -INFINITY ? 0.0f : m - kWeightUp<P>;
            if constexpr (D == 64) __builtin_amdgcn_s_setprio(1);
            u32x4 w[4];                                     // weights of 16 keys each, as the second product takes them
#pragma unroll
            for (uint32_t t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float a = exp2_of(fmaf(sc[t][j], unit, -from)), b = exp2_of(fmaf(sc[t][j + 1], unit, -from));
                    w[2 * t + j / 8][j % 8 / 2] = pack2<T>(a, b);
                    l = add2<T>(w[2 * t + j / 8][j % 8 / 2], l);
                }
            const uint32_t key_in = 4 * half + (lane % 16) / 4, piece_in = ((lane / 16) % 2) * 2 + (lane % 4) / 2, byte_in = (lane % 2) * 8;
            const uint32_t value_at = here(key_in * (2 * D) + value_piece<D>(key_in, piece_in) * 16 + byte_in);
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)                // channels 32 i .. of keys 16 t ..
#pragma unroll
                for (uint32_t i = 0; i < kOut; ++i) {
                    const char* at = values + (value_at ^ (64 * i));
                    const u32x2 lo = lds_transposed(at + 16 * t * (2 * D)), hi = lds_transposed(at + (16 * t + 8) * (2 * D));
                    o[i] = mfma32<T>(u32x4{lo[0], lo[1], hi[0], hi[1]}, w[t], o[i]);
                }
        }
        if constexpr (D == 64) __builtin_amdgcn_s_setprio(0);
        if (tile + 1 < last_tile) put(turn + 1);
        if (puts) put_places(turn + 2);
        wait_loads();
        __syncthreads();
    };
    if constexpr (kMixed) {                                 // loops of their own, so that neither moves the other's registers
        for (uint32_t tile = first_tile; tile < last_tile;) {
            for (; tile < last_tile && !odd_at(tile); ++tile) step(P{}, tile);
            for (; tile < last_tile && odd_at(tile); ++tile) step(E{}, tile);
        }
    } else {
        for (uint32_t tile = first_tile; tile < last_tile; ++tile) step(P{}, tile);
    }

    const float total = sum_halves(l);
    const uint32_t row = row0 + wave * 32 + here(col);
    if (alone) {
        // the halves of the wavefront have 4 channels each of every 8: they change every other 4, so that each has 8 in a row
        const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
        char* dst = p.out.data + (int64_t)(seq.first + (int32_t)token) * p.out.token_stride + (int64_t)(head * p.group + r - token * p.group) * p.out.head_stride + 16 * half;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
                const auto a = __builtin_amdgcn_permlane32_swap(pack2<E>(o[i][j] * inv, o[i][j + 1] * inv), pack2<E>(o[i][j + 4] * inv, o[i][j + 5] * inv), false, false);
                const auto b = __builtin_amdgcn_permlane32_swap(pack2<E>(o[i][j + 2] * inv, o[i][j + 3] * inv), pack2<E>(o[i][j + 6] * inv, o[i][j + 7] * inv), false, false);
                if (row < rows) *reinterpret_cast<u32x4*>(dst + 2 * (32 * i + 2 * j)) = u32x4{a[0], b[0], a[1], b[1]};
            }
    } else if (row < rows) {
        const uint64_t at = ((uint64_t)z * p.batch.n_tokens + (uint32_t)(seq.first + (int32_t)token)) * p.q_heads + head * p.group + r - token * p.group;
#pragma unroll
        for (uint32_t i = 0; i < kOut; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const f32x4 x = {o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]};
                *reinterpret_cast<f32x4*>(p.many_o + at * D + 32 * i + 2 * j + 4 * half) = x;
            }
        if (half == 0) p.many_ml[at] = f32x2{m - kWeightUp<P>, total};
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
