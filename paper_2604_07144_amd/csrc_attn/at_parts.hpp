// What both attention kernels share: their parameters, the part of the keys that rows can see, the matrix units, and the
// kernel that joins the parts of a key axis that was split.
#ifndef AT_PARTS_HPP
#define AT_PARTS_HPP

#include "at_common.hpp"

namespace {

constexpr uint32_t kFewKeys = 32;        // keys that a wavefront of the kernel of few rows takes at a time
constexpr uint32_t kManyKeys = 64;       // keys that a workgroup of the kernel of many rows takes at a time
constexpr uint32_t kManyRows = 128;      // rows of such a workgroup

struct AttnParams {
    Cache cache;
    Batch batch;
    Rows q, out;
    uint32_t q_heads, kv_heads, group;   // group = q_heads / kv_heads
    uint32_t group_magic, group_shift;   // row / group, as for pages
    uint32_t window, sinks;              // window 0: none
    float scale_log2;                    // scale * log2(e)
    uint32_t few_rows;                   // sequences with at most so many rows go to the kernel of few rows, the others to that of many
    uint32_t few_chunk, many_chunk;      // tiles of keys that a workgroup of either takes
    uint32_t few_stride;                 // rows that a (sequence, kv head) has in the workspace
    float *few_o, *many_o;               // what the chunks of a row found: [chunk][sequence][kv head][row][D], [chunk][new token][query head][D]
    f32x2 *few_ml, *many_ml;             // and its (m, l)
};

__device__ __forceinline__ uint32_t over_group(const AttnParams& p, uint32_t row) {
    return __umulhi(row * 2u, p.group_magic) >> p.group_shift;
}

// What the new tokens [i0, i1] of a sequence can see: the sinks [0, sink_end) and then [begin, end), as tiles of kTile keys.
struct Span {
    int32_t sink_end, begin, end;
    uint32_t sink_tiles, tiles;
};

template <uint32_t kTile>
__device__ __forceinline__ Span span_of(const AttnParams& p, const Seq& seq, int32_t i0, int32_t i1) {
    Span r;
    const int64_t last = (int64_t)seq.pos0 + i1;
    r.end = (int32_t)min((int64_t)seq.kv_len, max(last + 1, (int64_t)0));
    r.begin = 0;
    if (p.window) r.begin = (int32_t)min(max((int64_t)seq.pos0 + i0 - p.window + 1, (int64_t)0), (int64_t)r.end);
    r.sink_end = (int32_t)min((int64_t)p.sinks, (int64_t)r.begin);
    r.sink_tiles = (uint32_t)(r.sink_end + kTile - 1) / kTile;
    r.tiles = r.sink_tiles + (uint32_t)(r.end - r.begin + kTile - 1) / kTile;
    return r;
}

// First key of a tile and the end of its part.
template <uint32_t kTile> __device__ __forceinline__ void tile_at(const Span& sp, uint32_t tile, int32_t& base, int32_t& end) {
    const bool sink = tile < sp.sink_tiles;
    base = sink ? (int32_t)(tile * kTile) : sp.begin + (int32_t)((tile - sp.sink_tiles) * kTile);
    end = sink ? sp.sink_end : sp.end;
}

template <typename E> __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec8<bf16>, a), __builtin_bit_cast(Vec8<bf16>, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec8<fp16>, a), __builtin_bit_cast(Vec8<fp16>, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x2 lds_transposed(const char* at) {
    typedef __attribute__((address_space(3))) s16x4* Ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(at)));
}

__device__ __forceinline__ bool not_finite16(uint32_t two, uint32_t exponent) {
    return (two & exponent) == exponent || ((two >> 16) & exponent) == exponent;
}
template <typename E> constexpr uint32_t kExponent = std::is_same_v<E, bf16> ? 0x7F80u : 0x7C00u;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126: 0

// Joins the chunks of a row: a wavefront takes one row (token, head), a lane D / 64 of its channels.
template <typename E, uint32_t D>
__global__ __launch_bounds__(256) void k_attend_join(const AttnParams p) {
    const uint32_t lane = threadIdx.x & (kLanes - 1);
    const uint32_t per_token = (p.q_heads + 3) / 4;
    const uint32_t t = blockIdx.x / per_token, h = blockIdx.x % per_token * 4 + threadIdx.x / kLanes;
    if (h >= p.q_heads) return;
    const uint32_t s = seq_of(p.batch, t);
    if (s >= p.batch.n_seqs) return;
    const Seq seq = seq_at(p.batch, s);
    const int32_t n_new = min(seq.n_new, (int32_t)p.batch.max_new), i = (int32_t)t - seq.first;
    const uint32_t rows = (uint32_t)n_new * p.group;
    if (i < 0 || i >= n_new) return;
    const uint32_t head = h / p.group, row = (uint32_t)i * p.group + h - head * p.group;
    uint32_t n;
    const float* part_o;
    const f32x2* part_ml;
    uint64_t at, stride;
    if (rows <= p.few_rows) {
        part_o = p.few_o, part_ml = p.few_ml;
        at = ((uint64_t)s * p.kv_heads + head) * p.few_stride + row, stride = (uint64_t)p.batch.n_seqs * p.kv_heads * p.few_stride;
        n = (span_of<kFewKeys>(p, seq, 0, n_new - 1).tiles + p.few_chunk - 1) / p.few_chunk;
    } else {
        part_o = p.many_o, part_ml = p.many_ml;
        at = (uint64_t)t * p.q_heads + h, stride = (uint64_t)p.batch.n_tokens * p.q_heads;
        const uint32_t r0 = row / kManyRows * kManyRows, r1 = min(r0 + kManyRows, rows) - 1;
        n = (span_of<kManyKeys>(p, seq, (int32_t)(r0 / p.group), (int32_t)(r1 / p.group)).tiles + p.many_chunk - 1) / p.many_chunk;
    }
    if (n <= 1) return;                                     // written already
    float top = -INFINITY;
    for (uint32_t z = lane; z < n; z += kLanes) top = fmaxf(top, part_ml[at + z * stride][0]);
#pragma unroll
    for (uint32_t m = 1; m < kLanes; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    const float from = top == -INFINITY ? 0.0f : top;
    float total = 0.0f, acc[D / 64];
#pragma unroll
    for (uint32_t c = 0; c < D / 64; ++c) acc[c] = 0.0f;
#pragma unroll 4
    for (uint32_t z = 0; z < n; ++z) {
        const f32x2 ml = part_ml[at + z * stride];
        const float f = exp2_of(ml[0] - from);
        const float* src = part_o + (at + z * stride) * D + lane * (D / 64);
        total += f * ml[1];
#pragma unroll
        for (uint32_t c = 0; c < D / 64; ++c) acc[c] += ml[0] == -INFINITY ? 0.0f : f * src[c];
    }
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    char* dst = p.out.data + (int64_t)t * p.out.token_stride + (int64_t)h * p.out.head_stride;
    if constexpr (D == 128) reinterpret_cast<uint32_t*>(dst)[lane] = pack2<E>(acc[0] * inv, acc[1] * inv);
    else reinterpret_cast<E*>(dst)[lane] = (E)(acc[0] * inv);
}

}  // namespace

#endif  // AT_PARTS_HPP
