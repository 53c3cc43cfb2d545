// What both attention kernels share: their parameters, the part of the keys that rows can see, the matrix units, and the
// kernel that joins the parts of a key axis that was split.
#ifndef AT_PARTS_HPP
#define AT_PARTS_HPP

#include "at_common.hpp"

namespace {

constexpr uint32_t kFewKeys = 32;        // keys that a wavefront of the kernel of few rows takes at a time
constexpr uint32_t kManyKeys = 64;       // keys that a workgroup of the kernel of many rows takes at a time
constexpr uint32_t kManyWaves = 4, kManyThreads = kManyWaves * kLanes;
constexpr uint32_t kManyRows = 32 * kManyWaves;   // rows of such a workgroup

struct AttnParams {
    Cache cache;
    Batch batch;
    Rows q, out;
    uint32_t q_heads, kv_heads, group;   // group = q_heads / kv_heads
    uint32_t group_magic, group_shift;   // row / group, as for pages
    uint32_t window, sinks;              // window 0: none
    float scale_log2;                    // scale * log2(e)
    uint32_t few_rows;                   // sequences with at most so many rows go to the kernel of few rows, the others to that of many
    uint32_t few_waves, few_least;       // few rows: so many wavefronts share the line of tiles, at least so many tiles each
    uint32_t few_stride;                 // rows that a (sequence, kv head) has in the workspace
    uint32_t* few_plan;                  // null: a wavefront takes a whole (sequence, kv head); otherwise workspace: tiles of a wavefront, then the line (tiles of the sequences before each)
    float* few_o;                        // [wavefront][2][row][D]: what the pieces that do not cover their sequence found
    f32x2* few_ml;                       // and its (m, l)
    uint32_t many_chunk;                 // many rows: tiles of keys that a workgroup takes
    float* many_o;                       // [chunk][new token][query head][D]
    f32x2* many_ml;
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
template <typename E> constexpr uint32_t kExponentStep = std::is_same_v<E, bf16> ? 0x00800080u : 0x04000400u;   // 1 in both exponents of a dword
template <typename E> constexpr uint32_t kExponent = std::is_same_v<E, bf16> ? 0x7F80u : 0x7C00u;

// Weights in fp16 are held times 2^this: with a headroom of 2^8 their largest is 2^15, and what is lost of a weight by the type's
// range is below 2^-32 of the maximum's.
template <typename P> constexpr float kWeightUp = std::is_same_v<P, fp16> ? 7.0f : 0.0f;

// A power of two with the exponent e.
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The exponent above x > 0: x < 2^e.
__device__ __forceinline__ int exponent_above(float x) { return (int)(__float_as_uint(x) >> 23) - 126; }

// Weights are rounded to 16 bits because that is what the matrix units take beside values of 16 bits.  (What the rounding takes off could
// follow as a second operand; that is the second product twice, and makes NaN of an infinite value that such a row sees.)
// sum + both halves of a dword of weights, in 32 bits: what rows are divided by is the sum of the weights that meet the values, so
// that their rounding moves a row only by how values differ (and a row of one value alone is that value).  Adding them so takes 0.98 to
// 1.02 of the time of adding them before they are rounded; unpacked and added one by one 1.01 to 1.05.
template <typename E> __device__ __forceinline__ float add2(uint32_t two, float sum) {
    if constexpr (std::is_same_v<E, bf16>) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Vec2<bf16>, two), __builtin_bit_cast(Vec2<bf16>, 0x3F803F80u), sum, false);
    else return __builtin_amdgcn_fdot2(__builtin_bit_cast(Vec2<fp16>, two), __builtin_bit_cast(Vec2<fp16>, 0x3C003C00u), sum, false);
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126: 0

// Joins the parts of a row, which lie at `at(0)` .. `at(n - 1)`.  Each lane has the (m, l) of a part; then 16 lanes read the
// channels of a part, four parts at a time and four such rounds in flight, with the (m, l), so that a row costs two trips to
// memory however many parts it has (up to 16).
template <typename E, uint32_t D, typename F>
__device__ __forceinline__ void join_row(const float* __restrict__ o, const f32x2* __restrict__ ml, F at, uint32_t n, char* dst) {
    constexpr uint32_t kPer = D / 16;                       // channels of a lane
    const uint32_t lane = threadIdx.x & (kLanes - 1), set = lane / 16, c0 = lane % 16 * kPer;
    float top = -INFINITY, total = 0.0f, acc[kPer];
#pragma unroll
    for (uint32_t c = 0; c < kPer; ++c) acc[c] = 0.0f;
    for (uint32_t z0 = 0; z0 < n; z0 += kLanes) {
        const uint32_t here_n = min(n - z0, kLanes);
        const f32x2 mine = lane < here_n ? ml[at(z0 + lane)] : f32x2{-INFINITY, 0.0f};
        f32x4 x[4][kPer / 4];
        auto load = [&](uint32_t z) {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const f32x4* src = reinterpret_cast<const f32x4*>(o + at(z0 + min(z + 4 * i + set, here_n - 1)) * D + c0);
#pragma unroll
                for (uint32_t c = 0; c < kPer / 4; ++c) x[i][c] = src[c];
            }
        };
        load(0);
        float grown = mine[0];
#pragma unroll
        for (uint32_t m = 1; m < kLanes; m *= 2) grown = fmaxf(grown, __shfl_xor(grown, m));
        grown = fmaxf(grown, top);
        const float from = grown == -INFINITY ? 0.0f : grown, keep = exp2_of(top - from), weight = exp2_of(mine[0] - from);
        top = grown;
        total = total * keep + weight * mine[1];            // each lane has its parts' share
#pragma unroll
        for (uint32_t c = 0; c < kPer; ++c) acc[c] *= keep;
        for (uint32_t z = 0; z < here_n; z += 16) {
            if (z) load(z);
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const float f = __shfl(weight, z + 4 * i + set);     // 0 beyond the last part
#pragma unroll
                for (uint32_t c = 0; c < kPer; ++c) acc[c] += f == 0.0f ? 0.0f : f * x[i][c / 4][c % 4];
            }
        }
    }
#pragma unroll
    for (uint32_t m = 1; m < kLanes; m *= 2) total += __shfl_xor(total, m);
#pragma unroll
    for (uint32_t c = 0; c < kPer; ++c) {
        acc[c] += __shfl_xor(acc[c], 16);
        acc[c] += __shfl_xor(acc[c], 32);
    }
    const float inv = total > 0.0f || total != total ? 1.0f / total : 0.0f;
    if (set == 0) {
        uint32_t* to = reinterpret_cast<uint32_t*>(dst + 2 * c0);
#pragma unroll
        for (uint32_t c = 0; c < kPer; c += 2) to[c / 2] = pack2<E>(acc[c] * inv, acc[c + 1] * inv);
    }
}

}  // namespace

#endif  // AT_PARTS_HPP
