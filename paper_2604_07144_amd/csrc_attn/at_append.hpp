// Appending new tokens to the cache (rotation, and quantisation to 4 bits, on the way) and reading rows back.
//
// Both are one pass over the rows: what is read and written once is all there is to do, so memory bounds them.  A
// wavefront takes a token and some of its heads: lane = (head, unit), a unit being the 16 channels that one lane turns,
// two pieces of 16 bytes.  With pairs (i, i + rot/2) the two pieces lie rot/2 apart, so that both ends of a pair are in
// one lane and eight neighbouring lanes still read whole 128-byte lines; everywhere else they are neighbours.  The lane's
// eight (cos, sin) are loaded once and serve all of its heads.
//
// Measured, 128 channels: prompts of 40 heads on 40 in 16 bits 4.9 TB/s of 5.1 that a copy of 1 GiB moves; a prompt of 32768, 32 heads
// on 8, into 4 bits and read back 4.5.  One token for each of 64 slots 3.0 us in a graph; a call by the host costs 4 to 7.
#ifndef AT_APPEND_HPP
#define AT_APPEND_HPP

#include "at_common.hpp"

namespace {

constexpr uint32_t kAppendThreads = 256;

struct AppendParams {
    Cache cache;
    Batch batch;
    Rows k, v, q, q_out;
    const float* turn;                   // [position][rot / 2][2] or null
    uint32_t rot, q_heads, kv_heads, heads_per_wave;
};

template <typename E> constexpr float kLargest = std::is_same_v<E, bf16> ? 3.3895313892515355e38f : 65504.0f;

// The group of 64 channels: its lowest value, and the step rounded up to the 16-bit type, as raw bits.  The division is
// by 16ths of everything, which is exact and keeps the difference of two values of opposite sign in range.
template <typename E> __device__ __forceinline__ uint32_t group_pair(float lo, float hi, bool finite) {
    if (!finite) return std::is_same_v<E, bf16> ? 0x7FC07FC0u : 0x7E007E00u;
    const float want = (hi * 0.0625f - lo * 0.0625f) / 15.0f;
    float whole = want * 16.0f;
    E step = (E)whole;
    uint32_t bits = bits16(step);
    if ((float)step < whole) ++bits;
    if (!(fmaf(15.0f, low16<E>(bits), lo) <= kLargest<E>)) --bits;   // rounded down where 15 steps would leave the type's range
    return bits | (uint32_t)bits16((E)lo) << 16;
}

__device__ __forceinline__ uint32_t code_of(float x, float lo, float step) {
    const float c = rintf((x * 0.0625f - lo * 0.0625f) / (step * 0.0625f));
    return (uint32_t)fminf(fmaxf(c, 0.0f), 15.0f);       // a step of 0 (all values alike) gives NaN, and code 0
}

// kHalves: pairs (i, i + rot / 2); otherwise neighbours (or no rotation at all).
template <typename E, uint32_t D, uint32_t kBits, bool kHalves>
__global__ __launch_bounds__(kAppendThreads) void k_append(const AppendParams p) {
    constexpr uint32_t kUnits = D / 16, kHeadsAtOnce = kLanes / kUnits;
    const uint32_t lane = threadIdx.x & (kLanes - 1), unit = lane % kUnits;
    const uint32_t t = blockIdx.x * (kAppendThreads / kLanes) + threadIdx.x / kLanes;
    if (t >= p.batch.n_tokens) return;
    const uint32_t s = seq_of(p.batch, t);
    Seq seq{};
    int32_t pos = -1;
    if (s < p.batch.n_seqs) {
        seq = seq_at(p.batch, s);
        if ((int32_t)t >= seq.first && (int32_t)t < seq.first + seq.n_new) pos = seq.pos0 + ((int32_t)t - seq.first);
    }
    const bool held = pos >= 0 && pos < seq.kv_len;
    Place at{};
    if (held) at = place_of(p.cache, p.batch.table + (int64_t)s * p.batch.table_stride, (uint32_t)pos, (uint32_t)seq.kv_len);
    const bool there = held && at.there;

    const uint32_t turned = p.turn ? p.rot / 16u : 0u;     // units that turn
    const bool turns = unit < turned;
    const uint32_t piece0 = kHalves && turns ? unit : 2 * unit, piece1 = kHalves && turns ? unit + turned : 2 * unit + 1;
    float cs[8], sn[8];
    if (turns && held) {
        const f32x4* tab = reinterpret_cast<const f32x4*>(p.turn + (int64_t)pos * p.rot) + unit * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 x = tab[i];
            cs[2 * i] = x[0], sn[2 * i] = x[1], cs[2 * i + 1] = x[2], sn[2 * i + 1] = x[3];
        }
    }

    const uint32_t n_heads = 2 * p.kv_heads + p.q_heads;   // keys, values, queries
    const uint32_t begin = blockIdx.y * p.heads_per_wave, end = min(begin + p.heads_per_wave, n_heads);
    for (uint32_t base = begin; base < end; base += kHeadsAtOnce) {
        const uint32_t h = base + lane / kUnits;
        const bool live = h < end;
        const bool is_k = h < p.kv_heads, is_v = !is_k && h < 2 * p.kv_heads, is_q = !is_k && !is_v;
        const uint32_t head = is_k ? h : is_v ? h - p.kv_heads : h - 2 * p.kv_heads;
        u32x4 a{}, b{};
        if (live && (is_q || there)) {
            const Rows& src = is_k ? p.k : is_v ? p.v : p.q;
            const u32x4* row = reinterpret_cast<const u32x4*>(src.data + (int64_t)t * src.token_stride + (int64_t)head * src.head_stride);
            a = row[piece0], b = row[piece1];
        }
        if (turns && !is_v) {
            // products and their sum each rounded to 32 bits, as written: codes next to a border come out the same wherever this is computed
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (kHalves) {
                    const float x0 = low16<E>(a[i]), x1 = high16<E>(a[i]), y0 = low16<E>(b[i]), y1 = high16<E>(b[i]);
                    a[i] = pack2<E>(x0 * cs[2 * i] - y0 * sn[2 * i], x1 * cs[2 * i + 1] - y1 * sn[2 * i + 1]);
                    b[i] = pack2<E>(x0 * sn[2 * i] + y0 * cs[2 * i], x1 * sn[2 * i + 1] + y1 * cs[2 * i + 1]);
                } else {
                    const float x = low16<E>(a[i]), y = high16<E>(a[i]), u = low16<E>(b[i]), w = high16<E>(b[i]);
                    a[i] = pack2<E>(x * cs[i] - y * sn[i], x * sn[i] + y * cs[i]);
                    b[i] = pack2<E>(u * cs[i + 4] - w * sn[i + 4], u * sn[i + 4] + w * cs[i + 4]);
                }
            }
        }
        if (live && is_q) {
            if (!held) a = u32x4{}, b = u32x4{};
            u32x4* row = reinterpret_cast<u32x4*>(p.q_out.data + (int64_t)t * p.q_out.token_stride + (int64_t)head * p.q_out.head_stride);
            row[piece0] = a, row[piece1] = b;
        }
        char* const base_kv = is_k ? p.cache.k : p.cache.v;
        if constexpr (kBits == 16) {
            if (live && !is_q && there) {
                u32x4* row = reinterpret_cast<u32x4*>(base_kv + (int64_t)at.page * p.cache.page_stride + (int64_t)head * p.cache.head_stride +
                                                      (int64_t)at.slot * p.cache.slot_stride);
                row[piece0] = a, row[piece1] = b;
            }
        } else if (base < 2 * p.kv_heads) {
            // lowest and largest of each group of 64 over the lanes of the head; min / max leave NaN out, so finiteness is counted beside them
            constexpr uint32_t kGroups = D / 64;
            const uint32_t g0 = piece0 / 8, g1 = piece1 / 8;
            float lo[kGroups], hi[kGroups];
            uint32_t odd[kGroups];
#pragma unroll
            for (uint32_t g = 0; g < kGroups; ++g) lo[g] = INFINITY, hi[g] = -INFINITY, odd[g] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x[2] = {low16<E>(a[i]), high16<E>(a[i])}, y[2] = {low16<E>(b[i]), high16<E>(b[i])};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (uint32_t g = 0; g < kGroups; ++g) {
                        if (g0 == g) lo[g] = fminf(lo[g], x[j]), hi[g] = fmaxf(hi[g], x[j]), odd[g] |= !(fabsf(x[j]) < INFINITY);
                        if (g1 == g) lo[g] = fminf(lo[g], y[j]), hi[g] = fmaxf(hi[g], y[j]), odd[g] |= !(fabsf(y[j]) < INFINITY);
                    }
            }
#pragma unroll
            for (uint32_t m = 1; m < kUnits; m *= 2)
#pragma unroll
                for (uint32_t g = 0; g < kGroups; ++g) {
                    lo[g] = fminf(lo[g], __shfl_xor(lo[g], m)), hi[g] = fmaxf(hi[g], __shfl_xor(hi[g], m));
                    odd[g] |= __shfl_xor(odd[g], m);
                }
            uint32_t pair[kGroups];
#pragma unroll
            for (uint32_t g = 0; g < kGroups; ++g) pair[g] = group_pair<E>(lo[g], hi[g], !odd[g]);
            if (live && !is_q && there) {
                char* row = base_kv + (int64_t)at.page * p.cache.page_stride + (int64_t)head * p.cache.head_stride + (int64_t)at.slot * p.cache.slot_stride;
                char* pairs = (is_k ? p.cache.k_pairs : p.cache.v_pairs) + (int64_t)at.page * p.cache.pair_page_stride +
                              (int64_t)head * p.cache.pair_head_stride + (int64_t)at.slot * p.cache.pair_slot_stride;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const u32x4 x = half ? b : a;
                    const uint32_t g = half ? g1 : g0, pr = kGroups == 2 && g == 1 ? pair[kGroups - 1] : pair[0];
                    const float step = low16<E>(pr), low = high16<E>(pr);
                    uint32_t codes = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        codes |= code_of(low16<E>(x[i]), low, step) << (8 * i) | code_of(high16<E>(x[i]), low, step) << (8 * i + 4);
                    reinterpret_cast<uint32_t*>(row)[half ? piece1 : piece0] = codes;
                }
                if (unit < kGroups) reinterpret_cast<uint32_t*>(pairs)[unit] = kGroups == 2 && unit == 1 ? pair[kGroups - 1] : pair[0];
            }
        }
    }
}

// Rows of the cache as 16-bit values: lane = (head, piece of 16 bytes).
template <typename E, uint32_t D, uint32_t kBits>
__global__ __launch_bounds__(kAppendThreads) void k_read(const AppendParams p) {
    constexpr uint32_t kPieces = D / 8, kHeadsAtOnce = kLanes / kPieces;
    const uint32_t lane = threadIdx.x & (kLanes - 1), piece = lane % kPieces;
    const uint32_t t = blockIdx.x * (kAppendThreads / kLanes) + threadIdx.x / kLanes;
    if (t >= p.batch.n_tokens) return;
    const uint32_t s = seq_of(p.batch, t);
    bool there = false;
    Place at{};
    if (s < p.batch.n_seqs) {
        const Seq seq = seq_at(p.batch, s);
        const int32_t pos = seq.pos0 + ((int32_t)t - seq.first);
        if ((int32_t)t >= seq.first && (int32_t)t < seq.first + seq.n_new && pos >= 0 && pos < seq.kv_len) {
            at = place_of(p.cache, p.batch.table + (int64_t)s * p.batch.table_stride, (uint32_t)pos, (uint32_t)seq.kv_len);
            there = at.there;
        }
    }
    const uint32_t begin = blockIdx.y * p.heads_per_wave, end = min(begin + p.heads_per_wave, 2 * p.kv_heads);
    for (uint32_t h = begin + lane / kPieces; h < end; h += kHeadsAtOnce) {
        const bool is_k = h < p.kv_heads;
        const uint32_t head = is_k ? h : h - p.kv_heads;
        u32x4 x{};
        if (there) {
            const char* row = (is_k ? p.cache.k : p.cache.v) + (int64_t)at.page * p.cache.page_stride + (int64_t)head * p.cache.head_stride +
                              (int64_t)at.slot * p.cache.slot_stride;
            if constexpr (kBits == 16) {
                x = reinterpret_cast<const u32x4*>(row)[piece];
            } else {
                const char* pairs = (is_k ? p.cache.k_pairs : p.cache.v_pairs) + (int64_t)at.page * p.cache.pair_page_stride +
                                    (int64_t)head * p.cache.pair_head_stride + (int64_t)at.slot * p.cache.pair_slot_stride;
                const uint32_t pr = reinterpret_cast<const uint32_t*>(pairs)[piece / 8];
                x = decode8<E>(reinterpret_cast<const uint32_t*>(row)[piece], low16<E>(pr), high16<E>(pr));
            }
        }
        const Rows& dst = is_k ? p.k : p.v;
        reinterpret_cast<u32x4*>(dst.data + (int64_t)t * dst.token_stride + (int64_t)head * dst.head_stride)[piece] = x;
    }
}

}  // namespace

#endif  // AT_APPEND_HPP
