// Log probabilities of given tokens, entropy and the largest logits of rows: one pass over the logits, which bounds it.
//
// With a reference m near the largest logit, d = (x - m) scale log2(e):  S = sum 2^d,  Q = sum 2^d d,  and then
// log p = (x - m) scale - ln S,  entropy = ln S - ln 2 Q / S.  m is one number for a wavefront and is raised when a logit
// passes it by kRise in d, so that it is seldom raised: sums have room for terms of 2^kRise.
//
// Alternatives: a wavefront holds its 64 largest logits in order, one a lane, as whole numbers (value, then lowest token), and
// looks only at entries above the last place that is asked for.  Those are gathered in LDS and merged in when there are many.
// Wavefronts of a row, and pieces of a row where there are few rows, are joined in order at the end.
#ifndef LI_LOGPROBS_HPP
#define LI_LOGPROBS_HPP

#include "li_common.hpp"

namespace {

constexpr uint32_t kLogThreads = 256, kLogWaves = kLogThreads / kLanes, kMostTop = 64;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f, kRise = 8.0f;

struct LogParams {
    const char* logits;
    int64_t stride;
    uint32_t n_rows, vocab, top, pieces, piece;     // a row is cut into pieces of `piece` entries
    const int32_t* tokens;
    float scale;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_id;
    f32x4* part_sums;                               // [row][piece]: m, S, Q
    uint64_t* part_keys;                            // [row][piece][top]
};

struct Sums {
    float m, s, q;                                  // m is minus infinity where nothing was seen
};

// A logit and its token as a whole number that grows with the logit and, of equal ones, with a lower token; 0 is none.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) {
    const uint32_t bits = __float_as_uint(x + 0.0f);                   // -0 and 0 are one
    const uint32_t order = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return (uint64_t)order << 32 | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order);
}
__device__ __forceinline__ uint32_t token_of(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

template <typename E> struct Piece8 {                                  // eight entries
    u32x4 w[sizeof(E) / 2];
    __device__ __forceinline__ float operator[](uint32_t i) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[i / 4][i % 4]);
        else return i % 2 ? high16<E>(w[0][i / 2]) : low16<E>(w[0][i / 2]);
    }
};

// Entries at .. at + 7 of a row, counted from an address that is a multiple of 16: minus infinity outside of [begin, end).
template <typename E> __device__ __forceinline__ Piece8<E> load8(const char* base, int64_t at, int64_t begin, int64_t end) {
    Piece8<E> r;
    if (at >= begin && at + 8 <= end) {
#pragma unroll
        for (uint32_t i = 0; i < sizeof(E) / 2; ++i) r.w[i] = reinterpret_cast<const u32x4*>(base + at * (int64_t)sizeof(E))[i];
    } else {
        constexpr uint32_t kLeast = std::is_same_v<E, bf16> ? 0xFF80u : 0xFC00u;
#pragma unroll
        for (uint32_t i = 0; i < sizeof(E) / 2; ++i)
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                if constexpr (sizeof(E) == 4) {
                    const int64_t e = at + i * 4 + j;
                    r.w[i][j] = e >= begin && e < end ? reinterpret_cast<const uint32_t*>(base)[e] : 0xFF800000u;
                } else {
                    const int64_t e = at + j * 2;
                    const uint16_t* b = reinterpret_cast<const uint16_t*>(base);
                    const uint32_t lo = e >= begin && e < end ? b[e] : kLeast, hi = e + 1 >= begin && e + 1 < end ? b[e + 1] : kLeast;
                    r.w[i][j] = lo | hi << 16;
                }
            }
    }
    return r;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (uint32_t m = 1; m < kLanes; m *= 2) x = fmaxf(x, __shfl_xor(x, m));
    return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (uint32_t m = 1; m < kLanes; m *= 2) x += __shfl_xor(x, m);
    return x;
}

// What sums that were taken against `from` are worth against `to`, which is not below it.
__device__ __forceinline__ Sums moved(Sums x, float to, float c) {
    if (x.m == -INFINITY || x.m == to) return Sums{to, x.s, x.q};
    const float d = (x.m - to) * c, f = exp2f(d);
    return Sums{to, x.s * f, f > 0.0f ? fmaf(x.s, d, x.q) * f : x.q * f};
}
__device__ __forceinline__ Sums joined(Sums a, Sums b, float c) {
    const float m = fmaxf(a.m, b.m);
    a = moved(a, m, c), b = moved(b, m, c);
    return Sums{m, a.s + b.s, a.q + b.q};
}

// Keys in falling order over the lanes, from keys whose order falls and then rises, or rises and then falls.
__device__ __forceinline__ uint64_t settled(uint64_t key, uint32_t lane) {
#pragma unroll
    for (uint32_t m = kLanes / 2; m > 0; m /= 2) {
        const uint64_t other = __shfl_xor(key, m);
        key = (lane & m) ? min(key, other) : max(key, other);
    }
    return key;
}
// Any keys in rising order over the lanes.
__device__ __forceinline__ uint64_t rising(uint64_t key, uint32_t lane) {
#pragma unroll
    for (uint32_t n = 2; n <= kLanes; n *= 2)
#pragma unroll
        for (uint32_t m = n / 2; m > 0; m /= 2) {
            const uint64_t other = __shfl_xor(key, m);
            const bool up = (lane & n) == 0 || n == kLanes;
            key = ((lane & m) != 0) == up ? max(key, other) : min(key, other);
        }
    return key;
}
__device__ __forceinline__ uint64_t of_lane(uint64_t key, uint32_t lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(key >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)key, lane);
}

// What a row's sums and largest logits say.
template <typename E> __device__ __forceinline__ void answer(const LogParams& p, uint32_t row, Sums x, uint64_t key, uint32_t lane) {
    const float log = logf(x.s);
    if (lane == 0 && p.logprob) {
        const int32_t token = p.tokens[row];
        float r = 0.0f;
        if (token >= 0 && (uint32_t)token < p.vocab) {
            const float of = (float)reinterpret_cast<const E*>(p.logits + (int64_t)row * p.stride)[token];
            r = x.s == 0.0f ? -INFINITY : (of - x.m) * p.scale - log;
        }
        p.logprob[row] = r;
    }
    if (lane == 0 && p.entropy) p.entropy[row] = x.s == 0.0f ? 0.0f : log - kLn2 * (x.q / x.s);
    if (lane < p.top) {
        p.top_id[(uint64_t)row * p.top + lane] = key ? (int32_t)token_of(key) : -1;
        p.top_logprob[(uint64_t)row * p.top + lane] = x.s != x.s ? x.s : key ? (value_of(key) - x.m) * p.scale - log : -INFINITY;
    }
}

// The sums and keys of a workgroup's wavefronts, in the first of them.
__device__ __forceinline__ void gather(Sums* x, uint64_t* key, uint32_t wave, uint32_t lane, bool tops, float c) {
    __shared__ Sums lds_sums[kLogWaves];
    __shared__ uint64_t lds_keys[kLogWaves][kLanes];
    if (lane == 0) lds_sums[wave] = *x;
    if (tops) lds_keys[wave][lane] = *key;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (uint32_t w = 1; w < kLogWaves; ++w) {
        *x = joined(*x, lds_sums[w], c);
        if (tops) *key = settled(max(*key, lds_keys[w][kLanes - 1 - lane]), lane);
    }
}

template <typename E> __global__ __launch_bounds__(kLogThreads) void k_logprobs(const LogParams p) {
    constexpr uint32_t kAtOnce = 2;                                    // pieces of eight entries that a lane takes at once
    constexpr uint32_t kStride = kLogThreads * 8 * kAtOnce;
    __shared__ uint64_t lds_new[kLogWaves][2 * kLanes];
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes);
    const uint32_t row = blockIdx.x / p.pieces, z = blockIdx.x % p.pieces;
    const char* at = p.logits + (int64_t)row * p.stride;
    const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(at) % 16) / sizeof(E);     // entries to the last multiple of 16 bytes
    const char* base = at - odd * sizeof(E);
    const int64_t begin = (int64_t)odd + (int64_t)z * p.piece, end = min(begin + p.piece, (int64_t)odd + p.vocab);
    const float c = p.scale * kLog2e;

    Sums x{-INFINITY, 0.0f, 0.0f};
    float limit = -INFINITY, ref = 0.0f;
    float s = 0.0f, q = 0.0f;
    uint64_t key = 0;
    float least = -INFINITY;                                           // entries up to here are no alternatives
    uint32_t waiting = 0;
    uint64_t* const buf = lds_new[wave];
    auto merge = [&](uint32_t n) {
        uint64_t fresh = lane < n ? buf[lane] : 0;
        key = settled(max(key, rising(fresh, lane)), lane);
        const uint64_t last = of_lane(key, p.top - 1);
        if (last) least = value_of(last);
    };
    for (int64_t first = begin / 8 * 8 + wave * (8 * kLanes * kAtOnce); first < end; first += kStride) {
        Piece8<E> e[kAtOnce];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) e[u] = load8<E>(base, first + (u * kLanes + lane) * 8, begin, end);
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            float most = e[u][0];
#pragma unroll
            for (uint32_t i = 1; i < 8; ++i) most = fmaxf(most, e[u][i]);
            if (__any(most > limit)) {
                const float to = wave_max(fmaxf(most, x.m));
                const Sums r = moved(Sums{x.m, s, q}, to, c);
                x.m = to, s = r.s, q = r.q;
                ref = to > -INFINITY ? to : 0.0f, limit = to + kRise / c;
            }
            float s8 = 0.0f, q8 = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const float d = (e[u][i] - ref) * c, w = __builtin_amdgcn_exp2f(d);
                s8 += w, q8 = fmaf(w, fmaxf(d, -1000.0f), q8);         // minus infinity would make 0 times it no number
            }
            s += s8, q += q8;
            if (p.top && __any(most > least)) {
                const float before = least;                            // of equal ones a lower token may still come in this piece, not in later ones
                for (uint32_t i = 0; i < 8; ++i) {
                    float v = e[u][0];
#pragma unroll
                    for (uint32_t j = 1; j < 8; ++j) v = i == j ? e[u][j] : v;
                    const bool take = v > before;
                    const uint64_t who = __ballot(take);
                    if (!who) continue;
                    if (take) buf[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] =
                        key_of(v, (uint32_t)(first + (u * kLanes + lane) * 8 + i - odd));
                    waiting += (uint32_t)__popcll(who);
                    if (waiting >= kLanes) {
                        merge(kLanes);
                        waiting -= kLanes;
                        const uint64_t rest = lane < waiting ? buf[kLanes + lane] : 0;
                        buf[lane] = rest;
                    }
                }
            }
        }
    }
    if (p.top && waiting) merge(waiting);
    x.s = wave_sum(s), x.q = wave_sum(q);
    gather(&x, &key, wave, lane, p.top != 0, c);
    if (wave != 0) return;
    if (p.pieces == 1) {
        answer<E>(p, row, x, key, lane);
    } else {
        if (lane == 0) p.part_sums[blockIdx.x] = f32x4{x.m, x.s, x.q, 0.0f};
        if (lane < p.top) p.part_keys[(uint64_t)blockIdx.x * p.top + lane] = key;
    }
}

// The pieces of a row.
template <typename E> __global__ __launch_bounds__(kLogThreads) void k_join_logprobs(const LogParams p) {
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes), row = blockIdx.x;
    const float c = p.scale * kLog2e;
    Sums x{-INFINITY, 0.0f, 0.0f};
    uint64_t key = 0;
    for (uint32_t z = wave; z < p.pieces; z += kLogWaves) {
        const uint64_t at = (uint64_t)row * p.pieces + z;
        const f32x4 y = p.part_sums[at];
        x = joined(x, Sums{y[0], y[1], y[2]}, c);
        if (p.top) {
            const uint32_t from = kLanes - 1 - lane;                   // in rising order
            key = settled(max(key, from < p.top ? p.part_keys[at * p.top + from] : 0), lane);
        }
    }
    gather(&x, &key, wave, lane, p.top != 0, c);
    if (wave == 0) answer<E>(p, row, x, key, lane);
}

}  // namespace

#endif  // LI_LOGPROBS_HPP
