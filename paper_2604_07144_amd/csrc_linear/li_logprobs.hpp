// Log probabilities of given tokens, entropy and the largest logits of rows: one pass over the logits.
//
// In powers of two, with c = scale log2(e) and a reference m near the largest logit:  d = (x - m) c,  S = sum 2^d,  Q = sum 2^d d,  and then
// log p = scale (x - m) - log S,  entropy = log S - ln 2 Q / S.  m is one number for a wavefront and is raised when a logit passes it by kRise
// in d, so that it is seldom raised: sums have room for terms of 2^kRise.  (x c - m c by one multiply-add would spare a subtraction,
// but m c is rounded: a token that has all the probability would not get 0.)
//
// Alternatives: a wavefront holds its 64 largest logits in order, one a lane, as whole numbers (value, then lowest token), and
// looks only at entries above the last place that is asked for.  Those are gathered in LDS and merged in when there are many.
// Wavefronts of a row, and pieces of a row where there are few rows, are joined in order at the end.
//
// Measured, 128256 tokens, us a call among others: 2311 rows in bf16 with 8 alternatives 124.5 (4.8 TB/s; a copy 5.1; under a kernel trace
// 134), in 32 bits 220 (5.4 TB/s); 64 rows in 32 bits with 20 alternatives 19.5, 8 rows in bf16 with 5 12.3: a launch that joins (5) and finding
// the alternatives (64 rows without any 10), which is vector work of every wavefront, sorting networks of 64 keys.  So what a wavefront has in
// its registers, four spans, goes into the first bound at once: by the first span only 132 for 124, 21.8 for 19.7 and 13.2 for 11.9.
#ifndef LI_LOGPROBS_HPP
#define LI_LOGPROBS_HPP

#include "li_common.hpp"

namespace {

constexpr uint32_t kLogThreads = 256, kLogWaves = kLogThreads / kLanes, kMostTop = 64;
constexpr uint32_t kSpan = 8 * kLanes;              // entries that a wavefront looks at at once
constexpr float kLog2e = 1.44269504088896341f, kRise = 8.0f;
constexpr double kLn2 = 0.693147180559945309;
// The least c.  A logit may then be above m by 8 / c = 2^123 without passing it by more than kRise, and where (x - m) passes 32 bits below it
// d is under -2^8 and 2^d is no part of a sum in 32 bits.  With smaller ones differences that count would be infinite.
constexpr float kLeastScale = 0x1p-120f;

struct Sums {
    float m, s, q, unused;                          // m is minus infinity where nothing was seen
};

struct LogParams {
    const char* logits;
    int64_t stride;
    uint32_t n_rows, vocab, top, pieces, piece;     // a row is cut into pieces of `piece` entries
    const int32_t* tokens;
    float c;                                        // log2(e) scale, rounded
    double scale, beyond_c;                         // the scale as it was given; log2(e) scale / c - 1
    float *logprob, *entropy, *top_logprob;
    int32_t* top_id;
    Sums* part_sums;                                // [row][piece]
    uint64_t* part_keys;                            // [row][piece][top]
};

// A logit and its token as a whole number that grows with the logit and, of equal ones, with a lower token; 0 is none.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t bits = __float_as_uint(x + 0.0f);                   // -0 and 0 are one
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float from_order(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return (uint64_t)order_of(x) << 32 | (0xFFFFFFFFu - token); }
__device__ __forceinline__ float value_of(uint64_t key) { return from_order((uint32_t)(key >> 32)); }
__device__ __forceinline__ uint32_t token_of(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

// Eight entries of a lane.  In 16 bits they are neighbours; in 32 bits four and four, half a span apart, so that neighbouring lanes load
// what lies next to each other.
template <typename E> struct Piece8 {
    u32x4 w[sizeof(E) / 2];
    __device__ __forceinline__ float operator[](uint32_t i) const {
        if constexpr (sizeof(E) == 4) return __uint_as_float(w[i / 4][i % 4]);
        else return i % 2 ? high16<E>(w[0][i / 2]) : low16<E>(w[0][i / 2]);
    }
    static __device__ __forceinline__ uint32_t place(uint32_t lane, uint32_t i) { return sizeof(E) == 4 ? i / 4 * (kSpan / 2) + lane * 4 + i % 4 : lane * 8 + i; }
};

// The span from entry `at` on, counted from an address that is a multiple of 16; all of it is there.
template <typename E> __device__ __forceinline__ Piece8<E> load8(const char* base, int64_t at, uint32_t lane) {
    Piece8<E> r;
#pragma unroll
    for (uint32_t j = 0; j < sizeof(E) / 2; ++j)
        r.w[j] = *reinterpret_cast<const u32x4*>(base + (at + Piece8<E>::place(lane, 4 * j)) * (int64_t)sizeof(E));
    return r;
}
// Minus infinity outside of [begin, end).
template <typename E> __device__ __forceinline__ Piece8<E> load8_within(const char* base, int64_t at, uint32_t lane, int64_t begin, int64_t end) {
    Piece8<E> r{};
    constexpr uint32_t kLeast = sizeof(E) == 4 ? 0xFF800000u : std::is_same_v<E, bf16> ? 0xFF80u : 0xFC00u;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const int64_t e = at + Piece8<E>::place(lane, i);
        const bool in = e >= begin && e < end;
        if constexpr (sizeof(E) == 4) r.w[i / 4][i % 4] = in ? reinterpret_cast<const uint32_t*>(base)[e] : kLeast;
        else r.w[0][i / 2] |= (in ? (uint32_t)reinterpret_cast<const uint16_t*>(base)[e] : kLeast) << (16 * (i % 2));
    }
    return r;
}

__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, across<1>(x)), x = fmaxf(x, across<2>(x)), x = fmaxf(x, across<4>(x));
    return x = fmaxf(x, across<8>(x)), x = fmaxf(x, across<16>(x)), fmaxf(x, across<32>(x));
}
__device__ __forceinline__ float wave_sum(float x) {
    x += across<1>(x), x += across<2>(x), x += across<4>(x);
    return x += across<8>(x), x += across<16>(x), x + across<32>(x);
}

// Keys in falling order over the lanes, from keys whose order falls and then rises, or rises and then falls.
template <uint32_t M = kLanes / 2> __device__ __forceinline__ uint64_t settled(uint64_t key, uint32_t lane) {
    const uint64_t other = across<M>(key);
    key = (lane & M) ? min(key, other) : max(key, other);
    if constexpr (M > 1) return settled<M / 2>(key, lane);
    else return key;
}
// Any keys in rising order over the lanes.
template <uint32_t N = 2, uint32_t M = 1, typename K> __device__ __forceinline__ K rising(K key, uint32_t lane) {
    const K other = across<M>(key);
    const bool up = (lane & N) == 0 || N == kLanes;
    key = ((lane & M) != 0) == up ? max(key, other) : min(key, other);
    if constexpr (M > 1) return rising<N, M / 2>(key, lane);
    else if constexpr (N < kLanes) return rising<2 * N, N>(key, lane);
    else return key;
}
__device__ __forceinline__ uint64_t of_lane(uint64_t key, uint32_t lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(key >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)key, lane);
}

// Between what lanes of a wavefront write to LDS and what others read of it, or write in its place.  The LDS has a wavefront's operations in
// order; this keeps the compiler, for which lanes are threads of their own, from moving or merging them.  It costs no instruction.
__device__ __forceinline__ void in_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What sums that were taken against x.m are worth against `to`, which is not below it.
__device__ __forceinline__ Sums moved(Sums x, float to, float c) {
    if (x.m == to || x.m == -INFINITY) return Sums{to, x.s, x.q, 0.0f};
    const float d = (x.m - to) * c, f = exp2f(d);
    return Sums{to, x.s * f, f > 0.0f ? fmaf(x.s, d, x.q) * f : x.q * f, 0.0f};
}
__device__ __forceinline__ Sums joined(Sums a, Sums b, float c) {
    const float m = fmaxf(a.m, b.m);
    a = moved(a, m, c), b = moved(b, m, c);
    return Sums{m, a.s + b.s, a.q + b.q, 0.0f};
}

// The token that was given and its logit, two loads one after the other: asked for before there is anything to do with them.
struct Given {
    float logit;
    bool there;
};
template <typename E> __device__ __forceinline__ Given given(const LogParams& p, uint32_t row) {
    const int32_t token = p.tokens ? p.tokens[row] : -1;
    const bool there = token >= 0 && (uint32_t)token < p.vocab;
    return Given{there ? (float)reinterpret_cast<const E*>(p.logits + (int64_t)row * p.stride)[token] : 0.0f, there};
}

// log s to 64 bits, of a number above 0: with s = 2^k f, f from sqrt(1/2) to sqrt(2), it is k log 2 + 2 atanh z, z = (f - 1) / (f + 1), whose series
// (z^2 is at most 0.03) is left after z^21.  As short as it can be, since a row's last steps wait for it.
__device__ __forceinline__ double log_of(float s) {
    float f = __builtin_amdgcn_frexp_mantf(s);
    const bool low = f < 0.70710678f;
    f = low ? 2.0f * f : f;
    const double k = __builtin_amdgcn_frexp_expf(s) - (low ? 1 : 0), d = (double)f + 1.0;
    double inverse = __builtin_amdgcn_rcp(d);                          // to 2^-20 or so, then 2^-40 and 2^-52
    inverse = fma(fma(-d, inverse, 1.0), inverse, inverse);
    inverse = fma(fma(-d, inverse, 1.0), inverse, inverse);
    const double z = ((double)f - 1.0) * inverse, w = z * z, v = w * w;
    double even = 1.0 / 21, odd = 1.0 / 19;                            // from z^5 and z^3 on, in steps of z^4
    even = fma(even, v, 1.0 / 17), odd = fma(odd, v, 1.0 / 15);
    even = fma(even, v, 1.0 / 13), odd = fma(odd, v, 1.0 / 11);
    even = fma(even, v, 1.0 / 9), odd = fma(odd, v, 1.0 / 7);
    even = fma(even, v, 1.0 / 5), odd = fma(odd, v, 1.0 / 3);
    return fma(k, kLn2, 2.0 * fma(z * w, fma(even, w, odd), z));
}

// What a row's sums and largest logits say.  Once a row and so in 64 bits, with the scale itself: differences of logits that pass 32 bits are
// numbers here, and beside what the sums are off there is one rounding (8 rows of 128256: 12.35 us for 12.1 in 32 bits).  The sums were taken
// with c, which is rounded; what that makes of log S goes by the mean of d, to first order, and is put back.
template <typename E> __device__ __forceinline__ void answer(const LogParams& p, uint32_t row, Given t, Sums x, uint64_t key, uint32_t lane) {
    if (!(x.s < INFINITY)) x.s = __builtin_nanf("");                   // an infinity that no limit in 32 bits lay below was a weight, and not no number
    const double with_c = log_of(x.s), mean = x.q / x.s * kLn2, whole = fma(p.beyond_c, mean, with_c);
    auto log_p = [&](float logit) { return (float)fma((double)logit - (double)x.m, p.scale, -whole); };
    if (lane == 0 && p.logprob) p.logprob[row] = !t.there ? 0.0f : x.s == 0.0f ? -INFINITY : log_p(t.logit);
    if (lane == 0 && p.entropy) p.entropy[row] = x.s == 0.0f ? 0.0f : (float)(with_c - mean);
    if (lane < p.top) {
        p.top_id[(uint64_t)row * p.top + lane] = key ? (int32_t)token_of(key) : -1;
        p.top_logprob[(uint64_t)row * p.top + lane] = x.s != x.s ? x.s : key ? log_p(value_of(key)) : -INFINITY;
    }
}

// The sums and keys of a workgroup's W wavefronts, in the first of them: pairs of neighbours, then pairs of those.
template <uint32_t W> __device__ __forceinline__ void gather(Sums* x, uint64_t* key, uint32_t wave, uint32_t lane, bool tops, float c) {
    __shared__ Sums lds_sums[W];
    __shared__ uint64_t lds_keys[W][kLanes];
#pragma unroll
    for (uint32_t m = 1; m < W; m *= 2) {
        if (wave % (2 * m) == m) {
            if (lane == 0) lds_sums[wave] = *x;
            if (tops) lds_keys[wave][kLanes - 1 - lane] = *key;       // in rising order
        }
        __syncthreads();
        if (wave % (2 * m) == 0) {
            *x = joined(*x, lds_sums[wave + m], c);
            if (tops) *key = settled(max(*key, lds_keys[wave + m][lane]), lane);
        }
    }
}

// Registers for six wavefronts a SIMD (five in 32 bits): the 64 bits of the answer would take one too many.
template <typename E> __global__ __launch_bounds__(kLogThreads, sizeof(E) == 2 ? 6 : 5) void k_logprobs(const LogParams p) {
    constexpr uint32_t kAtOnce = 4;                                    // spans that a wavefront has on their way
    constexpr uint32_t kStride = kLogWaves * kSpan * kAtOnce;
    __shared__ uint64_t lds_new[kLogWaves][2 * kLanes];
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes);
    const uint32_t row = blockIdx.x / p.pieces, z = blockIdx.x % p.pieces;
    const char* at = p.logits + (int64_t)row * p.stride;
    const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(at) % 16) / sizeof(E);     // entries to the last multiple of 16 bytes
    const char* base = at - odd * sizeof(E);
    const int64_t begin = (int64_t)odd + (int64_t)z * p.piece, end = min(begin + p.piece, (int64_t)odd + p.vocab);
    const float c = p.c;

    Given token{};
    if (p.pieces == 1 && wave == 0) token = given<E>(p, row);
    Sums x{-INFINITY, 0.0f, 0.0f, 0.0f};
    float limit = -INFINITY, ref = 0.0f;                               // the last logit that m does for; m, or 0 while there is none
    float s = 0.0f, q = 0.0f;
    uint64_t key = 0;
    float least = -INFINITY;                                           // entries up to here are no alternatives
    uint32_t waiting = 0;
    bool begun = false;
    uint64_t* const buf = lds_new[wave];
    auto merge = [&](uint32_t n) {
        in_order();
        key = settled(max(key, rising(lane < n ? buf[lane] : 0, lane)), lane);
        const uint64_t last = of_lane(key, p.top - 1);
        if (last) least = value_of(last);
    };
    auto raise = [&](float largest) {
        const float to = wave_max(fmaxf(largest, x.m));
        const Sums r = moved(Sums{x.m, s, q, 0.0f}, to, c);
        x.m = to, s = r.s, q = r.q;
        ref = to > -INFINITY ? to : 0.0f, limit = to + kRise / c;
    };
    auto add = [&](const Piece8<E>& e) {
        float s8 = 0.0f, q8 = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const float d = (e[i] - ref) * c, w = __builtin_amdgcn_exp2f(d);
            s8 += w, q8 = fmaf(w, fmaxf(d, -1000.0f), q8);             // minus infinity would make 0 times it no number
        }
        s += s8, q += q8;
    };
    auto collect = [&](const Piece8<E>& e, int64_t first) {
        const float before = least;                                    // of equal ones a lower token may still come in this span, not in later ones
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const bool above = e[i] > before;
            const uint64_t who = __ballot(above);
            if (!who) continue;
            if (above) buf[waiting + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] =
                key_of(e[i], (uint32_t)(first + Piece8<E>::place(lane, i) - odd));
            waiting += (uint32_t)__popcll(who);
            if (waiting >= kLanes) {
                merge(kLanes);
                waiting -= kLanes;
                const uint64_t rest = lane < waiting ? buf[kLanes + lane] : 0;
                buf[lane] = rest;
                in_order();
            }
        }
    };
    for (int64_t first = begin / 8 * 8 + wave * (kSpan * kAtOnce); first < end; first += kStride) {
        Piece8<E> e[kAtOnce];
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            const int64_t from = first + u * kSpan;
            if (from >= begin && from + kSpan <= end) e[u] = load8<E>(base, from, lane);
            else e[u] = load8_within<E>(base, from, lane, begin, end);
        }
        float most[kAtOnce], largest = -INFINITY;
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u) {
            most[u] = e[u][0];
#pragma unroll
            for (uint32_t i = 1; i < 8; ++i) most[u] = fmaxf(most[u], e[u][i]);
            largest = fmaxf(largest, most[u]);
        }
        if (__any(largest > limit)) raise(largest);
#pragma unroll
        for (uint32_t u = 0; u < kAtOnce; ++u)
            if (first + u * kSpan < end) add(e[u]);
        if (p.top && __any(largest > least)) {
            if (!begun) {
                // Of the lanes' largest entries the one in the last place that is asked for: below it lies no alternative.
                const uint32_t last = (uint32_t)__builtin_amdgcn_readlane(rising(order_of(largest), lane), kLanes - p.top);
                if (from_order(last) > -INFINITY) least = from_order(last - (last == 0x80000000u ? 2 : 1));   // zero is two numbers
                begun = true;
            }
#pragma unroll
            for (uint32_t u = 0; u < kAtOnce; ++u)
                if (__any(most[u] > least)) collect(e[u], first + u * kSpan);
        }
    }
    if (p.top && waiting) merge(waiting);
    x.s = wave_sum(s), x.q = wave_sum(q);
    gather<kLogWaves>(&x, &key, wave, lane, p.top != 0, p.c);
    if (wave != 0) return;
    if (p.pieces == 1) {
        answer<E>(p, row, token, x, key, lane);
    } else {
        if (lane == 0) p.part_sums[blockIdx.x] = x;
        if (lane < p.top) p.part_keys[(uint64_t)blockIdx.x * p.top + lane] = key;
    }
}

// The pieces of a row.
template <typename E, uint32_t W> __global__ __launch_bounds__(W * kLanes) void k_join_logprobs(const LogParams p) {
    const uint32_t lane = threadIdx.x % kLanes, wave = uniform(threadIdx.x / kLanes), row = blockIdx.x;
    Given token{};
    if (wave == 0) token = given<E>(p, row);
    Sums x{-INFINITY, 0.0f, 0.0f, 0.0f};
    uint64_t key = 0;
    for (uint32_t z = wave; z < p.pieces; z += W) {
        const uint64_t at = (uint64_t)row * p.pieces + z;
        const uint32_t from = kLanes - 1 - lane;                       // in rising order
        const uint64_t theirs = from < p.top ? p.part_keys[at * p.top + from] : 0;
        x = joined(x, p.part_sums[at], p.c);
        if (p.top) key = settled(max(key, theirs), lane);
    }
    gather<W>(&x, &key, wave, lane, p.top != 0, p.c);
    if (wave == 0) answer<E>(p, row, token, x, key, lane);
}

}  // namespace

#endif  // LI_LOGPROBS_HPP
