// How a group of 16-bit values is held in 4 bits: a pair (step, lo) and whole numbers 0 .. 15.
#ifndef AT_CODES_HPP
#define AT_CODES_HPP

#include "at_common.hpp"

namespace {

template <typename E> constexpr float kLargest = std::is_same_v<E, bf16> ? 3.3895313892515355e38f : 65504.0f;

// A group: its lowest value, and the step rounded up to the 16-bit type, as raw bits.  The division is
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

}  // namespace

#endif  // AT_CODES_HPP
