// min-p's cut: the smallest logit whose weight is min_p or more, by the same arithmetic as on the device where it is compiled for the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dyspec {

// Ascending with x; -0 and 0 alike.
__host__ __device__ __forceinline__ uint32_t ordered_bits(float x)
{
    const uint32_t u = (uint32_t)__float_as_int(x + 0.0f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__host__ __device__ __forceinline__ float of_ordered_bits(uint32_t key) { return __int_as_float((int)(key & 0x80000000u ? key ^ 0x80000000u : ~key)); }

// The smallest key of lowest .. highest that is enough: enough(key) holds from it on, for `highest` without asking.  `near` is a guess: three
// questions where it is right to a key, else the rest of the range is halved, up to 34 in all.
template <typename F> __host__ __device__ __forceinline__ uint32_t first_enough(uint32_t lowest, uint32_t highest, uint32_t near, F&& enough)
{
    near = near < lowest ? lowest : near > highest ? highest : near;
    uint32_t a = near > lowest ? near - 1u : lowest, b = near < highest ? near + 1u : highest;
    if (a > lowest && enough(a)) {
        b = a;
        a = lowest;
    } else if (b < highest && !enough(b)) {
        a = b + 1u;
        b = highest;
    } else if (a > lowest) {
        ++a;
    }
#pragma unroll 1
    while (a < b) {
        const uint32_t mid = a + (b - a) / 2u;
        if (enough(mid)) b = mid;
        else a = mid + 1u;
    }
    return a;
}

// Of a row whose largest logit is `top`.  least: log2(min_p), per_nat: log2(e) / temperature.  Weights are numbers of 64 bits: those within
// 2^-54 of 1 are 1.  What is guessed from is off by the 64-bit rounding of its larger term, many keys where the cut lies near a logit of zero.
// asked: called at every question.
template <typename F> __host__ __device__ __forceinline__ float min_p_cut(float top, float temperature, double per_nat, double least, F&& asked)
{
    least -= 0x1p-54;
    const double top64 = (double)top;
    const float guess = (float)(top64 + least * ((double)temperature * 0.69314718055994530942));
    return of_ordered_bits(first_enough(ordered_bits(-3.402823466e38f), ordered_bits(top), ordered_bits(guess), [=](uint32_t key) __attribute__((always_inline)) {
        asked();
        return ((double)of_ordered_bits(key) - top64) * per_nat >= least;
    }));
}

}  // namespace dyspec
