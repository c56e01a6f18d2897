// cpes_powers.hpp -- the table of powers of 2 that the draws' pass over the logits adds
// its weights from, and where in it a logit's weight stands: the parts that the host checks
// as well.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace cpes {

// A weight 2^(c (x - base)) is that of a cell of 1/64 octave, of which there are kCells an octave, from
// kLow octaves on; the base moves before a logit is more than kRoom octaves above it.
constexpr int kLow = -56, kRoom = 7, kCells = 64;
constexpr int kPowers = (kRoom + 1 - kLow) * kCells;
constexpr double kExact = 2048.0;         // c base up to which the rounding of c base, 2^-42, is let through

// The largest logit that still adds to sums with this base: at most kRoom octaves above it, rounded
// down, since a step of 32 bits may be octaves itself (scale 1e6 at 20: 2.75; rounded to the nearest,
// a logit 8.26 octaves above the base passed, and its cell lay behind the table).  It is finite.
inline __host__ __device__ float last_above(float base, double c)
{
    const double most = (double)base + kRoom / c;
    const float last = (float)most;
    return (double)last > most ? nextafterf(last, -INFINITY) : last;
}

// A logit's place in the table, in cells, with `start` the product's part that all logits share.
inline __host__ __device__ double start_of(float base, double cells) { return cells * (double)base + kLow * kCells; }
inline __host__ __device__ bool start_is_near(double start) { return fabs(start) <= kExact * kCells; }
inline __host__ __device__ double cells_near(float x, double cells, double start) { return fma((double)x, cells, -start); }
inline __host__ __device__ double cells_far(float x, float base, double cells) { return ((double)x - (double)base) * cells - kLow * kCells; }

}  // namespace cpes
