// cpes_attend.hpp -- what the kernels of the attention of one new token per row and of
// trees of new tokens share: tiles, the softmax's arithmetic, how a wave holds its
// operands and state, and the shares of a line of tiles.  Internal to the library.
#pragma once

#include <type_traits>

#include "cpes_eval.hpp"

namespace cpes {

namespace {

typedef unsigned int V4u __attribute__((ext_vector_type(4)));
typedef unsigned int V2u __attribute__((ext_vector_type(2)));
typedef float V4f __attribute__((ext_vector_type(4)));
typedef __bf16 V8bf __attribute__((ext_vector_type(8)));
typedef V4u V4uAnywhere __attribute__((aligned(2)));          // caches and queries start at any element
typedef V2u V2uAnywhere __attribute__((aligned(2)));

constexpr float kLog2e = 1.44269504088896340736f;

template <typename T> struct Tile;
template <> struct Tile<uint16_t> { static constexpr int n = 32; };
template <> struct Tile<float> { static constexpr int n = 16; };

// e^x for x <= 0: the hardware's 2^x.  Scores and maxima stay in natural units,
// so that lse loses nothing on a way through base 2.  The product's rounding
// is |x| 2^-24 of the weight, which an fp32 cache's outputs would show; the lse of a
// bf16 cache carries it, as the mean of |x| 2^-24 under the weights.
template <typename T> __device__ __forceinline__ float weight(float x);
template <> __device__ __forceinline__ float weight<uint16_t>(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
template <> __device__ __forceinline__ float weight<float>(float x) { return expf(x); }

// x of the lanes that hold one query head's scores: rows of 16 lanes swapped
// pairwise, then halves, each pair holding both rows' values afterwards.
__device__ __forceinline__ void swap_rows(float x, float* y, float* z)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *y = __uint_as_float(r[0]);
    *z = __uint_as_float(r[1]);
}
__device__ __forceinline__ void swap_halves(float x, float* y, float* z)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    *y = __uint_as_float(r[0]);
    *z = __uint_as_float(r[1]);
}

__device__ __forceinline__ float max_over_lanes(float x)
{
    float y, z;
    swap_rows(x, &y, &z);
    swap_halves(fmaxf(y, z), &y, &z);
    return fmaxf(y, z);
}
__device__ __forceinline__ float sum_over_lanes(float x)
{
    float y, z;
    swap_rows(x, &y, &z);
    swap_halves(y + z, &y, &z);
    return y + z;
}

template <typename T, int DP> struct Layout;
// bf16: 8 elements of a key row per load; a lane's part of a value row
template <int DP> struct Layout<uint16_t, DP> {
    static constexpr int KV = DP / 32;            // key loads of 16 bytes per 16 positions
    static constexpr int VE = DP / 16;            // value elements of a lane's positions
    static constexpr int VD = DP / 32;            // their dwords
};
template <int DP> struct Layout<float, DP> {
    static constexpr int KV = DP / 16;
    static constexpr int VE = DP / 16;
    static constexpr int VD = DP / 16;
};

// One wave's state over the positions it has seen.
template <int DP> struct State {
    float m, l;              // of query head lane % 16; l is this lane's share
    V4f o[DP / 16];          // o[b][r]: dim DP/16 * (4 (lane / 16) + r) + b

    __device__ __forceinline__ void clear()
    {
        m = -__builtin_inff();
        l = 0.f;
#pragma unroll
        for (int b = 0; b < DP / 16; ++b) o[b] = V4f{0.f, 0.f, 0.f, 0.f};
    }
};

// Where the positions of one tile lie: element offsets of their rows from the
// head's first, and which are seen (bit j: position j of the tile).
//   kWhole: 16 positions share a page (its size is a multiple of 16), so a lane's
//   rows are a wave's base plus a fixed offset; otherwise each lane keeps the
//   rows of positions l % 16 and 16 + l % 16 and asks other lanes for the rest.
// Positions that are not seen point at some row of the cache, so that every
// load is inside it.
template <typename T, bool kWhole> struct Places {
    static constexpr int SUB = Tile<T>::n / 16;
    int64_t base[SUB];
    uint32_t seen;
};

// A tile's keys and values in a wave's registers.
template <typename T, int DP, bool kWhole> struct Operands {
    typedef Layout<T, DP> L;
    static constexpr int TILE = Tile<T>::n, SUB = TILE / 16, VROWS = TILE / 4;

    V4u key[SUB][L::KV];
    uint32_t val[VROWS][L::VD];

    // Row offset of value row j of this lane: position 4 (lane / 16) + j % 4 of the tile's 16 j / 4.
    template <typename A> static __device__ __forceinline__ int64_t value_row(const A& a, const Places<T, kWhole>& p, int j, int lane)
    {
        const int in16 = 4 * (lane >> 4) + (j & 3);
        if constexpr (kWhole) return p.base[j >> 2] + in16 * a.token_stride;
        const uint64_t x = (uint64_t)p.base[j >> 2];
        const uint32_t lo = __shfl((uint32_t)x, in16), hi = __shfl((uint32_t)(x >> 32), in16);
        return (int64_t)(((uint64_t)hi << 32) | lo);
    }

    template <typename A> __device__ __forceinline__ void load_keys(const A& a, const T* head, const Places<T, kWhole>& p, int lane)
    {
        constexpr int E = 16 / sizeof(T);
        const int d0 = E * (lane >> 4);
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const T* q = head + p.base[u] + (kWhole ? (lane & 15) * a.token_stride : 0);
#pragma unroll
            for (int i = 0; i < L::KV; ++i) {
                const int d = d0 + 4 * E * i;
                key[u][i] = *reinterpret_cast<const V4uAnywhere*>(q + (d < a.dim ? d : 0));
            }
        }
        if (a.dim != DP) {
            // dims the head does not have: zero against the query's zero, whatever the cache holds
#pragma unroll
            for (int i = 0; i < L::KV; ++i)
#pragma unroll
                for (int u = 0; u < SUB; ++u)
                    if (d0 + 4 * E * i >= a.dim) key[u][i] = V4u{0, 0, 0, 0};
        }
    }

    // Past the caches: a step reads each value once, and all layers' caches exceed
    // them (3 GB: 504 -> 454 us; 134 MB that could have stayed there: 31.2 -> 32.1 us).
    // A key row's line is completed by the next load, so keys take the usual way.
    // kOnce: nobody else reads them.
    template <bool kOnce = true, typename A> __device__ __forceinline__ void load_values(const A& a, const T* head, const Places<T, kWhole>& p, int lane)
    {
        constexpr int E = 16 / sizeof(T);
        const int d0 = L::VE * (lane & 15);
#pragma unroll
        for (int j = 0; j < VROWS; ++j) {
            const T* q = head + value_row(a, p, j, lane);
            if constexpr (L::VD == 2) {
                const V2uAnywhere* const from = reinterpret_cast<const V2uAnywhere*>(q + (d0 < a.dim ? d0 : 0));
                const V2u x = kOnce ? __builtin_nontemporal_load(from) : *from;
                val[j][0] = x[0];
                val[j][1] = x[1];
            } else {
#pragma unroll
                for (int i = 0; i < L::VD / 4; ++i) {
                    const V4uAnywhere* const from = reinterpret_cast<const V4uAnywhere*>(q + (d0 + E * i < a.dim ? d0 + E * i : 0));
                    const V4u x = kOnce ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
                    for (int e = 0; e < 4; ++e) val[j][4 * i + e] = x[e];
                }
            }
        }
    }

    // Values of positions that are not seen may be anything, and 0 times that is not 0.
    __device__ __forceinline__ void drop_unseen_values(uint32_t seen, int lane)
    {
#pragma unroll
        for (int j = 0; j < VROWS; ++j)
            if (!(seen >> (16 * (j >> 2) + 4 * (lane >> 4) + (j & 3)) & 1)) {
#pragma unroll
                for (int i = 0; i < L::VD; ++i) val[j][i] = 0;
            }
    }
};

template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t rounded<uint16_t>(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Four consecutive output values.
template <typename T> __device__ __forceinline__ void store4(T* p, V4f x);
template <> __device__ __forceinline__ void store4<float>(float* p, V4f x)
{
    *reinterpret_cast<V4uAnywhere*>(p) = __builtin_bit_cast(V4u, x);
}
template <> __device__ __forceinline__ void store4<uint16_t>(uint16_t* p, V4f x)
{
    typedef __bf16 V4bf __attribute__((ext_vector_type(4)));
    V4bf h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = (__bf16)x[e];
    *reinterpret_cast<V2uAnywhere*>(p) = __builtin_bit_cast(V2u, h);
}

// floor(x / y) of counts below 2^53: a third of the integer sequence's instructions.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y)
{
    int64_t q = (int64_t)((double)x / (double)y);
    const int64_t r = x - q * y;
    return r < 0 ? q - 1 : r >= y ? q + 1 : q;
}

// The line of `units` tiles in `waves` shares: share w begins at floor(units w / waves).
struct Shares {
    int64_t units, q;
    int32_t rest, waves;

    __device__ __forceinline__ Shares(int64_t u, int32_t n) : units(u), q(quotient(u, n)), rest((int32_t)(u - q * n)), waves(n) {}

    __device__ __forceinline__ int64_t begin(int32_t w) const
    {
        return q * w + (int64_t)((uint32_t)(rest * w) / (uint32_t)waves);     // both factors below 2^12
    }

    // The share that holds a unit.
    __device__ int32_t of(int64_t unit) const
    {
        int32_t w = min(waves - 1, (int32_t)((double)unit * waves / (double)units));      // or a neighbour
        while (begin(w) > unit) --w;
        while (w + 1 < waves && begin(w + 1) <= unit) ++w;
        return w;
    }
};

}  // namespace

}  // namespace cpes
