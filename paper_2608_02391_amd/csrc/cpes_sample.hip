// cpes_sample.hip -- gfx950 kernels that draw a token from each row of logits.
//
// Mathematics.  With c = scale log2 e and w_v = 2^(c (x_v - max x)), tokens in the order
// of descending x, then ascending v:
//   of the first top_k those in front of which less than top_p of their weight lies,
//   and of these the ones with ln w_v >= ln min_p, stay; the token is the lowest v with
//   sum_{v' <= v} w_v' > u sum w over those that stay.
// What stays is a beginning of that order, so one key, (x, ~v) as 64 bits, bounds it.
//
// Precision.  With V tokens there are V borders between 0 and 1, and sums that are off by
// e put u on the wrong side of one with a probability of up to V e: 32-bit sums of
// 151,936 logits would pick another token every few hundred rows.  Weights are
// therefore 64-bit, right to 2^-37.5 (2^t from a table of 64 cells an octave and a short
// polynomial), and so are their sums, always taken in one order.
//
// Split.  A row is cut into strips, one a wave, and these into blocks of 2^shift steps; a
// step is four 16-byte vectors of each lane, in token order.  The one pass over the
// logits (k_sample_read) leaves for each block its sum (where a sum over the whole row is
// needed: no filter, or top_p of everything), and otherwise for each of its lanes the
// maximum of what it has read, and one logit.  What is behind that (k_sample_join, a
// workgroup a row) looks at little again:
//   no filter:  the block in which u sum w lies, and in it the token;
//   filters:    the tokens from a bound on that the lanes' maxima give: the k-th largest of
//               them is reached by k tokens.  They are ranked, and what stays of them is known.
//   Only where that is too much (flat rows, thousands of tokens in top_p) is the row read
//   again, a few times: the bounding key is found by its digits, from histograms of weights
//   that begin where the logits that were noted put it.
// Two launches, because they want other registers and other numbers of waves; rows of up to
// four steps are one wave's, in one launch.
//
// What bounds it.  4,096 rows of 151,936 in bf16, 186 us of HBM: without a sum (top_k 20 or 50,
// min_p) 272-292 us, the notes and the second launch's dozen dependent trips; with sums and no
// filter the vector units, about 11 instructions a logit, 351 us; top_p of 0.95 where a seventh
// of the rows is flat 1,022-1,049 us, of which reading those again takes most.  One row is two
// launches of trips that wait for each other: 18-21 us, 50 where some hundred tokens stay and
// 229 where most do.
#include <algorithm>
#include <type_traits>

#include "cpes_eval.hpp"
#include "cpes_powers.hpp"

namespace cpes {

namespace {

typedef unsigned int V4u __attribute__((ext_vector_type(4)));
typedef unsigned int V2u __attribute__((ext_vector_type(2)));
typedef V4u V4uAnywhere __attribute__((aligned(2)));
typedef unsigned long long Key;

constexpr int kUnroll = 4;                // vectors of a lane and step
constexpr int kParts = 384;               // parts of blocks that are read again for them
constexpr int kFirstParts = 48;           // and how many at first, where top_p decides
constexpr int kCounted = 128;             // keys ranked by counting
constexpr int kDepth = 4;                 // vectors of a thread under way where the row is read again
constexpr int64_t kMaxGrid = 1 << 20;
constexpr int kFewRows = 256;
constexpr int kManyBlocks = 96;          // of a row among many
constexpr int kManyParts = 32;           // and parts, of 64 lanes
constexpr int kReadGroups = 1024;        // workgroups that read few rows
constexpr double kFar = -52.0;           // weights below 2^kFar of the largest count as 0

template <typename T> struct Vec { static constexpr int n = 16 / sizeof(T); };

template <typename T> __device__ __forceinline__ float value_of(T x);
template <> __device__ __forceinline__ float value_of<float>(float x) { return x; }
template <> __device__ __forceinline__ float value_of<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

template <typename T> __device__ __forceinline__ void unpack(V4u w, float* x);
template <> __device__ __forceinline__ void unpack<float>(V4u w, float* x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void unpack<uint16_t>(V4u w, float* x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// Descending value, ascending token; -inf and NaN have no key.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);       // -0 ties with 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_at(uint32_t order)
{
    return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order);
}
__device__ __forceinline__ Key key_of(float x, uint32_t token)
{
    return x > -__builtin_inff() ? ((Key)order_of(x) << 32) | (uint32_t)~token : 0;
}
__device__ __forceinline__ float key_value(Key k) { return value_at((uint32_t)(k >> 32)); }
__device__ __forceinline__ uint32_t key_token(Key k) { return ~(uint32_t)k; }

// The order of the least bf16 not below x.
__device__ __forceinline__ uint16_t note_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f), v = (u & 0x80000000u ? u : u + 0xFFFFu) >> 16;
    return (uint16_t)(v & 0x8000u ? ~v : v | 0x8000u);
}
constexpr uint16_t kNoteNothing = 0x007F;               // of -inf

// A maximum that a NaN gets through.
__device__ __forceinline__ float most_of(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// 2^(j / 32).
__device__ const double kTwoTo[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
};

// 2^t for -1022 < t < 1000 times what `add` is: t = k / 32 + r with |r| <= 1/64, 2^r from its
// series, e^y = 1 + y + .. + y^4 / 24, off by (ln 2 / 64)^5 / 120 = 1.2e-12 at most.
__device__ __forceinline__ double power(double t, const double* table)
{
    constexpr double kRound = 0x1.8p+47;                // 1.5 2^52 / 32: adding it leaves multiples of 1/32
    constexpr double a1 = 0.69314718055994530942, a2 = a1 * a1 / 2, a3 = a2 * a1 / 3, a4 = a3 * a1 / 4;
    const double y = t + kRound, r = t - (y - kRound);
    const uint32_t k = (uint32_t)__double_as_longlong(y);
    const double f = table[k & 31];
    const double p = r * fma(r, fma(r, fma(r, a4, a3), a2), a1);
    const double w = fma(f, p, f);
    return __longlong_as_double(__double_as_longlong(w) + ((long long)(int)(k & ~31u) << 47));
}

// The same for the pass over the logits, which does little else and is bound by it: t comes as cells of
// 1/64 octave from kLow on, whose beginnings are in a table that leaves no exponent to be put
// together; in a cell 2^(r / 64) = 1 + a1 r + a2 r^2 + a3 r^3, r < 1, off by 2^-37.5 at most (a minimax
// fit that is exact at 0).  The conversion takes what is below the table, -inf too, to its first entry,
// which is 0, and the fraction's clamp takes -inf's NaN to 0.  What is above the table must not come here.

template <int K> __device__ __forceinline__ void fill_powers(double* powers)
{
    for (int i = threadIdx.x; i < kPowers; i += K)
        powers[i] = i == 0 ? 0.0 : ldexp(kTwoTo[i % kCells / 2] * (i & 1 ? 0x1.02c9a3e778061p+0 : 1.0), i / kCells + kLow);
}

// sum + 2^t for N exponents t = cells(j) / 64 + kLow.  The table's entries of the next four are asked for
// before the last four are used: a wave waits for none of them (the pass over 4,096 rows of 151,936: 385 us
// with each asked for on its own, 345 so).
template <int N, typename F> __device__ __forceinline__ double add_powers(double sum, const double* powers, F cells)
{
    constexpr int G = 4;
    double f[2][G], r[2][G];
    auto ask = [&](int j) {
#pragma unroll
        for (int e = 0; e < G; ++e) {
            const double t = cells(j + e);
            uint32_t cell;
            asm("v_cvt_u32_f64_e32 %0, %1" : "=v"(cell) : "v"(t));
            asm("v_fract_f64_e64 %0, %1 clamp" : "=v"(r[j / G & 1][e]) : "v"(t));
            f[j / G & 1][e] = powers[cell];
        }
    };
    ask(0);
#pragma unroll
    for (int j = 0; j < N; j += G) {
        __builtin_amdgcn_sched_barrier(0);
        if (j + G < N) ask(j + G);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < G; ++e) {
            const double x = r[j / G & 1][e];
            sum = fma(f[j / G & 1][e], fma(x, fma(x, fma(x, 0x1.c90fc991be8ebp-23, 0x1.ebfa7f9763063p-15), 0x1.62e43029bdff8p-7), 1.0), sum);
        }
    }
    return sum;
}

// The logits of a vector one after the other, so that a loop over them need not be unrolled: most
// of what is behind the pass over the logits runs once a row, and what such code costs is its way
// into the instruction cache (one row's second launch: 27 us with all of it unrolled, 12 so).
template <typename T> struct Logits {
    V4u w;

    __device__ __forceinline__ float next()
    {
        if constexpr (std::is_same<T, uint16_t>::value) {
            const float x = __uint_as_float(w[0] << 16);
            w[0] = __builtin_amdgcn_alignbit(w[1], w[0], 16);
            w[1] = __builtin_amdgcn_alignbit(w[2], w[1], 16);
            w[2] = __builtin_amdgcn_alignbit(w[3], w[2], 16);
            w[3] >>= 16;
            return x;
        } else {
            const float x = __uint_as_float(w[0]);
            w[0] = w[1];
            w[1] = w[2];
            w[2] = w[3];
            return x;
        }
    }
};

// Vector i of a row of `count` logits; -inf behind its end.
template <typename T> __device__ __forceinline__ V4u vector_at(const T* x0, int64_t count, int64_t i)
{
    constexpr int N = Vec<T>::n;
    if ((i + 1) * N <= count) return *reinterpret_cast<const V4uAnywhere*>(x0 + i * N);
    constexpr uint32_t kNone = std::is_same<T, uint16_t>::value ? 0xFF80FF80u : 0xFF800000u;
    V4u w = {kNone, kNone, kNone, kNone};
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (i * N + j < count) {
            const T x = x0[i * N + j];
            if constexpr (std::is_same<T, uint16_t>::value)
                w[j >> 1] = j & 1 ? (w[j >> 1] & 0xFFFFu) | (uint32_t)x << 16 : (w[j >> 1] & 0xFFFF0000u) | x;
            else
                w[j] = __float_as_uint(x);
        }
    return w;
}

// x of the lane that the DPP control names, 0 where there is none.
template <int CONTROL, int ROWS, typename X> __device__ __forceinline__ X from_lane(X x)
{
    if constexpr (sizeof(X) == 4) {
        return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, ROWS, 0xF, false));
    } else {
        const V2u v = __builtin_bit_cast(V2u, x);
        V2u y;
        y[0] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v[0], CONTROL, ROWS, 0xF, false);
        y[1] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v[1], CONTROL, ROWS, 0xF, false);
        return __builtin_bit_cast(X, y);
    }
}

// Sum over the wave's lanes up to and including each: rows of 16 by shifts, then each row's last lane
// to the next row, and the second row's to the upper half.
template <typename X> __device__ __forceinline__ X wave_scan(X x)
{
    x += from_lane<0x111, 0xF>(x);
    x += from_lane<0x112, 0xF>(x);
    x += from_lane<0x114, 0xF>(x);
    x += from_lane<0x118, 0xF>(x);
    x += from_lane<0x142, 0xA>(x);
    x += from_lane<0x143, 0xC>(x);
    return x;
}

// The wave's sum, in lane 63.
template <typename X> __device__ __forceinline__ X wave_sum(X x) { return wave_scan(x); }

// What a strip's tokens are, as vectors: [first, last), with `behind` tokens short of whole ones.
template <typename T> struct Strip {
    int64_t first;        // vector
    int32_t steps;        // with anything in them

    __device__ __forceinline__ Strip(const SampleArgs& a, int32_t strip)
    {
        constexpr int N = Vec<T>::n;
        first = (int64_t)strip * a.strip_steps * (kSampleLanes * kUnroll);
        const int64_t vecs = ((int64_t)a.vocab + N - 1) / N - first;
        const int64_t all = vecs <= 0 ? 0 : (vecs + kSampleLanes * kUnroll - 1) / (kSampleLanes * kUnroll);
        steps = (int32_t)min(all, (int64_t)a.strip_steps);
    }
};

// 16 bits a part of each lane, stored for up to 8 parts together.  They cost more than their bytes: 39 MB of
// them, however stored, make the pass over 4,096 rows of 151,936 without sums 230 us long, 184 without
// any; so where rows are many a part is of 4 steps and more.
struct Notes {
    V4u w;

    __device__ __forceinline__ void push(uint16_t x)
    {
        w[0] = __builtin_amdgcn_alignbit(w[1], w[0], 16);
        w[1] = __builtin_amdgcn_alignbit(w[2], w[1], 16);
        w[2] = __builtin_amdgcn_alignbit(w[3], w[2], 16);
        w[3] = w[3] >> 16 | (uint32_t)x << 16;
    }
    // The last 2^group of them, a lane's beside each other.
    __device__ __forceinline__ void store(uint16_t* to, int32_t group, int lane) const
    {
        if (group == 3)
            reinterpret_cast<V4u*>(to)[lane] = w;
        else if (group == 2)
            reinterpret_cast<V2u*>(to)[lane] = V2u{w[2], w[3]};
        else if (group == 1)
            reinterpret_cast<uint32_t*>(to)[lane] = w[3];
        else
            to[lane] = (uint16_t)(w[3] >> 16);
    }
};

// One strip, by a wave: notes, samples, sums and what they are relative to, of its blocks;
// the strip's maximum is returned to all lanes.  NT: past the caches.
template <typename T, bool kSums, bool NT, bool kQuick>
__device__ float read_strip(const SampleArgs& a, const T* x0, int32_t strip, const double* powers, const double* table,
                            uint16_t* notes, uint16_t* samples, double* sums, float* refs)
{
    constexpr int N = Vec<T>::n;
    const int lane = threadIdx.x & 63;
    const Strip<T> s(a, strip);
    const int32_t per = 1 << a.shift, per_part = 1 << a.note_shift;
    Notes note = {}, sample = {};
    const int32_t whole = (int32_t)max((int64_t)0, min((int64_t)s.steps, ((int64_t)a.vocab / N - s.first) / (kSampleLanes * kUnroll)));
    float most = -__builtin_inff(), ref = -__builtin_inff(), last = -__builtin_inff(), noted = -__builtin_inff();
    double sum = 0.0, start = 0.0;
    const double cells = a.c * kCells;
    V4u w[kUnroll];
    auto load = [&](int32_t step, int u) {
        const V4uAnywhere* const at =
            reinterpret_cast<const V4uAnywhere*>(x0 + (s.first + (int64_t)step * (kSampleLanes * kUnroll) + u * kSampleLanes + lane) * N);
        w[u] = NT ? __builtin_nontemporal_load(at) : *at;
    };
    // the N logits of a vector, which may be changed
    auto take = [&](float* x) {
        float top = x[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = most_of(top, x[j]);
        noted = most_of(noted, top);
        if constexpr (kSums) {
            if (__any(!(top <= last))) {
                // a new base for all lanes; the block's sum so far moves to it.  With a NaN or +inf the row has no
                // token, and no logit beside it may reach the table's end: they count as nothing
                const bool broken = !(top < __builtin_inff());
                float high = broken ? -__builtin_inff() : top;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) high = fmaxf(high, __shfl_xor(high, d));
                if (high > last) {
                    const double t = a.c * ((double)ref - (double)high);
                    sum = t < 2 * kLow ? 0.0 : sum * power(t, table);
                    ref = high;
                    last = last_above(ref, a.c);
                    start = start_of(ref, cells);
                }
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = broken ? -__builtin_inff() : x[j];
            }
            auto add = [&](auto t) {
                if constexpr (kQuick) {
                    sum = add_powers<N>(sum, powers, t);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (t(j) > 0.0) sum += power(t(j) / kCells + kLow, table);
                }
            };
            if (start_is_near(start)) {
                if (ref > -__builtin_inff()) add([&](int j) { return cells_near(x[j], cells, start); });
            } else {
                add([&](int j) { return cells_far(x[j], ref, cells); });
            }
        }
    };
    const int32_t together = (1 << a.group) - 1;
    auto end_part = [&](int32_t p, uint16_t most_here, uint16_t one) {
        if (a.notes_kept) {
            note.push(most_here);
            if ((p & together) == together) note.store(notes + (p & ~together) * 64, a.group, lane);
        }
        if (a.samples_kept) {
            sample.push(one);
            if ((p & together) == together) sample.store(samples + (p & ~together) * 64, a.group, lane);
        }
    };
    auto end_block = [&](int32_t b) {
        if constexpr (kSums) {
            const double all = wave_sum(sum);
            if (lane == 63) {
                sums[b] = all;
                refs[b] = ref;
            }
            sum = 0.0;
        }
    };
    if (whole > 0) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) load(0, u);
    }
    for (int32_t step = 0; step < s.steps; ++step) {
        if (step >= whole) {
            // the row's last step
#pragma unroll 1
            for (int u = 0; u < kUnroll; ++u) {
                const V4u last = vector_at(x0, a.vocab, s.first + (int64_t)step * (kSampleLanes * kUnroll) + u * kSampleLanes + lane);
                w[0] = w[1];
                w[1] = w[2];
                w[2] = w[3];
                w[3] = last;
            }
        }
        float one = 0.f;
        if constexpr (kSums) {
            // a vector at a time: the registers are for the powers
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                float x[N];
                unpack<T>(w[u], x);
                if (step + 1 < whole) load(step + 1, u);
                if (u == 0) one = x[0];
                take(x);
            }
        } else {
            float x[kUnroll][N];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) unpack<T>(w[u], x[u]);
            if (step + 1 < whole) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) load(step + 1, u);
            }
            one = x[0][0];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) take(x[u]);
        }
        if ((step & (per - 1)) == per - 1 || step + 1 == s.steps) end_block(step >> a.shift);
        if ((step & (per_part - 1)) == per_part - 1 || step + 1 == s.steps) {
            most = most_of(most, noted);
            end_part(step >> a.note_shift, note_of(noted), note_of(one));
            noted = -__builtin_inff();
        }
    }
    static_assert(kUnroll == 4, "the last step fills w from behind");
    for (int32_t b = s.steps == 0 ? 0 : ((s.steps - 1) >> a.shift) + 1; b < a.slots; ++b) end_block(b);
    for (int32_t p = s.steps == 0 ? 0 : ((s.steps - 1) >> a.note_shift) + 1; p < a.note_slots; ++p) end_part(p, kNoteNothing, kNoteNothing);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = most_of(most, __shfl_xor(most, d));
    return most;
}

// What a row's work keeps in LDS.
template <int K, int BLOCKS, int PARTS, int BINS> struct Shared {
    static constexpr int kCandidates = BINS > 1024 ? BINS / 2 : 512;      // tokens that are ranked
    static constexpr int kBins = BINS;    // of a histogram
    alignas(16) uint16_t notes[PARTS * 64];           // maxima of parts
    double sums[BLOCKS];
    float refs[BLOCKS];
    int32_t ties[BLOCKS];
    double table[32];
    double wave[K / 64];
    uint32_t wave_count[K / 64];
    union {
        struct {
            Key keys[kCandidates], ranked[kCandidates];
        };
        struct {
            Key mass[BINS];               // of a bin's tokens, as whole numbers
            uint32_t count[BINS];
        };
    };
    int32_t number, place, token;
    float value;
    uint32_t found;
    double total;
};

// Sum over the workgroup's threads up to and including each; *total receives all.
template <int K, typename X> __device__ __forceinline__ X block_scan(X x, X* wave, X* total)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const X y = wave_scan(x);
    __syncthreads();
    if (lane == 63) wave[w] = y;
    __syncthreads();
    X before = 0, all = 0;
#pragma unroll 1
    for (int i = 0; i < K / 64; ++i) {
        const X z = wave[i];
        if (i < w) before += z;
        all += z;
    }
    *total = all;
    return before + y;
}

// What stays of a row: orders above `order`, and of those alike the first `ties`.
struct Cut {
    uint32_t order;
    int32_t ties;

    __device__ __forceinline__ Cut stricter(Cut o) const
    {
        return order != o.order ? (order > o.order ? *this : o) : Cut{order, min(ties, o.ties)};
    }
};
constexpr Cut kEverything = {0, 0};       // order 0 is a NaN's

template <typename T, typename S, int K> struct RowWork {
    static constexpr int N = Vec<T>::n, kBins = S::kBins, kCandidates = S::kCandidates;
    const SampleArgs& a;
    S& s;
    const T* x0;
    const uint16_t* samples;              // a logit of each part
    float m;                              // the row's largest logit
    int32_t blocks, parts;                // parts of 64 lanes
    int32_t tid;

    __device__ __forceinline__ double weight(float x) const
    {
        if (!(x > -__builtin_inff())) return 0.0;
        const double t = a.c * ((double)x - (double)m);
        return t < kFar ? 0.0 : power(t, s.table);
    }
    // whether ln w >= ln min_p
    __device__ __forceinline__ bool likely(float x) const { return a.scale * ((double)x - (double)m) >= a.least; }

    // First token of a block; blocks follow each other in token order.
    __device__ __forceinline__ int64_t block_begin(int32_t b) const
    {
        const int32_t strip = b / a.slots, i = b - strip * a.slots;
        return min((int64_t)a.vocab, ((int64_t)strip * a.strip_steps + min((int64_t)a.strip_steps, (int64_t)i << a.shift)) *
                                         (kSampleLanes * kUnroll * N));
    }

    // Of the tokens [from, to) that stay the first up to which more than `rest` lies; where
    // roundings leave none, the last that has a weight.  Into s.token, -1 if there is none, and its logit
    // into s.value.  `ties`: how many of the cut's ties before `from` stay.
    __device__ void locate(int64_t from, int64_t to, double rest, Cut cut, int32_t ties)
    {
        const float edge = cut.order ? value_at(cut.order) : -__builtin_inff();       // those above it stay
        if (tid == 0) s.token = -1;
#pragma unroll 1
        for (int64_t at = from; at < to; at += K * N) {
            const int64_t i = at / N + tid;
            const V4u w = vector_at(x0, to, i);
            uint32_t alike = 0, all_alike = 0;
            if (cut.order != 0) {
                Logits<T> x = {w};
#pragma unroll 1
                for (int j = 0; j < N; ++j) alike += x.next() == edge;
                alike = block_scan<K>(alike, s.wave_count, &all_alike) - alike + ties;
            }
            // the sum up to each token from `before` on: all of them, or up to the first above `limit`
            auto sum_from = [&](double before, double limit, int32_t* which, float* value) {
                Logits<T> x = {w};
                uint32_t tie = alike;
                double sum = before;
                *which = -1;
#pragma unroll 1
                for (int j = 0; j < N; ++j) {
                    const float y = x.next();
                    bool stays = y > edge;
                    if (cut.order != 0 && y == edge) stays = tie++ < (uint32_t)cut.ties;
                    const double v = stays && likely(y) ? weight(y) : 0.0;
                    if (v > 0.0) {
                        *which = j;
                        *value = y;
                        sum += v;
                        if (sum > limit) break;
                    }
                }
                return sum;
            };
            int32_t last;
            float value = 0.f;
            double total;
            const double mine = sum_from(0.0, __builtin_inf(), &last, &value);
            ties += all_alike;
            if (tid == 0) s.place = K;
            const double upto = block_scan<K>(mine, s.wave, &total);
            if (last >= 0) {
                atomicMax(&s.token, (int32_t)(i * N + last));
                if (upto > rest) atomicMin(&s.place, tid);
            }
            __syncthreads();
            const int32_t place = s.place;
            if (place < K ? tid == place : last >= 0 && s.token == (int32_t)(i * N + last)) {
                if (place < K) {
                    sum_from(upto - mine, rest, &last, &value);
                    s.token = (int32_t)(i * N + last);
                }
                s.value = value;
            }
            __syncthreads();
            if (place < K) return;
            rest -= total;
        }
    }

    // Sums of the blocks relative to the row's maximum; the sum up to each is left in s.sums, and all of them returned.
    __device__ double total_of_blocks()
    {
        double x = 0.0, total;
        if (tid < blocks && s.sums[tid] > 0.0) {
            // a block's largest weight may be above what its sum is relative to
            const double t = a.c * ((double)s.refs[tid] - (double)m);
            if (t >= kFar - (kRoom + 1)) x = s.sums[tid] * power(t, s.table);
        }
        const double upto = block_scan<K>(x, s.wave, &total);
        __syncthreads();
        if (tid < blocks) s.sums[tid] = upto;
        __syncthreads();
        return total;
    }

    // From the blocks' sums up to each the token; s.ties holds the ties before each block where there is a cut.
    // Inlined, because a call kept 240 bytes of its caller's state a lane in scratch where one wave does a row.
    __device__ __forceinline__ void pick(double total, Cut cut)
    {
        const double target = uniform() * total;
        if (tid == 0) s.place = blocks;
        __syncthreads();
        if (tid < blocks && s.sums[tid] > target) atomicMin(&s.place, tid);
        __syncthreads();
        int32_t b = s.place;
        __syncthreads();
        if (b == blocks) {
            // u sum w rounded up to the sum: the last block that has any
            if (tid == 0) s.place = 0;
            __syncthreads();
            if (tid < blocks && s.sums[tid] > (tid ? s.sums[tid - 1] : 0.0)) atomicMax(&s.place, tid);
            __syncthreads();
            b = s.place;
            __syncthreads();
        }
        int64_t from = block_begin(b), to = b + 1 < blocks ? block_begin(b + 1) : (int64_t)a.vocab;
        double rest = target - (b ? s.sums[b - 1] : 0.0);
        int32_t ties = cut.order ? s.ties[b] : 0;
#pragma unroll 1
        for (int turn = 0;; ++turn) {
            locate(from, to, rest, cut, ties);
            __syncthreads();
            if (s.token >= 0 || turn == 2) break;
            __syncthreads();
            // weights that count as 0 made that block's sum: the next token that has one, or else the last
            if (turn == 0) {
                from = to;
                to = a.vocab;
                rest = 0.0;
                ties = cut.order && b + 1 < blocks ? s.ties[b + 1] : 0;
            } else {
                to = from;
                from = 0;
                rest = __builtin_inf();
                ties = 0;
            }
        }
    }

    float u;                              // the number given
    uint32_t weights_from = 0;            // where not 0, s.mass holds the weights of bf16 logits of orders from here on
    __device__ __forceinline__ double uniform() const
    {
        constexpr double kLast = 1.0 - 0x1p-53;
        return u > 0.f ? fmin((double)u, kLast) : 0.0;      // a NaN is not above 0
    }

    // Calls f(x, token) for the logits of vectors [first, last) of a row that ends at `to`, THREADS
    // threads a vector each, kDepth of them under way.
    template <int THREADS, typename F> __device__ __forceinline__ void each_logit(int64_t first, int64_t last, int64_t to, int thread, F f)
    {
        const int64_t full = to / N;
#pragma unroll 1
        for (int64_t i0 = first + thread; i0 < last; i0 += THREADS * kDepth) {
            V4u w[kDepth];
#pragma unroll
            for (int d = 0; d < kDepth; ++d)
                if (i0 + d * THREADS < min(last, full)) w[d] = *reinterpret_cast<const V4uAnywhere*>(x0 + (i0 + d * THREADS) * N);
#pragma unroll 1
            for (int64_t i = i0; i < min(last, i0 + THREADS * kDepth); i += THREADS) {
                Logits<T> x = {w[0]};
                if (i >= full) x.w = vector_at(x0, to, i);
#pragma unroll 2
                for (int j = 0; j < N; ++j) f(x.next(), (uint32_t)(i * N + j));
#pragma unroll
                for (int d = 1; d < kDepth; ++d) w[d - 1] = w[d];
            }
        }
    }

    // Bins of the notes, by how far they are below the largest logit.
    static constexpr float kPerOctave = kBins / 64;
    __device__ __forceinline__ int note_bin(uint32_t order) const
    {
        // a note of fp32 logits may be rounded up beyond the largest
        return (int)fminf(fmaxf(m - value_at(order << 16), 0.f) * (float)a.c * kPerOctave, kBins - 1.f);
    }

    // Counts the notes in their bins: s.number receives the first bin up to which there are `rank` of
    // them and s.found how many there are; where these are more than `most`, the bin in front of the
    // first up to which there are so many, and the number up to there.  kBins - 1, and all of
    // them, if there are fewer than `rank`.
    __device__ void count_notes(uint32_t rank, uint32_t most)
    {
        for (int i = tid; i < kBins; i += K) s.count[i] = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < parts * 64; i += K) {
            const uint32_t order = s.notes[i];
            if (order > kNoteNothing) atomicAdd(&s.count[note_bin(order)], 1u);
        }
        __syncthreads();
        constexpr int PER = kBins / K;
        uint32_t mine = 0, all;
#pragma unroll 1
        for (int e = 0; e < PER; ++e) mine += s.count[tid * PER + e];
        uint32_t upto = block_scan<K>(mine, s.wave_count, &all) - mine;
        if (tid == 0) {
            s.number = kBins - 1;
            s.found = all;
        }
        __syncthreads();
#pragma unroll 1
        for (int e = 0; e < PER; ++e) {
            const uint32_t before = upto;
            upto += s.count[tid * PER + e];
            if (upto <= most ? before < rank && upto >= rank : before <= most && before < rank) {
                s.number = tid * PER + e - (upto <= most ? 0 : 1);
                s.found = upto <= most ? upto : before;
            }
        }
        __syncthreads();
    }

    // The least logit that the parts with notes in bins up to `bin` can have as their maximum.  All
    // tokens from it on lie in such parts, and each such part has one.
    __device__ __forceinline__ float least_of_bins(int bin) const
    {
        uint32_t o = note_of(m - (bin + 1) / ((float)a.c * kPerOctave));          // or near it
        while (o < 0xFF7F && note_bin(o) > bin) ++o;
        while (o > kNoteNothing + 1u && note_bin(o - 1) <= bin) --o;
        // a note above 0 is rounded up, one below is the beginning of what it stands for
        return value_at(o > 0x8000 ? ((o - 1) << 16) + 1 : o << 16);
    }

    // All tokens x >= bound of the parts whose notes lie in bins up to `bin` into s.keys; their number,
    // which may exceed what there is room for.  The parts are listed, and then read together.
    __device__ int32_t collect(int bin, float bound)
    {
        uint32_t* const list = reinterpret_cast<uint32_t*>(s.ranked);
        const uint32_t least = max((uint32_t)note_of(bound), kNoteNothing + 1u);
        if (tid == 0) s.number = s.place = 0;
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < parts * 64; i += K) {
            const uint32_t order = s.notes[i];
            if (order >= least && note_bin(order) <= bin) {
                const int at = atomicAdd(&s.place, 1);
                if (at < kParts) list[at] = i;
            }
        }
        __syncthreads();
        const int32_t listed = s.place;
        if (listed > kParts) return kCandidates + 1;
        const int32_t vectors = kUnroll << a.note_shift;
#pragma unroll 1
        for (int64_t item = tid; item < (int64_t)listed * vectors; item += K) {
            const int32_t part = (int32_t)(item >> (2 + a.note_shift)), v = (int32_t)(item & (vectors - 1)), i = list[part];
            // a strip's notes are groups of parts, of each group the lanes', of each lane the parts'
            const int32_t strip = i / (a.note_slots * 64), rest = i - strip * a.note_slots * 64, lane = rest >> a.group & 63;
            const int32_t in = ((rest >> (6 + a.group) << a.group) + (rest & ((1 << a.group) - 1))) << a.note_shift;
            if (in + v / kUnroll >= a.strip_steps) continue;
            const int64_t at = ((int64_t)strip * a.strip_steps + in) * (kSampleLanes * kUnroll) + v * kSampleLanes + lane;
            Logits<T> x = {vector_at(x0, a.vocab, at)};
#pragma unroll 1
            for (int j = 0; j < N; ++j) {
                const float y = x.next();
                if (y >= bound && y > -__builtin_inff()) {
                    const int32_t to = atomicAdd(&s.number, 1);
                    if (to < kCandidates) s.keys[to] = key_of(y, (uint32_t)(at * N + j));
                }
            }
        }
        __syncthreads();
        const int32_t found = s.number;
        __syncthreads();
        return found;
    }

    // The n keys in s.keys in descending order, in s.ranked.
    __device__ void rank(int32_t n)
    {
        if (n <= kCounted) {
            // each key's place is the number of larger ones
            for (int i = tid; i < n; i += K) {
                const Key mine = s.keys[i];
                int32_t place = 0;
#pragma unroll 4
                for (int j = 0; j < n; ++j) place += s.keys[j] > mine;
                s.ranked[place] = mine;
            }
            __syncthreads();
            return;
        }
        int size = 2 * kCounted;
        while (size < n) size *= 2;
        for (int i = tid; i < size; i += K) s.ranked[i] = i < n ? s.keys[i] : 0;
        __syncthreads();
        for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                for (int t = tid; t < size / 2; t += K) {
                    const int i = 2 * t - (t & (j - 1)), o = i + j;
                    const Key x = s.ranked[i], y = s.ranked[o];
                    if ((x < y) == ((i & k) == 0)) {
                        s.ranked[i] = y;
                        s.ranked[o] = x;
                    }
                }
                __syncthreads();
            }
    }

    // From the n tokens in s.keys, which are all from some key on: true, with the token in
    // s.token, its logit in s.value and the weight of those that stay in s.total, if they hold
    // all that stay.  bounded: nothing behind them stays.  total: the row's weight, where top_p
    // of it counts; *weighs receives that of the n.
    __device__ bool from_candidates(int32_t n, bool bounded, double total, double* weighs)
    {
        constexpr int PER = (kCandidates + K - 1) / K;
        rank(n);
        if (tid == 0) s.place = n;
        const int32_t first = a.top_k > 0 ? min(a.top_k, n) : n;
        double w[PER], mine = 0.0, all;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int32_t i = tid * PER + e;
            w[e] = i < first ? weight(key_value(s.ranked[i])) : 0.0;
            mine += w[e];
        }
        double upto = block_scan<K>(mine, s.wave, &all) - mine;
        *weighs = all;
        const double enough = a.top_p * (a.top_k > 0 ? all : total);
        const bool part = a.top_p < 1.0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int32_t i = tid * PER + e;
            if (i < first && i > 0 && ((part && !(upto < enough)) || !likely(key_value(s.ranked[i])))) atomicMin(&s.place, i);
            upto += w[e];
        }
        __syncthreads();
        const int32_t kept = min(s.place, first);
        // nothing of them was cut off: more may stay
        if (kept == n && !bounded && !(part && !(all < enough)) && !(a.top_k > 0 && n >= a.top_k)) return false;
        // in token order: keys that begin with the token
        for (int i = tid; i < kept; i += K) s.keys[i] = s.ranked[i] << 32 | s.ranked[i] >> 32;
        if (tid == 0) {
            s.token = -1;
            s.found = K;
        }
        __syncthreads();
        rank(kept);
        int32_t last = -1;
        mine = 0.0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int32_t i = tid * PER + e;
            w[e] = i < kept ? weight(value_at((uint32_t)s.ranked[i])) : 0.0;
            mine += w[e];
            if (w[e] > 0.0) last = i;
        }
        upto = block_scan<K>(mine, s.wave, &all);
        const double rest = uniform() * all;
        if (tid == 0) s.total = all;
        if (last >= 0) atomicMax(&s.token, last);
        if (upto > rest && last >= 0) atomicMin(&s.found, (uint32_t)tid);
        __syncthreads();
        const int32_t fallback = s.token;
        const uint32_t owner = s.found;
        __syncthreads();
        if (owner == K ? tid == 0 : tid == (int)owner) {
            int32_t at = fallback;
            double before = upto - mine;
            if (owner < K) {
                at = last;
                bool found = false;
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    before += w[e];
                    if (!found && w[e] > 0.0 && before > rest) {
                        at = tid * PER + e;
                        found = true;
                    }
                }
            }
            s.token = (int32_t)~(uint32_t)(s.ranked[at] >> 32);
            s.value = value_at((uint32_t)s.ranked[at]);
        }
        __syncthreads();
        return true;
    }

    // The cut that leaves the first `number` of the order (by_weight: as many as it takes to
    // reach `enough`), found by reading the row again: a histogram of what lies in [lo, hi] of
    // the orders, and of the bin it ends in again, until that is one order.  Weights in bins of
    // several orders are whole numbers, each off by up to half of 2^-44 of the heaviest, and 150,000 alike are off
    // alike.  Where that could decide, what lies above is summed again in 64 bits (`exact`: from the beginning,
    // for a caller who needs the weight): this says for certain whether the cut is in [lo, hi], and if not, the
    // orders on that side are looked at.  (Summed again in every round, 256 flat rows took 285 us, 257 so.)
    // *weight_left receives the weight that is left.
    __device__ Cut search(uint32_t lo, uint32_t hi, int64_t number, double enough, bool by_weight, bool exact, double* weight_left)
    {
        constexpr uint32_t kFirst = 0x00800000;      // of finite numbers
        // bf16 logits have 16 bits of order, and a bin may be one of them, whose weight is its number of times one weight
        constexpr int kLeast = std::is_same<T, uint16_t>::value ? 16 : 0;
        const auto logit = [](uint32_t o) { return value_at(kLeast > 0 && o < 0x80000000u ? o | 0xFFFFu : o); };
        const int64_t vecs = ((int64_t)a.vocab + N - 1) / N;
        double* const masses = reinterpret_cast<double*>(s.mass);
        // the cut lies in [bottom, ceiling]; weight, and number, of what lies above that, and how far that weight may be off
        const uint32_t highest = kLeast > 0 ? order_of(m) | 0xFFFFu : order_of(m);
        uint32_t bottom = kFirst, ceiling = highest;
        double above_ceiling = 0.0, doubt = 0.0;
        int64_t count_ceiling = 0;
        auto be_exact = [&] {
            exact = true;
            bottom = kFirst;
            ceiling = highest;
            above_ceiling = doubt = 0.0;
            count_ceiling = 0;
            __syncthreads();
        };
#pragma unroll 1
        while (true) {
            hi = max(min(hi, ceiling), bottom);
            lo = max(min(lo, hi), bottom);
            if (kLeast > 0) {
                lo &= 0xFFFF0000u;
                hi |= 0x0000FFFFu;
                // nothing lies above hi where the bins reach that far
                if (count_ceiling == 0 && (ceiling - lo) >> kLeast < kBins) hi = ceiling;
            }
            int sh = kLeast;
            while (((hi - lo) >> sh) >= kBins) ++sh;
            const bool alike = sh == kLeast;          // a bin is one order
            const float least = value_at(lo), most = value_at(hi), known_from = value_at(ceiling);
            // weights as whole numbers, so that their sums do not depend on the order: 2^units for the largest of them
            const int units = 62 - (32 - __clz((int)a.vocab));
            const double unit = (double)((uint64_t)1 << units) / fmax(weight(fminf(most, m)), 0x1p-100);
            for (int i = tid; i < kBins; i += K) {
                s.mass[i] = 0;
                s.count[i] = 0;
            }
            __syncthreads();
            double mine = 0.0;
            uint32_t mine_count = 0;
            each_logit<K>(0, vecs, a.vocab, tid, [&](float x, uint32_t) {
                if (!(x >= least) || x > known_from) return;
                if (x > most) {
                    mine += weight(x);
                    ++mine_count;
                } else {
                    const uint32_t bin = (order_of(x) - lo) >> sh;
                    if (!alike) atomicAdd(&s.mass[bin], (Key)(weight(x) * unit + 0.5));
                    atomicAdd(&s.count[bin], 1u);
                }
            });
            double above;                 // weight, and number, of what lies above hi
            uint32_t more;
            block_scan<K>(mine, s.wave, &above);
            block_scan<K>(mine_count, s.wave_count, &more);
            above += above_ceiling;
            int64_t above_count = count_ceiling + more;
            __syncthreads();
            // from the top: the bin in which the number or the weight is reached
            constexpr int PER = kBins / K;
            const int top = kBins - 1 - tid * PER;
            double mass = 0.0, all_mass;
            uint32_t count = 0, all_count;
#pragma unroll 1
            for (int e = 0; e < PER; ++e) {
                const int bin = top - e;
                const uint32_t n = s.count[bin];
                double w = 0.0;
                if (n) w = alike ? n * weight(logit(lo + ((uint32_t)bin << sh))) : (double)s.mass[bin] / unit;
                masses[bin] = w;
                mass += w;
                count += n;
            }
            double mass_upto = block_scan<K>(mass, s.wave, &all_mass) - mass;
            uint32_t count_upto = block_scan<K>(count, s.wave_count, &all_count) - count;
            const auto reached = [&](double x, uint32_t n) { return by_weight ? !(above + x < enough) : above_count + n >= number; };
            const bool before = reached(0.0, 0), inside = !before && reached(all_mass, all_count), none_above = above_count == 0;
            if (!inside && doubt > 0.0) {
                be_exact();
                continue;
            }
            if (before) {                 // above hi, which is below the ceiling
                lo = bottom = hi + 1;
                hi = ceiling;
                __syncthreads();
                continue;
            }
            ceiling = hi;
            above_ceiling = above;
            count_ceiling = above_count;
            if (!inside && lo > bottom) {
                hi = lo - 1;
                lo = bottom;
                __syncthreads();
                continue;
            }
            if (tid == 0) {
                s.found = 0;
                s.place = 0;
            }
            __syncthreads();
            // the first bin with anything in it that reaches it; where roundings leave none, the lowest one
#pragma unroll 1
            for (int e = 0; e < PER; ++e) {
                const int bin = top - e;
                const uint32_t n = s.count[bin];
                mass_upto += masses[bin];
                count_upto += n;
                if (n && reached(mass_upto, count_upto)) atomicMax(&s.found, (uint32_t)bin + 1);
                if (n && count_upto == all_count) s.place = bin + 1;
            }
            __syncthreads();
            const uint32_t found = inside && s.found ? s.found : s.place;
            if (found == 0) {             // nothing in [bottom, hi]: all that lies above stays
                *weight_left = above;
                return bottom == kFirst ? kEverything : Cut{bottom, 0};
            }
            const uint32_t bin = found - 1, here = s.count[bin];
            const double weighs = masses[bin];
            __syncthreads();
            // what lies above that bin
            mass = 0.0;
            count = 0;
#pragma unroll 1
            for (int e = 0; e < PER; ++e)
                if ((uint32_t)(top - e) > bin) {
                    mass += masses[top - e];
                    count += s.count[top - e];
                }
            block_scan<K>(mass, s.wave, &all_mass);
            block_scan<K>(count, s.wave_count, &all_count);
            above += all_mass;
            above_count += all_count;
            __syncthreads();
            const uint32_t from = lo;
            hi = min(hi, lo + (bin << sh) + ((1u << sh) - 1));
            lo += bin << sh;
            if (sh > kLeast) {
                if (!exact) {
                    ceiling = hi;
                    above_ceiling = above;
                    count_ceiling = above_count;
                    doubt += 0.5 * all_count / unit;
                }
                continue;
            }
            // `here` logits alike: as many of them as it takes, by the lowest tokens
            int64_t ties = here;
            if (inside) {
                if (by_weight) {
                    const double w = weighs / here;
                    auto needed = [&](double rest) {
                        return w > 0.0 ? max((int64_t)1, (int64_t)fmin(ceil(rest / w * (1 - 0x1p-50)), (double)here)) : (int64_t)here;
                    };
                    ties = needed(enough - above);
                    // one of them, or as many as there are, may stand for fewer or more
                    if (doubt > 0.0 && (enough - above <= doubt || enough - above + doubt > weighs || needed(enough - above + doubt) != needed(enough - above - doubt))) {
                        be_exact();
                        continue;
                    }
                } else {
                    ties = max((int64_t)1, min((int64_t)here, number - above_count));
                }
            }
            *weight_left = above + weighs * ((double)ties / here);
            if (kLeast > 0 && none_above) {
                // every token that stays lies in a bin: one weight each, for the sums that follow
                weights_from = from;
#pragma unroll 1
                for (int i = tid; i < kBins; i += K)
                    if (s.count[i]) masses[i] = weight(logit(from + ((uint32_t)i << kLeast)));
                __syncthreads();
            }
            return Cut{order_of(logit(lo)), (int32_t)ties};
        }
    }

    // Orders between which a share of the row's weight (or number) should end, from the
    // samples below `from`, whose tokens are known: `enough` of `all` lies below it.  Each
    // sample stands for its share of them; four standard deviations to either side.
    __device__ void guess(uint32_t from, double enough, double all, bool by_weight, uint32_t* lo, uint32_t* hi)
    {
        if (!a.samples_kept) {
            *lo = 0x00800000u;
            *hi = 0xFF7FFFFFu;
            return;
        }
        // bins of 1/32 octaves of weight below `from` (1/8 where there are few)
        constexpr double per = kBins / 64;
        const float top = value_at(from);
        for (int i = tid; i < kBins; i += K) {
            s.mass[i] = 0;
            s.count[i] = 0;
        }
        __syncthreads();
        auto bin_of = [&](float x) { return (int)fmin(a.c * ((double)top - (double)x) * per, kBins - 1.0); };
        for (int i = tid; i < parts * 64; i += K) {
            const uint32_t n = samples[i];
            if (n <= kNoteNothing || (n << 16) >= from) continue;
            const float x = value_at(n << 16);
            const int bin = bin_of(x);
            atomicAdd(&s.count[bin], 1u);
        }
        __syncthreads();
        constexpr int PER = kBins / K;
        double mass = 0.0, square = 0.0, all_mass, all_square;
        auto bin_weight = [&](int bin) { return by_weight ? power(-(double)bin / per, s.table) : 1.0; };
#pragma unroll 1
        for (int e = 0; e < PER; ++e) {
            const int bin = tid * PER + e;
            const double w = bin_weight(bin), n = s.count[bin];
            mass += n * w;
            square += n * w * w;
        }
        double upto = block_scan<K>(mass, s.wave, &all_mass) - mass;
        double upto_square = block_scan<K>(square, s.wave, &all_square) - square;
        const double target = enough / all * all_mass;
        if (tid == 0) {
            s.found = kBins;
            s.number = 0;
            s.place = kBins;
        }
        __syncthreads();
#pragma unroll 1
        for (int e = 0; e < PER; ++e) {
            const int bin = tid * PER + e;
            const double w = bin_weight(bin), n = s.count[bin];
            upto += n * w;
            upto_square += n * w * w;
            const double far = 4.0 * sqrt(upto_square) + 2.0 * w;
            if (upto + far < target) atomicMax(&s.number, bin);               // it ends behind this bin
            if (upto - far > target) atomicMin(&s.place, bin);                // it has ended
        }
        __syncthreads();
        const int first = s.number, last = s.place;
        __syncthreads();
        auto value_of_bin = [&](double bin) { return (float)((double)top - bin / per / a.c); };
        *hi = first == 0 ? from - 1 : order_of(value_of_bin(first));
        const float low = last >= kBins - 1 ? -__builtin_inff() : value_of_bin(last + 1);
        *lo = low > -3.4e38f ? order_of(low) : 0x00800000u;
        *lo = min(*lo, *hi);
    }

    // The row's sums once more, of the tokens that stay; s.ties receives the cut's ties before each block.
    __device__ double sums_of(Cut cut)
    {
        const int lane = tid & 63;
        const float above = cut.order ? value_at(cut.order) : -__builtin_inff(), edge = cut.order ? above : __builtin_nanf("");
        const bool least_matters = a.least > -__builtin_inf();
        const double* const weights = reinterpret_cast<const double*>(s.mass);
        __syncthreads();
        for (int32_t b = tid >> 6; b < blocks; b += K / 64) {
            const int64_t from = block_begin(b), to = b + 1 < blocks ? block_begin(b + 1) : (int64_t)a.vocab;
            double sum = 0.0;
            int32_t ties = 0;
            // blocks begin at whole vectors, but for those behind the row's end
            if (from < to)
                each_logit<64>(from / N, (to + N - 1) / N, to, lane, [&](float x, uint32_t) {
                    ties += x == edge;
                    if (x > above && (!least_matters || likely(x)))
                        sum += weights_from ? weights[(order_of(x) - weights_from) >> 16] : weight(x);
                });
            sum = wave_sum(sum);
            ties = wave_sum(ties);
            if (lane == 63) {
                s.sums[b] = sum;
                s.refs[b] = m;
                s.ties[b] = ties;
            }
        }
        __syncthreads();
        if (cut.order != 0) {
            uint32_t all;
            const int32_t mine = tid < blocks ? s.ties[tid] : 0;
            const int32_t before = (int32_t)block_scan<K>((uint32_t)mine, s.wave_count, &all) - mine;
            if (tid < blocks) {
                const float x = value_at(cut.order);
                const int32_t stay = max(0, min(mine, cut.ties - before));
                if (stay > 0 && likely(x)) s.sums[tid] += stay * weight(x);
                s.ties[tid] = before;
            }
            __syncthreads();
        }
        return total_of_blocks();
    }

    // Everything behind the pass over the logits.
    __device__ void finish(int64_t row, bool sums)
    {
        const float nan = __builtin_nanf("");
        const bool broken = !(m < __builtin_inff()), empty = m == -__builtin_inff();
        if (broken || empty) {
            if (tid == 0) {
                a.tokens[row] = -1;
                if (a.logp) a.logp[row] = broken ? nan : -__builtin_inff();
            }
            return;
        }
        double total = 0.0;
        if (sums) total = total_of_blocks();
        const bool filters = a.top_k > 0 || a.top_p < 1.0 || a.least > -__builtin_inf();
        if (!filters) {
            pick(total, kEverything);
        } else {
            bool done = false;
            // with min_p a bound is known
            float bound = -__builtin_inff();
            const bool known = a.least > -__builtin_inf() && !(a.top_k > 0 && a.top_p < 1.0);      // all of the first top_k count there
            if (known) {
                const double x = (double)m + a.least / a.scale * (1 + 1e-9) - 1e-30;
                if (x > -3.3e38) bound = nextafterf((float)x, -__builtin_inff());
            }
            uint32_t below = order_of(m) + 1;                   // orders from here on are known, and what they weigh
            double weighs = 0.0;
            if (a.top_k <= kParts) {
                // Each part has a token that reaches its note.  top_p alone may need few or many of them.
#pragma unroll 1
                for (int attempt = 0; attempt < 2 && !done; ++attempt) {
                    count_notes(a.top_k > 0 ? a.top_k : attempt == 0 ? kFirstParts : kParts, a.top_k > 0 && known ? 1u << 30 : kParts);
                    const int bin = s.number;
                    const uint32_t listed = s.found;
                    if (bin < 0 || (a.top_k > 0 && bin < kBins - 1 && listed < (uint32_t)a.top_k)) break;
                    // every note of these bins, and all tokens from the lowest value in them on
                    const bool all = bin == kBins - 1;
                    const float from = all ? -3.402823466e38f : least_of_bins(bin);
                    const bool bounded = all || (known && bound >= from);
                    const float least = known ? fmaxf(bound, from) : from;
                    __syncthreads();
                    const int32_t found = collect(bin, least);
                    if (found > kCandidates) break;
                    done = from_candidates(found, bounded, total, &weighs);
                    below = order_of(least);
                    if (a.top_k > 0 || all) break;
                }
            }
            if (!done) {
                Cut cut = kEverything;
                double among = total, ignored;
                uint32_t lo, hi;
                __syncthreads();
                if (a.top_k > 0) {
                    guess(order_of(m) + 1, a.top_k, a.vocab, false, &lo, &hi);
                    cut = search(lo, hi, a.top_k, 0.0, false, a.top_p < 1.0, &among);
                }
                if (a.top_p < 1.0) {
                    const double enough = a.top_p * among;
                    if (a.top_k > 0)
                        lo = cut.order ? cut.order : 0x00800000u, hi = 0xFF7FFFFFu;
                    else
                        guess(below, enough - weighs, total - weighs, true, &lo, &hi);
                    weights_from = 0;
                    cut = cut.stricter(search(lo, hi, 0, enough, true, false, &ignored));
                }
                total = sums_of(cut);
                pick(total, cut);
            } else {
                total = s.total;
            }
        }
        if (tid == 0) {
            const int32_t token = s.token;
            a.tokens[row] = token;
            if (a.logp) a.logp[row] = token < 0 ? nan : (float)(a.scale * ((double)s.value - (double)m) - log(total));
        }
    }
};

// A row of few steps, by one wave.
constexpr int kRowSteps = 4;
template <typename T, bool kSums> __global__ __launch_bounds__(64, 3) void k_sample(SampleArgs a)
{
    typedef Shared<64, kRowSteps, kRowSteps, 512> S;
    __shared__ S s;
    __shared__ alignas(16) uint16_t s_samples[kRowSteps * 64];
    const int tid = threadIdx.x;
    if (tid < 32) s.table[tid] = kTwoTo[tid];
    __syncthreads();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* const x0 = static_cast<const T*>(a.x) + row * a.stride;
        const float u = a.uniforms[row];
        const float m = read_strip<T, kSums, false, false>(a, x0, 0, nullptr, s.table, s.notes, s_samples, s.sums, s.refs);
        __syncthreads();
        RowWork<T, S, 64> work{a, s, x0, s_samples, m, a.slots, a.note_slots, tid, u};
        work.finish(row, kSums);
        __syncthreads();
    }
}

// A slice of a row: what its waves find out about their strips goes to the workspace.
constexpr int kReadThreads = 64 * kSampleWaves;
template <typename T, bool kSums, bool NT> __global__ __launch_bounds__(kReadThreads, 4) void k_sample_read(SampleArgs a)
{
    __shared__ double s_table[32], s_powers[kSums ? kPowers : 1];
    const int tid = threadIdx.x, wave = tid >> 6;
    if (kSums) {
        if (tid < 32) s_table[tid] = kTwoTo[tid];
        fill_powers<kReadThreads>(s_powers);
    }
    __syncthreads();
    const int32_t strips = a.slices * kSampleWaves;
    for (int64_t job = blockIdx.x; job < (int64_t)a.rows * a.slices; job += gridDim.x) {
        const int64_t row = job / a.slices;
        const int32_t strip = (int32_t)(job - row * a.slices) * kSampleWaves + wave;
        const int64_t at = (row * strips + strip) * a.slots, note = (row * strips + strip) * a.note_slots * 64;
        const float top = read_strip<T, kSums, NT, true>(a, static_cast<const T*>(a.x) + row * a.stride, strip, s_powers, s_table,
                                                         a.notes + note, a.samples + note, a.sums + at, a.refs + at);
        if ((tid & 63) == 0) a.most[row * strips + strip] = top;
    }
}

// The rest of such a row.
template <typename T, bool kSums, int K, int BLOCKS, int PARTS> __global__ __launch_bounds__(K, 4) void k_sample_join(SampleArgs a)
{
    typedef Shared<K, BLOCKS, PARTS, 2048> S;
    __shared__ S s;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    const int32_t strips = a.slices * kSampleWaves, blocks = strips * a.slots, parts = strips * a.note_slots;
    // at most 128 strips: two a lane
    const float* const most = a.most + row * strips;
    float m = lane < strips ? most[lane] : -__builtin_inff(), m2 = 64 + lane < strips ? most[64 + lane] : -__builtin_inff();
    const float u = a.uniforms[row];
    if (tid < 32) s.table[tid] = kTwoTo[tid];
    if (kSums && tid < blocks) {
        s.sums[tid] = a.sums[row * blocks + tid];
        s.refs[tid] = a.refs[row * blocks + tid];
    }
    if (a.notes_kept) {
        // eight notes to a load
        const V4u* const notes = reinterpret_cast<const V4u*>(a.notes + row * parts * 64);
        V4u n[PARTS * 8 / K];
#pragma unroll
        for (int v = 0; v < PARTS * 8 / K; ++v)
            if (v * K + tid < parts * 8) n[v] = notes[v * K + tid];
#pragma unroll
        for (int v = 0; v < PARTS * 8 / K; ++v)
            if (v * K + tid < parts * 8) reinterpret_cast<V4u*>(s.notes)[v * K + tid] = n[v];
    }
    m = most_of(m, m2);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = most_of(m, __shfl_xor(m, d));
    __syncthreads();
    RowWork<T, S, K> work{a, s, static_cast<const T*>(a.x) + row * a.stride, a.samples + row * parts * 64, m, blocks, parts, tid, u};
    work.finish(row, kSums);
}

constexpr double kCacheBytes = 256 << 20; // the last-level cache

template <typename T, bool kSums> hipError_t sample_as(const SampleArgs& a, hipStream_t s)
{
    if (a.slices == 0) {
        hipLaunchKernelGGL((k_sample<T, kSums>), dim3((unsigned)std::min<int64_t>(a.rows, kMaxGrid)), dim3(64), 0, s, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)a.rows * a.slices, kMaxGrid));
    if ((double)a.rows * a.vocab * sizeof(T) > kCacheBytes)
        hipLaunchKernelGGL((k_sample_read<T, kSums, true>), grid, dim3(kReadThreads), 0, s, a);
    else
        hipLaunchKernelGGL((k_sample_read<T, kSums, false>), grid, dim3(kReadThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.rows <= kFewRows)
        hipLaunchKernelGGL((k_sample_join<T, kSums, 1024, kSampleBlocks, kSampleBlocks>), dim3((unsigned)a.rows), dim3(1024), 0, s, a);
    else
        hipLaunchKernelGGL((k_sample_join<T, kSums, 256, kManyBlocks, kManyParts>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t sample_t(SampleArgs a, hipStream_t s)
{
    // the row's whole weight counts where nothing bounds it, or top_p of all of it does; its samples
    // help where many tokens may stay
    const bool filters = a.top_k > 0 || a.top_p < 1.0 || a.least > -__builtin_inf();
    a.notes_kept = filters;
    a.samples_kept = a.top_k > kParts || (a.top_p < 1.0 && a.top_k == 0);
    return !filters || (a.top_p < 1.0 && a.top_k == 0) ? sample_as<T, true>(a, s) : sample_as<T, false>(a, s);
}

}  // namespace

// How a row is cut.
SampleSplit sample_split(int32_t rows, int32_t vocab, int dtype)
{
    const int64_t step = kSampleLanes * kUnroll * (dtype == 0 ? Vec<uint16_t>::n : Vec<float>::n);
    const int64_t steps = (vocab + step - 1) / step;
    SampleSplit x = {0, 1, (int32_t)steps, 0, 0, 0, 0, 0};
    int64_t blocks = kRowSteps, parts = kRowSteps;
    if (steps > kRowSteps) {
        x.waves = kSampleWaves;
        const int64_t cut = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(32, kReadGroups / std::max(1, rows)), steps / kSampleWaves));
        x.strip_steps = (int32_t)((steps + cut * x.waves - 1) / (cut * x.waves));
        x.slices = (int32_t)((steps + (int64_t)x.strip_steps * x.waves - 1) / ((int64_t)x.strip_steps * x.waves));
        blocks = (rows <= kFewRows ? kSampleBlocks : kManyBlocks) / (x.slices * x.waves);
        parts = (rows <= kFewRows ? kSampleBlocks : kManyParts) / (x.slices * x.waves);
    }
    while ((x.slots = ((x.strip_steps - 1) >> x.shift) + 1) > blocks) ++x.shift;
    // as many parts as there is room for, rounded up to what is stored together
    for (x.note_shift = x.shift;; ++x.note_shift) {
        const int32_t n = ((x.strip_steps - 1) >> x.note_shift) + 1;
        for (x.group = 0; x.group < 3 && 1 << x.group < n; ++x.group) {}
        x.note_slots = (((n - 1) >> x.group) + 1) << x.group;
        if (x.note_slots <= parts) return x;
    }
}

hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t s)
{
    return dtype == 0 ? sample_t<uint16_t>(a, s) : sample_t<float>(a, s);
}

}  // namespace cpes
