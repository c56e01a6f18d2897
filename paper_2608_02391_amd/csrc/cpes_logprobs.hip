// cpes_logprobs.hip -- gfx950 kernels of the scores of given tokens under rows of
// logits: log probability, entropy, the most likely alternatives, and the
// gradient of the first two.
//
// Mathematics.  With z = scale x, M = max z, c = scale log2 e and t_v = c (x_v - max x) <= 0:
//   s = sum 2^(t_v) over all but the largest,  u = sum t_v 2^(t_v),
//   lse = M + ln (1 + s),  ln p_v = z_v - M - ln (1 + s),  entropy = ln (1 + s) - ln 2 u / (1 + s)
// (both terms of the entropy are positive: nothing cancels, and a near-certain
// token's numbers, of the size of s, keep their digits).  Pieces (max, s, u) of a row
// join by 2^(t of the smaller maximum), u moving by the terms times that exponent
// as well.  c rounded to fp32 is c (1 + r): to first order that adds r ln 2 u to s,
// which is taken back at the end.
//   dx_v = scale (g ([v = t] - p_v) - h p_v (ln p_v + entropy)).
//
// What bounds it: a logit is read once (and its gradient written once) for about
// six instructions, close to what the vector units do in the time its bytes take,
// so the loop holds no more than it must: one fused multiply-add for the exponent,
// the exponential, two sums, the maximum and the minimum by threes; the next step's
// loads are on their way meanwhile, and the alternatives cost a note of the step's
// maximum.  4,096 rows of 151,936 in bf16 with 5 alternatives: 201 us, 6.2 TB/s, with
// the vector units issuing in 79 % of cycles; the loop without its arithmetic takes
// 182.  The gradient of 2,000 rows of 50,257: 60 us, 6.7 TB/s read and written.
//
// Split.  A row is one workgroup's, of 64 to 256 threads by length and number of rows;
// where there are few long ones, they are cut into slices, joined by a second launch
// in slice order: one row of 151,936 with 20 alternatives in 15 us, latencies of a
// dozen trips to memory and barriers.
//
// Alternatives.  Order: value descending, then token ascending, as one 64-bit key,
// so no two are equal and the result does not depend on who writes first.  A
// thread keeps, with its running maximum, the step it first met it in, so the
// maximum's key lies between those of the step's last and first token.  Each wave
// ranks its lanes' lower ends; the least of the waves' k/4-th bounds the row's k-th
// largest key from below, and only threads whose upper end reaches that bound can
// hold a key from there on: k and a few.  Every thread notes each step's maximum in
// LDS, so of those threads only the steps that reach the bound are read again, about
// k x 64 bytes; reading all their logits again made 64 alternatives cost 180 us
// on 4,096 rows, now 10.  Rows of ties go through exact keys, and where even these
// overflow the buffer, through rounds that raise the bound.
#include <algorithm>
#include <type_traits>

#include "cpes_eval.hpp"

namespace cpes {

namespace {

typedef unsigned int V4u __attribute__((ext_vector_type(4)));
typedef V4u V4uAnywhere __attribute__((aligned(2)));
typedef unsigned long long Key;

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kFar = -1e4f;            // stands in for what is below, -inf too: its exponential is 0, and 0 times it

template <typename T> struct Vec { static constexpr int n = 16 / sizeof(T); };

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

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

// Descending value, ascending token.  0 is below every logit's key.
__device__ __forceinline__ Key key_of(float x, uint32_t token)
{
    const uint32_t u = __float_as_uint(x + 0.0f);       // -0 ties with 0
    const uint32_t v = u & 0x80000000u ? ~u : u | 0x80000000u;
    return ((Key)v << 32) | (uint32_t)~token;
}
__device__ __forceinline__ float key_value(Key k)
{
    const uint32_t v = (uint32_t)(k >> 32);
    return __uint_as_float(v & 0x80000000u ? v & 0x7FFFFFFFu : ~v);
}
__device__ __forceinline__ uint32_t key_token(Key k) { return ~(uint32_t)k; }

// Sums of a piece of a row, its largest logit's own term of 1 left out of s: a
// near-certain token's log probability is -ln (1 + s), and s may be far below the
// roundings of 1.  A piece of nothing but -inf has no such term, and s = u = 0.
struct Sums {
    float m, s, u;       // largest logit, sum 2^t of the others, sum t 2^t, with t = c (x - m)
};

__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const bool first = a.m >= b.m;
    const Sums hi = first ? a : b, lo = first ? b : a;
    const float d = lo.m == hi.m ? 0.f : fmaxf(c * (lo.m - hi.m), kFar), f = exp2_hw(d);
    const float all = lo.m == -__builtin_inff() ? lo.s : lo.s + 1.f;
    return Sums{hi.m, hi.s + f * all, hi.u + f * (lo.u + d * all)};
}

// The logit of a row's target, if it has one.
template <typename T> __device__ __forceinline__ float target_logit(const LogprobArgs& a, int64_t row, bool* valid)
{
    *valid = false;
    if (!a.logp) return 0.f;
    const int64_t v = a.targets[row];
    *valid = v >= 0 && v < a.vocab;
    return *valid ? value_of(static_cast<const T*>(a.x)[row * a.stride + v]) : 0.f;
}

// Writes a finished row's numbers; every thread gets what the alternatives need.  A
// row without a finite logit is empty, or broken if a NaN is among its logits: the
// maximum passes NaNs over, the sum does not.
__device__ __forceinline__ void finish(const LogprobArgs& a, int64_t row, Sums t, float target, bool valid, float* logsum,
                                       bool* broken)
{
    const float nan = __builtin_nanf("");
    const bool empty = t.m == -__builtin_inff();
    *broken = !(t.s >= 0.f) || t.m == __builtin_inff();
    t.s -= a.excess * t.u;
    *logsum = *broken ? nan : empty ? 0.f : log1pf(t.s);
    if (threadIdx.x != 0) return;
    if (a.logp) a.logp[row] = !valid ? 0.f : *broken ? nan : empty ? -__builtin_inff() : a.scale * (target - t.m) - *logsum;
    if (a.entropy) a.entropy[row] = *broken ? nan : empty ? 0.f : *logsum - t.u / (1.f + t.s) * kLn2;
    if (a.lse) a.lse[row] = *broken ? nan : a.scale * t.m + *logsum;
    if (a.stats) {
        a.stats[2 * row] = t.m;
        a.stats[2 * row + 1] = *logsum;
    }
}

// The alternative of rank j.
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t row, int j, Key k, float m, float logsum, bool broken)
{
    float x = -__builtin_inff();
    int64_t id = -1;
    if (broken) {
        x = __builtin_nanf("");
    } else if (k) {
        id = key_token(k);
        if (m != -__builtin_inff()) x = a.scale * (key_value(k) - m) - logsum;
    }
    a.top_logp[row * a.top + j] = x;
    a.top_ids[row * a.top + j] = id;
}

// How many of the n keys in LDS are larger than x: eight loads at a time are on
// their way.  Behind the n keys there is room, and 0, up to a multiple of eight.
__device__ __forceinline__ int larger(const Key* keys, int n, Key x)
{
    int place = 0;
    for (int j = 0; j < n; j += 8)
#pragma unroll
        for (int e = 0; e < 8; ++e) place += keys[j + e] > x;
    return place;
}

// 0 behind the n keys, up to a multiple of eight.
__device__ __forceinline__ void pad(Key* keys, int n)
{
    if (threadIdx.x < 8 && (n & 7) && (int)threadIdx.x >= (n & 7)) keys[(n & ~7) + threadIdx.x] = 0;
}

// The k largest of the n keys in LDS, descending, into best (0 where there are
// fewer): each key's place is the number of larger ones.  All threads; the keys
// are distinct.
template <int K> __device__ void largest(Key* keys, int n, int k, Key* best)
{
    for (int i = threadIdx.x; i < k; i += K) best[i] = 0;
    pad(keys, n);
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += K) {
        const Key x = keys[i];
        const int place = larger(keys, n, x);
        if (place < k) best[place] = x;
    }
    __syncthreads();
}

constexpr int kUnroll = 4;                // 16-byte loads of a thread and step
constexpr int kMaxTop = 64;
constexpr int kNoted = 32;                // maxima a thread notes: of a step each, or of 2, 4, .. steps of longer rows
constexpr int kItems = 512;               // of them whose steps are looked at again
// Threads that look at a vector each while candidates may have to be thinned out, and
// candidates' room: they can add 8 each to 256.  64 threads have less, so that sixteen
// such workgroups fit a CU.
template <int K> constexpr int kRound = K == 64 ? 32 : 64;
template <int K> constexpr int kCandidates = 256 + 8 * kRound<K>;
constexpr int kManyOwners = 3 * kMaxTop / 2;
constexpr float kHuge = 1e30f;
constexpr float kDominated = 1.f / 16;    // sum of the other logits' terms below which the largest one's thread is looked at again

// A thread's sums while it reads.  Exponents are one fused multiply-add, c x - b
// with b = c m rounded; what b lost is put right when the thread is done.  Where
// b does not fit (nothing but -inf so far, or the type's lowest value) they are
// c (x - m).
struct Running {
    float m, b, s, u;

    __device__ __forceinline__ bool far() const { return !(fabsf(b) < kHuge); }

    __device__ __forceinline__ void rise(float top, float c)
    {
        const float next = top * c;
        const float d = s == 0.f ? 0.f : fmaxf(far() || !(fabsf(next) < kHuge) ? c * (m - top) : b - next, kFar);
        const float f = exp2_hw(d);
        u = f * (u + d * s);
        s *= f;
        m = top;
        b = next;
    }

    // Adds N logits; true if one is a new maximum.  *most receives their own.
    template <int N> __device__ __forceinline__ bool take(const float* x, float c, float* most)
    {
        float top = x[0], least = x[0];
#pragma unroll
        for (int j = 1; j < N; ++j) {
            top = fmaxf(top, x[j]);
            least = fminf(least, x[j]);
        }
        const bool rises = top > m;
        *most = top;
        if (rises) rise(top, c);
        // 0 times an exponent of -inf is no number: such steps bound it
        if (__all(!far() && fmaf(least, c, -b) > -kHuge)) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = fmaf(x[j], c, -b), e = exp2_hw(t);
                s += e;
                u = fmaf(e, t, u);
            }
        } else {
            const float base = m == -__builtin_inff() ? 0.f : m;
            const bool apart = far();
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float t = apart ? c * (x[j] - base) : fmaf(x[j], c, -b), e = exp2_hw(t);
                s += e;
                u = fmaf(e, fmaxf(t, kFar), u);
            }
        }
        return rises;
    }

    __device__ __forceinline__ Sums done(float c) const
    {
        if (m == -__builtin_inff()) return Sums{m, s, 0.f};
        const float lost = far() ? 0.f : fmaf(m, c, -b), f = exp2_hw(-lost), rest = f * s - 1.f;
        return Sums{m, rest < 0.f ? 0.f : rest, f * (u - lost * s)};
    }
};

// The least bf16 not below x.
__device__ __forceinline__ uint16_t bf16_above(float x)
{
    const uint32_t u = __float_as_uint(x);
    return (uint16_t)((u & 0x80000000u ? u : u + 0xFFFFu) >> 16);
}

// The key that at least `top` threads' maxima reach, and the threads that may hold
// a key from there on, in s_owner; their number is returned.  low and high bound
// the key of this thread's maximum (0: no logits).  Each wave ranks its own lanes;
// the least of the waves' (top / waves)-th keys is reached by `top` of them.  All
// threads.
template <int K> __device__ int bound_by_waves(Key low, Key high, int top, Key* s_wave, int32_t* s_owner, int32_t* s_owners, Key* least)
{
    constexpr int kWaves = K / 64;
    const int each = (top + kWaves - 1) / kWaves;
    int place = 0;
#pragma unroll 8
    for (int j = 0; j < 64; ++j) {
        const Key other = ((Key)(uint32_t)__builtin_amdgcn_readlane((int)(low >> 32), j) << 32) |
                          (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)low, j);
        place += other > low;
    }
    if (threadIdx.x == 0) *s_owners = 0;
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = 0;
    __syncthreads();
    if (low && place == each - 1) s_wave[threadIdx.x >> 6] = low;
    __syncthreads();
    Key bound = s_wave[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) bound = min(bound, s_wave[w]);
    *least = max(bound, (Key)1);          // fewer logits than that: all of them
    if (high >= *least) s_owner[atomicAdd(s_owners, 1)] = threadIdx.x;
    __syncthreads();
    return *s_owners;
}

// The same exactly, from the exact keys of all threads' maxima: `top` owners, or all.
template <int K> __device__ int bound_exactly(Key key, int top, Key* s_keys, int32_t* s_owner, int32_t* s_owners, Key* least)
{
    s_keys[threadIdx.x] = key;
    if (threadIdx.x == 0) *s_owners = 0;
    __syncthreads();
    const int place = larger(s_keys, K, key);
    const bool mine = key && place < top;
    if (mine) s_owner[place] = threadIdx.x;
    if (mine) atomicAdd(s_owners, 1);
    __syncthreads();
    const int owners = *s_owners;
    *least = owners == top ? s_keys[s_owner[top - 1]] : 1;
    __syncthreads();
    return owners;
}

// One slice of one row.  NT: the logits exceed the last-level cache, and are read
// past the caches (622 million of bf16: 233 -> 206 us with 5 alternatives).
template <typename T, bool NT, int K>
__global__ __launch_bounds__(K, K == 64 ? 3 : 5) void k_logprobs(LogprobArgs a)
{
    constexpr int N = Vec<T>::n;
    __shared__ Sums s_sums[K / 64];
    __shared__ Key s_keys[kCandidates<K>], s_best[kMaxTop], s_wave[K / 64];
    __shared__ int32_t s_owner[K], s_count, s_owners, s_items;
    __shared__ uint16_t s_most[kNoted][K], s_item[kItems];
    const int tid = threadIdx.x;
    for (int64_t job = blockIdx.x; job < (int64_t)a.rows * a.slices; job += gridDim.x) {
        const int64_t row = job / a.slices;
        const int32_t slice = (int32_t)(job - row * a.slices);
        const int64_t begin = (int64_t)slice * a.per_slice;
        const int32_t len = (int32_t)min((int64_t)a.per_slice, a.vocab - begin);
        const T* const x0 = static_cast<const T*>(a.x) + row * a.stride + begin;
        const int32_t full = len / N, vecs = (len + N - 1) / N, steps = (vecs + kUnroll * K - 1) / (kUnroll * K);

        const int32_t whole = full / (kUnroll * K);

        // Vector i as floats; -inf behind the slice's end.
        auto floats_at = [&](int32_t i, float* x) {
            if (i < full) {
                unpack<T>(*reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)i * N), x);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    x[j] = -__builtin_inff();
                    if (i < vecs && i * N + j < len) x[j] = value_of(x0[(int64_t)i * N + j]);
                }
            }
        };

        bool valid = false;
        float target = 0.f;
        if (a.slices == 1 && tid == 0) target = target_logit<T>(a, row, &valid);
        Running run = {-__builtin_inff(), -__builtin_inff(), 0.f, 0.f};
        int32_t met = 0;                  // the step the maximum was first met in
        int32_t shift = 0;                // steps of a note
        while ((steps - 1) >> shift >= kNoted) ++shift;
        float most, noted = -__builtin_inff();
        auto note = [&](int32_t step, float x) {
            noted = step & ((1 << shift) - 1) ? fmaxf(noted, x) : x;
            s_most[step >> shift][tid] = bf16_above(noted);
        };
        V4u w[kUnroll];                   // the next step's, on their way while one is added
        auto load = [&](int32_t step) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const V4uAnywhere* const q =
                    reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)((step * kUnroll + u) * K + tid) * N);
                w[u] = NT ? __builtin_nontemporal_load(q) : *q;
            }
        };
        if (whole > 0) load(0);
        for (int32_t step = 0; step < whole; ++step) {
            float x[kUnroll * N];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) unpack<T>(w[u], x + u * N);
            if (step + 1 < whole) load(step + 1);
            if (run.take<kUnroll * N>(x, a.c, &most)) met = step;
            if (a.top > 0) note(step, most);
        }
        if (whole < steps) {
            float all = -__builtin_inff();
            int32_t i = whole * kUnroll * K + tid;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u)
                if (i + u * K < full) w[u] = *reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)(i + u * K) * N);
#pragma unroll 1
            for (int u = 0; u < kUnroll; ++u, i += K) {
                float x[N];
                if (i < full)
                    unpack<T>(w[0], x);
                else
                    floats_at(i, x);
                if (run.take<N>(x, a.c, &most)) met = whole;
                all = fmaxf(all, most);
#pragma unroll
                for (int v = 1; v < kUnroll; ++v) w[v - 1] = w[v];
            }
            if (a.top > 0) note(whole, all);
        }
        // the threads' sums join, in a fixed order
        Sums mine = run.done(a.c);
        auto joined = [&]() {
            Sums t = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1)
                t = join(t, Sums{__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.u, d)}, a.c);
            if ((tid & 63) == 0) s_sums[tid >> 6] = t;
            __syncthreads();
            t = s_sums[0];
#pragma unroll
            for (int v = 1; v < K / 64; ++v) t = join(t, s_sums[v], a.c);
            return t;
        };
        if (tid == 0) {
            s_count = s_items = 0;
            s_owner[0] = K;
        }
        Sums t = joined();
        if (t.s < kDominated && t.m > -__builtin_inff()) {
            // One logit dominates, and its thread's other terms have been rounded beside its 1: that thread's
            // logits again, all threads together, without it.
            if (run.m == t.m) atomicMin(&s_owner[0], tid);
            __syncthreads();
            const int32_t owner = s_owner[0];
            if (tid == owner) mine.s = mine.u = 0.f;
            Sums own = {t.m, 0.f, 0.f};
            for (int32_t i = tid * K + owner; i < vecs; i += K * K) {
                float x[N];
                floats_at(i, x);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float d = fmaxf(a.c * (x[j] - t.m), kFar), e = x[j] == t.m ? 0.f : exp2_hw(d);
                    own.s += e;
                    own.u += d * e;
                }
            }
            // the 1 of the largest stands in `mine`; these have none
            if (mine.m == t.m) {
                mine.s += own.s;
                mine.u += own.u;
            } else {
                const float d = fmaxf(a.c * (mine.m - t.m), kFar), f = exp2_hw(d), all = mine.m == -__builtin_inff() ? 0.f : mine.s + 1.f;
                mine = Sums{t.m, f * all + own.s, f * (mine.u + d * all) + own.u};
            }
            // now every thread's piece is relative to the largest, and they add up
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                mine.s += __shfl_xor(mine.s, d);
                mine.u += __shfl_xor(mine.u, d);
            }
            if ((tid & 63) == 0) s_sums[tid >> 6] = mine;
            __syncthreads();
            t.s = t.u = 0.f;
#pragma unroll
            for (int v = 0; v < K / 64; ++v) {
                t.s += s_sums[v].s;
                t.u += s_sums[v].u;
            }
        }
        float logsum = 0.f;
        bool broken = false;
        if (a.slices == 1)
            finish(a, row, t, target, valid, &logsum, &broken);
        else if (tid == 0)
            a.parts[job] = float4{t.m, t.s, t.u, 0.f};

        if (a.top > 0) {
            const int32_t first = met * kUnroll * K + tid;             // vectors of the step
            auto token = [&](int32_t i, int j) { return (uint32_t)(begin + (int64_t)i * N + j); };
            Key low = 0, high = 0, least;
            if (tid < vecs) {
                low = key_of(run.m, token(first + (kUnroll - 1) * K, N - 1));
                high = key_of(run.m, token(first, 0));
            }
            int owners = bound_by_waves<K>(low, high, a.top, s_wave, s_owner, &s_owners, &least);
            if (owners > kManyOwners) {
                // many maxima tie: find where each was met
                Key exact = 0;
                if (tid < vecs)
                    for (int u = kUnroll - 1; u >= 0; --u) {
                        float x[N];
                        floats_at(first + u * K, x);
#pragma unroll
                        for (int j = N - 1; j >= 0; --j)
                            if (x[j] == run.m && (first + u * K) * N + j < len)
                                exact = key_of(run.m, token(first + u * K, j));
                    }
                __syncthreads();
                owners = bound_exactly<K>(exact, a.top, s_keys, s_owner, &s_owners, &least);
            }
            // the owners' logits from the bound on
            auto collect = [&](const float* x, int32_t i) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Key k = key_of(x[j], token(i, j));
                    if (k >= least && i * N + j < len) {
                        const int at = atomicAdd(&s_count, 1);
                        if (at < kCandidates<K>) s_keys[at] = k;
                    }
                }
            };
            // only the steps of theirs whose notes reach the bound
            if (high >= least)
                for (int32_t at = 0; at <= (steps - 1) >> shift; ++at)
                    if (value_of(s_most[at][tid]) >= key_value(least) || least == 1) {
                        const int item = atomicAdd(&s_items, 1);
                        if (item < kItems) s_item[item] = (uint16_t)(at * K + tid);
                    }
            __syncthreads();
            const int noted_items = s_items, vectors = kUnroll << shift;
            bool whole_owners = noted_items > kItems;
            if (!whole_owners) {
                for (int at = tid; at < noted_items * vectors; at += K) {
                    const int32_t item = at / vectors, x = s_item[item];
                    const int32_t i = (x / K * vectors + at - item * vectors) * K + x % K;
                    if (i < vecs) {
                        float v[N];
                        floats_at(i, v);
                        collect(v, i);
                    }
                }
                __syncthreads();
                whole_owners = s_count > kCandidates<K>;
            }
            int n = s_count;
            if (whole_owners) {
                // more than there is room for: all of theirs, a round at a time, with the bound raised by what is there
                __syncthreads();
                if (tid == 0) s_count = 0;
                __syncthreads();
                const int32_t per = steps * kUnroll, items = owners * per;
                for (int32_t item0 = 0; item0 < items; item0 += kRound<K>) {
                    const int had = s_count;
                    __syncthreads();      // read by all before any candidate is added
                    if (had > kCandidates<K> - 8 * kRound<K>) {
                        largest<K>(s_keys, had, a.top, s_best);
                        if (tid < a.top) s_keys[tid] = s_best[tid];
                        if (tid == 0) s_count = a.top;
                        least = s_best[a.top - 1];
                        __syncthreads();
                    }
                    const int32_t item = item0 + tid, o = item / per;
                    if (tid < kRound<K> && item < items) {
                        const int32_t i = (item - o * per) * K + s_owner[o];
                        if (i < vecs) {
                            float x[N];
                            floats_at(i, x);
                            collect(x, i);
                        }
                    }
                    __syncthreads();
                }
                n = s_count;
            }
            largest<K>(s_keys, n, a.top, s_best);
            if (tid < a.top) {
                if (a.slices == 1)
                    write_top(a, row, tid, s_best[tid], t.m, logsum, broken);
                else
                    a.keys[job * a.top + tid] = s_best[tid];
            }
        }
        __syncthreads();                  // shared memory is free for the next row
    }
}

// Joins the slices of a row.
constexpr int kJoinKeys = kMaxSlices * kMaxTop;
// Keys from the bound on: k of the lists' first few, and behind them only in lists whose
// few, at least two, all are among these.
constexpr int kJoinCandidates = kMaxTop + kMaxTop / 2 * kMaxTop;

template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprobs_join(LogprobArgs a)
{
    __shared__ Key s_all[kJoinKeys], s_keys[kJoinCandidates], s_best[kMaxTop], s_least;
    __shared__ int32_t s_count;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    float4 p = {-__builtin_inff(), 0.f, 0.f, 0.f};
    if (lane < a.slices) p = a.parts[row * a.slices + lane];
    const Key* const keys = a.keys + row * a.slices * a.top;
    for (int i = tid; i < a.slices * a.top; i += kThreads) s_all[i] = keys[i];
    bool valid;
    const float target = target_logit<T>(a, row, &valid);
    Sums t = Sums{p.x, p.y, p.z};
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        t = join(t, Sums{__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.u, d)}, a.c);
    t = Sums{__shfl(t.m, 0), __shfl(t.s, 0), __shfl(t.u, 0)};
    float logsum;
    bool broken;
    finish(a, row, t, target, valid, &logsum, &broken);
    if (a.top == 0) return;
    // the k-th largest of the slices' first few keys, twice as many as k, bounds what can be among the row's k largest
    const int few = min(a.top, 2 * ((a.top + a.slices - 1) / a.slices)), heads = a.slices * few;
    if (tid == 0) {
        s_count = 0;
        s_least = 1;
    }
    __syncthreads();
    for (int i = tid; i < heads; i += kThreads) s_keys[i] = s_all[i / few * a.top + i % few];
    pad(s_keys, heads);
    __syncthreads();
    for (int i = tid; i < heads; i += kThreads) {
        const Key head = s_keys[i];
        if (head && larger(s_keys, heads, head) == a.top - 1) s_least = head;
    }
    __syncthreads();
    const Key least = s_least;
    for (int i = tid; i < a.slices * a.top; i += kThreads)
        if (s_all[i] >= least) s_keys[atomicAdd(&s_count, 1)] = s_all[i];
    __syncthreads();
    largest<kThreads>(s_keys, s_count, a.top, s_best);
    if (tid < a.top) write_top(a, row, tid, s_best[tid], t.m, logsum, broken);
}

// --------------------------------------------------------------- gradient --
constexpr int64_t kMaxGrid = 1 << 20;     // workgroups per launch; larger jobs loop
constexpr double kCacheBytes = 256 << 20; // the last-level cache
constexpr int64_t kSliceBytes = kUnroll * kThreads * 16;      // one step of all threads

template <typename T> __device__ __forceinline__ V4u pack(const float* x);
template <> __device__ __forceinline__ V4u pack<float>(const float* x)
{
    V4u w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
    return w;
}
template <> __device__ __forceinline__ V4u pack<uint16_t>(const float* x)
{
    typedef __bf16 V8bf __attribute__((ext_vector_type(8)));
    V8bf h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (__bf16)x[i];
    return __builtin_bit_cast(V4u, h);
}

// Large gradients are written past the caches, and logits that exceed them read so
// too, four vectors a thread then (622 million of bf16: 444 -> 402 us); logits that
// the forward call has left in the caches are read from there (100 million: 72 ->
// 60 us with the stores alone).
template <typename T, bool kFarLoad, bool kFarStore>
__global__ __launch_bounds__(kThreads) void k_logprobs_backward(LogprobGradArgs a)
{
    constexpr int kGradUnroll = kFarLoad ? 4 : 2;
    constexpr int N = Vec<T>::n;
    const int32_t full = a.vocab / N, vecs = full + (a.vocab % N != 0);      // any vocabulary the argument holds
    const int64_t chunks = (vecs + kGradUnroll * kThreads - 1) / (kGradUnroll * kThreads);
    for (int64_t job = blockIdx.x; job < (int64_t)a.rows * chunks; job += gridDim.x) {
        const int64_t row = job / chunks;
        const int32_t i0 = (int32_t)(job - row * chunks) * kGradUnroll * kThreads + threadIdx.x;
        const T* const x0 = static_cast<const T*>(a.x) + row * a.stride;
        T* const d0 = static_cast<T*>(a.dx) + row * a.dx_stride;
        const float m = a.stats[2 * row], logsum = a.stats[2 * row + 1];
        const float g = a.d_logp ? a.scale * a.d_logp[row] : 0.f, h = a.d_entropy ? a.scale * a.d_entropy[row] : 0.f;
        const float entropy = a.d_entropy ? a.entropy[row] : 0.f;
        int64_t target = -1;
        if (a.d_logp) target = a.targets[row];
        const bool valid = target >= 0 && target < a.vocab;
        const float gp = valid ? g : 0.f;
        const bool empty = m == -__builtin_inff() && logsum == 0.f;
        auto gradient = [&](float x, int64_t v) {
            const float logp = a.scale * (x - m) - logsum, p = exp2_hw(logp * kLog2e);
            // p = 0: no gradient, whatever ln p is
            float d = p == 0.f || empty ? 0.f : -p * (gp + h * (logp + entropy));
            // g (1 - p) without the difference, which a near-certain target would lose
            if (v == target && !empty) d = (p == 0.f ? 0.f : -p * h * (logp + entropy)) - gp * expm1f(logp);
            return d;
        };
        V4u w[kGradUnroll];
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u)
            if (i0 + u * kThreads < full) {
                const V4uAnywhere* const q = reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)(i0 + u * kThreads) * N);
                w[u] = kFarLoad ? __builtin_nontemporal_load(q) : *q;
            }
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) {
            const int32_t i = i0 + u * kThreads;
            if (i < full) {
                float x[N];
                unpack<T>(w[u], x);
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = gradient(x[j], (int64_t)i * N + j);
                V4uAnywhere* const q = reinterpret_cast<V4uAnywhere*>(d0 + (int64_t)i * N);
                if (kFarStore)
                    __builtin_nontemporal_store(pack<T>(x), q);
                else
                    *q = pack<T>(x);
            } else if (i < vecs) {
                for (int64_t v = (int64_t)i * N; v < a.vocab; ++v) {
                    const float d = gradient(value_of(x0[v]), v);
                    if constexpr (std::is_same<T, float>::value)
                        d0[v] = d;
                    else
                        d0[v] = __builtin_bit_cast(uint16_t, (__bf16)d);
                }
            }
        }
    }
}

template <typename T, int K>
void logprobs_as(const LogprobArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)std::min((int64_t)a.rows * a.slices, kMaxGrid)), block(K);
    if ((double)a.rows * a.vocab * sizeof(T) > kCacheBytes)
        hipLaunchKernelGGL((k_logprobs<T, true, K>), grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_logprobs<T, false, K>), grid, block, 0, s, a);
}

// Threads of a row (or slice).  Few rows: as many as have a few vectors each.  More: so
// few that they all run at once, sixteen to a CU by 64 threads, while their starts
// and ends count; longer ones only where the logits exceed the last-level cache.  us by
// 64, 128, 256 threads, 20 alternatives:
//   8,192 rows of 1,000       28    46   114      8,192 rows of 32,768    106   117   124
//   2,000 rows of 24,000      27    28    35      4,096 rows of 100,000   144   161   153
//   1,000 rows of 12,000      17    16    18      5,000 rows of 100,000   195   192   184
//     300 rows of 12,000      14    13    14      1,300 rows of 151,936    97    89    83
// The range between, where the logits fit the cache, by the same three, of logits that
// are there and of others:
//   rows of 50,257             2,000                          1,000
//   20 alternatives       44  49  52    56  57  59       30  28  33    33  31  34
//   none                  35  41  40    47  48  49       21  21  25    25  24  27
//   and the gradient     102 105 100   114 119 112       62  57  57    68  69  68
// 256 threads, which the rule takes there, are 1 % faster where a gradient follows and
// 5 to 20 % slower for scores alone; it does not tell the two apart.  For many
// alternatives 64 maxima bound too little (64 of 2,000 rows of 12,000: 112, 29, 38).
int logprob_threads(int64_t jobs, int64_t bytes, int top)
{
    constexpr int64_t kCUs = 256;
    const bool far = (double)jobs * bytes > kCacheBytes;
    int64_t by64 = 48 << 10, by128 = 48 << 10;           // the longest
    if (jobs <= 2 * kCUs)
        by64 = 4 << 10, by128 = 12 << 10;
    else if (jobs <= 4 * kCUs)
        by64 = 16 << 10;
    else if (far && jobs >= 6 * kCUs)
        by64 = jobs <= 16 * kCUs ? 200 << 10 : 64 << 10;
    if (top > 40) by64 = 1 << 10;
    return bytes <= by64 ? 64 : bytes <= by128 ? 128 : 256;
}

template <typename T>
hipError_t logprobs_t(const LogprobArgs& a, hipStream_t s)
{
    switch (logprob_threads((int64_t)a.rows * a.slices, (int64_t)a.per_slice * sizeof(T), a.top)) {
    case 64: logprobs_as<T, 64>(a, s); break;
    case 128: logprobs_as<T, 128>(a, s); break;
    default: logprobs_as<T, 256>(a, s); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.slices == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T, bool kFarLoad, bool kFarStore>
void backward_as(const LogprobGradArgs& a, hipStream_t s)
{
    const int64_t per = (int64_t)(kFarLoad ? 4 : 2) * kThreads * Vec<T>::n, jobs = a.rows * ((a.vocab + per - 1) / per);
    hipLaunchKernelGGL((k_logprobs_backward<T, kFarLoad, kFarStore>), dim3((unsigned)std::min(jobs, kMaxGrid)),
                       dim3(kThreads), 0, s, a);
}

template <typename T>
hipError_t backward_t(const LogprobGradArgs& a, hipStream_t s)
{
    const double bytes = (double)a.rows * a.vocab * sizeof(T);
    if (bytes > kCacheBytes)
        backward_as<T, true, true>(a, s);
    else if (2 * bytes > kCacheBytes)
        backward_as<T, false, true>(a, s);
    else
        backward_as<T, false, false>(a, s);
    return hipGetLastError();
}

}  // namespace

// Slices of a row.  A second launch and its join cost 4 to 6 us, so only long rows
// that leave CUs idle are cut, into two workgroups a CU at most and not below a
// step of all threads: 100 rows of 151,936 12 us (17 whole, 17 in six workgroups a CU),
// one row 8 (20 whole); 200 rows of 50,257 9.5 whole and 12.5 in two, 48 of 32,768 6.3 and 9.
int logprob_slices(int32_t rows, int32_t vocab, int dtype, int32_t* per_slice)
{
    const int n = dtype == 0 ? Vec<uint16_t>::n : Vec<float>::n;
    const int64_t bytes = (int64_t)vocab * 16 / n;
    int64_t slices = 1;
    if (rows > 0 && rows <= kMaxSlicedRows && bytes >= 8 * kSliceBytes)
        slices = std::min<int64_t>(std::min<int64_t>(kMaxSlices, 512 / rows), bytes / kSliceBytes);
    const int64_t per = ((vocab + slices - 1) / slices + n - 1) / n * n;
    *per_slice = (int32_t)std::min<int64_t>(per, INT32_MAX / n * n);
    return (int)((vocab + per - 1) / per);
}

hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t s)
{
    return dtype == 0 ? logprobs_t<uint16_t>(a, s) : logprobs_t<float>(a, s);
}

hipError_t launch_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t s)
{
    return dtype == 0 ? backward_t<uint16_t>(a, s) : backward_t<float>(a, s);
}

}  // namespace cpes
