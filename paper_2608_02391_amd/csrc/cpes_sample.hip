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
// therefore 64-bit, of 40 bits and more (2^t from a table of 32 and a polynomial of degree 4),
// and so are their sums, always taken in one order.
//
// Split.  A row is cut into strips, one a wave, and these into blocks of 2^shift steps; a
// step is four 16-byte vectors of each lane, in token order.  The one pass over the
// logits leaves for each block its sum (where a sum over the whole row is needed: no
// filter, or top_p of everything) and for each of its lanes the maximum of what it has
// read.  What is behind that looks at little again:
//   no filter:  the block in which u sum w lies, and in it the token;
//   filters:    the tokens from a bound on that the lanes' maxima give: the k-th largest of
//               them is reached by k tokens.  They are ranked, and what stays of them is known.
//   Only where that is too much (flat rows, thousands of tokens in top_p) is the row read
//   again, a few times: the bounding key is found by its digits, from histograms of weights.
// A workgroup does a row; where there are few long rows, several read one, and a second
// launch does the rest.
#include <algorithm>
#include <type_traits>

#include "cpes_eval.hpp"

namespace cpes {

namespace {

typedef unsigned int V4u __attribute__((ext_vector_type(4)));
typedef V4u V4uAnywhere __attribute__((aligned(2)));
typedef unsigned long long Key;

constexpr int kWaves = 4;                 // of a reading workgroup, a strip each
constexpr int kUnroll = 4;                // vectors of a lane and step
constexpr int kCandidates = 512;          // tokens that are ranked
constexpr int kDigit = 11;                // bits of a key that one reading settles
constexpr int kBins = 1 << kDigit;
constexpr int64_t kMaxGrid = 1 << 20;
constexpr double kExact = 2048.0;         // c x up to which the rounding of c max x, 2^-42, is let through
constexpr double kFar = -900.0;           // weights below 2^kFar of the largest count as 0

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

// Vector i of a row as floats; -inf behind the row's end.
template <typename T> __device__ __forceinline__ void floats_at(const T* x0, int32_t vocab, int64_t i, float* x)
{
    constexpr int N = Vec<T>::n;
    if ((i + 1) * N <= vocab) {
        unpack<T>(*reinterpret_cast<const V4uAnywhere*>(x0 + i * N), x);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = i * N + j < vocab ? value_of(x0[i * N + j]) : -__builtin_inff();
    }
}

__device__ __forceinline__ int32_t blocks_of_strip(const SampleArgs& a)
{
    return ((a.strip_steps - 1) >> a.shift) + 1;
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}

// One strip, by a wave: notes, sums and what they are relative to, of its blocks; the
// strip's maximum is returned to all lanes.
template <typename T, bool kSums>
__device__ float read_strip(const SampleArgs& a, const T* x0, int32_t strip, const double* table, uint16_t* notes, double* sums,
                            float* refs)
{
    constexpr int N = Vec<T>::n, M = kUnroll * N;
    const int lane = threadIdx.x & 63;
    const Strip<T> s(a, strip);
    const int32_t blocks = blocks_of_strip(a), per = 1 << a.shift;
    const int32_t whole = (int32_t)max((int64_t)0, min((int64_t)s.steps, ((int64_t)a.vocab / N - s.first) / (kSampleLanes * kUnroll)));
    float most = -__builtin_inff(), ref = -__builtin_inff(), noted = -__builtin_inff();
    double sum = 0.0, base = 0.0;
    // exponents up to 64 above what they are relative to are let through
    const float room = (float)fmin(64.0 / a.c, 1e38);
    V4u w[kUnroll];
    auto load = [&](int32_t step) {
        const T* const q = x0 + (s.first + (int64_t)step * (kSampleLanes * kUnroll) + lane) * N;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) w[u] = *reinterpret_cast<const V4uAnywhere*>(q + u * kSampleLanes * N);
    };
    auto take = [&](const float* x) {
        float top = x[0];
#pragma unroll
        for (int j = 1; j < M; ++j) top = most_of(top, x[j]);
        most = most_of(most, top);
        noted = most_of(noted, top);
        if constexpr (kSums) {
            if (__any(top > ref + room)) {
                // a new base for all lanes; the block's sum so far moves to it
                float high = top > -__builtin_inff() ? top : -__builtin_inff();
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) high = fmaxf(high, __shfl_xor(high, d));
                if (high < __builtin_inff()) {
                    if (ref > -__builtin_inff()) sum *= power(fmax(a.c * ((double)ref - (double)high), kFar), table);
                    ref = high;
                    base = a.c * (double)ref;
                }
            }
            if (fabs(base) <= kExact) {
                if (ref > -__builtin_inff()) {
#pragma unroll
                    for (int j = 0; j < M; ++j) sum += power(fmax(fma((double)x[j], a.c, -base), kFar - 100.0), table);
                }
            } else {
#pragma unroll
                for (int j = 0; j < M; ++j) sum += power(fmax(((double)x[j] - (double)ref) * a.c, kFar - 100.0), table);
            }
        }
    };
    auto end_block = [&](int32_t step) {
        const int32_t b = step >> a.shift;
        notes[b * 64 + lane] = note_of(noted);
        noted = -__builtin_inff();
        if constexpr (kSums) {
            const double all = wave_sum(sum);
            if (lane == 0) {
                sums[b] = all < 0x1p-900 ? 0.0 : all;           // nothing but -inf, each of which has added 2^-1000
                refs[b] = ref;
            }
            sum = 0.0;
        }
    };
    if (whole > 0) load(0);
    for (int32_t step = 0; step < whole; ++step) {
        float x[M];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) unpack<T>(w[u], x + u * N);
        if (step + 1 < whole) load(step + 1);
        take(x);
        if ((step & (per - 1)) == per - 1 || step + 1 == s.steps) end_block(step);
    }
    if (whole < s.steps) {
        float x[M];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            floats_at(x0, a.vocab, s.first + (int64_t)whole * (kSampleLanes * kUnroll) + u * kSampleLanes + lane, x + u * N);
        take(x);
        end_block(whole);
    }
    for (int32_t b = s.steps == 0 ? 0 : ((s.steps - 1) >> a.shift) + 1; b < blocks; ++b) {
        notes[b * 64 + lane] = kNoteNothing;
        if (kSums && lane == 0) {
            sums[b] = 0.0;
            refs[b] = -__builtin_inff();
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = most_of(most, __shfl_xor(most, d));
    return most;
}

// What the rest of a row's work keeps in LDS.
template <int K, int BLOCKS> struct Shared {
    uint16_t notes[BLOCKS * 64];
    double sums[BLOCKS];
    float refs[BLOCKS];
    float most[BLOCKS];                   // of strips
    double table[32];
    double wave[K / 64];
    Key wave_mass[K / 64];
    uint32_t wave_count[K / 64];
    union {
        struct {
            Key keys[kCandidates], ranked[kCandidates];
            double weights[kCandidates];
        };
        struct {
            Key mass[kBins];              // of a digit's tokens, in units of 2^-units
            uint32_t count[kBins];
        };
    };
    uint32_t bins[256];
    int32_t number, place, token;
    uint32_t found;
    double rest, total;
    Key bound;
};

// Sum over the workgroup's threads up to and including each; *total receives all.
template <int K, typename X> __device__ X block_scan(X x, X* wave, X* total)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    X y = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const X z = __shfl_up(y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();
    if (lane == 63) wave[w] = y;
    __syncthreads();
    X before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < K / 64; ++i) {
        if (i < w) before += wave[i];
        all += wave[i];
    }
    *total = all;
    return before + y;
}

template <typename T, int K, int BLOCKS> struct RowWork {
    typedef Shared<K, BLOCKS> S;
    static constexpr int N = Vec<T>::n;
    const SampleArgs& a;
    S& s;
    const T* x0;
    float m;                              // the row's largest logit
    int32_t blocks;
    int32_t tid;

    __device__ __forceinline__ double weight(float x) const
    {
        if (!(x > -__builtin_inff())) return 0.0;
        const double t = a.c * ((double)x - (double)m);
        return t < kFar ? 0.0 : power(t, s.table);
    }
    // whether ln w >= ln min_p
    __device__ __forceinline__ bool likely(float x) const { return a.scale * ((double)x - (double)m) >= a.least; }
    // whether a token is among those that stay, given the least key
    __device__ __forceinline__ bool stays(float x, uint32_t token, Key least) const
    {
        return key_of(x, token) >= least && likely(x);
    }

    // First token of a block; blocks follow each other in token order.
    __device__ __forceinline__ int64_t block_begin(int32_t b) const
    {
        const int32_t per_strip = blocks_of_strip(a), strip = b / per_strip, i = b - strip * per_strip;
        return min((int64_t)a.vocab, ((int64_t)strip * a.strip_steps + min((int64_t)a.strip_steps, (int64_t)i << a.shift)) *
                                         (kSampleLanes * kUnroll * N));
    }

    // Of the tokens [from, to) that stay the first up to which more than `rest` lies; where
    // roundings leave none, the last that has a weight.  Into s.token, -1 if there is none.
    __device__ void locate(int64_t from, int64_t to, double rest, Key least)
    {
        if (tid == 0) s.token = -1;
        for (int64_t at = from; at < to; at += K * N) {
            const int64_t i = at / N + tid;
            float x[N];
            floats_at(x0, (int32_t)min((int64_t)a.vocab, to), i, x);
            double w[N], mine = 0.0, total;
            int32_t last = -1;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                w[j] = stays(x[j], (uint32_t)(i * N + j), least) ? weight(x[j]) : 0.0;
                mine += w[j];
                if (w[j] > 0.0) last = j;
            }
            if (tid == 0) s.place = K;
            const double upto = block_scan<K>(mine, s.wave, &total);
            if (last >= 0) atomicMax(&s.token, (int32_t)(i * N + last));
            if (upto > rest && last >= 0) atomicMin(&s.place, tid);
            __syncthreads();
            const bool found = s.place < K;
            if (found && tid == s.place) {
                double before = upto - mine;
                int32_t j = last;
#pragma unroll
                for (int e = N - 1; e >= 0; --e) {
                    // the sum up to e, as it was added
                    double sum = before;
#pragma unroll
                    for (int f = 0; f <= e; ++f) sum += w[f];
                    if (w[e] > 0.0 && sum > rest) j = e;
                }
                s.token = (int32_t)(i * N + j);
            }
            __syncthreads();
            if (found) return;
            rest -= total;
        }
    }

    // Sums of the blocks relative to the row's maximum; the sum up to each is left in s.sums, and all of them returned.
    __device__ double total_of_blocks()
    {
        double x = 0.0, total;
        if (tid < blocks && s.sums[tid] > 0.0) {
            const double t = a.c * ((double)s.refs[tid] - (double)m);
            if (t >= kFar) x = s.sums[tid] * power(t, s.table);
        }
        const double upto = block_scan<K>(x, s.wave, &total);
        __syncthreads();
        if (tid < blocks) s.sums[tid] = upto;
        __syncthreads();
        return total;
    }

    // From the blocks' sums up to each the token.
    __device__ void pick(double total, Key least)
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
        const double before = b ? s.sums[b - 1] : 0.0;
        locate(block_begin(b), b + 1 < blocks ? block_begin(b + 1) : (int64_t)a.vocab, target - before, least);
        __syncthreads();
        // weights at the edge of what counts as 0 made that block: the first token that has one
        if (s.token < 0) {
            __syncthreads();
            locate(0, a.vocab, 0.0, least);
            __syncthreads();
        }
    }

    float u;
    __device__ __forceinline__ double uniform() const
    {
        constexpr double kLast = 1.0 - 0x1p-53;
        return u > 0.f ? fmin((double)u, kLast) : 0.0;      // a NaN is not above 0
    }

    // The order of the r-th largest note (0: fewer have any tokens), and how many notes reach it.
    __device__ uint32_t note_of_rank(int32_t r)
    {
        uint32_t prefix = 0;
        int32_t left = r;
        for (int level = 0; level < 2; ++level) {
            for (int i = tid; i < 256; i += K) s.bins[i] = 0;
            if (tid == 0) s.found = 0;
            __syncthreads();
            for (int i = tid; i < blocks * 64; i += K) {
                const uint32_t n = s.notes[i];
                if (n > kNoteNothing && (level == 0 || n >> 8 == prefix)) atomicAdd(&s.bins[level == 0 ? n >> 8 : n & 255], 1);
            }
            __syncthreads();
            if (tid < 64) {
                // four bins a lane, from the top
                uint32_t c[4], mine = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) mine += c[e] = s.bins[255 - 4 * tid - e];
                uint32_t upto = mine;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const uint32_t y = __shfl_up(upto, d);
                    if (tid >= d) upto += y;
                }
                uint32_t before = upto - mine;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if ((int32_t)before < left && (int32_t)(before + c[e]) >= left) {
                        s.found = 256 + 255 - 4 * tid - e;
                        s.number = left - (int32_t)before;
                    }
                    before += c[e];
                }
            }
            __syncthreads();
            const uint32_t found = s.found;
            if (found == 0) return 0;
            prefix = (prefix << 8) | (found - 256);
            left = s.number;
            __syncthreads();
        }
        return prefix;
    }

    // All tokens from `bound` on into s.keys; their number, which may exceed what there is room for.
    __device__ int32_t collect(float bound, uint32_t note)
    {
        if (tid == 0) s.number = 0;
        __syncthreads();
        const int32_t per_strip = blocks_of_strip(a);
        for (int i = tid; i < blocks * 64; i += K) {
            if (s.notes[i] < note || s.notes[i] <= kNoteNothing) continue;
            const int32_t b = i >> 6, lane = i & 63, strip = b / per_strip, in = (b - strip * per_strip) << a.shift;
            const int32_t steps = min(1 << a.shift, a.strip_steps - in);
            for (int32_t v = 0; v < steps * kUnroll; ++v) {
                const int64_t at = ((int64_t)strip * a.strip_steps + in) * (kSampleLanes * kUnroll) + v * kSampleLanes + lane;
                float x[N];
                floats_at(x0, a.vocab, at, x);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (x[j] >= bound && x[j] > -__builtin_inff()) {
                        const int32_t n = atomicAdd(&s.number, 1);
                        if (n < kCandidates) s.keys[n] = key_of(x[j], (uint32_t)(at * N + j));
                    }
            }
        }
        __syncthreads();
        const int32_t n = s.number;
        __syncthreads();
        return n;
    }

    // From the n tokens in s.keys, which are all from some key on: true, with the token in
    // s.token and the weight of those that stay in s.total, if they hold all that stay.
    // total: the row's weight, where top_p of it counts.
    __device__ bool from_candidates(int32_t n, bool bounded, double total)
    {
        constexpr int PER = (kCandidates + K - 1) / K;
        // ranks: how many are larger
#pragma unroll 1
        for (int i = tid; i < n; i += K) {
            const Key mine = s.keys[i];
            int32_t place = 0;
            for (int j = 0; j < n; ++j) place += s.keys[j] > mine;
            s.ranked[place] = mine;
        }
        if (tid == 0) s.place = n;
        __syncthreads();
        const int32_t first = a.top_k > 0 ? min(a.top_k, n) : n;
        double w[PER], mine = 0.0, all;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int32_t i = tid * PER + e;
            w[e] = i < first ? weight(key_value(s.ranked[i])) : 0.0;
            mine += w[e];
        }
        double upto = block_scan<K>(mine, s.wave, &all) - mine;
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
        // in token order
#pragma unroll 1
        for (int i = tid; i < kept; i += K) {
            const Key k = s.ranked[i];
            const uint32_t token = key_token(k);
            int32_t place = 0;
            for (int j = 0; j < kept; ++j) place += key_token(s.ranked[j]) < token;
            s.keys[place] = k;
        }
        if (tid == 0) {
            s.token = -1;
            s.place = K;
        }
        __syncthreads();
        int32_t last = -1;
        mine = 0.0;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int32_t i = tid * PER + e;
            w[e] = i < kept ? weight(key_value(s.keys[i])) : 0.0;
            mine += w[e];
            if (w[e] > 0.0) last = i;
        }
        upto = block_scan<K>(mine, s.wave, &all);
        const double rest = uniform() * all;
        if (tid == 0) s.total = all;
        if (last >= 0) atomicMax(&s.token, last);
        if (upto > rest && last >= 0) atomicMin(&s.place, tid);
        __syncthreads();
        const int32_t fallback = s.token;
        __syncthreads();
        if (s.place == K ? tid == 0 : tid == s.place) {
            int32_t at = fallback;
            double before = upto - mine;
            if (s.place < K) {
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
            s.token = (int32_t)key_token(s.keys[at]);
        }
        __syncthreads();
        return true;
    }

    // The least key of those that stay, found digit by digit from histograms of the row:
    // by number (the first `number` of the order) or by weight (as many as it takes to
    // reach share of `total`).  *weight receives the weight from that key on.
    __device__ Key search(int64_t number, double enough, bool by_weight, double* weight_from)
    {
        // weights as whole numbers, so that their sums do not depend on the order: 2^units for the largest
        const int units = min(44, 62 - (32 - __clz((int)a.vocab)));
        const double unit = (double)((uint64_t)1 << units);
        const int64_t vecs = ((int64_t)a.vocab + N - 1) / N;
        const double target = by_weight ? enough * unit : 0.0;
        Key prefix = 0, above_mass = 0;
        int64_t above = 0;
        int shift = 64;
        // digits of 11, 11 and 10 bits of the value, then of the token
        while (shift > 0) {
            const int bits = shift == 42 || shift == 10 ? 10 : kDigit, low = shift - bits;
            for (int i = tid; i < kBins; i += K) {
                s.mass[i] = 0;
                s.count[i] = 0;
            }
            if (tid == 0) s.found = 0;
            __syncthreads();
            for (int64_t i = tid; i < vecs; i += K) {
                float x[N];
                floats_at(x0, a.vocab, i, x);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Key k = key_of(x[j], (uint32_t)(i * N + j));
                    if (k != 0 && (shift == 64 || k >> shift == prefix)) {
                        const uint32_t bin = (uint32_t)(k >> low) & ((1u << bits) - 1);
                        atomicAdd(&s.mass[bin], (Key)(weight(x[j]) * unit + 0.5));
                        atomicAdd(&s.count[bin], 1u);
                    }
                }
            }
            __syncthreads();
            // from the top: the bin in which the number or the weight is reached; where roundings leave
            // none, the lowest with anything in it
            constexpr int PER = kBins / K;
            const int top = (1 << bits) - 1 - tid * PER;
            Key mass = 0, all_mass;
            uint32_t count = 0, all_count;
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (top - e >= 0) {
                    mass += s.mass[top - e];
                    count += s.count[top - e];
                }
            Key mass_upto = above_mass + block_scan<K>(mass, s.wave_mass, &all_mass) - mass;
            int64_t count_upto = above + block_scan<K>(count, s.wave_count, &all_count) - count;
            const auto reached = [&](Key x, int64_t n) { return by_weight ? !((double)x < target) : n >= number; };
            const bool none = !reached(above_mass + all_mass, above + all_count);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int bin = top - e;
                if (bin < 0 || s.count[bin] == 0) continue;
                const Key m1 = mass_upto + s.mass[bin];
                const int64_t n1 = count_upto + s.count[bin];
                const bool first = mass_upto == above_mass && count_upto == above;       // nothing above it in here
                if (none ? n1 == above + all_count : reached(m1, n1) && (first || !reached(mass_upto, count_upto))) {
                    s.found = bin + 1;
                    s.bound = mass_upto;
                    s.number = (int32_t)count_upto;
                }
                mass_upto = m1;
                count_upto = n1;
            }
            __syncthreads();
            const uint32_t found = s.found;
            if (found == 0) return 1;                        // no tokens at all
            const uint32_t bin = found - 1;
            above_mass = s.bound;
            above = s.number;
            prefix = (prefix << bits) | bin;
            shift = low;
            const bool single = s.count[bin] == 1 || (!by_weight && above + s.count[bin] == number);
            const Key here = s.mass[bin];
            __syncthreads();
            if (single || shift == 0) {
                *weight_from = (double)(above_mass + here) / unit;
                return max(prefix << shift, (Key)1);
            }
        }
        return 1;
    }

    // The row's sums once more, of the tokens that stay.
    __device__ double sums_of(Key least)
    {
        const int lane = tid & 63;
        __syncthreads();
        for (int32_t b = tid >> 6; b < blocks; b += K / 64) {
            const int64_t from = block_begin(b), to = b + 1 < blocks ? block_begin(b + 1) : (int64_t)a.vocab;
            double sum = 0.0;
            // blocks begin at whole vectors, but for those behind the row's end
            for (int64_t i = from / N + lane; from < to && i * N < to; i += 64) {
                float x[N];
                floats_at(x0, (int32_t)to, i, x);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (stays(x[j], (uint32_t)(i * N + j), least)) sum += weight(x[j]);
            }
            sum = wave_sum(sum);
            if (lane == 0) {
                s.sums[b] = sum;
                s.refs[b] = m;
            }
        }
        __syncthreads();
        return total_of_blocks();
    }

    // Everything behind the pass over the logits.
    __device__ void finish(int64_t row, float most, bool sums)
    {
        const float nan = __builtin_nanf("");
        m = most;
        const bool broken = !(m < __builtin_inff()), empty = m == -__builtin_inff();
        if (broken || empty) {
            if (tid == 0) {
                a.tokens[row] = -1;
                if (a.logp) a.logp[row] = broken ? nan : -__builtin_inff();
            }
            return;
        }
        u = a.uniforms[row];
        double total = 0.0;
        if (sums) total = total_of_blocks();
        const bool filters = a.top_k > 0 || a.top_p < 1.0 || a.least > -__builtin_inf();
        if (!filters) {
            pick(total, 1);
        } else {
            bool done = false;
            const bool many = a.top_k > 3 * kCandidates / 4;
            // with min_p a bound is known
            float bound = -__builtin_inff();
            const bool known = a.least > -__builtin_inf() && !(a.top_k > 0 && a.top_p < 1.0);      // all of the first top_k count there
            if (known) {
                const double x = (double)m + a.least / a.scale * (1 + 1e-9) - 1e-30;
                if (x > -3.3e38) bound = nextafterf((float)x, -__builtin_inff());
            }
            for (int attempt = 0; attempt < 2 && !done && !many; ++attempt) {
                const int32_t rank = a.top_k > 0 ? a.top_k : attempt == 0 ? 96 : 3 * kCandidates / 4;
                const uint32_t order = note_of_rank(rank);
                // notes of fp32 logits are rounded up: the one below is exceeded
                float from = -3.402823466e38f;
                if (order > 0) from = value_at((std::is_same<T, float>::value ? order - 1 : order) << 16);
                if (order > 0 && order - 1 <= kNoteNothing) from = -3.402823466e38f;
                const bool all = order == 0;
                const bool bounded = all || (known && bound >= from);
                const float least = known ? fmaxf(bound, from) : from;
                const int32_t n = collect(least, note_of(least));
                if (n > kCandidates) break;
                done = from_candidates(n, bounded, total);
                if (a.top_k > 0) break;
            }
            if (!done) {
                Key least = 1;
                double among = total;
                if (a.top_k > 0) least = search(a.top_k, 0.0, false, &among);
                if (a.top_p < 1.0) {
                    double ignored;
                    least = max(least, search(0, a.top_p * among, true, &ignored));
                }
                const double kept = sums_of(least);
                pick(kept, least);
                total = kept;
            } else {
                total = s.total;
            }
        }
        if (tid == 0) {
            const int32_t token = s.token;
            a.tokens[row] = token;
            if (a.logp) a.logp[row] = token < 0 ? nan : (float)(a.scale * ((double)value_of(x0[token]) - (double)m) - log(total));
        }
    }
};

template <typename T, bool kSums> __global__ __launch_bounds__(64 * kWaves) void k_sample(SampleArgs a)
{
    constexpr int K = 64 * kWaves, BLOCKS = kSampleBlocks / 2;
    __shared__ Shared<K, BLOCKS> s;
    const int tid = threadIdx.x, wave = tid >> 6;
    if (tid < 32) s.table[tid] = kTwoTo[tid];
    __syncthreads();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* const x0 = static_cast<const T*>(a.x) + row * a.stride;
        const int32_t per = blocks_of_strip(a);
        const float top = read_strip<T, kSums>(a, x0, wave, s.table, s.notes + wave * per * 64, s.sums + wave * per, s.refs + wave * per);
        if ((tid & 63) == 0) s.most[wave] = top;
        __syncthreads();
        float m = s.most[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = most_of(m, s.most[w]);
        RowWork<T, K, BLOCKS> work{a, s, x0, 0.f, per * kWaves, tid, 0.f};
        work.finish(row, m, kSums);
        __syncthreads();
    }
}

// A slice of a row.
template <typename T, bool kSums> __global__ __launch_bounds__(64 * kWaves) void k_sample_read(SampleArgs a)
{
    __shared__ double s_table[32];
    const int tid = threadIdx.x, wave = tid >> 6;
    if (tid < 32) s_table[tid] = kTwoTo[tid];
    __syncthreads();
    const int64_t row = blockIdx.x / a.slices;
    const int32_t strips = a.slices * kWaves, strip = (int32_t)(blockIdx.x - row * a.slices) * kWaves + wave;
    const int32_t per = blocks_of_strip(a);
    const int64_t at = (row * strips + strip) * per;
    const float top = read_strip<T, kSums>(a, static_cast<const T*>(a.x) + row * a.stride, strip, s_table, a.notes + at * 64,
                                           a.sums + at, a.refs + at);
    if ((tid & 63) == 0) a.most[row * strips + strip] = top;
}

// The rest of a row that several workgroups have read.
constexpr int kJoinThreads = 1024;
template <typename T, bool kSums> __global__ __launch_bounds__(kJoinThreads) void k_sample_join(SampleArgs a)
{
    __shared__ Shared<kJoinThreads, kSampleBlocks> s;
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int32_t strips = a.slices * kWaves, per = blocks_of_strip(a), blocks = strips * per;
    if (tid < 32) s.table[tid] = kTwoTo[tid];
    if (tid < strips) s.most[tid] = a.most[row * strips + tid];
    if (kSums && tid < blocks) {
        s.sums[tid] = a.sums[row * blocks + tid];
        s.refs[tid] = a.refs[row * blocks + tid];
    }
    const uint32_t* const notes = reinterpret_cast<const uint32_t*>(a.notes + row * blocks * 64);
    for (int i = tid; i < blocks * 32; i += kJoinThreads) reinterpret_cast<uint32_t*>(s.notes)[i] = notes[i];
    __syncthreads();
    float m = s.most[0];
    for (int i = 1; i < strips; ++i) m = most_of(m, s.most[i]);
    RowWork<T, kJoinThreads, kSampleBlocks> work{a, s, static_cast<const T*>(a.x) + row * a.stride, 0.f, blocks, tid, 0.f};
    work.finish(row, m, kSums);
}

template <typename T, bool kSums> hipError_t sample_as(const SampleArgs& a, hipStream_t s)
{
    const dim3 block(64 * kWaves);
    if (a.slices == 1) {
        hipLaunchKernelGGL((k_sample<T, kSums>), dim3((unsigned)std::min<int64_t>(a.rows, kMaxGrid)), block, 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_sample_read<T, kSums>), dim3((unsigned)(a.rows * a.slices)), block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_sample_join<T, kSums>), dim3((unsigned)a.rows), dim3(kJoinThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t sample_t(const SampleArgs& a, hipStream_t s)
{
    // the row's whole weight counts where nothing bounds it, or top_p of all of it does
    const bool filters = a.top_k > 0 || a.top_p < 1.0 || a.least > -__builtin_inf();
    return !filters || (a.top_p < 1.0 && a.top_k == 0) ? sample_as<T, true>(a, s) : sample_as<T, false>(a, s);
}

}  // namespace

// How a row is cut: workgroups, steps of a wave's strip, steps of a block.
void sample_split(int32_t rows, int32_t vocab, int dtype, int32_t* slices, int32_t* strip_steps, int32_t* shift)
{
    const int64_t step = kSampleLanes * kUnroll * (dtype == 0 ? Vec<uint16_t>::n : Vec<float>::n);
    const int64_t steps = (vocab + step - 1) / step;
    int64_t cut = 1;
    if (rows > 0 && rows <= kMaxSlicedRows && steps >= 8 * kWaves / 4)
        cut = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(32, 512 / rows), steps / kWaves));
    const int64_t per = (steps + cut * kWaves - 1) / (cut * kWaves);
    *slices = (int32_t)((steps + per * kWaves - 1) / (per * kWaves));
    *strip_steps = (int32_t)per;
    const int64_t most = (*slices == 1 ? kSampleBlocks / 2 : kSampleBlocks) / (*slices * kWaves);
    *shift = 0;
    while (((per - 1) >> *shift) + 1 > most) ++*shift;
}

hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t s)
{
    return dtype == 0 ? sample_t<uint16_t>(a, s) : sample_t<float>(a, s);
}

}  // namespace cpes
