// cpes_logprobs.hip -- gfx950 kernels of the scores of given tokens under rows of
// logits: log probability, entropy, the most likely alternatives, and the
// gradient of the first two.
//
// Mathematics.  With z = scale x, M = max z, c = scale log2 e and t_v = c (x_v - max x) <= 0:
//   s = sum 2^(t_v),  u = sum t_v 2^(t_v),
//   lse = M + ln s,  ln p_v = z_v - M - ln s,  entropy = ln s - ln 2 u / s
// (both terms of the entropy are positive: nothing cancels).  Pieces (max, s, u) of
// a row join by 2^(t of the smaller maximum), u moving by s times that exponent as
// well.  c rounded to fp32 is c (1 + r): to first order that adds r ln 2 u to s, which
// is taken back at the end.
//   dx_v = scale (g ([v = t] - p_v) - h p_v (ln p_v + entropy)).
//
// What bounds it: a logit is read once (and its gradient written once) for about
// ten operations, close to what the vector units do in the time its bytes take,
// so the loop holds no more than it must: one subtraction, product, exponential
// and three sums a logit, the maximum by threes, and the alternatives cost nothing
// until the row's end (below).
//
// Split.  A row is one workgroup's where there are rows for the GPU; few rows are cut
// into slices, joined by a second launch in slice order.
//
// Alternatives.  Order: value descending, then token ascending, as one 64-bit key,
// so no two are equal and the result does not depend on who writes first.  A
// thread keeps, with its running maximum, the step it first met it in, so the
// maximum's key lies between those of the step's last and first token.  The k-th
// largest of the 256 threads' lower ends bounds the row's k-th largest key from
// below, and only threads whose upper end reaches that bound can hold a key from
// there on: k of them, and a few that tie, whose logits, about k / 256 of the row,
// are looked at again (from the caches).
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

// Sums of a piece of a row.
struct Sums {
    float m, s, u;       // largest logit, sum 2^t, sum t 2^t with t = c (x - m)
};

__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m);
    // a piece of nothing but -inf has s = u = 0 and moves nothing
    const float da = a.m == m ? 0.f : fmaxf(c * (a.m - m), kFar), db = b.m == m ? 0.f : fmaxf(c * (b.m - m), kFar);
    const float fa = exp2_hw(da), fb = exp2_hw(db);
    return Sums{m, fa * a.s + fb * b.s, fa * (a.u + da * a.s) + fb * (b.u + db * b.s)};
}

// Writes a finished row's numbers; every thread gets what the alternatives need.
template <typename T>
__device__ __forceinline__ void finish(const LogprobArgs& a, int64_t row, Sums t, float* logsum, bool* broken)
{
    const float nan = __builtin_nanf("");
    const bool empty = t.s == 0.f;        // nothing but -inf
    *broken = !(t.s >= 0.f) || t.m == __builtin_inff();
    t.s -= a.excess * t.u;
    *logsum = *broken ? nan : empty ? 0.f : logf(t.s);
    if (threadIdx.x != 0) return;
    if (a.logp) {
        const int64_t v = a.targets[row];
        float x = 0.f;
        if (v >= 0 && v < a.vocab) {
            x = value_of(static_cast<const T*>(a.x)[row * a.stride + v]);
            x = empty ? -__builtin_inff() : a.scale * (x - t.m) - *logsum;
        }
        a.logp[row] = x;
    }
    if (a.entropy) a.entropy[row] = empty ? 0.f : *logsum - t.u / t.s * kLn2;
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

// The k largest of the n keys in LDS, descending, into best (0 where there are
// fewer): each key's place is the number of larger ones.  All threads; the keys
// are distinct.
__device__ void largest(const Key* keys, int n, int k, Key* best)
{
    for (int i = threadIdx.x; i < k; i += kThreads) best[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const Key x = keys[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += keys[j] > x;
        if (place < k) best[place] = x;
    }
    __syncthreads();
}

constexpr int kUnroll = 4;                // 16-byte loads of a thread and step
constexpr int kMaxTop = 64;
constexpr int kSoft = 256;                // candidates from which on they are thinned out
constexpr int kCandidates = kSoft + kThreads * 8;

// One slice of one row.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprobs(LogprobArgs a)
{
    constexpr int N = Vec<T>::n;
    constexpr uint32_t kNone = std::is_same<T, float>::value ? 0xFF800000u : 0xFF80FF80u;   // -inf
    __shared__ Sums s_sums[kThreads / 64];
    __shared__ Key s_keys[kCandidates], s_best[kMaxTop];
    __shared__ int32_t s_owner[kThreads], s_count, s_owners;
    const int tid = threadIdx.x;
    for (int64_t job = blockIdx.x; job < (int64_t)a.rows * a.slices; job += gridDim.x) {
        const int64_t row = job / a.slices;
        const int32_t slice = (int32_t)(job - row * a.slices);
        const int64_t begin = (int64_t)slice * a.per_slice;
        const int32_t len = (int32_t)min((int64_t)a.per_slice, a.vocab - begin);
        const T* const x0 = static_cast<const T*>(a.x) + row * a.stride + begin;
        const int32_t full = len / N, vecs = (len + N - 1) / N, steps = (vecs + kUnroll * kThreads - 1) / (kUnroll * kThreads);

        auto vector_at = [&](int32_t i) {
            if (i < full) return (V4u)*reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)i * N);
            V4u w = {kNone, kNone, kNone, kNone};
            if (i < vecs) {
                T* const e = reinterpret_cast<T*>(&w);
                for (int j = 0; j < N; ++j)
                    if (i * N + j < len) e[j] = x0[(int64_t)i * N + j];
            }
            return w;
        };

        Sums t = {-__builtin_inff(), 0.f, 0.f};
        int32_t met = 0;                  // the step the maximum was first met in
        for (int32_t step = 0; step < steps; ++step) {
            V4u w[kUnroll];
            const int32_t i0 = step * kUnroll * kThreads + tid;
            if ((step + 1) * kUnroll * kThreads <= full) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    w[u] = *reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)(i0 + u * kThreads) * N);
            } else {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) w[u] = vector_at(i0 + u * kThreads);
            }
            float x[kUnroll * N], top = t.m;
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) unpack<T>(w[u], x + u * N);
#pragma unroll
            for (int j = 0; j < kUnroll * N; ++j) top = fmaxf(top, x[j]);
            if (top > t.m) {
                const float d = t.s == 0.f ? 0.f : fmaxf(a.c * (t.m - top), kFar), f = exp2_hw(d);
                t.u = f * (t.u + d * t.s);
                t.s *= f;
                t.m = top;
                met = step;
            }
            const float base = t.m == -__builtin_inff() ? 0.f : t.m;
#pragma unroll
            for (int j = 0; j < kUnroll * N; ++j) {
                const float d = a.c * (x[j] - base), e = exp2_hw(d);
                t.s += e;
                t.u += e * fmaxf(d, kFar);
            }
        }
        // the threads' sums join, in a fixed order; the maximum a thread met stays its own
        const float mine = t.m;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1)
            t = join(t, Sums{__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.u, d)}, a.c);
        if ((tid & 63) == 0) s_sums[tid >> 6] = t;
        if (a.top > 0 && tid == 0) s_count = s_owners = 0;
        Key low = 0, high = 0;            // no more and no less than the key of this thread's maximum
        if (a.top > 0) {
            const int64_t first = begin + ((int64_t)(met * kUnroll) * kThreads + tid) * N;
            if (tid < vecs) {
                low = key_of(mine, (uint32_t)(first + (kUnroll - 1) * kThreads * N + N - 1));
                high = key_of(mine, (uint32_t)first);
            }
            s_keys[tid] = low;
        }
        __syncthreads();
        t = s_sums[0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) t = join(t, s_sums[w], a.c);
        float logsum = 0.f;
        bool broken = false;
        if (a.slices == 1)
            finish<T>(a, row, t, &logsum, &broken);
        else if (tid == 0)
            a.parts[job] = float4{t.m, t.s, t.u, 0.f};

        if (a.top > 0) {
            // the k-th largest lower end, and the threads that reach it
            int place = 0;
            for (int j = 0; j < kThreads; ++j) place += s_keys[j] > low;
            if (tid == 0) s_best[0] = 1;
            __syncthreads();
            if (low && place == a.top - 1) s_best[0] = low;
            __syncthreads();
            Key least = s_best[0];
            if (high >= least) s_owner[atomicAdd(&s_owners, 1)] = tid;
            __syncthreads();
            const int owners = s_owners;
            // their logits from there on
            const int32_t per = steps * kUnroll, items = owners * per;
            for (int32_t item0 = 0; item0 < items; item0 += kThreads) {
                const int n = s_count;
                __syncthreads();          // read by all before any candidate is added
                if (n > kSoft) {
                    largest(s_keys, n, a.top, s_best);
                    if (tid < a.top) s_keys[tid] = s_best[tid];
                    if (tid == 0) s_count = a.top;
                    least = s_best[a.top - 1];
                    __syncthreads();
                }
                const int32_t item = item0 + tid, o = item / per;
                if (item < items) {
                    const int32_t i = (item - o * per) * kThreads + s_owner[o];
                    if (i < vecs) {
                        const V4u w = vector_at(i);
                        float x[N];
                        unpack<T>(w, x);
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            const Key k = key_of(x[j], (uint32_t)(begin + (int64_t)i * N + j));
                            if (i * N + j < len && k >= least) s_keys[atomicAdd(&s_count, 1)] = k;
                        }
                    }
                }
                __syncthreads();
            }
            largest(s_keys, s_count, a.top, s_best);
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
template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprobs_join(LogprobArgs a)
{
    __shared__ Key s_keys[kMaxSlices * kMaxTop], s_head[kMaxSlices], s_best[kMaxTop], s_least;
    __shared__ int32_t s_count;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    Sums t = {-__builtin_inff(), 0.f, 0.f};
    if (lane < a.slices) {
        const float4 p = a.parts[row * a.slices + lane];
        t = Sums{p.x, p.y, p.z};
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        t = join(t, Sums{__shfl_xor(t.m, d), __shfl_xor(t.s, d), __shfl_xor(t.u, d)}, a.c);
    t = Sums{__shfl(t.m, 0), __shfl(t.s, 0), __shfl(t.u, 0)};
    float logsum;
    bool broken;
    finish<T>(a, row, t, &logsum, &broken);
    if (a.top == 0) return;
    // the k-th largest of the slices' first keys bounds what can be among the row's k largest
    const Key* const keys = a.keys + row * a.slices * a.top;
    const Key head = tid < a.slices ? keys[tid * a.top] : 0;
    if (tid < kMaxSlices) s_head[tid] = head;
    if (tid == 0) {
        s_count = 0;
        s_least = 1;
    }
    __syncthreads();
    if (tid < a.slices) {
        int place = 0;
        for (int j = 0; j < a.slices; ++j) place += s_head[j] > head;
        if (place == a.top - 1 && head) s_least = head;
    }
    __syncthreads();
    const Key least = s_least;
    for (int i = tid; i < a.slices * a.top; i += kThreads)
        if (keys[i] >= least) s_keys[atomicAdd(&s_count, 1)] = keys[i];
    __syncthreads();
    largest(s_keys, s_count, a.top, s_best);
    if (tid < a.top) write_top(a, row, tid, s_best[tid], t.m, logsum, broken);
}

// --------------------------------------------------------------- gradient --
constexpr int kGradUnroll = 2;
constexpr int64_t kMaxGrid = 1 << 20;     // workgroups per launch; larger jobs loop

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

template <typename T>
__global__ __launch_bounds__(kThreads) void k_logprobs_backward(LogprobGradArgs a)
{
    constexpr int N = Vec<T>::n;
    const int32_t vecs = (a.vocab + N - 1) / N, full = a.vocab / N;
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
            if (v == target) d += empty ? 0.f : gp;
            return d;
        };
        V4u w[kGradUnroll];
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u)
            if (i0 + u * kThreads < full)
                w[u] = *reinterpret_cast<const V4uAnywhere*>(x0 + (int64_t)(i0 + u * kThreads) * N);
#pragma unroll
        for (int u = 0; u < kGradUnroll; ++u) {
            const int32_t i = i0 + u * kThreads;
            if (i < full) {
                float x[N];
                unpack<T>(w[u], x);
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = gradient(x[j], (int64_t)i * N + j);
                *reinterpret_cast<V4uAnywhere*>(d0 + (int64_t)i * N) = pack<T>(x);
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

template <typename T>
hipError_t logprobs_t(const LogprobArgs& a, hipStream_t s)
{
    const int64_t jobs = (int64_t)a.rows * a.slices;
    hipLaunchKernelGGL(k_logprobs<T>, dim3((unsigned)std::min(jobs, kMaxGrid)), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.slices == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const LogprobGradArgs& a, hipStream_t s)
{
    const int64_t per = (int64_t)kGradUnroll * kThreads * Vec<T>::n, jobs = a.rows * ((a.vocab + per - 1) / per);
    hipLaunchKernelGGL(k_logprobs_backward<T>, dim3((unsigned)std::min(jobs, kMaxGrid)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

// Slices of a row: none where the rows alone fill the GPU, otherwise enough for
// six workgroups a CU, of at least a thread's vector each.
int logprob_slices(int32_t rows, int32_t vocab, int dtype, int32_t* per_slice)
{
    const int n = dtype == 0 ? Vec<uint16_t>::n : Vec<float>::n;
    int64_t slices = 1;
    if (rows > 0 && rows < 768)
        slices = std::min<int64_t>(std::min<int64_t>(kMaxSlices, (1536 + rows - 1) / rows), std::max(1, vocab / (kThreads * n)));
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
