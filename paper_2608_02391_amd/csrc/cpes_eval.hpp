// cpes_eval.hpp -- argument blocks and launchers of the operators that evaluate
// a member (cache pages, attention, token scores), shared by the host runtime
// (cpes_eval_api.hip) and the kernels.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cpes {

// Pages and sequences of a pool, as include/cpes.h describes them.
struct PoolArgs {
    int32_t* table;
    int32_t* lengths;
    int32_t* refs;
    int64_t table_stride;
    int32_t sequences, width, pages, page_size;
};

// Division of counts below 2^31 by a divisor known on the host: one multiplication.
// With l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1, floor(n m / 2^(31 + l)) is
// floor(n / d), since n (m - 2^(31 + l) / d) < 2^(31 + l) / d.
struct Divisor {
    uint32_t d, m, shift;

    Divisor() = default;
    explicit Divisor(uint32_t divisor) : d(divisor), m(0), shift(0)
    {
        int l = 0;
        while (((uint64_t)1 << l) < d) ++l;
        if (l > 0) {
            m = (uint32_t)(((uint64_t)1 << (31 + l)) / d + 1);
            shift = l - 1;
        }
    }

    __device__ __forceinline__ uint32_t of(uint32_t n) const { return m ? __umulhi(n, m) >> shift : n; }
};

// One page as `runs` pieces of `run` consecutive 16-byte units: layer, keys or
// values, and the outer and inner of heads and tokens that do not join up.
struct PageArgs {
    char* k;
    char* v;
    int64_t page_bytes, layer_bytes, outer_bytes, inner_bytes;   // strides
    Divisor outers, inners;
    Divisor run;                 // units of a run
    uint32_t units;              // units of a page: 2 * layers * outers * inners * run
};

constexpr int kPlanBlock = 1024;         // the bookkeeping kernels are one workgroup
constexpr int kPagesHeader = 16;         // int32 words in front of a workspace's lists

struct AppendArgs {
    PoolArgs pool;
    char* k;                     // of the layer
    char* v;
    const char* k_new;
    const char* v_new;
    const int32_t* seqs;
    const int32_t* positions;
    int64_t page_bytes, head_bytes, token_bytes, new_bytes, new_head_bytes;   // strides
    int32_t n, heads;
    Divisor run, token;          // 16-byte units of one head, and of all heads, of one token
};

constexpr int kAttendHeads = 16;         // query heads of a workgroup: the columns of a matrix instruction
constexpr int kAttendWaves = 4;          // of a workgroup, each with a share of the tiles

struct AttendArgs {
    const void* k;               // of the layer
    const void* v;
    const void* q;
    void* out;
    float* lse;
    const int32_t* seqs;
    const int32_t* table;
    const int32_t* lengths;
    float* parts;                // partial results, two per share
    int2* joins;                 // per row and head block: the shares it begins and ends in
    int64_t page_stride, head_stride, token_stride, table_stride;
    int64_t q_stride, q_head_stride, out_stride, out_head_stride;
    int32_t rows, heads, group, blocks;      // q_heads = heads * group, in `blocks` blocks of kAttendHeads
    int32_t dim, page_size, page_shift, pages, width, sequences;   // page_shift < 0: no power of two
    int32_t window, sinks;
    int32_t groups;              // workgroups launched
    float scale;
};

// One partial result: kAttendHeads maxima, as many sums, then the output rows.
inline __host__ __device__ int64_t attend_part_floats(int dim)
{
    return 2 * kAttendHeads + (int64_t)kAttendHeads * dim;
}

constexpr int kMaxSlices = 64;           // workgroups of one row of logits at most
constexpr int kMaxSlicedRows = 256;      // more rows are not cut into slices

struct LogprobArgs {
    const void* x;
    const int64_t* targets;
    float* logp;
    float* entropy;
    float* lse;
    float* stats;
    float* top_logp;
    int64_t* top_ids;
    float4* parts;               // [rows][slices]: maximum, sum, weighted sum
    unsigned long long* keys;    // [rows][slices][top]
    int64_t stride;
    int32_t rows, vocab, top;
    int32_t slices, per_slice;   // per_slice: a multiple of the vector
    float scale;
    float c;                     // scale log2 e
    float excess;                // (c / (scale log2 e) - 1) ln 2
};

struct LogprobGradArgs {
    const void* x;
    void* dx;
    const int64_t* targets;
    const float* stats;
    const float* entropy;
    const float* d_logp;
    const float* d_entropy;
    int64_t stride, dx_stride;
    int32_t rows, vocab;
    float scale;
};

hipError_t launch_pages_reserve(const PoolArgs& p, int32_t n, const int32_t* seqs, const int32_t* new_lengths,
                                int32_t* ws, int32_t* status, hipStream_t s);
hipError_t launch_pages_fork(const PageArgs& c, const PoolArgs& p, int32_t n, const int32_t* parents,
                             const int32_t* children, int32_t* ws, int32_t* status, hipStream_t s);
hipError_t launch_pages_free(const PoolArgs& p, int32_t n, const int32_t* seqs, int32_t* status, hipStream_t s);
hipError_t launch_pages_copy(const PageArgs& c, int32_t pages, int32_t n, const int32_t* src, const int32_t* dst,
                             hipStream_t s);
hipError_t launch_pages_compact(const PageArgs& c, const PoolArgs& p, const PoolArgs& packed, int32_t* ws,
                                int32_t* moved, hipStream_t s);
hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_attend(int dtype, const AttendArgs& a, hipStream_t s);
int logprob_slices(int32_t rows, int32_t vocab, int dtype, int32_t* per_slice);
hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t s);
hipError_t launch_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t s);

}  // namespace cpes
