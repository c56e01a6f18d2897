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

constexpr int kMaxTree = 256;            // CPES_MAX_TREE

// The end of a step with drafted tokens: what stays of them moves together.
struct KeepArgs {
    PoolArgs pool;
    char* k;
    char* v;
    const int32_t* seqs;
    const int32_t* starts;
    const int32_t* kept;
    const int32_t* path;
    int32_t* ws;                 // whether the call goes on; per row where its drafted tokens begin and how many stay; their pages
    int64_t page_bytes, layer_bytes, head_bytes, token_bytes;   // strides
    int32_t n, longest;
    int32_t span;                // pages that `longest` tokens may touch
    Divisor run, heads;          // 16-byte units of one head of a token; heads
    uint32_t units;              // of a token: 2 * layers * heads * run
};

inline __host__ __device__ int64_t keep_words(int64_t n, int64_t span)
{
    return kPagesHeader + n * (2 + span);
}

struct AcceptArgs {
    const int32_t* starts;
    const int32_t* parents;
    const int64_t* drafted;
    const int64_t* sampled;
    int32_t* kept;
    int32_t* path;
    int64_t* next;
    int32_t rows, tokens, longest;
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

struct TreeArgs {
    const void* k;               // of the layer
    const void* v;
    const void* q;
    void* out;
    float* lse;
    const int32_t* seqs;
    const int32_t* starts;
    const int32_t* parents;
    const int32_t* table;
    const int32_t* lengths;
    float* parts;                // partial results, two per share
    int2* joins;                 // per job: the shares it begins and ends in
    int64_t page_stride, head_stride, token_stride, table_stride;
    int64_t q_stride, q_head_stride, out_stride, out_head_stride;
    int32_t rows, tokens, longest;
    int32_t heads, group;        // q_heads = heads * group
    int32_t columns;             // queries of a job: 16 * sets * beside
    bool wide;
    int32_t sets;                // of 16 queries, of a wave
    int32_t beside;              // waves of a job on the same positions
    int32_t job_heads, blocks;   // a group's query heads in `blocks` blocks of job_heads
    int32_t job_tokens, pieces;  // a row's tokens in pieces of job_tokens, `pieces` at most
    int32_t dim, page_size, page_shift, pages, width, sequences;   // page_shift < 0: no power of two
    int32_t window, sinks;
    int32_t groups;              // workgroups launched for shares
    float scale;
};

// How jobs are cut, from what the host knows.
struct TreeShape {
    bool wide;                   // more than 32 queries, up to 128 dims: through shared memory, where the call lets it
    int32_t sets, beside, columns, job_heads, blocks, job_tokens, pieces;
};

inline TreeShape tree_shape(bool bf16, bool shared, int32_t longest, int32_t group, int32_t dim)
{
    TreeShape t;
    const int64_t queries = (int64_t)longest * group;
    t.wide = bf16 && shared && dim <= 128 && queries > 32;
    t.sets = bf16 && dim <= 128 && queries > 16 ? 2 : 1;        // what fits a wave's registers
    t.beside = 1;
    while (t.beside < (t.wide ? 8 : 4) && 16 * t.sets * t.beside < queries) t.beside *= 2;
    t.columns = 16 * t.sets * t.beside;
    t.job_heads = group < t.columns ? group : t.columns;
    t.blocks = (group + t.job_heads - 1) / t.job_heads;
    t.job_tokens = t.columns / t.job_heads;
    t.pieces = (longest + t.job_tokens - 1) / t.job_tokens;
    return t;
}

// One partial result of a wave: 16 * sets maxima, as many sums, then the output rows.
inline __host__ __device__ int64_t tree_part_floats(int sets, int dim)
{
    return 16 * (int64_t)sets * (2 + dim);
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

constexpr int kSampleLanes = 64;
constexpr int kSampleWaves = 4;          // strips of a slice, where a row is cut into slices
constexpr int kSampleBlocks = 256;       // blocks of such a row at most
constexpr int kSampleRows = 1024;        // more rows are all cut alike
constexpr int kSampleAtOnce = 8192;      // rows that a workspace holds

// How a row of logits is cut: into slices of a workgroup (0: one wave does the row) and strips
// of a wave; a strip into blocks of 2^shift steps, of which there are `slots`, and parts of
// 2^note_shift, room for note_slots of which, stored 2^group together.
struct SampleSplit {
    int32_t slices, waves, strip_steps, shift, slots, note_shift, note_slots, group;

    int32_t strips() const { return (slices > 0 ? slices : 1) * waves; }
};

struct SampleArgs {
    const void* x;
    const float* uniforms;
    int64_t* tokens;
    float* logp;
    uint16_t* notes;             // [rows][strips][note_slots / 2^group][64][2^group]: maxima of the lanes' parts
    uint16_t* samples;           // a logit of each of these parts
    double* sums;                // [rows][strips][slots]
    float* refs;                 // [rows][strips][slots]: what the sums' exponents are relative to
    float* most;                 // [rows][strips]: maxima, NaN where there is one
    int64_t stride;
    int32_t rows, vocab;
    int32_t slices, strip_steps, shift, slots, note_shift, note_slots, group;
    bool notes_kept, samples_kept;
    int32_t top_k;               // 0: all
    double top_p;
    double least;                // ln min_p, or -inf
    double scale, c;             // c = scale log2 e
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
hipError_t launch_pages_keep(const KeepArgs& a, int32_t* status, hipStream_t s);
hipError_t launch_tree_accept(const AcceptArgs& a, hipStream_t s);
hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_attend(int dtype, const AttendArgs& a, hipStream_t s);
int logprob_slices(int32_t rows, int32_t vocab, int dtype, int32_t* per_slice);
hipError_t launch_attend_tree(int dtype, const TreeArgs& a, hipStream_t s);
SampleSplit sample_split(int32_t rows, int32_t vocab, int dtype);
hipError_t launch_sample(int dtype, const SampleArgs& a, hipStream_t s);
hipError_t launch_logprobs(int dtype, const LogprobArgs& a, hipStream_t s);
hipError_t launch_logprobs_backward(int dtype, const LogprobGradArgs& a, hipStream_t s);

}  // namespace cpes
