// cpes_attend.hip -- gfx950 kernels of the attention of one new token per row
// over a paged key-value cache.
//
// Mathematics.  For the heads i of one key-value head, with x_ij = scale q_i k_j:
//   m_i = max_j x_ij,  l_i = sum_j e^(x_ij - m_i),  o_i = sum_j e^(x_ij - m_i) v_j,
// kept for the positions seen so far and rescaled by e^(m_old - m_new) when the
// maximum grows; pieces (m, l, o) of any split of the positions join the same
// way, out = o / l and lse = m + ln l.
//
// What bounds it: every key and value is read once, 2 D elements for 4 D
// operations per query head, far below what the matrix instructions do; the
// kernel is a stream from HBM, so the work is arranged for many wide loads in
// flight and none of it waits on another wave.  8 rows of 65 to 131 thousand positions,
// 32 heads on 8 of 128 in bf16 (2.95 GB): 446 us, 6.6 TB/s, as fast as a large copy;
// 40 rows of up to 8,191 (306 MB): 51 us and 5.6 for the join, 6.0 TB/s while it
// streams; the matrix units are busy 5 to 7 % of the time.  In fp32, 24 rows through a
// window of 4,096 (591 MB): 96 us, 6.1 TB/s.
//
// Tiles.  A wave takes 32 positions (16 in fp32), about 16 KiB at D = 128.
// Scores come out of the matrix instructions transposed, S^T = K Q^T with the
// positions as rows: lane l then holds, for query head l % 16, positions
// 4 (l / 16) .. + 3 of each 16, which is just where the second product
// O^T = V^T P^T wants its right operand, whose inner index may be numbered at
// will as long as V's rows are numbered alike.  So the weights never leave their
// lane, and m, l and the rescaling are per lane.  A lane loads 16 bytes of keys
// (rows of 64 bytes per load and position) and whole 16-byte pieces of its
// positions' values, dims D/16 (l % 16) .., and in bf16 pairs two positions'
// values with one byte permutation per two elements: no shared memory and no
// transposition anywhere in the loop.  The weights of a bf16 cache go in as a
// bf16 value and its bf16 remainder, 16 bits of mantissa for one more matrix
// instruction in a kernel that has them to spare; scores, maxima, sums and
// outputs are fp32.
//
// Split.  All rows' tiles, for every key-value head, form one line, cut into equal
// shares, one per wave, whatever the lengths: a share may end one row and begin
// others, and its loads run on across them.  A row (and head) that lies in one
// share is written by its wave; otherwise each wave leaves its piece, and a
// second launch joins the pieces in order, so the result does not depend on
// timing.  Where no row can have more than a few tiles, a workgroup takes a row
// (and head), its waves join in shared memory, and there is one launch.
#include <algorithm>
#include <type_traits>

#include "cpes_attend.hpp"

namespace cpes {

namespace {

constexpr int kWaves = kAttendWaves;
constexpr int kThreads = 64 * kWaves;
constexpr int kShareTiles = 2;            // tiles of a wave's share at least
constexpr int64_t kMaxGrid = 1 << 20;     // workgroups of the short and the join launch

// Tiles of one row: [0, sinks_tiles) from position 0 on, the rest from `from`.
struct Row {
    int32_t n;            // its tokens
    int32_t sink_tiles;
    int32_t from;
    int32_t tiles;        // at least one: an empty row is written too
    int32_t seq;

    // First position of tile i.
    __device__ __forceinline__ int32_t begin(int32_t i, int tile) const
    {
        return i < sink_tiles ? i * tile : from + (i - sink_tiles) * tile;
    }
};

template <int TILE>
__device__ __forceinline__ Row row_at(const AttendArgs& a, int32_t r)
{
    Row x;
    x.seq = a.seqs ? a.seqs[r] : r;
    x.n = 0;
    if (x.seq >= 0 && x.seq < a.sequences) {
        const int64_t cap = (int64_t)a.width * a.page_size;
        const int32_t most = cap > INT32_MAX - 64 ? INT32_MAX - 64 : (int32_t)cap;
        x.n = min(max(a.lengths[x.seq], 0), most);
    }
    x.sink_tiles = 0;
    x.from = 0;
    if (a.window > 0 && x.n > a.window) {
        const int32_t begin = (x.n - a.window) / TILE, sinks = min((a.sinks - 1) / TILE + (a.sinks > 0), begin);
        // where the sinks reach the window's first tile there is nothing to leave out
        if (sinks < begin) {
            x.sink_tiles = sinks;
            x.from = begin * TILE;
        }
    }
    x.tiles = max(1, x.sink_tiles + (x.n - x.from + TILE - 1) / TILE);
    return x;
}

// The page ids of a tile's positions, asked for long before they are needed.
template <typename T, bool kWhole> struct Pages {
    static constexpr int SUB = Tile<T>::n / 16;
    int32_t id[SUB], slot[SUB];

    __device__ __forceinline__ void ask(const AttendArgs& a, const Row& row, const int32_t* table, int32_t pos0, int lane)
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const int32_t pos = pos0 + 16 * u + (kWhole ? 0 : lane & 15);
            const int32_t at = a.page_shift >= 0 ? pos >> a.page_shift : pos / a.page_size;
            slot[u] = pos - at * a.page_size;
            id[u] = -1;
            if (pos < row.n) id[u] = table[at];          // row.n is at most what the table holds
        }
    }

    __device__ __forceinline__ Places<T, kWhole> places(const AttendArgs& a, const Row& row, int32_t pos0)
    {
        Places<T, kWhole> p;
        p.seen = 0;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            int32_t page = id[u], at = slot[u];
            if constexpr (kWhole) page = __builtin_amdgcn_readfirstlane(page);
            const bool there = page >= 0 && page < a.pages;
            p.base[u] = there ? page * a.page_stride + at * a.token_stride : 0;
            if constexpr (kWhole)
                p.seen |= there ? 0xFFFFu << (16 * u) : 0u;
            else
                p.seen |= (uint32_t)(__ballot(there) & 0xFFFF) << (16 * u);
        }
        const int32_t left = row.n - pos0;
        if (left < 32) p.seen &= left > 0 ? (1u << left) - 1u : 0u;
        if (a.window > 0) {
            // seen: before `sinks`, or from n - window on
            const int32_t skip = row.n - a.window - pos0, sinks = a.sinks - pos0;
            uint32_t keep = skip <= 0 ? ~0u : skip >= 32 ? 0u : ~0u << skip;
            if (sinks > 0) keep |= sinks >= 32 ? ~0u : (1u << sinks) - 1u;
            p.seen &= keep;
        }
        return p;
    }
};

template <typename T, int DP, bool kWhole> struct Work : Operands<T, DP, kWhole> {
    typedef Operands<T, DP, kWhole> O;
    typedef typename O::L L;
    using O::key;
    using O::val;
    using O::SUB;
    using O::TILE;
    using O::VROWS;

    // Scores of the tile, unseen ones -inf: x[4 u + r] is position 16 u + 4 (lane / 16) + r.
    __device__ __forceinline__ void scores(const AttendArgs& a, const V4u* q, uint32_t seen, int lane, float x[VROWS])
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            V4f s;
            if constexpr (std::is_same<T, uint16_t>::value) {
                s = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::KV; ++i)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8bf, key[u][i]),
                                                                __builtin_bit_cast(V8bf, q[i]), s, 0, 0, 0);
            } else {
                // four sums: a quarter of the roundings in line, and of the instructions that wait for each other
                V4f part[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e] = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::KV; ++i) {
                    const V4f k4 = __builtin_bit_cast(V4f, key[u][i]), q4 = __builtin_bit_cast(V4f, q[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[e], q4[e], part[e], 0, 0, 0);
                }
                s = (part[0] + part[1]) + (part[2] + part[3]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * u + r] = s[r] * a.scale;
        }
        if (seen != (TILE == 32 ? ~0u : 0xFFFFu)) {
#pragma unroll
            for (int j = 0; j < VROWS; ++j)
                if (!(seen >> (16 * (j >> 2) + 4 * (lane >> 4) + (j & 3)) & 1)) x[j] = -__builtin_inff();
        }
    }

    // Folds the tile's values, with weights e^x, into the state.
    __device__ __forceinline__ void fold(State<DP>& st, float x[VROWS])
    {
        float top = x[0];
#pragma unroll
        for (int j = 1; j < VROWS; ++j) top = fmaxf(top, x[j]);
        const float m = fmaxf(st.m, max_over_lanes(top));
        // nothing seen yet: any finite base gives weights of 0
        const float base = m == -__builtin_inff() ? 0.f : m;
        const float keep = weight<T>(st.m - base);
        float l = 0.f;
#pragma unroll
        for (int j = 0; j < VROWS; ++j) {
            x[j] = weight<T>(x[j] - base);
            l += x[j];
        }
        st.l = st.l * keep + l;
        st.m = m;
        if (__any(keep != 1.f)) {
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) st.o[b] *= keep;
        }
        if constexpr (std::is_same<T, uint16_t>::value) {
            V8bf hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                hi[j] = (__bf16)x[j];
                lo[j] = (__bf16)(x[j] - (float)hi[j]);
            }
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) {
                V4u v;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = __builtin_amdgcn_perm(val[2 * i + 1][b >> 1], val[2 * i][b >> 1],
                                                 b & 1 ? 0x07060302u : 0x05040100u);
                const V8bf v8 = __builtin_bit_cast(V8bf, v);
                st.o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, hi, st.o[b], 0, 0, 0);
                st.o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, lo, st.o[b], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int b = 0; b < DP / 16; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    st.o[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(val[j][b]), x[j], st.o[b], 0, 0, 0);
        }
    }
};

// A key-value head with kAttendHeads of its query heads, or what is left of them.
struct Job {
    int32_t kv, head0, heads;
};

__device__ __forceinline__ Job job_at(const AttendArgs& a, int32_t hh)
{
    Job j;
    j.kv = hh / a.blocks;
    const int32_t block = hh - j.kv * a.blocks;
    j.head0 = j.kv * a.group + block * kAttendHeads;
    j.heads = min(kAttendHeads, a.group - block * kAttendHeads);
    return j;
}

// The queries of a row, as the right operand of the first product.
template <typename T, int DP>
__device__ __forceinline__ void load_queries(const AttendArgs& a, int32_t r, const Job& job, int lane, V4u* q)
{
    constexpr int E = 16 / sizeof(T);
    const int head = lane & 15;
    const T* const p = static_cast<const T*>(a.q) + (int64_t)r * a.q_stride + (job.head0 + min(head, job.heads - 1)) * a.q_head_stride;
#pragma unroll
    for (int i = 0; i < Layout<T, DP>::KV; ++i) {
        const int d = E * (lane >> 4) + 4 * E * i;
        q[i] = *reinterpret_cast<const V4uAnywhere*>(p + (d < a.dim ? d : 0));
        if (d >= a.dim || head >= job.heads) q[i] = V4u{0, 0, 0, 0};
    }
}

template <typename T>
__device__ __forceinline__ T* out_row(const AttendArgs& a, int32_t row, int32_t head)
{
    return static_cast<T*>(a.out) + (int64_t)row * a.out_stride + head * a.out_head_stride;
}

__device__ __forceinline__ void write_lse(const AttendArgs& a, int32_t row, int32_t head, float m, float l)
{
    if (a.lse) a.lse[(int64_t)row * a.heads * a.group + head] = l == 0.f ? -__builtin_inff() : m + logf(l);
}

// A tile of the line: row, key-value head and block, and its place in the row.
struct Cursor {
    Row row;
    int32_t r, hh, i;

    template <int TILE> __device__ __forceinline__ void next(const AttendArgs& a)
    {
        if (++i < row.tiles) return;
        i = 0;
        if (++r == a.rows) {
            r = 0;
            ++hh;
        }
        row = row_at<TILE>(a, r);
    }
};

template <typename T, int DP, bool kWhole>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void k_attend(AttendArgs a)
{
    typedef Work<T, DP, kWhole> W;
    constexpr int TILE = Tile<T>::n;
    __shared__ int64_t s_sum[kWaves], s_before[kWaves];
    __shared__ int32_t s_row[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // Every row's tiles, and where this workgroup's waves begin on their line.  Up
    // to 64 rows a wave finds its own place, a lane to a row; more are spread over
    // the workgroup's threads.
    const bool few = a.rows <= 64;
    const int32_t threads = few ? 64 : kThreads, thread = few ? lane : tid;
    const int32_t each = (a.rows + threads - 1) / threads, r0 = min(a.rows, thread * each), r1 = min(a.rows, r0 + each);
    int64_t mine = 0;
    for (int32_t r = r0; r < r1; ++r) mine += row_at<TILE>(a, r).tiles;
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
    }
    int64_t tiles = __shfl(upto, 63);
    if (!few) {
        if (lane == 63) s_sum[wave] = upto;
        __syncthreads();
        tiles = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) upto += s_sum[w];
            tiles += s_sum[w];
        }
    }
    const int64_t units = tiles * a.heads * a.blocks;
    const int32_t waves = (int32_t)max((int64_t)1, min((int64_t)a.groups * kWaves, units / kShareTiles));
    // Consecutive shares to the waves of a workgroup -- or, where there are no more than
    // workgroups, one to each, on as many CUs (one row of 2,000: 13.1 -> 12.3 us).  Token-major
    // pages take the second order too: a workgroup's waves are then a head or two apart at the
    // same positions, whose heads lie side by side in memory (64 rows: 104 -> 98 us; long
    // rows of head-major pages are 2 % faster in the first), and so do more query heads of a
    // key-value head than a wave takes, which read the same pages (32 on 1: 38.4 -> 37.3).
    const bool apart = waves <= (int32_t)gridDim.x || a.head_stride < a.token_stride || a.blocks > 1;
    const int32_t share0 = apart ? blockIdx.x : blockIdx.x * kWaves, step = apart ? gridDim.x : 1;
    const int32_t me = share0 + wave * step;
    if (share0 >= waves) return;
    const Shares shares(units, waves);
    if (!few) {
#pragma unroll 1
        for (int w = 0; w < kWaves; ++w) {
            const int32_t share = share0 + w * step;
            if (share >= waves) break;
            const int64_t at = shares.begin(share), t = at - quotient(at, tiles) * tiles;
            if (t >= upto - mine && t < upto) {
                int64_t before = upto - mine;
                int32_t r = r0;
                for (; r < r1; ++r) {
                    const int32_t n = row_at<TILE>(a, r).tiles;
                    if (t < before + n) break;
                    before += n;
                }
                s_row[w] = r;
                s_before[w] = before;
            }
        }
        __syncthreads();
    }
    if (me >= waves) return;
    const int64_t at = shares.begin(me), hh = quotient(at, tiles), t = at - hh * tiles;
    const int32_t share = __builtin_amdgcn_readfirstlane((int32_t)(shares.begin(me + 1) - at));
    int32_t left = share;
    if (left == 0) return;

    Cursor cur;
    int64_t before;
    if (few) {
        const int from = __ffsll(__ballot(t < upto)) - 1;    // the first row that ends behind it
        cur.r = from;
        before = __shfl(upto - mine, from);
    } else {
        cur.r = s_row[wave];
        before = s_before[wave];
    }
    cur.r = __builtin_amdgcn_readfirstlane(cur.r);
    cur.hh = __builtin_amdgcn_readfirstlane((int32_t)hh);
    cur.i = __builtin_amdgcn_readfirstlane((int32_t)(t - before));
    cur.row = row_at<TILE>(a, cur.r);

    // Three tiles are under way: the scores and values of one, the keys and values
    // of the next, the page ids of the one behind.
    W work;
    State<DP> st;
    V4u q[W::L::KV], q_next[W::L::KV];
    Pages<T, kWhole> pages;
    auto table_of = [&](const Row& row) { return a.table + (int64_t)max(row.seq, 0) * a.table_stride; };
    auto keys_of = [&](int32_t hh) { return static_cast<const T*>(a.k) + hh / a.blocks * a.head_stride; };
    auto values_of = [&](int32_t hh) { return static_cast<const T*>(a.v) + hh / a.blocks * a.head_stride; };

    load_queries<T, DP>(a, cur.r, job_at(a, cur.hh), lane, q);
    pages.ask(a, cur.row, table_of(cur.row), cur.row.begin(cur.i, TILE), lane);
    Places<T, kWhole> p = pages.places(a, cur.row, cur.row.begin(cur.i, TILE));
    work.load_keys(a, keys_of(cur.hh), p, lane);
    work.load_values(a, values_of(cur.hh), p, lane);
    Cursor nxt = cur;
    if (left > 1) {
        nxt.next<TILE>(a);
        pages.ask(a, nxt.row, table_of(nxt.row), nxt.row.begin(nxt.i, TILE), lane);
    }
    st.clear();
    int32_t first = cur.i;                // of this row in this share
    while (true) {
        const bool more = left > 1, turns = cur.i + 1 == cur.row.tiles;
        Places<T, kWhole> pn = p;
        Cursor far = nxt;
        if (more) {
            pn = pages.places(a, nxt.row, nxt.row.begin(nxt.i, TILE));
            if (turns) load_queries<T, DP>(a, nxt.r, job_at(a, nxt.hh), lane, q_next);
            if (left > 2) {
                far.next<TILE>(a);
                pages.ask(a, far.row, table_of(far.row), far.row.begin(far.i, TILE), lane);
            }
        }
        float x[W::VROWS];
        work.scores(a, q, p.seen, lane, x);
        if (more) work.load_keys(a, keys_of(nxt.hh), pn, lane);
        if (p.seen != (TILE == 32 ? ~0u : 0xFFFFu)) work.drop_unseen_values(p.seen, lane);
        work.fold(st, x);
        if (more) work.load_values(a, values_of(nxt.hh), pn, lane);

        if (turns || !more) {
            // the row, or this share of it, is done
            const Job job = job_at(a, cur.hh);
            const int head = lane & 15;
            const bool begins = first == 0;
            const float l = sum_over_lanes(st.l);
            const int64_t index = (int64_t)cur.r * (a.heads * a.blocks) + cur.hh;
            if (begins && lane == 0) {
                // which shares hold the rest of it
                const int64_t stop = at + (share - left) - cur.i + cur.row.tiles - 1;
                a.joins[index] = int2{me, turns ? me : shares.of(stop)};
            }
            if (head < job.heads) {
                const int d0 = DP / 16 * 4 * (lane >> 4);
                if (begins && turns) {
                    T* const out = out_row<T>(a, cur.r, job.head0 + head);
                    const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int b = 0; b < DP / 16; b += 4) {
                            const int d = d0 + DP / 16 * e + b;
                            if (d < a.dim)
                                store4<T>(out + d, l == 0.f ? V4f{0.f, 0.f, 0.f, 0.f}
                                                            : V4f{st.o[b][e], st.o[b + 1][e], st.o[b + 2][e], st.o[b + 3][e]} * f);
                        }
                    if (lane < 16) write_lse(a, cur.r, job.head0 + head, st.m, l);
                } else {
                    float* const part = a.parts + (2 * (int64_t)me + (begins ? 1 : 0)) * attend_part_floats(a.dim);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int b = 0; b < DP / 16; b += 4) {
                            const int d = d0 + DP / 16 * e + b;
                            if (d < a.dim)
                                *reinterpret_cast<V4f*>(part + 2 * kAttendHeads + head * a.dim + d) =
                                    V4f{st.o[b][e], st.o[b + 1][e], st.o[b + 2][e], st.o[b + 3][e]};
                        }
                    if (lane < 16) {
                        part[head] = st.m;
                        part[kAttendHeads + head] = l;
                    }
                }
            }
            if (!more) break;
            st.clear();
            first = 0;
#pragma unroll
            for (int i = 0; i < W::L::KV; ++i) q[i] = q_next[i];
        }
        p = pn;
        cur = nxt;
        nxt = far;
        --left;
    }
}

// A workgroup to a row and key-value head: its waves take every WAVES-th tile, and
// their pieces join in shared memory.
template <typename T, int DP, bool kWhole, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP == 256 || WAVES == 8 ? 1 : 2) void k_attend_short(AttendArgs a)
{
    typedef Work<T, DP, kWhole> W;
    constexpr int TILE = Tile<T>::n;
    __shared__ float s_o[WAVES][kAttendHeads][DP + 4];
    __shared__ float s_m[WAVES][kAttendHeads], s_l[WAVES][kAttendHeads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, head = lane & 15;
    const int32_t each = a.heads * a.blocks, r = blockIdx.x / each, hh = blockIdx.x - r * each;
    const Job job = job_at(a, hh);
    V4u q[W::L::KV];
    load_queries<T, DP>(a, r, job, lane, q);
    const Row row = row_at<TILE>(a, r);
    const int32_t* const table = a.table + (int64_t)max(row.seq, 0) * a.table_stride;
    const T* const keys = static_cast<const T*>(a.k) + job.kv * a.head_stride;
    const T* const values = static_cast<const T*>(a.v) + job.kv * a.head_stride;
    State<DP> st;
    st.clear();
    int32_t i = __builtin_amdgcn_readfirstlane(wave);
    if (i < row.tiles) {
        W work;
        Pages<T, kWhole> pages;
        pages.ask(a, row, table, row.begin(i, TILE), lane);
        Places<T, kWhole> p = pages.places(a, row, row.begin(i, TILE));
        work.load_keys(a, keys, p, lane);
        work.load_values(a, values, p, lane);
        if (i + WAVES < row.tiles) pages.ask(a, row, table, row.begin(i + WAVES, TILE), lane);
        while (true) {
            const bool more = i + WAVES < row.tiles;
            Places<T, kWhole> pn = p;
            if (more) {
                pn = pages.places(a, row, row.begin(i + WAVES, TILE));
                if (i + 2 * WAVES < row.tiles) pages.ask(a, row, table, row.begin(i + 2 * WAVES, TILE), lane);
            }
            float x[W::VROWS];
            work.scores(a, q, p.seen, lane, x);
            if (more) work.load_keys(a, keys, pn, lane);
            if (p.seen != (TILE == 32 ? ~0u : 0xFFFFu)) work.drop_unseen_values(p.seen, lane);
            work.fold(st, x);
            if (!more) break;
            work.load_values(a, values, pn, lane);
            p = pn;
            i += WAVES;
        }
    }
    const float l = sum_over_lanes(st.l);
    if (lane < 16) {
        s_m[wave][lane] = st.m;
        s_l[wave][lane] = l;
    }
    if (head < job.heads) {
#pragma unroll
        for (int b = 0; b < DP / 16; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_o[wave][head][DP / 16 * (4 * (lane >> 4) + e) + b] = st.o[b][e];
    }
    __syncthreads();
    for (int x = tid; x < job.heads * a.dim; x += 64 * WAVES) {
        const int g = x / a.dim, d = x - g * a.dim;
        float m = s_m[0][g];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, s_m[w][g]);
        const float base = m == -__builtin_inff() ? 0.f : m;
        float sum = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = weight<T>(s_m[w][g] - base);
            sum += f * s_l[w][g];
            o += f * s_o[w][g][d];
        }
        out_row<T>(a, r, job.head0 + g)[d] = rounded<T>(sum == 0.f ? 0.f : o / sum);
        if (d == 0) write_lse(a, r, job.head0 + g, m, sum);
    }
}

// Joins the pieces of a row and head that lie in more than one share: the second
// part of the share it begins in and the first parts of the ones behind it.  Eight
// groups of threads take every eighth piece, four dims a thread, each with a
// running maximum of its own, and join in shared memory: two trips to memory.
constexpr int kJoinGroups = 8;
constexpr int kMaxDim = 256;

template <typename T>
__global__ __launch_bounds__(kThreads) void k_attend_join(AttendArgs a)
{
    __shared__ float s_m[kJoinGroups], s_l[kJoinGroups];
    __shared__ V4f s_o[kJoinGroups][kMaxDim / 4];
    const int32_t each = a.heads * a.blocks, tid = threadIdx.x;
    const int64_t size = attend_part_floats(a.dim);
    const int quads = a.dim / 4, groups = min(kJoinGroups, kThreads / quads), group = tid / quads, d4 = tid - group * quads;
    for (int64_t index = blockIdx.x; index < (int64_t)a.rows * each; index += gridDim.x) {
        const int2 held = a.joins[index];
        const int32_t pieces = held.y - held.x + 1;
        if (pieces == 1) continue;
        const int32_t r = (int32_t)quotient(index, each);
        const Job job = job_at(a, (int32_t)(index - (int64_t)r * each));
        const float* const first = a.parts + (2 * (int64_t)held.x + 1) * size;
        for (int g = blockIdx.y; g < job.heads; g += gridDim.y) {
            float m = -__builtin_inff(), l = 0.f;
            V4f o = {0.f, 0.f, 0.f, 0.f};
            if (group < groups)
#pragma unroll 4
                for (int32_t i = group; i < pieces; i += groups) {
                    const float* const part = i == 0 ? first : first + (2 * (int64_t)i - 1) * size;
                    const float mi = part[g], li = part[kAttendHeads + g];
                    const V4f oi = *reinterpret_cast<const V4f*>(part + 2 * kAttendHeads + g * a.dim + 4 * d4);
                    const float top = fmaxf(m, mi), base = top == -__builtin_inff() ? 0.f : top;
                    const float f = weight<T>(m - base), fi = weight<T>(mi - base);
                    l = l * f + li * fi;
                    o = o * f + oi * fi;
                    m = top;
                }
            if (group < groups) {
                s_o[group][d4] = o;
                if (d4 == 0) {
                    s_m[group] = m;
                    s_l[group] = l;
                }
            }
            __syncthreads();
            if (tid < quads) {
                for (int i = 1; i < groups; ++i) m = fmaxf(m, s_m[i]);
                const float base = m == -__builtin_inff() ? 0.f : m;
                l = 0.f;
                o = V4f{0.f, 0.f, 0.f, 0.f};
                for (int i = 0; i < groups; ++i) {
                    const float f = weight<T>(s_m[i] - base);
                    l += s_l[i] * f;
                    o += s_o[i][tid] * f;
                }
                const float f = l == 0.f ? 0.f : 1.f / l;
                store4<T>(out_row<T>(a, r, job.head0 + g) + 4 * tid, l == 0.f ? V4f{0.f, 0.f, 0.f, 0.f} : o * f);
                if (tid == 0) write_lse(a, r, job.head0 + g, m, l);
            }
            __syncthreads();
        }
    }
}

template <typename T, int DP, bool kWhole>
hipError_t attend_shares(const AttendArgs& a, int64_t jobs, hipStream_t s)
{
    const dim3 block(kThreads);
    hipLaunchKernelGGL((k_attend<T, DP, kWhole>), dim3((unsigned)a.groups), block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_attend_join<T>, dim3((unsigned)std::min(jobs, kMaxGrid), (unsigned)std::min(a.group, kAttendHeads)),
                       block, 0, s, a);
    return hipGetLastError();
}

// Tiles of the longest row up to which a workgroup takes a row (and head), with few rows
// and heads, and with so many that they nearly fill the GPU: shares balance any lengths,
// but cost a search and a second launch, 6 to 8 us.  us by shares and so, 32 heads on 8, rows
// as long as the table, and where two numbers follow, of 1/30 to all of it:
//   head_dim  64, bf16:   1 row of 1,200  10.9, 10.4    1 of 1,600  11.4, 12.2    32 of 1,700  24, 21 (17, 15)
//   head_dim 128, bf16:   1 row of 800    12.3, 12.0    1 of 1,000  11.8, 14.9    32 of 1,200  31, 28 (21, 19)
//   head_dim 128, fp32:   1 row of 250    12.2, 11.0    1 of 500    13.2, 19.5    32 of 500    35, 27 (23, 21)
//   head_dim 256, bf16:   1 row of 200    14.8, 12.4    1 of 300    13.3, 15.6    32 of 500    32, 27 (23, 21)
struct RowTiles {
    int32_t few, many;
};
template <typename T, int DP>
constexpr RowTiles kRowTiles = DP == 256                          ? RowTiles{8, 16}
                               : std::is_same<T, uint16_t>::value ? (DP == 64 ? RowTiles{40, 64} : RowTiles{26, 40})
                                                                  : (DP == 64 ? RowTiles{32, 64} : RowTiles{20, 32});
constexpr int64_t kManyJobs = 160;
// Tiles from which on eight waves share a row, where one such workgroup a CU is enough:
// 1 row of 500 of head_dim 64 6.4 us by four and 6.0 by eight, 32 rows of 800 13.6 and
// 12.0, but 64 rows of 400 of head_dim 128 20.7 and 23.8.  The widest fp32 pieces take
// longer to join than they save (250 positions of head_dim 128: 11.0 and 11.8).
template <typename T, int DP> constexpr int kEightWaves = std::is_same<T, float>::value && DP == 128 ? 16 : 4;
constexpr int64_t kEightJobs = 256;

// Tiles a row has at most: its table's, or its window's and sinks'.  A window begins
// inside a tile and may end inside another.  us by the table's alone (shares) and so,
// rows of 4,000 in bf16, 32 heads on 8 of 128, 4 sinks: 1 row, window of 193  11.5, 5.8;
// 32 rows, 449  19.8, 12.1;  96 rows, 449  45.4, 32.2, and 1,217  87.6, 72.8.
template <int TILE>
int64_t most_tiles(const AttendArgs& a)
{
    const int64_t table = ((int64_t)a.width * a.page_size + TILE - 1) / TILE;
    if (a.window == 0) return table;
    const int64_t window = ((int64_t)a.window + 2 * TILE - 2) / TILE, sinks = ((int64_t)a.sinks + TILE - 1) / TILE;
    return std::min(table, window + sinks);
}

template <typename T, int DP, bool kWhole>
hipError_t attend_as(const AttendArgs& a, hipStream_t s)
{
    const int64_t jobs = (int64_t)a.rows * a.heads * a.blocks;
    const int64_t most = most_tiles<Tile<T>::n>(a);
    if (jobs > kMaxGrid || most > (jobs >= kManyJobs ? kRowTiles<T, DP>.many : kRowTiles<T, DP>.few))
        return attend_shares<T, DP, kWhole>(a, jobs, s);
    if constexpr (DP <= 128) {            // eight waves of the widest heads would not fit the registers
        if (most > kEightWaves<T, DP> && jobs <= kEightJobs) {
            hipLaunchKernelGGL((k_attend_short<T, DP, kWhole, 8>), dim3((unsigned)jobs), dim3(512), 0, s, a);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((k_attend_short<T, DP, kWhole, 4>), dim3((unsigned)jobs), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t attend_dim(const AttendArgs& a, hipStream_t s)
{
    return a.page_size % 16 == 0 ? attend_as<T, DP, true>(a, s) : attend_as<T, DP, false>(a, s);
}

template <typename T>
hipError_t attend_t(const AttendArgs& a, hipStream_t s)
{
    if (a.dim <= 64) return attend_dim<T, 64>(a, s);
    if (a.dim <= 128) return attend_dim<T, 128>(a, s);
    return attend_dim<T, 256>(a, s);
}

}  // namespace

hipError_t launch_attend(int dtype, const AttendArgs& a, hipStream_t s)
{
    return dtype == 0 ? attend_t<uint16_t>(a, s) : attend_t<float>(a, s);
}

}  // namespace cpes
