// cpes_tree.hip -- gfx950 kernels of the attention of several new tokens per sequence,
// a tree or a chain of them, over a paged key-value cache.
//
// Mathematics.  As in cpes_attend.hip, for every query (a new token's query head): scores
// x_j = scale q k_j over the positions it sees, a running maximum m, l = sum e^(x - m) and o =
// sum e^(x - m) v, rescaled as m grows; pieces (m, l, o) of any split of the positions join
// the same way.  A query sees the b tokens in front of the new ones, as far as its window
// reaches, and of the new ones its ancestors and itself: a bit each, found by walking up
// the parents once.
//
// Tiles.  A wave takes 32 positions (16 in fp32) at a time and one or two sets of 16
// queries, which use the keys and values that it holds in registers in the layout of
// cpes_attend.hpp: S^T = K Q^T leaves the weights where O^T = V^T P^T wants them.  With more
// queries up to four waves of a workgroup take the same positions and other queries, and
// the first one's loads leave the others' in the caches.  Two sets are for bf16 up to 128 dims
// (8 nodes on 64 rows of 8,000, when they were chosen: 440 us, 476 with one; now 383).  In fp32 they
// leave room for one wave a SIMD (32 nodes on 8 rows of 8,000: 505 us, 378 with one), and above 128
// dims they spill (16 nodes of 256 in bf16 340 us and 203, in fp32 2,520 and 502).  Above 32 queries a bf16 cache
// goes through shared memory (below, "many queries").  The weights of a bf16 cache go in as a
// bf16 value and its remainder, as there: a bf16 weight alone is off by 2^-9, which the
// outputs of long contexts would show.
//
// What a tile's queries see differs only where the new tokens are and at the edges of
// windows.  Such tiles mask scores per query.  A value that one query sees and another does
// not may be infinite or NaN, and 0 times it is not 0: where that is so, those positions
// are left out of the matrix products and added by themselves.
//
// Work.  Either a workgroup does a job (the queries of a row's piece and KV head that go
// together), or the jobs' tiles are laid in a line, cut into as many shares as workgroups are
// resident, and what lies in several shares is joined by a second launch.
#include <algorithm>
#include <type_traits>

#include "cpes_attend.hpp"

namespace cpes {

namespace {

constexpr int kWaves = kAttendWaves;
constexpr int kThreads = 64 * kWaves;
constexpr int64_t kMaxGrid = 1 << 20;
constexpr int kWords = kMaxTree / 32;

// A row's sequence and new tokens.
struct Row {
    int32_t seq;
    int32_t first;        // its tokens' first row of q and out
    int32_t tokens;       // 0: left out
    int32_t base;         // tokens in front of them; negative: the sequence does not have them
};

__device__ __forceinline__ Row row_at(const TreeArgs& a, int32_t r)
{
    Row x;
    const int64_t begin = a.starts[r], tokens = (int64_t)a.starts[r + 1] - begin;
    const bool there = begin >= 0 && tokens > 0 && tokens <= a.longest && begin + tokens <= a.tokens;
    x.first = (int32_t)begin;
    x.tokens = there ? (int32_t)tokens : 0;
    x.seq = a.seqs ? a.seqs[r] : r;
    x.base = -1;
    if (x.seq >= 0 && x.seq < a.sequences) {
        const int64_t cap = (int64_t)a.width * a.page_size;
        const int32_t most = cap > INT32_MAX - 64 ? INT32_MAX - 64 : (int32_t)cap;
        x.base = max(min(max(a.lengths[x.seq], 0), most) - x.tokens, -1);
    }
    if (x.base < 0) x.seq = 0;
    return x;
}

// A job: `count` tokens of a row from token `from` on, for one block of one key-value
// head's query heads, and the tiles of positions that any of them sees: [0, sink_tiles)
// from position 0 on, the rest from `begin`.
struct Span {
    int32_t from, count;
    int32_t end;          // positions behind which nothing is seen
    int32_t sink_tiles, begin;
    int32_t tiles;        // at least one: what sees nothing is written too

    __device__ __forceinline__ int32_t at(int32_t i, int tile) const
    {
        return i < sink_tiles ? i * tile : begin + (i - sink_tiles) * tile;
    }
};

template <int TILE> __device__ __forceinline__ Span span_at(const TreeArgs& a, const Row& row, int32_t piece)
{
    Span x;
    x.from = piece * a.job_tokens;
    x.count = min(a.job_tokens, row.tokens - x.from);
    x.end = row.base < 0 ? 0 : row.base + x.from + x.count;
    x.sink_tiles = 0;
    x.begin = 0;
    if (a.window > 0 && x.end > 0) {
        // the first position that the window of any of them reaches: in a tree all may hang from the context
        const int64_t low = (int64_t)row.base + (a.parents ? 0 : x.from) + 1 - a.window;
        if (low > 0) {
            const int32_t begin = (int32_t)(low / TILE), sinks = min((a.sinks - 1) / TILE + (a.sinks > 0), begin);
            if (sinks < begin) {
                x.sink_tiles = sinks;
                x.begin = begin * TILE;
            }
        }
    }
    x.tiles = max(1, x.sink_tiles + (x.end - x.begin + TILE - 1) / TILE);
    return x;
}

__device__ __forceinline__ int32_t pieces_of(const TreeArgs& a, const Row& row)
{
    return (row.tokens + a.job_tokens - 1) / a.job_tokens;
}

template <int TILE> __device__ __forceinline__ int64_t row_tiles(const TreeArgs& a, const Row& row)
{
    int64_t sum = 0;
    const int32_t n = pieces_of(a, row);
    for (int32_t i = 0; i < n; ++i) sum += span_at<TILE>(a, row, i).tiles;
    return sum;
}

// The page ids of a tile's positions, asked for before they are needed.
template <typename T, bool kWhole> struct Pages {
    static constexpr int SUB = Tile<T>::n / 16;
    int32_t id[SUB], slot[SUB];

    __device__ __forceinline__ void ask(const TreeArgs& a, int32_t end, const int32_t* table, int32_t pos0, int lane)
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            const int32_t pos = pos0 + 16 * u + (kWhole ? 0 : lane & 15);
            const int32_t at = a.page_shift >= 0 ? pos >> a.page_shift : pos / a.page_size;
            slot[u] = pos - at * a.page_size;
            id[u] = -1;
            if (pos < end) id[u] = table[at];            // end is at most what the table holds
        }
    }

    // `seen`: positions that lie in front of `end` and have a page.
    __device__ __forceinline__ Places<T, kWhole> places(const TreeArgs& a, int32_t end, int32_t pos0)
    {
        Places<T, kWhole> p;
        p.seen = 0;
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            int32_t page = id[u];
            if constexpr (kWhole) page = __builtin_amdgcn_readfirstlane(page);
            const bool there = page >= 0 && page < a.pages;
            p.base[u] = there ? page * a.page_stride + slot[u] * a.token_stride : 0;
            if constexpr (kWhole)
                p.seen |= there ? 0xFFFFu << (16 * u) : 0u;
            else
                p.seen |= (uint32_t)(__ballot(there) & 0xFFFF) << (16 * u);
        }
        const int32_t left = end - pos0;
        if (left < 32) p.seen &= left > 0 ? (1u << left) - 1u : 0u;
        return p;
    }
};

// Bits [0, n) of 32.
__device__ __forceinline__ uint32_t bits_below(int32_t n)
{
    return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u;
}

// What a wave keeps in shared memory about its job's queries.
template <int NQ> struct Family {
    int16_t parent[kMaxTree];
    int32_t depth[16 * NQ];
    uint32_t above[16 * NQ][kWords + 1];  // ancestors and itself that the window lets through; the last word is 0
};

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <typename T, int DP, bool kWhole, int NQ> struct Work : Operands<T, DP, kWhole> {
    typedef Operands<T, DP, kWhole> O;
    typedef typename O::L L;
    using O::key;
    using O::val;
    using O::SUB;
    using O::TILE;
    using O::VROWS;
    static constexpr uint32_t kAll = TILE == 32 ? ~0u : 0xFFFFu;

    const TreeArgs& a;
    Family<NQ>& family;
    const int lane, sub;                  // of the waves beside each other

    Row row;
    Span span;
    int32_t kv, block;
    V4u q[NQ][L::KV];
    int32_t low[NQ], high[NQ];            // of the lane's queries: positions [low, high) are seen, and those before `sinks`
    bool valid[NQ];
    int32_t every_high, every_low;        // all of them see [every_low, every_high)
    State<DP> st[NQ];

    __device__ __forceinline__ Work(const TreeArgs& args, Family<NQ>& f, int l, int s) : a(args), family(f), lane(l), sub(s) {}

    __device__ __forceinline__ int32_t token_of(int32_t column) const { return column / a.job_heads; }

    __device__ __forceinline__ void begin(const Row& r, const Span& x, int32_t hh)
    {
        row = r;
        span = x;
        kv = hh / a.blocks;
        block = hh - kv * a.blocks;
        constexpr int E = 16 / sizeof(T);
        const bool tree = a.parents != nullptr;
        if (tree) {
            wave_sync();                  // the last job's are no longer read
            const int32_t last = span.from + span.count;
            for (int32_t i = lane; i < last; i += 64) {
                const int32_t parent = a.parents[row.first + i];
                family.parent[i] = (int16_t)(parent >= 0 && parent < i ? parent : -1);
            }
            wave_sync();
            if (lane < 16 * NQ) {
                const int32_t token = token_of(sub * 16 * NQ + lane);
                const int32_t i = span.from + min(token, span.count - 1);
                int32_t depth = 0;
                for (int32_t j = family.parent[i]; j >= 0; j = family.parent[j]) ++depth;
                family.depth[lane] = depth;
#pragma unroll
                for (int w = 0; w <= kWords; ++w) family.above[lane][w] = 0;
                int32_t at = depth;
                for (int32_t j = i; j >= 0; j = family.parent[j], --at)
                    if (a.window == 0 || depth - at < a.window || (int64_t)row.base + at < a.sinks)
                        family.above[lane][j >> 5] |= 1u << (j & 31);
            }
            wave_sync();
        }
        every_low = 0;
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const int32_t column = (sub * NQ + s) * 16 + (lane & 15), token = token_of(column);
            const int32_t head = block * a.job_heads + column - token * a.job_heads;
            valid[s] = token < span.count && head < a.group;
            const int32_t i = span.from + min(token, span.count - 1);
            const int32_t depth = tree ? family.depth[s * 16 + (lane & 15)] : i;
            high[s] = row.base < 0 ? 0 : tree ? row.base : row.base + i + 1;
            // below 0 where the window holds all
            low[s] = a.window > 0 && row.base >= 0 ? (int32_t)max((int64_t)row.base + depth + 1 - a.window, (int64_t)0) : 0;
            const T* const p = static_cast<const T*>(a.q) + (int64_t)(row.first + i) * a.q_stride +
                               (int64_t)(kv * a.group + min(head, a.group - 1)) * a.q_head_stride;
#pragma unroll
            for (int e = 0; e < L::KV; ++e) {
                const int d = E * (lane >> 4) + 4 * E * e;
                q[s][e] = *reinterpret_cast<const V4uAnywhere*>(p + (d < a.dim ? d : 0));
                if (d >= a.dim || !valid[s]) q[s][e] = V4u{0, 0, 0, 0};
            }
            st[s].clear();
        }
        every_high = row.base < 0 ? 0 : tree ? row.base : row.base + span.from + 1;
        if (a.window > 0 && row.base >= 0)
            every_low = (int32_t)max((int64_t)row.base + (tree ? span.from + span.count : span.from + span.count - 1) + 1 - a.window, (int64_t)0);
    }

    // Whether all queries see all of a tile's positions that have a page.
    __device__ __forceinline__ bool whole(int32_t pos0) const
    {
        return pos0 + TILE <= every_high && (pos0 >= every_low || pos0 + TILE <= a.sinks);
    }

    // Positions of the tile that set s's query of this lane sees.
    __device__ __forceinline__ uint32_t seen_by(int s, int32_t pos0) const
    {
        uint32_t seen = bits_below(high[s] - pos0) & ~(bits_below(low[s] - pos0) & ~bits_below(a.sinks - pos0));
        if (a.parents && row.base >= 0) {
            const int32_t off = pos0 - row.base;
            if (off > -32 && off < kMaxTree) {
                const int32_t w = off >> 5, shift = off & 31;
                const uint32_t* const above = family.above[s * 16 + (lane & 15)];
                const uint32_t lo = w >= 0 ? above[w] : 0u, hi = above[w + 1];
                seen |= shift ? lo >> shift | hi << (32 - shift) : lo;
            }
        }
        return valid[s] ? seen : 0u;
    }

    // Scores of the tile: x[4 u + r] is position 16 u + 4 (lane / 16) + r.
    __device__ __forceinline__ void scores(int s, float x[VROWS])
    {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
            V4f t;
            if constexpr (std::is_same<T, uint16_t>::value) {
                t = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::KV; ++i)
                    t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8bf, key[u][i]),
                                                                __builtin_bit_cast(V8bf, q[s][i]), t, 0, 0, 0);
            } else {
                // four sums: a quarter of the roundings in line, and of the instructions that wait for each other
                V4f part[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) part[e] = V4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < L::KV; ++i) {
                    const V4f k4 = __builtin_bit_cast(V4f, key[u][i]), q4 = __builtin_bit_cast(V4f, q[s][i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[e], q4[e], part[e], 0, 0, 0);
                }
                t = (part[0] + part[1]) + (part[2] + part[3]);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * u + r] = t[r] * a.scale;
        }
    }

    __device__ __forceinline__ void hide(uint32_t seen, float x[VROWS])
    {
#pragma unroll
        for (int j = 0; j < VROWS; ++j)
            if (!(seen >> (16 * (j >> 2) + 4 * (lane >> 4) + (j & 3)) & 1)) x[j] = -__builtin_inff();
    }

    // Scores to weights, and the state's sums moved to the new maximum.
    __device__ __forceinline__ void weigh(int s, float x[VROWS])
    {
        State<DP>& t = st[s];
        float top = x[0];
#pragma unroll
        for (int j = 1; j < VROWS; ++j) top = fmaxf(top, x[j]);
        const float m = fmaxf(t.m, max_over_lanes(top));
        // nothing seen yet: any finite base gives weights of 0
        const float base = m == -__builtin_inff() ? 0.f : m;
        const float keep = weight<T>(t.m - base);
        float l = 0.f;
#pragma unroll
        for (int j = 0; j < VROWS; ++j) {
            x[j] = weight<T>(x[j] - base);
            l += x[j];
        }
        t.l = t.l * keep + l;
        t.m = m;
        if (__any(keep != 1.f)) {
#pragma unroll
            for (int b = 0; b < DP / 16; ++b) t.o[b] *= keep;
        }
    }

    // Positions of the tile whose values, seen by some and not by others, are not finite.
    __device__ __forceinline__ uint32_t odd_values(uint32_t partly) const
    {
        uint32_t odd = 0;
#pragma unroll
        for (int j = 0; j < VROWS; ++j) {
            bool here = false;
#pragma unroll
            for (int i = 0; i < L::VD; ++i) {
                const uint32_t v = val[j][i];
                if constexpr (std::is_same<T, uint16_t>::value)
                    here |= (v & 0x7F80u) == 0x7F80u || (v & 0x7F800000u) == 0x7F800000u;
                else
                    here |= (v & 0x7F800000u) == 0x7F800000u;
            }
            const uint64_t those = __ballot(here);
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (those >> (16 * g) & 0xFFFF) odd |= 1u << (16 * (j >> 2) + 4 * g + (j & 3));
        }
        return odd & partly;
    }

    // The tile's values, as the left operand of block b of the second product (bf16).
    __device__ __forceinline__ V8bf values8(int b) const
    {
        V4u v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = __builtin_amdgcn_perm(val[2 * i + 1][b >> 1], val[2 * i][b >> 1], b & 1 ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(V8bf, v);
    }

    // Block b of the product of the values with set s's weights, added to o.
    __device__ __forceinline__ V4f product(int b, const float x[VROWS], V8bf hi, V8bf lo, V4f o) const
    {
        if constexpr (std::is_same<T, uint16_t>::value) {
            const V8bf v8 = values8(b);
            o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, hi, o, 0, 0, 0);
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, lo, o, 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(val[j][b]), x[j], o, 0, 0, 0);
            return o;
        }
    }

    // Folds the tile into the state: scores, weights, and the products with the values.
    // `next` is called when the keys are no longer needed.
    template <typename F> __device__ __forceinline__ void tile(const Places<T, kWhole>& p, int32_t pos0, const T* values, F next)
    {
        float x[NQ][VROWS];
#pragma unroll
        for (int s = 0; s < NQ; ++s) scores(s, x[s]);
        next();
        uint32_t some = kAll, odd = 0, seen[NQ];
        const bool all = p.seen == kAll && whole(pos0);
        if (!all) {
            uint32_t every = ~0u;
            some = 0;
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                seen[s] = seen_by(s, pos0) & p.seen;
                hide(seen[s], x[s]);
                some |= seen[s];
                every &= valid[s] ? seen[s] : ~0u;
            }
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) {
                some |= __shfl_xor(some, d);
                every &= __shfl_xor(every, d);
            }
            odd = odd_values(some & ~every);
            this->drop_unseen_values(some & ~odd, lane);
        }
#pragma unroll
        for (int s = 0; s < NQ; ++s) weigh(s, x[s]);
        V8bf hi[NQ], lo[NQ];
        if constexpr (std::is_same<T, uint16_t>::value) {
#pragma unroll
            for (int s = 0; s < NQ; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hi[s][j] = (__bf16)x[s][j];
                    lo[s][j] = (__bf16)(x[s][j] - (float)hi[s][j]);
                }
        }
#pragma unroll
        for (int b = 0; b < DP / 16; ++b)
#pragma unroll
            for (int s = 0; s < NQ; ++s) st[s].o[b] = product(b, x[s], hi[s], lo[s], st[s].o[b]);
        // the odd positions one by one: their products reach only the queries that see them
        while (__builtin_expect(odd != 0, 0)) {
            const int j = __builtin_amdgcn_readfirstlane(__ffs(odd) - 1);
            odd &= odd - 1;
            this->template load_values<false>(a, values, p, lane);
            this->drop_unseen_values(1u << j, lane);
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                const bool sees = seen[s] >> j & 1;
#pragma unroll
                for (int b = 0; b < DP / 16; ++b) {
                    const V4f o = product(b, x[s], hi[s], lo[s], V4f{0.f, 0.f, 0.f, 0.f});
                    if (sees) st[s].o[b] += o;
                }
            }
        }
    }

    // The row of q and out, and the query head, of set s's query of this lane.
    __device__ __forceinline__ void place_of(int s, int32_t* token, int32_t* head) const
    {
        const int32_t column = (sub * NQ + s) * 16 + (lane & 15), t = token_of(column);
        *token = row.first + span.from + t;
        *head = kv * a.group + block * a.job_heads + column - t * a.job_heads;
    }

    __device__ __forceinline__ void write_out()
    {
        const int d0 = DP / 16 * 4 * (lane >> 4);
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const float l = sum_over_lanes(st[s].l);
            if (!valid[s]) continue;
            int32_t token, head;
            place_of(s, &token, &head);
            T* const out = static_cast<T*>(a.out) + (int64_t)token * a.out_stride + (int64_t)head * a.out_head_stride;
            const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < DP / 16; b += 4) {
                    const int d = d0 + DP / 16 * e + b;
                    if (d < a.dim)
                        store4<T>(out + d, l == 0.f ? V4f{0.f, 0.f, 0.f, 0.f}
                                                    : V4f{st[s].o[b][e], st[s].o[b + 1][e], st[s].o[b + 2][e], st[s].o[b + 3][e]} * f);
                }
            if (lane < 16 && a.lse)
                a.lse[(int64_t)token * a.heads * a.group + head] = l == 0.f ? -__builtin_inff() : st[s].m + logf(l);
        }
    }

    __device__ __forceinline__ void write_part(float* part)
    {
        const int d0 = DP / 16 * 4 * (lane >> 4);
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            const float l = sum_over_lanes(st[s].l);
            const int column = s * 16 + (lane & 15);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < DP / 16; b += 4) {
                    const int d = d0 + DP / 16 * e + b;
                    if (d < a.dim)
                        *reinterpret_cast<V4f*>(part + 32 * NQ + column * a.dim + d) =
                            V4f{st[s].o[b][e], st[s].o[b + 1][e], st[s].o[b + 2][e], st[s].o[b + 3][e]};
                }
            if (lane < 16) {
                part[column] = st[s].m;
                part[16 * NQ + column] = l;
            }
        }
    }
};

// A row as a wave goes through it, in scalar registers.
__device__ __forceinline__ Row wave_row(const TreeArgs& a, int32_t r)
{
    const Row x = row_at(a, r);
    return Row{__builtin_amdgcn_readfirstlane(x.seq), __builtin_amdgcn_readfirstlane(x.first),
               __builtin_amdgcn_readfirstlane(x.tokens), __builtin_amdgcn_readfirstlane(x.base)};
}

// A tile of the line: row, piece of its tokens, key-value head and block, and its place in the job.
struct Cursor {
    Row row;
    Span span;
    int32_t r, piece, hh, i;

    template <int TILE> __device__ __forceinline__ void next(const TreeArgs& a)
    {
        if (++i < span.tiles) return;
        i = 0;
        if (++piece * a.job_tokens >= row.tokens) {
            piece = 0;
            do {
                if (++r == a.rows) {
                    r = 0;
                    ++hh;
                }
                row = wave_row(a, r);
            } while (row.tokens == 0);    // one row at least has tokens
        }
        span = span_at<TILE>(a, row, piece);
    }
};

__device__ __forceinline__ int64_t job_index(const TreeArgs& a, int32_t r, int32_t piece, int32_t hh)
{
    return ((int64_t)r * a.pieces + piece) * (a.heads * a.blocks) + hh;
}

// Every row's tiles: a thread's share of them before, and after, its rows.
template <int TILE, int WAVES> struct Line {
    int32_t r0, r1;
    int64_t mine, upto, tiles;

    // All threads.
    __device__ __forceinline__ Line(const TreeArgs& a, int64_t* s_sum)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int32_t each = (a.rows + 64 * WAVES - 1) / (64 * WAVES);
        r0 = min(a.rows, tid * each);
        r1 = min(a.rows, r0 + each);
        mine = 0;
        for (int32_t r = r0; r < r1; ++r) mine += row_tiles<TILE>(a, row_at(a, r));
        upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t y = __shfl_up(upto, d);
            if (lane >= d) upto += y;
        }
        if (lane == 63) s_sum[wave] = upto;
        __syncthreads();
        tiles = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) upto += s_sum[w];
            tiles += s_sum[w];
        }
    }

    // The thread that holds tile t of the rows' says in which of them it lies, and what is before that row.
    __device__ __forceinline__ void find(const TreeArgs& a, int64_t t, int32_t* s_row, int64_t* s_before) const
    {
        if (t < upto - mine || t >= upto) return;
        int64_t before = upto - mine;
        int32_t r = r0;
        for (; r < r1; ++r) {
            const int64_t n = row_tiles<TILE>(a, row_at(a, r));
            if (t < before + n) break;
            before += n;
        }
        *s_row = r;
        *s_before = before;
    }
};

// All jobs' tiles form one line, cut into equal shares, one for `beside` waves.
template <typename T, int DP, bool kWhole, int NQ>
__global__ __launch_bounds__(kThreads, DP == 256 || NQ > 1 ? 1 : 2) void k_tree(TreeArgs a)
{
    typedef Work<T, DP, kWhole, NQ> W;
    constexpr int TILE = Tile<T>::n;
    __shared__ Family<NQ> s_family[kWaves];
    __shared__ int64_t s_sum[kWaves], s_before[kWaves];
    __shared__ int32_t s_row[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int teams = kWaves / a.beside, team = wave / a.beside, sub = wave - team * a.beside;

    const Line<TILE, kWaves> line(a, s_sum);
    const int64_t tiles = line.tiles, units = tiles * a.heads * a.blocks;
    constexpr int kShareTiles = 2 * NQ;
    const int32_t shares_n = (int32_t)max((int64_t)1, min((int64_t)a.groups * teams, units / kShareTiles));
    const bool apart = shares_n <= (int32_t)gridDim.x;
    const int32_t share0 = apart ? blockIdx.x : blockIdx.x * teams, step = apart ? gridDim.x : 1;
    const int32_t me = share0 + team * step;
    if (share0 >= shares_n || units == 0) return;
    const Shares shares(units, shares_n);
#pragma unroll 1
    for (int w = 0; w < teams; ++w) {
        const int32_t share = share0 + w * step;
        if (share >= shares_n) break;
        const int64_t at = shares.begin(share);
        line.find(a, at - quotient(at, tiles) * tiles, &s_row[w], &s_before[w]);
    }
    __syncthreads();
    if (me >= shares_n) return;
    const int64_t at = shares.begin(me), hh = quotient(at, tiles), t = at - hh * tiles;
    const int32_t share = __builtin_amdgcn_readfirstlane((int32_t)(shares.begin(me + 1) - at));
    int32_t left = share;
    if (left == 0) return;

    Cursor cur;
    cur.r = __builtin_amdgcn_readfirstlane(s_row[team]);
    cur.hh = __builtin_amdgcn_readfirstlane((int32_t)hh);
    cur.row = wave_row(a, cur.r);
    int64_t in_row = t - s_before[team];
    cur.piece = 0;
    cur.span = span_at<TILE>(a, cur.row, 0);
    while (in_row >= cur.span.tiles) {
        in_row -= cur.span.tiles;
        cur.span = span_at<TILE>(a, cur.row, ++cur.piece);
    }
    cur.piece = __builtin_amdgcn_readfirstlane(cur.piece);
    cur.i = __builtin_amdgcn_readfirstlane((int32_t)in_row);
    cur.span = span_at<TILE>(a, cur.row, cur.piece);

    W work(a, s_family[wave], lane, sub);
    Pages<T, kWhole> pages;
    auto table_of = [&](const Row& row) { return a.table + (int64_t)row.seq * a.table_stride; };
    auto keys_of = [&](int32_t hh) { return static_cast<const T*>(a.k) + hh / a.blocks * a.head_stride; };
    auto values_of = [&](int32_t hh) { return static_cast<const T*>(a.v) + hh / a.blocks * a.head_stride; };
    work.begin(cur.row, cur.span, cur.hh);
    pages.ask(a, cur.span.end, table_of(cur.row), cur.span.at(cur.i, TILE), lane);
    Places<T, kWhole> p = pages.places(a, cur.span.end, cur.span.at(cur.i, TILE));
    work.load_keys(a, keys_of(cur.hh), p, lane);
    work.template load_values<false>(a, values_of(cur.hh), p, lane);
    Cursor nxt = cur;
    if (left > 1) {
        nxt.next<TILE>(a);
        pages.ask(a, nxt.span.end, table_of(nxt.row), nxt.span.at(nxt.i, TILE), lane);
    }
    int32_t first = cur.i;                // of this job in this share
    while (true) {
        const bool more = left > 1, turns = cur.i + 1 == cur.span.tiles;
        Places<T, kWhole> pn = p;
        Cursor far = nxt;
        if (more) {
            pn = pages.places(a, nxt.span.end, nxt.span.at(nxt.i, TILE));
            if (left > 2) {
                far.next<TILE>(a);
                pages.ask(a, far.span.end, table_of(far.row), far.span.at(far.i, TILE), lane);
            }
        }
        work.tile(p, cur.span.at(cur.i, TILE), values_of(cur.hh),
                  [&] { if (more) work.load_keys(a, keys_of(nxt.hh), pn, lane); });
        if (more) work.template load_values<false>(a, values_of(nxt.hh), pn, lane);
        if (turns || !more) {
            // the job, or this share of it, is done
            const bool begins = first == 0;
            if (begins && lane == 0 && sub == 0) {
                // which shares hold the rest of it
                const int64_t stop = at + (share - left) - cur.i + cur.span.tiles - 1;
                a.joins[job_index(a, cur.r, cur.piece, cur.hh)] = int2{me, turns ? me : shares.of(stop)};
            }
            if (begins && turns)
                work.write_out();
            else
                work.write_part(a.parts + ((2 * (int64_t)me + (begins ? 1 : 0)) * a.beside + sub) * tree_part_floats(NQ, a.dim));
            if (!more) break;
            work.begin(nxt.row, nxt.span, nxt.hh);
            first = 0;
        }
        p = pn;
        cur = nxt;
        nxt = far;
        --left;
    }
}

// Row and piece of job slot j: a row's slots begin at starts / job_tokens + row, which
// leaves one too many here and there.
__device__ __forceinline__ bool find_job(const TreeArgs& a, int64_t j, int32_t* r, int32_t* piece)
{
    // the last row that begins at or before it: 64 of them looked at together
    const int lane = threadIdx.x & 63;
    auto begins = [&](int32_t x) { return (int64_t)(min(max(a.starts[x], 0), a.tokens) / a.job_tokens) + x; };
    int32_t lo = 0, n = a.rows;
    while (n > 1) {
        const int32_t step = (n + 63) / 64, x = lo + lane * step;
        const uint64_t before = __ballot(lane * step < n && begins(x) <= j);
        const int32_t last = before ? 63 - __clzll((long long)before) : 0;
        lo += last * step;
        n = min(step, n - last * step);
        if (step == 1) break;
    }
    *r = __builtin_amdgcn_readfirstlane(lo);
    *piece = __builtin_amdgcn_readfirstlane((int32_t)(j - begins(lo)));
    return *piece >= 0;
}

// A workgroup to a job: `beside` waves on the same positions, kWaves / beside of them
// taking turns at the tiles, whose pieces join in shared memory.
template <typename T, int DP, bool kWhole, int NQ>
__global__ __launch_bounds__(kThreads, DP == 256 || NQ > 1 ? 1 : 2) void k_tree_jobs(TreeArgs a)
{
    typedef Work<T, DP, kWhole, NQ> W;
    constexpr int TILE = Tile<T>::n;
    __shared__ Family<NQ> s_family[kWaves];
    __shared__ float s_o[kWaves / 2][16 * NQ][DP + 4];
    __shared__ float s_m[kWaves / 2][16 * NQ], s_l[kWaves / 2][16 * NQ];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), head = lane & 15;
    const int teams = kWaves / a.beside, team = wave / a.beside, sub = wave - team * a.beside;
    const int32_t each = a.heads * a.blocks, hh = blockIdx.x % each;
    const int64_t slots = gridDim.x / each;
    int32_t r, piece;
    if (!find_job(a, slots - 1 - blockIdx.x / each, &r, &piece)) return;
    const Row row = wave_row(a, r);
    if ((int64_t)piece * a.job_tokens >= row.tokens) return;
    const Span span = span_at<TILE>(a, row, piece);
    const int32_t* const table = a.table + (int64_t)row.seq * a.table_stride;
    W work(a, s_family[wave], lane, sub);
    work.begin(row, span, hh);
    const T* const keys = static_cast<const T*>(a.k) + work.kv * a.head_stride;
    const T* const values = static_cast<const T*>(a.v) + work.kv * a.head_stride;
    int32_t i = team;
    if (i < span.tiles) {
        Pages<T, kWhole> pages;
        pages.ask(a, span.end, table, span.at(i, TILE), lane);
        Places<T, kWhole> p = pages.places(a, span.end, span.at(i, TILE));
        work.load_keys(a, keys, p, lane);
        work.template load_values<false>(a, values, p, lane);
        if (i + teams < span.tiles) pages.ask(a, span.end, table, span.at(i + teams, TILE), lane);
        while (true) {
            const bool more = i + teams < span.tiles;
            Places<T, kWhole> pn = p;
            if (more) {
                pn = pages.places(a, span.end, span.at(i + teams, TILE));
                if (i + 2 * teams < span.tiles) pages.ask(a, span.end, table, span.at(i + 2 * teams, TILE), lane);
            }
            work.tile(p, span.at(i, TILE), values, [&] { if (more) work.load_keys(a, keys, pn, lane); });
            if (!more) break;
            work.template load_values<false>(a, values, pn, lane);
            p = pn;
            i += teams;
        }
    }
    // pieces join pairwise: the upper half of the teams hands its own to the lower
    for (int half = teams / 2; half > 0; half /= 2) {
        const bool gives = team >= half && team < 2 * half;
        const int slot = (gives ? team - half : team) * a.beside + sub;
        if (gives) {
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                const float l = sum_over_lanes(work.st[s].l);
                if (lane < 16) {
                    s_m[slot][s * 16 + lane] = work.st[s].m;
                    s_l[slot][s * 16 + lane] = l;
                }
#pragma unroll
                for (int b = 0; b < DP / 16; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s_o[slot][s * 16 + head][DP / 16 * (4 * (lane >> 4) + e) + b] = work.st[s].o[b][e];
            }
        }
        __syncthreads();
        if (team < half) {
#pragma unroll
            for (int s = 0; s < NQ; ++s) {
                State<DP>& t = work.st[s];
                const float mi = s_m[slot][s * 16 + head], top = fmaxf(t.m, mi), base = top == -__builtin_inff() ? 0.f : top;
                const float f = weight<T>(t.m - base), fi = weight<T>(mi - base);
                // this lane's share of l: the other piece's sum is whole, and a quarter of it its share
                t.l = t.l * f + (lane < 16 ? s_l[slot][s * 16 + head] * fi : 0.f);
                t.m = top;
#pragma unroll
                for (int b = 0; b < DP / 16; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        t.o[b][e] = t.o[b][e] * f + s_o[slot][s * 16 + head][DP / 16 * (4 * (lane >> 4) + e) + b] * fi;
            }
        }
        __syncthreads();
    }
    if (team == 0) work.write_out();
}

// ------------------------------------------------------------ many queries --
// bf16, more than 32 queries a job: the workgroup's waves share tiles of 64 positions in
// shared memory, 32 queries a wave, on the 32 x 32 matrix instruction.  A key and a value
// are read from memory once for up to 256 queries: eight waves, a workgroup a CU.  Up to 128
// queries four waves, two workgroups a CU; up to 64 of them two waves take a half of each
// tile for the same queries, and join at the end.
//
// The next tile goes straight into the other buffer while one is folded (through registers
// it took 32 of them, and as many instructions as the softmax).  A wave folds both halves of
// a tile together: their products interleave, one base serves both, and one's weights are
// taken beside the other's products (prompts 712 -> 656 us).  The values come out of shared
// memory turned, four positions of a dim to a lane, so no lane sorts them (109 -> 87 us for
// ragged trees of 12, with the next two).  The base of the weights moves only when it is 2^4
// behind, which in most tiles it is not, and saves scaling the outputs.
//
// Bound: 24 products of 32 clocks and about 150 vector instructions of 4 a wave and half a
// tile; a SIMD's two waves overlap them in part (matrix units 36 - 41 % busy, vector units 41 - 45 %).
// 8 prompts of up to 4,095 tokens, 32 heads on 8 of 128: 578 us, 617 TFLOP/s of the scores' and
// outputs' products, 925 with the remainders'.  4 rows of 65 - 131 thousand tokens with up to 64
// nodes: 571 us, of which the join is 15; 2.8 TB/s and 505 TFLOP/s.  Both vary by 5 % from one GPU to the
// next, and by 15 % with its clock.
typedef float V16f __attribute__((ext_vector_type(16)));
typedef float V2f __attribute__((ext_vector_type(2)));
typedef __bf16 V2bf __attribute__((ext_vector_type(2)));
typedef short V4s __attribute__((ext_vector_type(4)));

constexpr int kWideTile = 64;
constexpr int kWideShare = 4;             // tiles of a workgroup's share at least
constexpr int kWideColumns = 32;          // of a wave
constexpr float kAhead = 4.f;             // powers of 2 that a weight may be above 1, and that the outputs' range is short of

template <int DP, int WAVES> struct WideShared {
    // Rows in pieces of 16 bytes.  32 lanes read one piece each of as many keys, or 4 positions' values of 16 dims
    // twice: which piece stands where in a row depends on its number, so that they lie in different banks.
    uint16_t keys[2][kWideTile * DP];
    uint16_t values[2][kWideTile * DP];
    uint32_t odd[2];                      // positions with values that are not finite, where not all queries see all of a tile
    Family<2> family[WAVES];

    static __device__ __forceinline__ int key_swap(int r) { return DP == 128 ? r & 15 : r >> 1 & 7; }
    static __device__ __forceinline__ int value_swap(int r) { return DP == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2; }
    static __device__ __forceinline__ int value(int r, int d) { return r * DP + (((d >> 3) ^ value_swap(r)) << 3) + (d & 7); }
};

template <int DP, int WAVES, int TEAMS, bool kLean> struct Wide {
    static constexpr int PIECES = DP / 8, BLOCKS = DP / 32;
    static constexpr int ROWS = 64 / PIECES, LOADS = kWideTile / ROWS / WAVES;     // of a wave's load, and how many of them

    const TreeArgs& a;
    WideShared<DP, WAVES>& s;
    const int tid, lane, wave, sub, team;

    Row row;
    Span span;
    int32_t kv, block;
    bool busy;                            // the wave has queries of the job
    bool valid;                           // the lane's query: column sub * 32 + lane % 32
    int32_t low, high, every_low, every_high;
    V4u q[DP / 16];
    float unit;                           // of the scores, as powers of 2
    float m, l;                           // l is this lane's share
    V16f o[BLOCKS];                       // o[b][i]: dim 32 b + 8 (i / 4) + 4 (lane / 32) + i % 4

    __device__ __forceinline__ Wide(const TreeArgs& args, WideShared<DP, WAVES>& shared)
        : a(args), s(shared), tid(threadIdx.x), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
          sub(wave % (WAVES / TEAMS)), team(wave / (WAVES / TEAMS))
    {
    }

    __device__ __forceinline__ const uint16_t* keys_at() const { return static_cast<const uint16_t*>(a.k) + kv * a.head_stride; }
    __device__ __forceinline__ const uint16_t* values_at() const { return static_cast<const uint16_t*>(a.v) + kv * a.head_stride; }

    __device__ __forceinline__ void begin(const Row& r, const Span& x, int32_t hh)
    {
        row = r;
        span = x;
        kv = hh / a.blocks;
        block = hh - kv * a.blocks;
        const bool tree = a.parents != nullptr;
        Family<2>& family = s.family[wave];
        const int32_t column = sub * kWideColumns + (lane & 31), token = column / a.job_heads;
        const int32_t head = block * a.job_heads + column - token * a.job_heads;
        const int32_t i = span.from + min(token, span.count - 1);
        valid = token < span.count && head < a.group;
        busy = sub * kWideColumns < span.count * a.job_heads;
        int32_t depth = i;
        if (tree) {
            wave_sync();                  // the last job's are no longer read
            const int32_t last = span.from + span.count;
            for (int32_t j = lane; j < last; j += 64) {
                const int32_t parent = a.parents[row.first + j];
                family.parent[j] = (int16_t)(parent >= 0 && parent < j ? parent : -1);
            }
            wave_sync();
            depth = 0;
            for (int32_t j = family.parent[i]; j >= 0; j = family.parent[j]) ++depth;
            if (lane < kWideColumns) {
#pragma unroll
                for (int w = 0; w <= kWords; ++w) family.above[lane][w] = 0;
                int32_t at = depth;
                for (int32_t j = i; j >= 0; j = family.parent[j], --at)
                    if (a.window == 0 || depth - at < a.window || (int64_t)row.base + at < a.sinks)
                        family.above[lane][j >> 5] |= 1u << (j & 31);
            }
            wave_sync();
        }
        high = row.base < 0 ? 0 : tree ? row.base : row.base + i + 1;
        low = a.window > 0 && row.base >= 0 ? (int32_t)max((int64_t)row.base + depth + 1 - a.window, (int64_t)0) : 0;
        const uint16_t* const p = static_cast<const uint16_t*>(a.q) + (int64_t)(row.first + i) * a.q_stride +
                                  (int64_t)(kv * a.group + min(head, a.group - 1)) * a.q_head_stride;
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) {
            const int d = 8 * (lane >> 5) + 16 * e;
            q[e] = *reinterpret_cast<const V4uAnywhere*>(p + (d < a.dim ? d : 0));
            if (d >= a.dim || !valid) q[e] = V4u{0, 0, 0, 0};
            if (a.scale < 0.f) q[e] ^= 0x80008000u;       // of -q with -scale
        }
        unit = fabsf(a.scale) * kLog2e;
        every_high = row.base < 0 ? 0 : tree ? row.base : row.base + span.from + 1;
        every_low = 0;
        if (a.window > 0 && row.base >= 0)
            every_low = (int32_t)max((int64_t)row.base + (tree ? span.from + span.count : span.from + span.count - 1) + 1 - a.window, (int64_t)0);
        m = -__builtin_inff();
        l = 0.f;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] = 0.f;
    }

    // Whether all queries of the job see all of a tile's positions that have a page.
    __device__ __forceinline__ bool whole(int32_t pos0) const
    {
        return pos0 + kWideTile <= every_high && (pos0 >= every_low || pos0 + kWideTile <= a.sinks);
    }

    // Positions pos0 .. + 31 that the lane's query sees.
    __device__ __forceinline__ uint32_t seen_from(int32_t pos0) const
    {
        uint32_t seen = bits_below(high - pos0) & ~(bits_below(low - pos0) & ~bits_below(a.sinks - pos0));
        if (a.parents && row.base >= 0) {
            const int32_t off = pos0 - row.base;
            if (off > -32 && off < kMaxTree) {
                const int32_t w = off >> 5, shift = off & 31;
                const uint32_t* const above = s.family[wave].above[lane & 31];
                const uint32_t lo = w >= 0 ? above[w] : 0u, hi = above[w + 1];
                seen |= shift ? lo >> shift | hi << (32 - shift) : lo;
            }
        }
        return valid ? seen : 0u;
    }

    // The lane's position of a tile: its row's offset in the cache, -1 without a page.
    __device__ __forceinline__ int32_t ask(int32_t pos0) const
    {
        const int32_t pos = pos0 + lane, at = a.page_shift >= 0 ? pos >> a.page_shift : pos / a.page_size;
        int32_t id = -1;
        if (pos < span.end) id = (a.table + (int64_t)row.seq * a.table_stride)[at];
        return id;
    }
    __device__ __forceinline__ int64_t place(int32_t id, int32_t pos0) const
    {
        const int32_t pos = pos0 + lane, at = a.page_shift >= 0 ? pos >> a.page_shift : pos / a.page_size;
        return id >= 0 && id < a.pages ? id * a.page_stride + (pos - at * a.page_size) * a.token_stride : -1;
    }

    // A tile's rows that have a page go to a buffer, in 1 KiB a wave and load.  Written out, because the compiler would
    // wait for them before any other read of shared memory; arrived() waits.
    __device__ __forceinline__ void load(int buffer, int64_t at)
    {
        typedef __attribute__((address_space(3))) uint16_t Lds;
        // what follows from the lane is found again for each tile where the folding needs the registers
        int again = lane;
        if constexpr (kLean) asm volatile("" : "+v"(again));
        const int in = again / PIECES, piece = again % PIECES;
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int first = (wave + k * WAVES) * ROWS, r = first + in;
            const uint32_t lo = __shfl((uint32_t)(uint64_t)at, r), hi = __shfl((uint32_t)((uint64_t)at >> 32), r);
            const int64_t from = (int64_t)(((uint64_t)hi << 32) | lo);
            const int kp = 8 * (piece ^ s.key_swap(r)), vp = 8 * (piece ^ s.value_swap(r));
            const uint32_t key_to = (uint32_t)(uintptr_t)(Lds*)&s.keys[buffer][first * DP];
            const uint32_t value_to = (uint32_t)(uintptr_t)(Lds*)&s.values[buffer][first * DP];
            if (from >= 0 && kp < a.dim)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(key_to), "v"(keys_at() + from + kp)
                             : "memory", "m0");
            if (from >= 0 && vp < a.dim)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(value_to), "v"(values_at() + from + vp)
                             : "memory", "m0");
        }
    }
    __device__ __forceinline__ void arrived()
    {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }

    // Rows without a page become zeros, those with values that are not finite are marked.
    __device__ __forceinline__ void clean(int buffer, uint64_t there)
    {
#pragma unroll 1
        for (int i = tid; i < kWideTile * PIECES; i += 64 * WAVES) {
            const int r = i / PIECES;
            V4u* const v = reinterpret_cast<V4u*>(s.values[buffer]) + i;
            if (!(there >> r & 1)) {
                *v = V4u{0, 0, 0, 0};
                reinterpret_cast<V4u*>(s.keys[buffer])[i] = V4u{0, 0, 0, 0};
                continue;
            }
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= ((*v)[e] & 0x7F80u) == 0x7F80u || ((*v)[e] & 0x7F800000u) == 0x7F800000u;
            if (odd) atomicOr(&s.odd[r >> 5], 1u << (r & 31));
        }
    }

    // Folds the team's part of the tile in a buffer into the state: all of it, or a half.
    __device__ __forceinline__ void fold(int buffer, int32_t pos0, bool edge, uint64_t there)
    {
        constexpr int PARTS = 2 / TEAMS;
        const int h = lane >> 5, r0 = 32 * team;
        V16f x[PARTS];
        const int krow = (r0 + (lane & 31)) * DP + 8 * (h ^ s.key_swap(lane & 31));
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[p][e] = 0.f;
#pragma unroll
        for (int i0 = 0; i0 < DP / 16; i0 += 8 / PARTS) {
            // eight pieces of keys asked for at once: more do not fit the registers
            V4u k[PARTS][8 / PARTS];
#pragma unroll
            for (int i = 0; i < 8 / PARTS; ++i)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    if (i0 + i < DP / 16) k[p][i] = *reinterpret_cast<const V4u*>(&s.keys[buffer][(krow ^ (16 * (i0 + i))) + 32 * p * DP]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 8 / PARTS; ++i)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    if (i0 + i < DP / 16)
                        x[p] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(V8bf, k[p][i]), __builtin_bit_cast(V8bf, q[i0 + i]), x[p],
                                                                       0, 0, 0);
        }
        // the values are on their way during the softmax: dim lane % 32 of each 32, positions 8 t + {0 .. 3} + 4 h of the part
        V2u v[PARTS][BLOCKS][4];
        auto values = [&](int p) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const uint16_t* const from = &s.values[buffer][s.value(r0 + 4 * h + (lane >> 2 & 3), 32 * b + (lane & 16) + 4 * (lane & 3))];
#pragma unroll
                for (int t = 0; t < 4; ++t) v[p][b][t] = turned(from + (32 * p + 8 * t) * DP);
            }
        };
        values(0);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t seen[PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            seen[p] = ~0u;
            if (edge) {
                seen[p] = seen_from(pos0 + r0 + 32 * p) & (uint32_t)(there >> (r0 + 32 * p));
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!(seen[p] >> (8 * (e >> 2) + 4 * h + (e & 3)) & 1)) x[p][e] = -__builtin_inff();
            }
        }
        float top = x[0][0];
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, x[p][e]);
        float y, z;
        swap_halves(top, &y, &z);
        top = fmaxf(y, z);
        // weights may come to 2^kAhead: then only is the base moved, and what is there scaled
        const bool moves = (top - m) * unit > kAhead;
        if (__any(moves)) {
            const float next = moves ? top : m, keep = moves ? __builtin_amdgcn_exp2f((m - next) * unit) : 1.f;
            m = next;
            l *= keep;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) o[b] *= keep;
        }
        // nothing seen yet: any finite base gives weights of 0
        const float shift = m == -__builtin_inff() ? 0.f : -m * unit;
        if (edge && __builtin_amdgcn_readfirstlane(s.odd[0] | s.odd[1])) {
            // values that are not finite: for the queries that see them only, and then no longer there
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll 1
                for (uint32_t left = __builtin_amdgcn_readfirstlane(s.odd[team + p]); left; left &= left - 1) {
                    const int r = __builtin_ctz(left);
                    float w = x[p][0];
#pragma unroll
                    for (int e = 1; e < 16; ++e)
                        if (e == 4 * (r >> 3) + (r & 3)) w = x[p][e];
                    w = __builtin_amdgcn_exp2f(fmaf(__shfl(w, (lane & 31) + 32 * (r >> 2 & 1)), unit, shift));
                    if (seen[p] >> r & 1) {
#pragma unroll
                        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                o[b][e] = fmaf(w, __uint_as_float((uint32_t)s.values[buffer][s.value(r0 + 32 * p + r, 32 * b + 8 * (e >> 2) + 4 * h + (e & 3))] << 16), o[b][e]);
                    }
                }
            clear_odd(buffer);
            values(0);
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            if (p > 0) values(p);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[p][e] = __builtin_amdgcn_exp2f(fmaf(x[p][e], unit, shift));
                sum[e & 1] += x[p][e];
            }
            V4u hi[2], lo[2];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const uint32_t both = pair(x[p][e], x[p][e + 1]);
                hi[e >> 3][e >> 1 & 3] = both;
                lo[e >> 3][e >> 1 & 3] = pair(x[p][e] - __uint_as_float(both << 16), x[p][e + 1] - __uint_as_float(both & 0xFFFF0000u));
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    const V2u v0 = v[p][b][2 * t], v1 = v[p][b][2 * t + 1];
                    const V8bf v8 = __builtin_bit_cast(V8bf, V4u{v0[0], v0[1], v1[0], v1[1]});
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v8, __builtin_bit_cast(V8bf, hi[t]), o[b], 0, 0, 0);
                    o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v8, __builtin_bit_cast(V8bf, lo[t]), o[b], 0, 0, 0);
                }
        }
        l += sum[0] + sum[1];
    }

    // All waves, when what the marked positions add has been added: their values become zeros.
    __device__ __forceinline__ void clear_odd(int buffer)
    {
        __syncthreads();
#pragma unroll 1
        for (int i = tid; i < kWideTile * PIECES; i += 64 * WAVES)
            if (s.odd[i / PIECES >> 5] >> (i / PIECES & 31) & 1) reinterpret_cast<V4u*>(s.values[buffer])[i] = V4u{0, 0, 0, 0};
        __syncthreads();
    }

    static __device__ __forceinline__ uint32_t pair(float a, float b)
    {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(V2f{a, b}, V2bf));
    }
    // Four values of a position a lane: of 16 lanes, lane i gets the i-th value of what lanes i / 4, 4 + i / 4, .. name,
    // i.e. a dim's four positions.
    static __device__ __forceinline__ V2u turned(const uint16_t* p)
    {
        using At = __attribute__((address_space(3))) V4s*;
        return __builtin_bit_cast(V2u, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p)));
    }

    // Tiles [first, last) of the job.
    __device__ __forceinline__ void run(int32_t first, int32_t last)
    {
        __syncthreads();                  // the buffers are no longer read
        if (tid < 2) s.odd[tid] = 0;
        if (a.dim < DP) {
            // what no load writes
            for (int i = tid; i < 2 * kWideTile * PIECES; i += 64 * WAVES)
                reinterpret_cast<V4u*>(s.keys)[i] = reinterpret_cast<V4u*>(s.values)[i] = V4u{0, 0, 0, 0};
            __syncthreads();
        }
        int32_t pos0 = span.at(first, kWideTile);
        int64_t at = place(ask(pos0), pos0);
        load(0, at);
        int32_t id = -1;
        if (first + 1 < last) id = ask(span.at(first + 1, kWideTile));
#pragma unroll 1
        for (int32_t i = first; i < last; ++i) {
            const int buffer = (i - first) & 1;
            const uint64_t there = __ballot(at >= 0);
            const bool edge = there != ~0ull || !whole(pos0);
            arrived();
            __syncthreads();              // the tile is there, and the other buffer free
            int32_t next = 0;
            if (i + 1 < last) {
                next = span.at(i + 1, kWideTile);
                at = place(id, next);
                load(buffer ^ 1, at);
                if (i + 2 < last) id = ask(span.at(i + 2, kWideTile));
            }
            if (edge) {
                clean(buffer, there);
                __syncthreads();
            }
            if (busy)
                fold(buffer, pos0, edge, there);
            else if (edge && __builtin_amdgcn_readfirstlane(s.odd[0] | s.odd[1]))
                clear_odd(buffer);
            if (edge) {
                __syncthreads();
                if (tid < 2) s.odd[tid] = 0;
            }
            pos0 = next;
        }
        // two waves with the same queries: the second hands its piece to the first
        if constexpr (TEAMS == 2) {
            __syncthreads();
            float* const to = reinterpret_cast<float*>(&s) + sub * 64 * (16 * BLOCKS + 2);
            if (team == 1) {
                to[lane] = m;
                to[64 + lane] = l;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) to[(2 + 16 * b + e) * 64 + lane] = o[b][e];
            }
            __syncthreads();
            if (team == 0) {
                const float mi = to[lane], top = fmaxf(m, mi), base = top == -__builtin_inff() ? 0.f : top;
                const float f = __builtin_amdgcn_exp2f((m - base) * unit), fi = __builtin_amdgcn_exp2f((mi - base) * unit);
                l = l * f + to[64 + lane] * fi;
                m = top;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[b][e] = o[b][e] * f + to[(2 + 16 * b + e) * 64 + lane] * fi;
            }
        }
    }

    __device__ __forceinline__ float whole_sum() const
    {
        float y, z;
        swap_halves(l, &y, &z);
        return y + z;
    }

    template <typename F> __device__ __forceinline__ void each_dims(F f) const
    {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const int d = 32 * b + 2 * e + 4 * (lane >> 5);
                if (d < a.dim) f(d, V4f{o[b][e], o[b][e + 1], o[b][e + 2], o[b][e + 3]});
            }
    }

    __device__ __forceinline__ void write_out()
    {
        const float sum = whole_sum();
        if (team != 0 || !valid) return;
        const int32_t column = sub * kWideColumns + (lane & 31), token = column / a.job_heads;
        const int64_t at = row.first + span.from + token;
        const int32_t head = kv * a.group + block * a.job_heads + column - token * a.job_heads;
        uint16_t* const out = static_cast<uint16_t*>(a.out) + at * a.out_stride + (int64_t)head * a.out_head_stride;
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        each_dims([&](int d, V4f v) { store4<uint16_t>(out + d, sum == 0.f ? V4f{0.f, 0.f, 0.f, 0.f} : v * f); });
        if (lane < 32 && a.lse) a.lse[at * a.heads * a.group + head] = sum == 0.f ? -__builtin_inff() : m * fabsf(a.scale) + logf(sum);
    }

    // As the parts of the other kernels: a wave's maxima, sums and rows, here of two sets.
    __device__ __forceinline__ void write_part(float* part)
    {
        const float sum = whole_sum();
        if (team != 0) return;
        float* const to = part + sub * tree_part_floats(2, a.dim);
        const int column = lane & 31;
        each_dims([&](int d, V4f v) { *reinterpret_cast<V4f*>(to + 64 + column * a.dim + d) = v; });
        if (lane < 32) {
            to[column] = m == -__builtin_inff() ? m : m * fabsf(a.scale);
            to[32 + column] = sum;
        }
    }
};

// Where a workgroup is in its share.  Kept in shared memory: what it held in registers while tiles are folded would
// cost the folding its own.
struct Progress {
    int64_t unit, end, units;
    int32_t r, hh, piece, i;
};

__device__ __forceinline__ int32_t held(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <int DP, int WAVES, int TEAMS> __global__ __launch_bounds__(64 * WAVES, 2) void k_tree_wide(TreeArgs a)
{
    __shared__ alignas(256) WideShared<DP, WAVES> s;
    __shared__ int64_t s_sum[WAVES], s_before;
    __shared__ int32_t s_row;
    __shared__ Progress s_at[2];
    const int32_t me = blockIdx.x;
    auto number = [&](int64_t units) { return (int32_t)max((int64_t)1, min((int64_t)a.groups, units / kWideShare)); };
    {
        const Line<kWideTile, WAVES> line(a, s_sum);
        Progress x;
        x.units = line.tiles * a.heads * a.blocks;
        if (me >= number(x.units) || x.units == 0) return;
        const Shares shares(x.units, number(x.units));
        x.unit = shares.begin(me);
        x.end = shares.begin(me + 1);
        x.hh = (int32_t)quotient(x.unit, line.tiles);
        int64_t t = x.unit - x.hh * line.tiles;
        line.find(a, t, &s_row, &s_before);
        __syncthreads();
        x.r = held(s_row);
        x.piece = 0;
        const Row row = wave_row(a, x.r);
        t -= s_before;
        for (int32_t n; t >= (n = span_at<kWideTile>(a, row, x.piece).tiles); ++x.piece) t -= n;
        x.i = (int32_t)t;
        if (threadIdx.x == 0) s_at[0] = x;
        __syncthreads();
    }
    Wide<DP, WAVES, TEAMS, DP == 128> work(a, s);
#pragma unroll 1
    for (int slot = 0;; slot ^= 1) {
        bool begins, turns;
        {
            const Progress& x = s_at[slot];
            const Row row = wave_row(a, held(x.r));
            const int32_t piece = held(x.piece), i = held(x.i), hh = held(x.hh);
            const Span span = span_at<kWideTile>(a, row, piece);
            const int32_t take = (int32_t)min(x.end - x.unit, (int64_t)(span.tiles - i));
            begins = i == 0;
            turns = i + take == span.tiles;
            if (begins && threadIdx.x == 0) {
                // which shares hold the rest of it
                const int32_t last = turns ? me : Shares(x.units, number(x.units)).of(x.unit + span.tiles - 1);
                a.joins[job_index(a, x.r, piece, hh)] = int2{me, last};
            }
            work.begin(row, span, hh);
            work.run(i, held(i + take));
        }
        if (begins && turns)
            work.write_out();
        else
            work.write_part(a.parts + (2 * (int64_t)me + (begins ? 1 : 0)) * a.beside * tree_part_floats(2, a.dim));
        {
            Progress x = s_at[slot];
            Cursor cur;
            cur.r = held(x.r);
            cur.hh = held(x.hh);
            cur.piece = held(x.piece);
            cur.row = wave_row(a, cur.r);
            cur.span = span_at<kWideTile>(a, cur.row, cur.piece);
            const int32_t take = (int32_t)min(x.end - x.unit, (int64_t)(cur.span.tiles - x.i));
            cur.i = held(x.i + take - 1);
            x.unit += take;
            if (x.unit >= x.end) return;
            cur.template next<kWideTile>(a);
            x.r = cur.r;
            x.hh = cur.hh;
            x.piece = cur.piece;
            x.i = cur.i;
            if (threadIdx.x == 0) s_at[slot ^ 1] = x;
        }
        __syncthreads();
    }
}

template <int DP, int WAVES, int TEAMS> __global__ __launch_bounds__(64 * WAVES, 2) void k_tree_wide_jobs(TreeArgs a)
{
    __shared__ alignas(256) WideShared<DP, WAVES> s;
    const int32_t each = a.heads * a.blocks, hh = blockIdx.x % each;
    const int64_t slots = gridDim.x / each;
    int32_t r, piece;
    // a row's last pieces see most: they begin first
    if (!find_job(a, slots - 1 - blockIdx.x / each, &r, &piece)) return;
    const Row row = wave_row(a, r);
    if ((int64_t)piece * a.job_tokens >= row.tokens) return;
    Wide<DP, WAVES, TEAMS, false> work(a, s);
    work.begin(row, span_at<kWideTile>(a, row, piece), hh);
    work.run(0, work.span.tiles);
    work.write_out();
}

// Joins the pieces of a job that lies in more than one share, as the join of one new
// token a row does, four dims a thread: of many pieces eight groups of threads take every
// eighth one of a column, of few each group joins a column of its own (32 ragged trees of 12,
// 256 jobs of 3 pieces: 16.6 us with eight groups a column, 10.1 so).
constexpr int kJoinGroups = 8;
constexpr int kFewPieces = 16;
constexpr int kMaxDim = 256;

template <typename T> __global__ __launch_bounds__(kThreads) void k_tree_join(TreeArgs a)
{
    __shared__ float s_m[kJoinGroups], s_l[kJoinGroups];
    __shared__ V4f s_o[kJoinGroups][kMaxDim / 4];
    const int32_t each = a.heads * a.blocks, tid = threadIdx.x;
    const int64_t size = tree_part_floats(a.sets, a.dim) * a.beside;
    const int quads = a.dim / 4, groups = min(kJoinGroups, kThreads / quads), group = tid / quads, d4 = tid - group * quads;
    for (int64_t index = blockIdx.x; index < (int64_t)a.rows * a.pieces * each; index += gridDim.x) {
        const int64_t job = quotient(index, each);
        const int32_t r = (int32_t)quotient(job, a.pieces), piece = (int32_t)(job - (int64_t)r * a.pieces);
        const int32_t hh = (int32_t)(index - job * each), kv = hh / a.blocks, block = hh - kv * a.blocks;
        const Row row = row_at(a, r);
        if ((int64_t)piece * a.job_tokens >= row.tokens) continue;
        const int2 held = a.joins[index];
        const int32_t pieces = held.y - held.x + 1;
        if (pieces == 1) continue;
        const int32_t heads = min(a.job_heads, a.group - block * a.job_heads);
        const int32_t from = piece * a.job_tokens, count = min(a.job_tokens, row.tokens - from);
        float m, l;
        V4f o;
        const float* first;
        int32_t token, head, in;
        auto begin = [&](int32_t c) {
            token = c / heads;
            head = c - token * heads;
            const int32_t column = token * a.job_heads + head, sub = column / (16 * a.sets);
            in = column - sub * 16 * a.sets;
            first = a.parts + (2 * (int64_t)held.x + 1) * size + sub * tree_part_floats(a.sets, a.dim);
            m = -__builtin_inff();
            l = 0.f;
            o = V4f{0.f, 0.f, 0.f, 0.f};
        };
        auto add = [&](int32_t i) {
            const float* const part = i == 0 ? first : first + (2 * (int64_t)i - 1) * size;
            const float mi = part[in], li = part[16 * a.sets + in];
            const V4f oi = *reinterpret_cast<const V4f*>(part + 32 * a.sets + in * a.dim + 4 * d4);
            const float top = fmaxf(m, mi), base = top == -__builtin_inff() ? 0.f : top;
            const float f = weight<T>(m - base), fi = weight<T>(mi - base);
            l = l * f + li * fi;
            o = o * f + oi * fi;
            m = top;
        };
        auto write = [&] {
            const float f = l == 0.f ? 0.f : 1.f / l;
            const int64_t at = row.first + from + token;
            const int32_t to = kv * a.group + block * a.job_heads + head;
            store4<T>(static_cast<T*>(a.out) + at * a.out_stride + (int64_t)to * a.out_head_stride + 4 * d4,
                      l == 0.f ? V4f{0.f, 0.f, 0.f, 0.f} : o * f);
            if (d4 == 0 && a.lse) a.lse[at * a.heads * a.group + to] = l == 0.f ? -__builtin_inff() : m + logf(l);
        };
        if (pieces <= kFewPieces) {
            if (group >= groups) continue;
            for (int32_t c = blockIdx.y * groups + group; c < count * heads; c += gridDim.y * groups) {
                begin(c);
#pragma unroll 4
                for (int32_t i = 0; i < pieces; ++i) add(i);
                write();
            }
            continue;
        }
        for (int32_t c = blockIdx.y; c < count * heads; c += gridDim.y) {
            begin(c);
            if (group < groups) {
#pragma unroll 4
                for (int32_t i = group; i < pieces; i += groups) add(i);
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
                write();
            }
            __syncthreads();
        }
    }
}

// Workgroups for a job's columns: some thousands in all.
unsigned join_columns(int64_t jobs, int32_t columns)
{
    return (unsigned)std::min<int64_t>(columns, std::max<int64_t>(16, 4096 / jobs));
}

// Tiles a job has at most: its table's, or its window's and sinks'.
template <int TILE> int64_t most_tiles(const TreeArgs& a)
{
    const int64_t table = ((int64_t)a.width * a.page_size + TILE - 1) / TILE;
    if (a.window == 0) return table;
    const int64_t span = a.parents ? a.longest : std::min(a.longest, a.job_tokens);
    const int64_t window = ((int64_t)a.window + span + 2 * TILE - 2) / TILE, sinks = ((int64_t)a.sinks + TILE - 1) / TILE;
    return std::min(table, window + sinks);
}

template <typename T, int DP, bool kWhole, int NQ> hipError_t tree_as(const TreeArgs& a, hipStream_t s)
{
    const int32_t each = a.heads * a.blocks;
    // as many as find_job counts
    const int64_t jobs = ((int64_t)a.tokens / a.job_tokens + a.rows) * each;
    const int64_t most = most_tiles<Tile<T>::n>(a);
    // Measured with a workgroup a job and with shares, bf16 trees of 5: one row of 500 tokens 18 and 24 us, of 1,000 24
    // and 25, of 2,000 37 and 29; 32 rows of 4,000 134 and 118, 64 of 8,000 377 and 368, 128 of 4,000 350 and 388, 256 of
    // 100 - 8,000 458 and 475.  Prompts in fp32, one of 1,000 (504 jobs) 149 and 173, of 2,000 427 and 533, 4 of 1,000 149
    // and 213, 8 of 2,000 452 and 788; 500 tokens on each of 4 rows of up to 4,000 (520 jobs) 633 and 515.  fp32 trees of 5
    // lose by it, 128 rows of 4,000 1,019 and 856, until jobs are more, 256 of 2,000 895 and 885.
    if ((jobs >= (a.parents ? 1024 : 512) || most <= 32) && jobs <= INT32_MAX / kThreads) {
        hipLaunchKernelGGL((k_tree_jobs<T, DP, kWhole, NQ>), dim3((unsigned)jobs), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_tree<T, DP, kWhole, NQ>), dim3((unsigned)a.groups), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t all = (int64_t)a.rows * a.pieces * each;
    hipLaunchKernelGGL(k_tree_join<T>, dim3((unsigned)std::min(all, kMaxGrid), join_columns(all, a.columns)), dim3(kThreads),
                       0, s, a);
    return hipGetLastError();
}

template <typename T, int DP, bool kWhole> hipError_t tree_sets(const TreeArgs& a, hipStream_t s)
{
    if constexpr (std::is_same<T, uint16_t>::value && DP < 256)
        if (a.sets == 2) return tree_as<T, DP, kWhole, 2>(a, s);
    return tree_as<T, DP, kWhole, 1>(a, s);
}

template <int DP, int WAVES, int TEAMS> hipError_t tree_wide(const TreeArgs& a, hipStream_t s)
{
    const int32_t each = a.heads * a.blocks;
    const int64_t jobs = ((int64_t)a.tokens / a.job_tokens + a.rows) * each, most = most_tiles<kWideTile>(a);
    // Shares balance rows of any length, but each pays for its beginning and the join.  Measured with a workgroup a job
    // and with shares: one prompt of 512 tokens 32 and 59 us, of 2,048 97 and 138, of 8,000 (1,000 jobs) 842 and
    // 1,013; trees of 24 on 32 rows of up to 1,000 49 and 59, of 4,000 (256 jobs) 164 and 129, on 64 rows 246 and
    // 238, on 128 426 and 430.  A prompt's many jobs are of all lengths, the longest first; a tree's job is a row.
    if ((jobs >= (a.parents ? 4 : 2) * (int64_t)a.groups || most <= 32) && jobs <= INT32_MAX / (64 * WAVES)) {
        hipLaunchKernelGGL((k_tree_wide_jobs<DP, WAVES, TEAMS>), dim3((unsigned)jobs), dim3(64 * WAVES), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((k_tree_wide<DP, WAVES, TEAMS>), dim3((unsigned)a.groups), dim3(64 * WAVES), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t all = (int64_t)a.rows * a.pieces * each;
    hipLaunchKernelGGL(k_tree_join<uint16_t>, dim3((unsigned)std::min(all, kMaxGrid), join_columns(all, a.columns)), dim3(kThreads), 0,
                       s, a);
    return hipGetLastError();
}

template <typename T, int DP> hipError_t tree_dim(const TreeArgs& a, hipStream_t s)
{
    if constexpr (std::is_same<T, uint16_t>::value && DP <= 128)
        if (a.wide) return a.beside > 4 ? tree_wide<DP, 8, 1>(a, s) : a.beside > 2 ? tree_wide<DP, 4, 1>(a, s) : tree_wide<DP, 4, 2>(a, s);

    return a.page_size % 16 == 0 ? tree_sets<T, DP, true>(a, s) : tree_sets<T, DP, false>(a, s);
}

template <typename T> hipError_t tree_t(const TreeArgs& a, hipStream_t s)
{
    if (a.dim <= 64) return tree_dim<T, 64>(a, s);
    if (a.dim <= 128) return tree_dim<T, 128>(a, s);
    return tree_dim<T, 256>(a, s);
}

}  // namespace

hipError_t launch_attend_tree(int dtype, const TreeArgs& a, hipStream_t s)
{
    return dtype == 0 ? tree_t<uint16_t>(a, s) : tree_t<float>(a, s);
}

}  // namespace cpes
