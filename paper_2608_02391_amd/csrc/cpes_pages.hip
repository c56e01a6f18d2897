// cpes_pages.hip -- gfx950 kernels of the key-value cache's pages: handing out,
// forking, freeing, copying and compacting them, the entry of new tokens, and of
// drafted ones the walk that finds which stay and their way together.
//
// The bookkeeping (which pages are free, who gets which) is one workgroup of 1,024
// threads, or 256, that walks the reference counts in ascending order, 16 pages
// a thread and step, so the result is the same on every run: the lowest free
// pages, in list order.  It is a chain of trips to memory and of barriers, and that
// is its time: about 4.6 us for a few sequences, 2.6 of them any launch's.  A
// sequence it works on is claimed by a mark in its length, which finds sequences
// listed twice and is taken back when the call fails.  Data moves in a second
// launch over the whole GPU; without any, the call is one launch.
#include <algorithm>

#include "cpes_eval.hpp"

namespace cpes {

namespace {

constexpr int32_t kClaim = INT32_MIN;    // the mark: a length's sign bit
constexpr int kOk = 0, kShort = 1, kBadSequence = 2;

typedef unsigned int V4u __attribute__((ext_vector_type(4)));
typedef V4u V4uAnywhere __attribute__((aligned(2)));          // tensors start at any element
typedef int V4i __attribute__((ext_vector_type(4)));
typedef V4i V4iAnywhere __attribute__((aligned(4)));

__device__ __forceinline__ V4u load16(const char* p)
{
    return *reinterpret_cast<const V4uAnywhere*>(p);
}
__device__ __forceinline__ void store16(char* p, V4u v)
{
    *reinterpret_cast<V4uAnywhere*>(p) = v;
}

// Most tokens a sequence of the pool can hold.
__device__ __forceinline__ int64_t capacity(const PoolArgs& p)
{
    return (int64_t)p.width * p.page_size;
}

// Pages that hold n tokens (n at most the capacity, counted in 32 bits).
__device__ __forceinline__ int32_t pages_of(int32_t n, int32_t page_size)
{
    return n / page_size + (n % page_size != 0);
}

__device__ __forceinline__ bool known(const PoolArgs& p, int32_t s)
{
    return s >= 0 && s < p.sequences;
}

__device__ __forceinline__ int32_t* row_of(const PoolArgs& p, int32_t s)
{
    return p.table + (int64_t)s * p.table_stride;
}

// A sequence's length as far as its table can hold it.
__device__ __forceinline__ int32_t held_tokens(const PoolArgs& p, int32_t length)
{
    const int64_t cap = capacity(p);
    return length < 0 ? 0 : (int64_t)length > cap ? (int32_t)cap : length;
}

// Exclusive sum of x over the workgroup; *total receives the sum.  All threads.
template <int BLOCK> __device__ int32_t block_scan(int32_t x, int32_t* total)
{
    __shared__ int32_t wave_sum[BLOCK / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t inc = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t y = __shfl_up(inc, d);
        if (lane >= d) inc += y;
    }
    __syncthreads();                      // the last call's sums have been read
    if (lane == 63) wave_sum[wave] = inc;
    __syncthreads();
    int32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < BLOCK / 64; ++w) {
        const int32_t y = wave_sum[w];
        if (w < wave) before += y;
        all += y;
    }
    *total = all;
    return before + inc - x;
}

// Reference counts of 16 consecutive pages; beyond the pool `beyond`.
__device__ __forceinline__ void load_refs(const PoolArgs& p, int64_t first, int32_t beyond, int32_t r[16])
{
    if (first + 16 <= p.pages) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const V4i x = *reinterpret_cast<const V4iAnywhere*>(p.refs + first + 4 * u);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[4 * u + e] = x[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) r[e] = first + e < p.pages ? p.refs[first + e] : beyond;
    }
}

// The lowest `want` free pages, ascending, into list (fewer if there are not
// that many); their number is returned.  r holds the counts of the first step's
// pages, 16 a thread.  All threads.
template <int BLOCK> __device__ int32_t lowest_free(const PoolArgs& p, int32_t r[16], int32_t want, int32_t* list)
{
    int32_t found = 0;
    for (int64_t base = 0; base < p.pages && found < want; base += 16 * BLOCK) {
        const int64_t first = base + 16 * (int64_t)threadIdx.x;
        int32_t mine = 0, total;
        if (base > 0) load_refs(p, first, 1, r);
#pragma unroll
        for (int e = 0; e < 16; ++e) mine += r[e] <= 0;
        int32_t at = found + block_scan<BLOCK>(mine, &total);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (r[e] <= 0) {
                if (at < want) list[at] = (int32_t)(first + e);
                ++at;
            }
        found += total;
    }
    __syncthreads();                      // the list is written
    return found < want ? found : want;
}

// ---------------------------------------------------------------- reserve --
// Claims every listed sequence, sums what they lack, takes that many of the
// lowest free pages and hands them out, one wave per sequence at a time.  A
// thread's first entry of the list stays in registers, and the first reference
// counts are on their way while the sequences are claimed.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_pages_reserve(PoolArgs p, int32_t n, const int32_t* seqs,
                                                              const int32_t* new_lengths, int32_t* ws, int32_t* status)
{
    __shared__ int32_t s_seq[BLOCK], s_from[BLOCK], s_need[BLOCK], s_at[BLOCK];
    int32_t* const list = ws + kPagesHeader;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t r[16];
    load_refs(p, 16 * (int64_t)tid, 1, r);
    bool bad = false, claimed = false;
    // A length that was negative before looks like a claim.  Up to a list entry a
    // thread each knows what it claimed; of longer lists none is claimed then.
    if (n > BLOCK) {
        for (int32_t i = tid; i < n; i += BLOCK) bad |= known(p, seqs[i]) && p.lengths[seqs[i]] < 0;
        if (__syncthreads_or(bad)) {
            if (tid == 0 && status) *status = kBadSequence;
            return;
        }
    }
    int32_t seq0 = 0, len0 = 0, old0 = 0;               // of entry tid
    for (int32_t i = tid; i < n; i += BLOCK) {
        const int32_t s = seqs[i], len = new_lengths[i];
        if (!known(p, s) || len < 0 || (int64_t)len > capacity(p)) {
            bad = true;
            continue;
        }
        const int32_t old = atomicOr(&p.lengths[s], kClaim);
        bad |= old < 0;
        if (i == tid) {
            seq0 = s;
            len0 = len;
            old0 = old & ~kClaim;
            claimed = old >= 0;
        }
    }
    bad = __syncthreads_or(bad);
    auto entry = [&](int32_t i, int32_t* s, int32_t* len, int32_t* old) {
        if (i == tid) {
            *s = seq0;
            *len = len0;
            *old = old0;
        } else {
            *s = seqs[i];
            *len = new_lengths[i];
            *old = p.lengths[*s] & ~kClaim;
        }
        const int32_t from = pages_of(held_tokens(p, *old), p.page_size);
        s_from[tid] = from;
        return max(0, pages_of(*len, p.page_size) - from);
    };
    // pages lacking in all, and in front of this thread's first entry; two sums of 16 bits where one could overflow
    const bool wide = p.width >= 1 << 20;
    int64_t want = 0;
    int32_t need0 = 0, at0 = 0;
    for (int32_t base = 0; base < n && !bad; base += BLOCK) {
        int32_t need = 0, lo, hi = 0, s, len, old;
        if (base + tid < n) need = entry(base + tid, &s, &len, &old);
        const int32_t at = block_scan<BLOCK>(wide ? need & 0xFFFF : need, &lo);
        if (wide) block_scan<BLOCK>(need >> 16, &hi);
        want += ((int64_t)hi << 16) + lo;
        if (base == 0) {
            need0 = need;
            at0 = at;
        }
    }
    const bool once = n <= BLOCK && !wide;          // then these are all there is to know
    const bool enough = !bad && want <= p.pages && lowest_free<BLOCK>(p, r, (int32_t)want, list) == (int32_t)want;
    if (!enough) {
        for (int32_t i = tid; i < n; i += BLOCK)
            if (n > BLOCK ? known(p, seqs[i]) : claimed) atomicAnd(&p.lengths[seqs[i]], ~kClaim);
        if (tid == 0 && status) *status = bad ? kBadSequence : kShort;
        return;
    }
    int32_t given = 0;
    for (int32_t base = 0; base < n; base += BLOCK) {
        int32_t need = need0, at = at0, total = 0, s = seq0, len = len0, old = old0;
        if (!once) {
            need = 0;
            if (base + tid < n) need = entry(base + tid, &s, &len, &old);
            at = given + block_scan<BLOCK>(need, &total);
        }
        if (base + tid < n) p.lengths[s] = max(old, len);
        s_seq[tid] = s;
        s_need[tid] = need;
        s_at[tid] = at;
        __syncthreads();
        const int32_t here = min(n - base, BLOCK);
        for (int32_t i = wave; i < here; i += BLOCK / 64) {
            int32_t* const row = row_of(p, s_seq[i]) + s_from[i];
            for (int32_t j = lane; j < s_need[i]; j += 64) {
                const int32_t page = list[s_at[i] + j];
                row[j] = page;
                p.refs[page] = 1;
            }
        }
        given += total;
        __syncthreads();
    }
    if (tid == 0 && status) *status = kOk;
}

// ------------------------------------------------------------- page copies --

// Byte offset of unit u of a page, and whether it belongs to the values.
__device__ __forceinline__ int64_t unit_offset(const PageArgs& c, uint32_t u, bool* values)
{
    uint32_t run = c.run.of(u);
    int64_t at = (int64_t)(u - run * c.run.d) * 16;
    uint32_t rest = c.inners.of(run);
    at += (int64_t)(run - rest * c.inners.d) * c.inner_bytes;
    run = rest;
    rest = c.outers.of(run);
    at += (int64_t)(run - rest * c.outers.d) * c.outer_bytes;
    *values = rest & 1;
    return at + (int64_t)(rest >> 1) * c.layer_bytes;
}

constexpr int kCopyBlock = 256;
constexpr int kCopyUnits = 4;             // 16-byte units a thread has in flight

// Units [piece * kCopyBlock * kCopyUnits, ...) of page src to page dst: a copy, bound
// by HBM, 16 bytes a lane and four of them under way.  259 MB of a pool's pages, runs
// of 8 KiB, move in 94 us, 5.5 TB/s read and written, against 6.7 of one large copy; the
// tails of 256 rollouts, 47 MB from a few pages, in 13.5 us.  Eight under way
// are half as fast, two or one-piece workgroups no faster.  NT: past the caches, for
// copies that exceed them.
template <bool NT>
__device__ __forceinline__ void copy_piece(const PageArgs& c, int32_t src, int32_t dst, uint32_t piece)
{
    const uint32_t u0 = piece * (kCopyBlock * kCopyUnits) + threadIdx.x;
    const int64_t from = src * c.page_bytes, to = dst * c.page_bytes;
    V4u x[kCopyUnits];
    char* q[kCopyUnits];
#pragma unroll
    for (int i = 0; i < kCopyUnits; ++i) {
        const uint32_t u = u0 + i * kCopyBlock;
        if (u < c.units) {
            bool values;
            const int64_t at = unit_offset(c, u, &values);
            char* const base = (values ? c.v : c.k) + at;
            x[i] = NT ? __builtin_nontemporal_load(reinterpret_cast<const V4uAnywhere*>(base + from)) : load16(base + from);
            q[i] = base + to;
        }
    }
#pragma unroll
    for (int i = 0; i < kCopyUnits; ++i)
        if (u0 + i * kCopyBlock < c.units) {
            if (NT)
                __builtin_nontemporal_store(x[i], reinterpret_cast<V4uAnywhere*>(q[i]));
            else
                store16(q[i], x[i]);
        }
}

__device__ __host__ __forceinline__ uint32_t pieces_of(const PageArgs& c)
{
    return (c.units + kCopyBlock * kCopyUnits - 1) / (kCopyBlock * kCopyUnits);
}

__global__ __launch_bounds__(kCopyBlock) void k_pages_copy(PageArgs c, int32_t pages, int32_t n, const int32_t* src,
                                                           const int32_t* dst)
{
    const uint32_t pieces = pieces_of(c);
    for (int64_t job = blockIdx.x; job < (int64_t)n * pieces; job += gridDim.x) {
        const int32_t i = (int32_t)(job / pieces), a = src[i], b = dst[i];
        if (a >= 0 && a < pages && b >= 0 && b < pages) copy_piece<false>(c, a, b, (uint32_t)(job - (int64_t)i * pieces));
    }
}

// ------------------------------------------------------------------- fork --
// The plan claims the children (an empty one's length becomes the mark), takes
// the lowest free page for each partly filled last page, writes it into the
// child's table and sets the child's length; ws[0] says whether it went well.  A
// thread's first entry and the first reference counts are in registers, as there.
template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_pages_fork_plan(PoolArgs p, int32_t n, const int32_t* parents,
                                                                const int32_t* children, int32_t* ws, int32_t* status)
{
    int32_t* const list = ws + kPagesHeader;
    const int tid = threadIdx.x;
    int32_t r[16];
    load_refs(p, 16 * (int64_t)tid, 1, r);
    bool bad = false, claimed = false;
    if (n > BLOCK) {                      // a length that is the mark already, as there
        for (int32_t i = tid; i < n; i += BLOCK) bad |= known(p, children[i]) && p.lengths[children[i]] != 0;
        if (__syncthreads_or(bad)) {
            if (tid == 0) {
                ws[0] = 0;
                if (status) *status = kBadSequence;
            }
            return;
        }
    }
    int32_t child0 = 0, len0 = 0;         // of entry tid
    for (int32_t i = tid; i < n; i += BLOCK) {
        const int32_t a = parents[i], c = children[i];
        if (!known(p, a) || !known(p, c)) {
            bad = true;
            continue;
        }
        // a parent that is itself a child of this call is empty, or carries the mark: it counts as empty
        const int32_t len = held_tokens(p, p.lengths[a]);
        const bool mine = atomicCAS(&p.lengths[c], 0, kClaim) == 0;
        bad |= !mine;
        if (i == tid) {
            child0 = c;
            len0 = len;
            claimed = mine;
        }
    }
    bad = __syncthreads_or(bad);
    auto length = [&](int32_t i) { return i == tid ? len0 : held_tokens(p, p.lengths[parents[i]]); };
    int32_t want = 0, at0 = 0;
    for (int32_t base = 0; base < n && !bad; base += BLOCK) {
        int32_t total;
        const int32_t at = block_scan<BLOCK>(base + tid < n && length(base + tid) % p.page_size != 0, &total);
        if (base == 0) at0 = at;
        want += total;
    }
    const bool enough = !bad && lowest_free<BLOCK>(p, r, want, list) == want;
    if (!enough) {
        // only a child that was empty and claimed here carries the mark alone
        for (int32_t i = tid; i < n; i += BLOCK)
            if (n > BLOCK ? known(p, children[i]) : claimed) atomicCAS(&p.lengths[children[i]], kClaim, 0);
        if (tid == 0) {
            ws[0] = 0;
            if (status) *status = bad ? kBadSequence : kShort;
        }
        return;
    }
    int32_t given = 0;
    for (int32_t base = 0; base < n; base += BLOCK) {
        int32_t total = 0, len = 0, c = child0;
        const bool mine = base + tid < n;
        if (mine) {
            len = length(base + tid);
            if (base > 0) c = children[base + tid];
        }
        const int32_t last = len / p.page_size;
        const bool tail = len - last * p.page_size != 0;
        const int32_t at = n <= BLOCK ? at0 : given + block_scan<BLOCK>(tail, &total);
        if (tail) {
            row_of(p, c)[last] = list[at];
            p.refs[list[at]] = 1;
        }
        // the mark stays on while entries behind may read this length as a parent's
        if (mine) p.lengths[c] = n > BLOCK ? len | kClaim : len;
        given += total;
    }
    if (n > BLOCK) {
        __syncthreads();                  // every parent's length has been read
        for (int32_t i = tid; i < n; i += BLOCK) p.lengths[children[i]] &= ~kClaim;
    }
    if (tid == 0) {
        ws[0] = 1;
        if (status) *status = kOk;
    }
}

// The children's tables, the references of shared pages and the copies of the
// last pages: `per` workgroups a child.
__global__ __launch_bounds__(kCopyBlock) void k_pages_fork(PageArgs c, PoolArgs p, int32_t per, const int32_t* parents,
                                                           const int32_t* children, const int32_t* ws)
{
    if (ws[0] == 0) return;
    const int32_t i = blockIdx.x / per, part = blockIdx.x - i * per;
    const int32_t len = p.lengths[children[i]], full = len / p.page_size;
    const int32_t* const from = row_of(p, parents[i]);
    int32_t* const to = row_of(p, children[i]);
    for (int64_t j = part * kCopyBlock + threadIdx.x; j < full; j += (int64_t)per * kCopyBlock) {
        const int32_t page = from[j];
        to[j] = page;
        if (page >= 0 && page < p.pages) atomicAdd(&p.refs[page], 1);
    }
    if (len % p.page_size == 0) return;
    const int32_t src = from[full], dst = to[full];
    if (src < 0 || src >= p.pages || dst < 0 || dst >= p.pages) return;
    for (uint32_t piece = part; piece < pieces_of(c); piece += per) copy_piece<false>(c, src, dst, piece);
}

// ------------------------------------------------------------------- free --
// One workgroup a sequence; taking its length makes the sequence this
// workgroup's, so one listed twice is freed once.
__global__ __launch_bounds__(kCopyBlock) void k_pages_free(PoolArgs p, int32_t n, const int32_t* seqs, int32_t* status)
{
    __shared__ int32_t s_len;
    if (blockIdx.x == 0 && status) {
        bool bad = false;
        for (int32_t i = threadIdx.x; i < n; i += kCopyBlock) bad |= !known(p, seqs[i]);
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) *status = bad ? kBadSequence : kOk;
    }
    if ((int64_t)blockIdx.x >= n) return;
    const int32_t s = seqs[blockIdx.x];
    if (!known(p, s)) return;
    if (threadIdx.x == 0) s_len = atomicExch(&p.lengths[s], 0);
    __syncthreads();
    int32_t* const row = row_of(p, s);
    const int32_t pages = pages_of(held_tokens(p, s_len), p.page_size);
    for (int32_t j = threadIdx.x; j < pages; j += kCopyBlock) {
        const int32_t page = row[j];
        row[j] = -1;
        if (page >= 0 && page < p.pages) atomicSub(&p.refs[page], 1);
    }
}

// ---------------------------------------------------------------- compact --
// ws: [0] pages that move, [1] live pages; then where they go, where they come
// from, and for every page behind the live ones' count its place in the list.
struct CompactLists {
    int32_t* header;
    int32_t* dst;
    int32_t* src;
    int32_t* place;
};

__device__ __host__ __forceinline__ CompactLists compact_lists(int32_t* ws, int32_t pages)
{
    CompactLists l;
    l.header = ws;
    l.dst = ws + kPagesHeader;
    l.src = l.dst + pages / 2;
    l.place = l.src + pages / 2;
    return l;
}

template <int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_pages_compact_plan(PoolArgs p, int32_t* ws, int32_t* moved)
{
    const CompactLists l = compact_lists(ws, p.pages);
    const bool once = p.pages <= 16 * BLOCK;        // the counts of the one step stay in registers
    int32_t live = 0, r[16];
    for (int64_t base = 0; base < p.pages; base += 16 * BLOCK) {
        int32_t mine = 0, total;
        load_refs(p, base + 16 * (int64_t)threadIdx.x, 0, r);
#pragma unroll
        for (int e = 0; e < 16; ++e) mine += r[e] > 0;
        block_scan<BLOCK>(mine, &total);
        live += total;
    }
    int32_t holes = 0, movers = 0;
    for (int64_t base = 0; base < p.pages; base += 16 * BLOCK) {
        const int64_t first = base + 16 * (int64_t)threadIdx.x;
        int32_t mine = 0, total;
        if (!once) load_refs(p, first, 0, r);
        // both counts of a step fit 16 bits: one sum
#pragma unroll
        for (int e = 0; e < 16; ++e) mine += first + e < live ? r[e] <= 0 : r[e] > 0 ? 1 << 16 : 0;
        const int32_t before = block_scan<BLOCK>(mine, &total);
        int32_t hole = holes + (before & 0xFFFF), mover = movers + (before >> 16);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int64_t page = first + e;
            if (page < live) {
                if (r[e] <= 0) l.dst[hole++] = (int32_t)page;
            } else if (page < p.pages) {
                l.place[page] = r[e] > 0 ? mover : -1;
                if (r[e] > 0) l.src[mover++] = (int32_t)page;
            }
        }
        holes += total & 0xFFFF;
        movers += total >> 16;
    }
    if (threadIdx.x == 0) {
        l.header[0] = movers;             // as many as holes: what is live behind the front is missing in it
        l.header[1] = live;
        if (moved) *moved = movers;
    }
}

// Data, reference counts, tables and lengths.  In place, each count that
// changes is written by one thread: the hole's and the mover's by the thread of
// their pair; the thread of a page writes only what the page had.
template <bool NT>
__global__ __launch_bounds__(kCopyBlock) void k_pages_compact(PageArgs c, PoolArgs p, PoolArgs packed, int32_t* ws)
{
    const CompactLists l = compact_lists(ws, p.pages);
    const int32_t moved = l.header[0], live = l.header[1];
    const uint32_t pieces = pieces_of(c);
    for (int64_t job = blockIdx.x; job < (int64_t)moved * pieces; job += gridDim.x) {
        const int32_t i = (int32_t)(job / pieces);
        copy_piece<NT>(c, l.src[i], l.dst[i], (uint32_t)(job - (int64_t)i * pieces));
    }
    const int64_t thread = (int64_t)blockIdx.x * kCopyBlock + threadIdx.x, threads = (int64_t)gridDim.x * kCopyBlock;
    for (int64_t page = thread; page < p.pages; page += threads) {
        const int32_t r = p.refs[page];
        if (page < live ? r > 0 : r <= 0) packed.refs[page] = max(r, 0);
    }
    for (int64_t i = thread; i < moved; i += threads) {
        const int32_t r = p.refs[l.src[i]];
        packed.refs[l.dst[i]] = r;
        packed.refs[l.src[i]] = 0;
    }
    for (int64_t s = blockIdx.x; s < p.sequences; s += gridDim.x) {
        const int32_t length = p.lengths[s], held = pages_of(held_tokens(p, length), p.page_size);
        const int32_t* const from = row_of(p, (int32_t)s);
        int32_t* const to = row_of(packed, (int32_t)s);
        for (int32_t j = threadIdx.x; j < p.width; j += kCopyBlock) {
            int32_t page = from[j];
            if (j < held && page >= live && page < p.pages) {
                const int32_t at = l.place[page];
                if (at >= 0) page = l.dst[at];
            }
            to[j] = page;
        }
        if (threadIdx.x == 0) packed.lengths[s] = length;
    }
}

// ------------------------------------------------------------------- keep --
// The plan claims the sequences as a reservation does, checks them and their paths,
// and then, a thread to a page of a row's drafted tokens, notes the page for the
// second launch and gives it back where the kept ones end before it.  In ws: whether it
// went well; per row where its drafted tokens begin and how many stay; their pages.
template <int BLOCK> __global__ __launch_bounds__(BLOCK) void k_pages_keep_plan(KeepArgs a, int32_t* status)
{
    const PoolArgs& p = a.pool;
    int32_t* const rows = a.ws + kPagesHeader;
    int32_t* const pages = rows + 2 * (int64_t)a.n;
    const int tid = threadIdx.x;
    auto seq_of = [&](int32_t i) { return a.seqs ? a.seqs[i] : i; };
    bool bad = false, claimed = false;
    if (a.n > BLOCK) {                    // a length that is negative before, as in a reservation
        for (int32_t i = tid; i < a.n; i += BLOCK) bad |= known(p, seq_of(i)) && p.lengths[seq_of(i)] < 0;
        if (__syncthreads_or(bad)) {
            if (tid == 0) {
                a.ws[0] = 0;
                if (status) *status = kBadSequence;
            }
            return;
        }
    }
    for (int32_t i = tid; i < a.n; i += BLOCK) {
        const int32_t s = seq_of(i), kept = a.kept[i];
        const int64_t drafted = (int64_t)a.starts[i + 1] - a.starts[i];
        if (!known(p, s) || drafted < 0 || drafted > a.longest || kept < 0 || kept > drafted) {
            bad = true;
            continue;
        }
        const int32_t old = atomicOr(&p.lengths[s], kClaim), length = old & ~kClaim;
        if (i == tid) claimed = old >= 0;
        bad |= old < 0 || length < drafted || (int64_t)length > capacity(p);
        int32_t last = -1;
        for (int32_t j = 0; j < kept; ++j) {
            const int32_t node = a.path[(int64_t)i * a.longest + j];
            bad |= node <= last || node >= drafted;
            last = node;
        }
        rows[2 * (int64_t)i] = length - (int32_t)drafted;
        rows[2 * (int64_t)i + 1] = kept;
    }
    bad = __syncthreads_or(bad);          // and the rows are written
    if (bad) {
        for (int32_t i = tid; i < a.n; i += BLOCK)
            if (a.n > BLOCK ? known(p, seq_of(i)) : claimed) atomicAnd(&p.lengths[seq_of(i)], ~kClaim);
    } else {
        for (int64_t at = tid; at < (int64_t)a.n * a.span; at += BLOCK) {
            const int32_t i = (int32_t)(at / a.span), j = (int32_t)(at - (int64_t)i * a.span), s = seq_of(i);
            const int32_t base = rows[2 * (int64_t)i], length = base + rows[2 * (int64_t)i + 1];
            const int32_t old = p.lengths[s] & ~kClaim, slot = base / p.page_size + j;
            int32_t page = -1;
            if (slot < pages_of(old, p.page_size)) {
                int32_t* const entry = row_of(p, s) + slot;
                page = *entry;
                if (slot >= pages_of(length, p.page_size)) {
                    *entry = -1;
                    if (page >= 0 && page < p.pages) atomicSub(&p.refs[page], 1);
                }
            }
            pages[at] = page;
        }
        __syncthreads();                  // every length has been read
        for (int32_t i = tid; i < a.n; i += BLOCK) p.lengths[seq_of(i)] = rows[2 * (int64_t)i] + rows[2 * (int64_t)i + 1];
    }
    if (tid == 0) {
        a.ws[0] = !bad;
        if (status) *status = bad ? kBadSequence : kOk;
    }
}

// The moves, `per` workgroups a row: a thread takes a 16-byte unit of all the row's
// tokens that move, in ascending order.  None is written to that is still to be read: the
// j-th of an ascending path lies at j or behind it, and its place is j.
constexpr int kKeepMoves = 4;             // of a thread under way

__global__ __launch_bounds__(kCopyBlock) void k_pages_keep(KeepArgs a, int32_t per)
{
    __shared__ int64_t s_from[kMaxTree], s_to[kMaxTree];
    __shared__ int32_t s_moves;
    if (a.ws[0] == 0) return;
    const int32_t page_size = a.pool.page_size;
    const int32_t* const rows = a.ws + kPagesHeader;
    for (int64_t job = blockIdx.x; job < (int64_t)a.n * per; job += gridDim.x) {
        const int32_t i = (int32_t)(job / per), part = (int32_t)(job - (int64_t)i * per);
        const int32_t base = rows[2 * (int64_t)i], kept = rows[2 * (int64_t)i + 1], first = base / page_size;
        const int32_t* const pages = rows + 2 * (int64_t)a.n + (int64_t)i * a.span;
        const int32_t j = threadIdx.x;
        int64_t from = -1, to = -1;
        if (j < kept) {
            const int32_t node = a.path[(int64_t)i * a.longest + j];
            if (node != j) {
                auto place = [&](int32_t pos) -> int64_t {
                    const int32_t at = pos / page_size, page = pages[at - first];
                    return page >= 0 && page < a.pool.pages ? page * a.page_bytes + (pos - at * page_size) * a.token_bytes : -1;
                };
                from = place(base + node);
                to = place(base + j);
            }
        }
        // the moves in order: each wave's behind the ones before
        const bool moves = from >= 0 && to >= 0;
        const uint64_t mine = __ballot(moves);
        if (threadIdx.x == 0) s_moves = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kCopyBlock / 64; ++w) {
            if ((threadIdx.x >> 6) == w) {
                const int32_t at = s_moves + __popcll(mine & ((1ull << (threadIdx.x & 63)) - 1));
                if (moves) {
                    s_from[at] = from;
                    s_to[at] = to;
                }
                if ((threadIdx.x & 63) == 0) s_moves += __popcll(mine);
            }
            __syncthreads();
        }
        const int32_t count = s_moves;
        for (uint32_t u = part * kCopyBlock + threadIdx.x; count > 0 && u < a.units; u += per * kCopyBlock) {
            const uint32_t run = a.run.of(u), rest = a.heads.of(run);
            const int64_t at = (int64_t)(u - run * a.run.d) * 16 + (int64_t)(run - rest * a.heads.d) * a.head_bytes +
                               (int64_t)(rest >> 1) * a.layer_bytes;
            char* const q = (rest & 1 ? a.v : a.k) + at;
            for (int32_t m0 = 0; m0 < count; m0 += kKeepMoves) {
                V4u x[kKeepMoves];
#pragma unroll
                for (int m = 0; m < kKeepMoves; ++m)
                    if (m0 + m < count) x[m] = load16(q + s_from[m0 + m]);
#pragma unroll
                for (int m = 0; m < kKeepMoves; ++m)
                    if (m0 + m < count) store16(q + s_to[m0 + m], x[m]);
            }
        }
        __syncthreads();                  // the moves have been read
    }
}

// ------------------------------------------------------------------ accept --
// A wave a row: a lane holds up to four nodes' parents and drafted tokens, and each step
// of the walk is a comparison and a ballot per 64 nodes.  Bound by the launch and two
// trips to memory.
__global__ __launch_bounds__(64) void k_tree_accept(AcceptArgs a)
{
    __shared__ int64_t s_sampled[kMaxTree];
    __shared__ int32_t s_path[kMaxTree];
    const int32_t r = blockIdx.x, lane = threadIdx.x;
    const int64_t begin = a.starts[r], nodes = a.starts[r + 1] - begin;
    int32_t* const path = a.path + (int64_t)r * a.longest;
    int32_t kept = 0;
    int64_t next = -1;
    if (begin >= 0 && nodes > 0 && nodes <= a.longest && begin + nodes <= a.tokens) {
        int32_t parent[kMaxTree / 64];
        int64_t drafted[kMaxTree / 64];
#pragma unroll
        for (int b = 0; b < kMaxTree / 64; ++b) {
            const int32_t i = b * 64 + lane;
            parent[b] = -1;
            drafted[b] = 0;
            if (i < nodes) {
                parent[b] = a.parents ? a.parents[begin + i] : i - 1;
                if (parent[b] >= i) parent[b] = -1;
                drafted[b] = a.drafted[begin + i];
                s_sampled[i] = a.sampled[begin + i];
            }
        }
        __syncthreads();
        int32_t at = 0;
        while (at >= 0) {
            next = s_sampled[at];
            if (lane == 0) s_path[kept] = at;
            ++kept;
            int32_t below = -1;
#pragma unroll
            for (int b = 0; b < kMaxTree / 64; ++b) {
                // a node hangs from one before it, so the walk ascends and ends
                const uint64_t those = __ballot(parent[b] == at && drafted[b] == next);
                if (below < 0 && those) below = b * 64 + __ffsll((unsigned long long)those) - 1;
            }
            at = below;
        }
        __syncthreads();
    }
    for (int32_t j = lane; j < a.longest; j += 64) path[j] = j < kept ? s_path[j] : -1;
    if (lane == 0) {
        a.kept[r] = kept;
        a.next[r] = next;
    }
}

// ----------------------------------------------------------------- append --
// `per` tokens a workgroup; where each goes is found once and kept in LDS, then
// the threads move the tokens' 16-byte units, key and value together.  Bound by HBM, or
// by the launch: 6,700 tokens of 4 KiB in 9.9 us (5.6 TB/s read and written), one token
// of 48 rollouts in 2.9 us.
constexpr int kAppendTokens = 64;         // most tokens of a workgroup
constexpr int kAppendUnits = 4;           // units of keys (and of values) a thread should get

__global__ __launch_bounds__(kCopyBlock) void k_append(AppendArgs a, int32_t per)
{
    __shared__ int64_t s_to[kAppendTokens];
    for (int64_t first = (int64_t)blockIdx.x * per; first < a.n; first += (int64_t)gridDim.x * per) {
        const int32_t here = (int32_t)min((int64_t)per, a.n - first);
        if ((int)threadIdx.x < here) {
            const int32_t i = (int32_t)first + threadIdx.x, pos = a.positions[i], s = a.seqs ? a.seqs[i] : i;
            int64_t to = -1;
            if (known(a.pool, s) && pos >= 0 && (int64_t)pos < capacity(a.pool)) {
                const int32_t at = pos / a.pool.page_size, page = row_of(a.pool, s)[at];
                if (page >= 0 && page < a.pool.pages)
                    to = page * a.page_bytes + (pos - at * a.pool.page_size) * a.token_bytes;
            }
            s_to[threadIdx.x] = to;
        }
        __syncthreads();
        const uint32_t all = a.token.d * here;
        for (uint32_t u = threadIdx.x; u < all; u += kCopyBlock) {
            const uint32_t t = a.token.of(u), rest = u - t * a.token.d, h = a.run.of(rest), x = rest - h * a.run.d;
            const int64_t to = s_to[t];
            if (to < 0) continue;
            const int64_t from = (first + t) * a.new_bytes + h * a.new_head_bytes + x * 16;
            const V4u k = load16(a.k_new + from), v = load16(a.v_new + from);
            store16(a.k + to + h * a.head_bytes + x * 16, k);
            store16(a.v + to + h * a.head_bytes + x * 16, v);
        }
        __syncthreads();                  // the places have been read
    }
}

// Workgroups of a launch whose jobs are counted on the device, or are many.
constexpr int kCopyGrid = 4096;
constexpr int kAppendGrid = 1 << 20;
constexpr double kCacheBytes = 256 << 20; // the last-level cache

// Where 256 threads see all pages and sequences in one step, their plan is done
// sooner: free, reserve and fork of four rollouts 19.6 us with 1,024, 17.5 so.  A
// reservation's pages are written by a wave a sequence, so more than a few
// sequences want all waves (32 of up to 125 pages: 8.0 us with 256, 6.7 with 1,024).
constexpr int kSmallPlan = 256;
constexpr int kSmallReserve = 16;
bool small_plan(const PoolArgs& p, int32_t n, int32_t most)
{
    return n <= most && p.pages <= 16 * kSmallPlan;
}

}  // namespace

hipError_t launch_pages_reserve(const PoolArgs& p, int32_t n, const int32_t* seqs, const int32_t* new_lengths,
                                int32_t* ws, int32_t* status, hipStream_t s)
{
    if (small_plan(p, n, kSmallReserve))
        hipLaunchKernelGGL(k_pages_reserve<kSmallPlan>, dim3(1), dim3(kSmallPlan), 0, s, p, n, seqs, new_lengths, ws, status);
    else
        hipLaunchKernelGGL(k_pages_reserve<kPlanBlock>, dim3(1), dim3(kPlanBlock), 0, s, p, n, seqs, new_lengths, ws, status);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PageArgs& c, const PoolArgs& p, int32_t n, const int32_t* parents,
                             const int32_t* children, int32_t* ws, int32_t* status, hipStream_t s)
{
    if (small_plan(p, n, kSmallPlan))
        hipLaunchKernelGGL(k_pages_fork_plan<kSmallPlan>, dim3(1), dim3(kSmallPlan), 0, s, p, n, parents, children, ws, status);
    else
        hipLaunchKernelGGL(k_pages_fork_plan<kPlanBlock>, dim3(1), dim3(kPlanBlock), 0, s, p, n, parents, children, ws, status);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 0) return e;
    const int32_t most = std::max<int32_t>((int32_t)pieces_of(c), p.width / kCopyBlock);
    const int32_t per = std::max(1, std::min(most, kCopyGrid / n));
    hipLaunchKernelGGL(k_pages_fork, dim3((unsigned)((int64_t)n * per)), dim3(kCopyBlock), 0, s, c, p, per, parents,
                       children, ws);
    return hipGetLastError();
}

hipError_t launch_pages_free(const PoolArgs& p, int32_t n, const int32_t* seqs, int32_t* status, hipStream_t s)
{
    hipLaunchKernelGGL(k_pages_free, dim3((unsigned)std::max(1, n)), dim3(kCopyBlock), 0, s, p, n, seqs, status);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const PageArgs& c, int32_t pages, int32_t n, const int32_t* src, const int32_t* dst,
                             hipStream_t s)
{
    const int64_t jobs = (int64_t)n * pieces_of(c);
    hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)std::min<int64_t>(jobs, 4 * kCopyGrid)), dim3(kCopyBlock), 0, s, c,
                       pages, n, src, dst);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const PageArgs& c, const PoolArgs& p, const PoolArgs& packed, int32_t* ws,
                                int32_t* moved, hipStream_t s)
{
    if (small_plan(p, 0, kSmallPlan))
        hipLaunchKernelGGL(k_pages_compact_plan<kSmallPlan>, dim3(1), dim3(kSmallPlan), 0, s, p, ws, moved);
    else
        hipLaunchKernelGGL(k_pages_compact_plan<kPlanBlock>, dim3(1), dim3(kPlanBlock), 0, s, p, ws, moved);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // half of the pages move at most
    const int64_t jobs = std::max<int64_t>((int64_t)(p.pages / 2) * pieces_of(c), p.sequences);
    const dim3 grid((unsigned)std::max<int64_t>(1, std::min<int64_t>(jobs, 4 * kCopyGrid))), block(kCopyBlock);
    if ((double)p.pages * c.units * 16 > kCacheBytes)
        hipLaunchKernelGGL(k_pages_compact<true>, grid, block, 0, s, c, p, packed, ws);
    else
        hipLaunchKernelGGL(k_pages_compact<false>, grid, block, 0, s, c, p, packed, ws);
    return hipGetLastError();
}

hipError_t launch_pages_keep(const KeepArgs& a, int32_t* status, hipStream_t s)
{
    if (small_plan(a.pool, a.n, kSmallPlan))
        hipLaunchKernelGGL(k_pages_keep_plan<kSmallPlan>, dim3(1), dim3(kSmallPlan), 0, s, a, status);
    else
        hipLaunchKernelGGL(k_pages_keep_plan<kPlanBlock>, dim3(1), dim3(kPlanBlock), 0, s, a, status);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n == 0) return e;
    const int32_t per = std::max<int32_t>(1, std::min<int64_t>((a.units + kCopyBlock - 1) / kCopyBlock, 4 * kCopyGrid / a.n));
    hipLaunchKernelGGL(k_pages_keep, dim3((unsigned)std::min<int64_t>((int64_t)a.n * per, 4 * kCopyGrid)), dim3(kCopyBlock), 0,
                       s, a, per);
    return hipGetLastError();
}

hipError_t launch_tree_accept(const AcceptArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(k_tree_accept, dim3((unsigned)a.rows), dim3(64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s)
{
    const int64_t token = a.token.d;
    // one token a workgroup while they are few, then enough for every thread's units
    const int64_t full = std::max<int64_t>(1, std::min<int64_t>(kAppendTokens, kCopyBlock * kAppendUnits / token));
    const int32_t per = (int32_t)std::min<int64_t>(full, std::max(1, a.n / 1024));
    hipLaunchKernelGGL(k_append, dim3((unsigned)std::min<int64_t>((a.n + (int64_t)per - 1) / per, kAppendGrid)),
                       dim3(kCopyBlock), 0, s, a, per);
    return hipGetLastError();
}

}  // namespace cpes
