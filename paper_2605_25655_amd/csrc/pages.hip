// Page bookkeeping of a paged cache, on the device and without a host round trip: forking (with freeing and taking pages) and
// compaction.  State is a count of references per page, nothing else: a page is free where the count is zero, and free pages are
// taken in the order of their numbers, so results do not depend on the order in which workgroups run (the only atomics add
// whole numbers).  Tables and counts are read from one set of arrays and written to another.
//
// Small pools and tables: one launch, in which every workgroup makes the whole plan for itself (a bit per page in LDS, prefix sums of the bits) and
// then its share of the copies.  Large ones: one workgroup plans, a second launch writes tables and counts and copies.
#include "kv4.h"

namespace thi {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64, PLAN_PER = 8;          // counts per thread and step of the plan
constexpr int APPLY_THREADS = 256;

// Exclusive prefix sum over the workgroup; `total` to every thread.
template <class T>
__device__ __forceinline__ T block_prefix(T v, T& total)
{
    __shared__ T s_wave[PLAN_WAVES];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    T x = v;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
        const T y = __shfl_up(x, sh);
        if (lane >= sh) x += y;
    }
    __syncthreads();                     // (the last call's sums have been read)
    if (lane == 63) s_wave[wv] = x;
    __syncthreads();
    T before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
        const T s = s_wave[w];
        before += w < wv ? s : 0;
        all += s;
    }
    total = all;
    return before + x - v;
}

__device__ __forceinline__ int clamp_len(const PagesArgs& a, int len)
{
    const long most = (long)a.max_pages * KV4_PAGE;
    return len < 0 ? 0 : len > most ? (int)most : len;
}
__device__ __forceinline__ int pages_of(int len) { return (int)(((long)len + KV4_PAGE - 1) / KV4_PAGE); }

// A row of the new table: its parent, positions, whole pages, pages in use, entries that may be a page.
struct Row {
    int parent, len, full, used, limit;
    bool first;            // the lowest row of this parent: takes over what only that parent has
};
__device__ __forceinline__ Row row_of(const PagesArgs& a, int i)      // (but for `first`)
{
    Row r{a.parents[i], 0, 0, 0, 0, false};
    const int room = a.headroom ? a.headroom[i] : 0;
    if (r.parent < 0 || r.parent >= a.rows_in) r.parent = -1;
    else r.len = clamp_len(a, a.lens_in[r.parent]);
    r.full = r.len / KV4_PAGE;
    r.used = pages_of(r.len);
    const long want = ((long)r.len + (room > 0 ? room : 0) + KV4_PAGE - 1) / KV4_PAGE;
    const int most = want < a.max_pages ? (int)want : a.max_pages;
    r.limit = most > r.used ? most : r.used;
    return r;
}
// What entry j >= full of a row becomes: the parent's page (kept), a fresh one (copied from the parent's where that is the partly filled
// one), or none.
struct Entry {
    int src;               // the parent's page, -1: none
    bool fresh;
};
template <class Single>      // is a page's count 1?
__device__ __forceinline__ Entry entry_of(const PagesArgs& a, const Row& r, int j, Single single)
{
    Entry e{-1, false};
    if (j >= r.limit) return e;
    if (r.parent >= 0 && (r.first || j < r.used)) {      // (what only the first row may take over concerns no other)
        e.src = a.table_in[(size_t)r.parent * a.max_pages + j];
        if (e.src < 0 || e.src >= a.num_pages) e.src = -1;
    }
    const bool mine = e.src >= 0 && r.first && single(e.src);
    e.fresh = !mine && (j >= r.used || e.src >= 0);
    return e;
}
__device__ __forceinline__ Row row_of_lane(const Row& r, int lane)
{
    return Row{__shfl(r.parent, lane), __shfl(r.len, lane), __shfl(r.full, lane), __shfl(r.used, lane), __shfl(r.limit, lane), __shfl((int)r.first, lane) != 0};
}

// The entries behind a row's whole pages, a row per lane: up to TAIL of them (the usual one or two) by the lane itself, all loads together; more
// by the whole wave, 64 entries at a time.
constexpr int TAIL = 4;
struct Tail {
    int src[TAIL];
    unsigned fresh;        // bits
};
template <class Single>
__device__ __forceinline__ int count_fresh(const PagesArgs& a, const Row& r, Tail& t, Single single)
{
    const int n = r.limit - r.full, lane = threadIdx.x & 63;
    t.fresh = 0;
    int count = 0;
    if (n <= TAIL) {
#pragma unroll
        for (int k = 0; k < TAIL; ++k) {
            const Entry e = entry_of(a, r, r.full + k, single);
            t.src[k] = e.src;
            t.fresh |= e.fresh ? 1u << k : 0u;
        }
        count = __builtin_popcount(t.fresh);
    }
    for (unsigned long long long_ones = __builtin_amdgcn_ballot_w64(n > TAIL); long_ones; long_ones &= long_ones - 1) {
        const int of = __builtin_ctzll(long_ones);
        const Row o = row_of_lane(r, of);
        int total = 0;
        for (int j = o.full; j < o.limit; j += 64) total += __builtin_popcountll(__builtin_amdgcn_ballot_w64(entry_of(a, o, j + lane, single).fresh));
        if (lane == of) {
            count = total;
            t.src[0] = o.full < o.used ? a.table_in[(size_t)o.parent * a.max_pages + o.full] : -1;
            t.fresh = o.full < o.used && entry_of(a, o, o.full, single).fresh ? 1u : 0u;
        }
    }
    return count;
}
// Does the partly filled page need a copy?  (Of t.src[0], to the row's first fresh page.)
__device__ __forceinline__ bool copies_page(const Row& r, const Tail& t) { return r.full < r.used && (t.fresh & 1u); }

// workspace words: first[rows_in], rank[rows_out] (fresh pages of the rows before), free[num_pages], counts
struct ForkWs {
    int *first, *rank, *free, *free_count;
};
__device__ __forceinline__ ForkWs fork_ws(const PagesArgs& a)
{
    ForkWs w;
    w.free_count = a.ws;
    w.first = a.ws + 64;
    w.rank = w.first + a.rows_in;
    w.free = w.rank + a.rows_out;
    return w;
}
__device__ __forceinline__ Row planned_row(const PagesArgs& a, const ForkWs& w, int i)
{
    Row r = row_of(a, i);
    if (r.parent >= 0) r.first = __hip_atomic_load(w.first + r.parent, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
    return r;
}
struct Counted {           // counts as they stand in memory
    const int* refs;
    __device__ __forceinline__ bool operator()(int page) const { return refs[page] == 1; }
};

__global__ __launch_bounds__(PLAN_THREADS) void fork_plan(PagesArgs a)
{
    const ForkWs w = fork_ws(a);
    const int tid = threadIdx.x;
    for (int i = tid; i < a.rows_in; i += PLAN_THREADS) w.first[i] = 0x7fffffff;
    __threadfence_block();
    __syncthreads();
    for (int i = tid; i < a.rows_out; i += PLAN_THREADS) {
        const int p = a.parents[i];
        if (p >= 0 && p < a.rows_in) atomicMin(w.first + p, i);
    }
    __threadfence();
    __syncthreads();
    int carry = 0;
    for (int i0 = 0; i0 < a.rows_out; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        Row r{-1, 0, 0, 0, 0, false};
        if (i < a.rows_out) r = planned_row(a, w, i);
        Tail t;
        const int fresh = count_fresh(a, r, t, Counted{a.refs_in});
        int total;
        const int before = block_prefix(fresh, total);
        if (i < a.rows_out) w.rank[i] = carry + before;
        carry += total;
    }
    const int wanted = carry;
    carry = 0;
    for (int p0 = 0; p0 < a.num_pages; p0 += PLAN_THREADS * PLAN_PER) {
        int n = 0, refs[PLAN_PER];
#pragma unroll
        for (int k = 0; k < PLAN_PER; ++k) {
            const int p = p0 + tid * PLAN_PER + k;
            refs[k] = p < a.num_pages ? a.refs_in[p] : 1;
            n += refs[k] == 0 ? 1 : 0;
        }
        int total, at = carry + block_prefix(n, total);
#pragma unroll
        for (int k = 0; k < PLAN_PER; ++k) {
            const int p = p0 + tid * PLAN_PER + k;
            if (p < a.num_pages) {
                a.refs_out[p] = refs[k];
                if (refs[k] == 0) w.free[at++] = p;
            }
        }
        carry += total;
    }
    if (tid == 0) {
        w.free_count[0] = carry;
        if (a.info) {
            a.info[0] = wanted < carry ? wanted : carry;
            a.info[1] = wanted < carry ? 0 : wanted - carry;
        }
    }
}

// Bytes [at, end) of one layer's page src to page dst, `step` apart from one 16-byte load of a thread to its next (`at` the thread's first); eight loads in flight.
__device__ __forceinline__ void copy_page(const PagesArgs& a, int src, int dst, int layer, size_t at, size_t end, size_t step)
{
    const char* const from = a.pages + layer * a.layer_bytes + (size_t)src * a.page_bytes;
    char* const to = a.pages + layer * a.layer_bytes + (size_t)dst * a.page_bytes;
    for (; at < end; at += 8 * step) {
        uintx4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at + k * step < end) x[k] = *reinterpret_cast<const uintx4*>(from + at + k * step);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at + k * step < end) *reinterpret_cast<uintx4*>(to + at + k * step) = x[k];
    }
}

// Blocks (row, y): y = 0 writes a row of the new table and adds its references, y = 1 takes a row of the old table's away, y >= 2
// copies the row's partly filled page in layer y - 2, if it needs a copy.
__global__ __launch_bounds__(APPLY_THREADS) void fork_apply(PagesArgs a)
{
    const ForkWs w = fork_ws(a);
    const int i = blockIdx.x, y = blockIdx.y, tid = threadIdx.x;
    if (y == 1) {
        if (i < a.rows_in)
            for (int j = tid; j < a.max_pages; j += APPLY_THREADS) {
                const int e = a.table_in[(size_t)i * a.max_pages + j];
                if (e >= 0 && e < a.num_pages) atomicSub(a.refs_out + e, 1);
            }
        return;
    }
    if (i >= a.rows_out) return;
    const Row r = planned_row(a, w, i);
    const int free_count = w.free_count[0], rank = w.rank[i];
    if (y >= 2) {
        if (r.full == r.used) return;
        const Entry e = entry_of(a, r, r.full, Counted{a.refs_in});
        if (e.fresh && rank < free_count) copy_page(a, e.src, w.free[rank], y - 2, tid * 16, a.page_bytes, APPLY_THREADS * 16);
        return;
    }
    int* const out = a.table_out + (size_t)i * a.max_pages;
    for (int j = tid; j < r.full; j += APPLY_THREADS) {
        int e = a.table_in[(size_t)r.parent * a.max_pages + j];
        if (e < 0 || e >= a.num_pages) e = -1;
        out[j] = e;
        if (e >= 0) atomicAdd(a.refs_out + e, 1);
    }
    if (tid < 64) {
        int at = rank;
        for (int j0 = r.full; j0 < a.max_pages; j0 += 64) {
            const int j = j0 + tid;
            Entry e{-1, false};
            if (j < a.max_pages) e = entry_of(a, r, j, Counted{a.refs_in});
            const unsigned long long mask = __builtin_amdgcn_ballot_w64(e.fresh);
            const int k = at + __builtin_popcountll(mask & ((1ull << tid) - 1ull));
            at += __builtin_popcountll(mask);
            if (j < a.max_pages) {
                const int page = e.fresh ? (k < free_count ? w.free[k] : -1) : e.src;
                out[j] = page;
                if (page >= 0) atomicAdd(a.refs_out + page, 1);
            }
        }
        if (tid == 0) a.lens_out[i] = r.len;
    }
}

// workspace words: counts (live, moved), to[num_pages], hole[num_pages], mover[num_pages]
struct CompactWs {
    int *count, *to, *hole, *mover;
};
__device__ __forceinline__ CompactWs compact_ws(const PagesArgs& a)
{
    CompactWs w;
    w.count = a.ws;
    w.to = a.ws + 64;
    w.hole = w.to + a.num_pages;
    w.mover = w.hole + a.num_pages;
    return w;
}

__global__ __launch_bounds__(PLAN_THREADS) void compact_plan(PagesArgs a)
{
    const CompactWs w = compact_ws(a);
    const int tid = threadIdx.x;
    int mine = 0, live, total;
    for (int p = tid; p < a.num_pages; p += PLAN_THREADS) mine += a.refs_in[p] > 0 ? 1 : 0;
    block_prefix(mine, live);
    int holes = 0, movers = 0;
    for (int p0 = 0; p0 < a.num_pages; p0 += PLAN_THREADS) {
        const int p = p0 + tid;
        const bool in = p < a.num_pages, used = in && a.refs_in[p] > 0;
        const bool hole = in && !used && p < live, mover = used && p >= live;
        const int h = holes + block_prefix(hole ? 1 : 0, total);
        holes += total;
        const int m = movers + block_prefix(mover ? 1 : 0, total);
        movers += total;
        if (hole) w.hole[h] = p;
        if (mover) w.mover[m] = p;
        if (in) {
            w.to[p] = used && p < live ? p : -1;
            a.refs_out[p] = used && p < live ? a.refs_in[p] : 0;
        }
    }
    __threadfence();
    __syncthreads();
    for (int m = tid; m < movers; m += PLAN_THREADS) {
        const int p = w.mover[m], h = w.hole[m];
        w.to[p] = h;
        a.refs_out[h] = a.refs_in[p];
    }
    if (tid == 0) {
        w.count[0] = live;
        w.count[1] = movers;
        if (a.info) {
            a.info[0] = live;
            a.info[1] = movers;
        }
    }
}

__global__ __launch_bounds__(APPLY_THREADS) void compact_apply(PagesArgs a)
{
    const CompactWs w = compact_ws(a);
    const size_t entries = (size_t)a.rows_in * a.max_pages, stride = (size_t)gridDim.x * APPLY_THREADS;
    for (size_t i = (size_t)blockIdx.x * APPLY_THREADS + threadIdx.x; i < entries; i += stride) {
        const int e = a.table_in[i];
        a.table_out[i] = e >= 0 && e < a.num_pages ? w.to[e] : -1;
    }
    const long jobs = (long)w.count[1] * a.layers;
    for (long k = blockIdx.x; k < jobs; k += gridDim.x) {
        const int m = (int)(k / a.layers), layer = (int)(k % a.layers);
        copy_page(a, w.mover[m], w.hole[m], layer, threadIdx.x * 16, a.page_bytes, APPLY_THREADS * 16);
    }
}

// ---- one launch ---------------------------------------------------------------------------------------------------
//
// A bit per page of what `is` holds for, and the bits in front of each word: rank() and select() in a handful of LDS reads, so that no list is
// written, no workspace read, and no workgroup waits for another.
template <int WORDS> struct PageBits {
    unsigned long long word[WORDS + 1];
    int before[WORDS + 1];
    __device__ __forceinline__ int rank(int p) const      // bits in front of p
    {
        return before[p >> 6] + __builtin_popcountll(word[p >> 6] & ((1ull << (p & 63)) - 1ull));
    }
    // The page of the k-th bit that is set (SET) or not; there has to be one.
    template <bool SET> __device__ __forceinline__ int select(int k) const
    {
        int w = 0;
#pragma unroll
        for (int step = WORDS / 2; step; step >>= 1) {
            const int front = SET ? before[w + step] : 64 * (w + step) - before[w + step];
            if (front <= k) w += step;
        }
        unsigned long long m = SET ? word[w] : ~word[w];
        int r = k - (SET ? before[w] : 64 * w - before[w]), p = 64 * w;
#pragma unroll
        for (int width = 32; width; width >>= 1) {
            const int low = __builtin_popcountll(m & ((1ull << width) - 1ull));
            if (r >= low) {
                r -= low;
                m >>= width;
                p += width;
            }
        }
        return p;
    }
};
// The counts of all pages, 64 a word, every PLAN_WAVES-th word of them a wave's; -1 where there is no page.
template <int WORDS> struct Counts {
    int refs[WORDS / PLAN_WAVES];
};
template <int WORDS>
__device__ __forceinline__ void ask_counts(const PagesArgs& a, Counts<WORDS>& c)
{
    static_assert((WORDS & (WORDS - 1)) == 0 && WORDS % 64 == 0, "");
#pragma unroll
    for (int k = 0; k < WORDS / PLAN_WAVES; ++k) {
        const int p = k * PLAN_THREADS + (int)threadIdx.x;
        c.refs[k] = p < a.num_pages ? a.refs_in[p] : -1;
    }
}
template <int WORDS, class Is>
__device__ __forceinline__ void put_words(const Counts<WORDS>& c, unsigned long long* word, Is is)
{
#pragma unroll
    for (int k = 0; k < WORDS / PLAN_WAVES; ++k) {
        const unsigned long long m = __builtin_amdgcn_ballot_w64(is(c.refs[k]));
        if ((threadIdx.x & 63) == 0) word[k * PLAN_WAVES + (threadIdx.x >> 6)] = m;
    }
}
template <int WORDS, class Is>
__device__ __forceinline__ void make_bits(const Counts<WORDS>& c, PageBits<WORDS>& bits, Is is)
{
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    put_words(c, bits.word, is);
    __syncthreads();
    if (wv == 0) {
        constexpr int PER = WORDS / 64;
        int n[PER], sum = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            n[k] = __builtin_popcountll(bits.word[lane * PER + k]);
            sum += n[k];
        }
        int x = sum;
#pragma unroll
        for (int sh = 1; sh < 64; sh <<= 1) {
            const int y = __shfl_up(x, sh);
            if (lane >= sh) x += y;
        }
        int at = x - sum;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            bits.before[lane * PER + k] = at;
            at += n[k];
        }
        if (lane == 63) {
            bits.before[WORDS] = at;
            bits.word[WORDS] = 0;
        }
    }
    __syncthreads();
}

// Copies of `jobs` pages in every layer, dealt to the waves in equal runs of SLICE bytes; places(k, src, dst) are those of the k-th.
constexpr int SLICE = 1024;
template <class Places>
__device__ __forceinline__ void copy_share(const PagesArgs& a, int jobs, int block, int blocks, Places places)
{
    const int lane = threadIdx.x & 63;
    const unsigned wave = (unsigned)block * PLAN_WAVES + (unsigned)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = (unsigned)blocks * PLAN_WAVES;
    const size_t slices = (a.page_bytes + SLICE - 1) / SLICE, total = (size_t)jobs * a.layers * slices, per = total / waves, more = total % waves;
    size_t s = wave * per + (wave < more ? wave : more);
    const size_t s1 = s + per + (wave < more ? 1 : 0);
    if (s >= s1) return;
    const size_t job = s / slices;
    size_t in = s % slices;
    int k = (int)(job / (size_t)a.layers), layer = (int)(job % (size_t)a.layers), src, dst;
    places(k, src, dst);
    for (;;) {
        const size_t n = s1 - s < slices - in ? s1 - s : slices - in, end = (in + n) * SLICE < a.page_bytes ? (in + n) * SLICE : a.page_bytes;
        copy_page(a, src, dst, layer, in * SLICE + lane * 16, end, SLICE);
        s += n;
        in = 0;
        if (s >= s1) return;
        if (++layer == a.layers) {
            layer = 0;
            places(++k, src, dst);
        }
    }
}

constexpr int COMPACT_WORDS = 256, COMPACT_ENTRIES = 1 << 22;          // 16384 pages
__global__ __launch_bounds__(PLAN_THREADS, 8) void compact_one(PagesArgs a)
{
    __shared__ PageBits<COMPACT_WORDS> live;
    Counts<COMPACT_WORDS> counts;
    ask_counts(a, counts);
    make_bits(counts, live, [](int refs) { return refs > 0; });
    const int L = live.before[COMPACT_WORDS], front = live.rank(L), moved = L - front;      // as many holes in front of L as live pages behind
    const int tid = blockIdx.x * PLAN_THREADS + threadIdx.x, stride = gridDim.x * PLAN_THREADS;
    auto is_live = [&](int p) { return (live.word[p >> 6] >> (p & 63) & 1ull) != 0; };
    for (int i = tid; i < a.rows_in * a.max_pages; i += stride) {
        const int e = a.table_in[i];
        int to = -1;
        if (e >= 0 && e < a.num_pages && is_live(e)) to = e < L ? e : live.select<false>(live.rank(e) - front);
        a.table_out[i] = to;
    }
    for (int p = tid; p < a.num_pages; p += stride) {
        int refs = 0;
        if (p < L) refs = a.refs_in[is_live(p) ? p : live.select<true>(front + (p - live.rank(p)))];
        a.refs_out[p] = refs;
    }
    if (tid == 0 && a.info) {
        a.info[0] = L;
        a.info[1] = moved;
    }
    copy_share(a, moved, blockIdx.x, gridDim.x, [&](int k, int& src, int& dst) {
        src = __builtin_amdgcn_readfirstlane(live.select<true>(front + k));
        dst = __builtin_amdgcn_readfirstlane(live.select<false>(k));
    });
}

// The first workgroup writes tables, lengths and counts (which it sums in LDS), the others copy.
constexpr int FORK_WORDS = 128, FORK_PAGES = FORK_WORDS * 64, FORK_ROWS = PLAN_THREADS, FORK_ENTRIES = 1 << 16;
__global__ __launch_bounds__(PLAN_THREADS, 4) void fork_one(PagesArgs a)
{
    __shared__ PageBits<FORK_WORDS> free;
    __shared__ int s_first[FORK_ROWS], s_copies;
    __shared__ int s_src[FORK_ROWS], s_dst[FORK_ROWS];       // copies; of the first workgroup the rows' parents and whole pages
    __shared__ int s_limit[FORK_ROWS], s_refs[FORK_PAGES];   // of the first workgroup
    __shared__ unsigned long long s_single[FORK_WORDS];      // pages with a count of 1
    const int i = threadIdx.x;
    const bool books = blockIdx.x == 0;
    Counts<FORK_WORDS> counts;
    ask_counts(a, counts);
    Row r{-1, 0, 0, 0, 0, false};
    if (i < a.rows_out) r = row_of(a, i);
    s_first[i] = 0x7fffffff;
    if (i == 0) s_copies = 0;
    if (books) {
#pragma unroll
        for (int k = 0; k < FORK_PAGES / PLAN_THREADS; ++k) s_refs[k * PLAN_THREADS + i] = counts.refs[k];
    }
    __syncthreads();
    if (r.parent >= 0) atomicMin(&s_first[r.parent], i);
    put_words(counts, s_single, [](int refs) { return refs == 1; });
    make_bits(counts, free, [](int refs) { return refs == 0; });      // (a barrier behind the minima)
    if (r.parent >= 0) r.first = s_first[r.parent] == i;
    auto single = [&](int page) { return (s_single[page >> 6] >> (page & 63) & 1ull) != 0; };
    Tail t;
    const int fresh = count_fresh(a, r, t, single), free_count = free.before[FORK_WORDS];
    const bool copies = copies_page(r, t);
    // fresh pages and copies of the rows in front, in one sum; where pages run out they do for the rows behind as well
    long long total;
    const long long before = block_prefix((long long)fresh << 16 | (copies ? 1 : 0), total);
    const int rank = (int)(before >> 16), wanted = (int)(total >> 16);
    if (!books) {
        if (copies && rank < free_count) {
            const int k = (int)(before & 0xffff);
            s_src[k] = t.src[0];
            s_dst[k] = free.select<true>(rank);
            atomicAdd(&s_copies, 1);
        }
        __syncthreads();
        copy_share(a, s_copies, blockIdx.x - 1, gridDim.x - 1, [&](int k, int& src, int& dst) {
            src = __builtin_amdgcn_readfirstlane(s_src[k]);
            dst = __builtin_amdgcn_readfirstlane(s_dst[k]);
        });
        return;
    }
    s_src[i] = r.parent;
    s_dst[i] = r.full;
    s_limit[i] = r.limit;
    __syncthreads();
    constexpr int AHEAD = 8;                 // loads in flight
    for (int k0 = i; k0 < a.rows_in * a.max_pages; k0 += AHEAD * PLAN_THREADS) {
        int e[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) e[k] = k0 + k * PLAN_THREADS < a.rows_in * a.max_pages ? a.table_in[k0 + k * PLAN_THREADS] : -1;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (e[k] >= 0 && e[k] < a.num_pages) atomicSub(&s_refs[e[k]], 1);
    }
    for (int k0 = i; k0 < a.rows_out * a.max_pages; k0 += AHEAD * PLAN_THREADS) {
        int e[AHEAD];
        bool shared[AHEAD], none[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int at = k0 + k * PLAN_THREADS, row = at / a.max_pages, j = at - row * a.max_pages;
            const bool in = row < a.rows_out;
            shared[k] = in && j < s_dst[row];
            none[k] = in && j >= s_limit[row];
            e[k] = shared[k] ? a.table_in[s_src[row] * a.max_pages + j] : -1;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (e[k] < 0 || e[k] >= a.num_pages) e[k] = -1;
            if (shared[k] || none[k]) a.table_out[k0 + k * PLAN_THREADS] = e[k];
            if (e[k] >= 0) atomicAdd(&s_refs[e[k]], 1);
        }
    }
    auto put = [&](int row, int j, const Entry& e, int k) {      // k: fresh pages in front
        const int page = e.fresh ? (k < free_count ? free.select<true>(k) : -1) : e.src;
        a.table_out[row * a.max_pages + j] = page;
        if (page >= 0) atomicAdd(&s_refs[page], 1);
    };
    const int n = r.limit - r.full, lane = i & 63;
    if (n <= TAIL) {
#pragma unroll
        for (int k = 0; k < TAIL; ++k)
            if (k < n) put(i, r.full + k, Entry{t.src[k], (t.fresh >> k & 1u) != 0}, rank + __builtin_popcount(t.fresh & ((1u << k) - 1u)));
    }
    for (unsigned long long long_ones = __builtin_amdgcn_ballot_w64(n > TAIL); long_ones; long_ones &= long_ones - 1) {
        const int of = __builtin_ctzll(long_ones), row = (i & ~63) + of;
        const Row o = row_of_lane(r, of);
        int at = __shfl(rank, of);
        for (int j = o.full; j < o.limit; j += 64) {
            const Entry e = entry_of(a, o, j + lane, single);
            const unsigned long long mask = __builtin_amdgcn_ballot_w64(e.fresh);
            if (j + lane < o.limit) put(row, j + lane, e, at + __builtin_popcountll(mask & ((1ull << lane) - 1ull)));
            at += __builtin_popcountll(mask);
        }
    }
    if (i < a.rows_out) a.lens_out[i] = r.len;
    if (i == 0 && a.info) {
        a.info[0] = wanted < free_count ? wanted : free_count;
        a.info[1] = wanted < free_count ? 0 : wanted - free_count;
    }
    __syncthreads();
    for (int p = i; p < a.num_pages; p += PLAN_THREADS) a.refs_out[p] = s_refs[p];
}

// Workgroups that copy: as many as fit beside each other (one more cost a fork 5.5 us: a second round), or as have a share of 64 KiB of the most that there can be to copy.
unsigned copy_blocks(const PagesArgs& a, long pages, unsigned most)
{
    const double bytes = (double)pages * a.layers * (double)a.page_bytes;
    return bytes >= 65536.0 * most ? most : (unsigned)(bytes / 65536.0) + 1u;
}

}  // namespace

size_t pages_workspace_words(int rows_in, int rows_out, int num_pages)
{
    const size_t fork = 64 + (size_t)rows_in + rows_out + num_pages, compact = 64 + 3 * (size_t)num_pages;
    return fork > compact ? fork : compact;
}

// One launch up to what its LDS holds, and as many table entries as one workgroup goes through while the others copy.  One launch / two: 16 rows, 8192 pages 8.4 / 20.7 us
// (the call's own 8 among them); 256 rows, ten layers of 70 KB pages 22.5 / 33; 1000 rows of 32 entries, a layer 22.6 / 22.9, six 27.0 / 37.6.
hipError_t launch_kv4_fork(const PagesArgs& a, int num_cus, hipStream_t stream)
{
    if (a.rows_in <= FORK_ROWS && a.rows_out <= FORK_ROWS && a.num_pages <= FORK_PAGES && ((long)a.rows_in + a.rows_out) * a.max_pages <= FORK_ENTRIES) {
        hipLaunchKernelGGL(fork_one, dim3(1 + copy_blocks(a, a.rows_out, num_cus > 1 ? (unsigned)num_cus - 1u : 1u)), dim3(PLAN_THREADS), 0, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(fork_plan, dim3(1), dim3(PLAN_THREADS), 0, stream, a);
    const dim3 grid((unsigned)(a.rows_in > a.rows_out ? a.rows_in : a.rows_out), (unsigned)(2 + a.layers));
    hipLaunchKernelGGL(fork_apply, grid, dim3(APPLY_THREADS), 0, stream, a);
    return hipGetLastError();
}

// One launch / two at 16384 pages: 4 rows 8.6 / 35 us, 1000 rows (285 MB moved) 70 / 100; 2000 pages in ten layers (468 MB) 101 / 109.
hipError_t launch_kv4_compact(const PagesArgs& a, int num_cus, hipStream_t stream)
{
    if (a.num_pages <= 64 * COMPACT_WORDS && (long)a.rows_in * a.max_pages <= COMPACT_ENTRIES) {
        hipLaunchKernelGGL(compact_one, dim3(copy_blocks(a, a.num_pages / 2 + 1, 2u * (unsigned)num_cus)), dim3(PLAN_THREADS), 0, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(compact_plan, dim3(1), dim3(PLAN_THREADS), 0, stream, a);
    hipLaunchKernelGGL(compact_apply, dim3((unsigned)num_cus * 8), dim3(APPLY_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
