// Page bookkeeping of a paged cache, on the device and without a host round trip: forking (with freeing and taking pages) and
// compaction.  State is a count of references per page, nothing else: a page is free where the count is zero, and free pages are
// taken in the order of their numbers, so results do not depend on the order in which workgroups run (the only atomics add
// whole numbers).  Tables and counts are read from one set of arrays and written to another.
//
// Two launches each: one workgroup plans (which pages are free, which row gets which: prefix sums), then the chip writes the
// tables and counts and copies pages.
#include "kv4.h"

namespace thi {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_PER = 8;          // counts per thread and step of the plan
constexpr int APPLY_THREADS = 256;

// Exclusive prefix sum over the workgroup; `total` to every thread.
__device__ __forceinline__ int block_prefix(int v, int& total)
{
    __shared__ int s_wave[PLAN_THREADS / 64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
        const int y = __shfl_up(x, sh);
        if (lane >= sh) x += y;
    }
    __syncthreads();                     // (the last call's sums have been read)
    if (lane == 63) s_wave[wv] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        const int s = s_wave[w];
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

// A row of the new table: its parent, positions, whole pages, pages in use, pages wanted.
struct Row {
    int parent, len, full, used, want;
    bool first;            // the lowest row of this parent: takes over what only that parent has
};
__device__ __forceinline__ Row row_of(const PagesArgs& a, const int* first, int i)
{
    Row r{a.parents[i], 0, 0, 0, 0, false};
    if (r.parent < 0 || r.parent >= a.rows_in) r.parent = -1;
    else {
        r.len = clamp_len(a, a.lens_in[r.parent]);
        r.first = __hip_atomic_load(first + r.parent, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == i;
    }
    r.full = r.len / KV4_PAGE;
    r.used = pages_of(r.len);
    const int room = a.headroom ? a.headroom[i] : 0;
    const long want = ((long)r.len + (room > 0 ? room : 0) + KV4_PAGE - 1) / KV4_PAGE;
    r.want = want < a.max_pages ? (int)want : a.max_pages;
    return r;
}
// What entry j >= full of a row becomes: the parent's page (kept), a fresh one (copied from the parent's where that is the partly filled
// one), or none.
struct Entry {
    int src;               // the parent's page, -1: none
    bool fresh;
};
__device__ __forceinline__ Entry entry_of(const PagesArgs& a, const Row& r, int j)
{
    Entry e{-1, false};
    if (r.parent >= 0) {
        e.src = a.table_in[(size_t)r.parent * a.max_pages + j];
        if (e.src < 0 || e.src >= a.num_pages) e.src = -1;
    }
    if (j >= r.want && j >= r.used) { e.src = -1; return e; }
    const bool mine = e.src >= 0 && r.first && a.refs_in[e.src] == 1;
    e.fresh = !mine && (j >= r.used || e.src >= 0);
    return e;
}

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
        int fresh = 0;
        if (i < a.rows_out) {
            const Row r = row_of(a, w.first, i);
            for (int j = r.full; j < (r.want > r.used ? r.want : r.used); ++j) fresh += entry_of(a, r, j).fresh ? 1 : 0;
        }
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

__device__ __forceinline__ void copy_page(const PagesArgs& a, int src, int dst, int layer, int part, int parts)
{
    const uintx4* const from = reinterpret_cast<const uintx4*>(a.pages + layer * a.layer_bytes + (size_t)src * a.page_bytes);
    uintx4* const to = reinterpret_cast<uintx4*>(a.pages + layer * a.layer_bytes + (size_t)dst * a.page_bytes);
    const size_t n = a.page_bytes / 16;
    for (size_t i = (size_t)part * APPLY_THREADS + threadIdx.x; i < n; i += (size_t)parts * APPLY_THREADS) to[i] = from[i];
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
    const Row r = row_of(a, w.first, i);
    const int free_count = w.free_count[0], rank = w.rank[i];
    if (y >= 2) {
        if (r.full == r.used) return;
        const Entry e = entry_of(a, r, r.full);
        if (e.fresh && rank < free_count) copy_page(a, e.src, w.free[rank], y - 2, 0, 1);
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
            if (j < a.max_pages) e = entry_of(a, r, j);
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
        copy_page(a, w.mover[m], w.hole[m], layer, 0, 1);
    }
}

}  // namespace

size_t pages_workspace_words(int rows_in, int rows_out, int num_pages)
{
    const size_t fork = 64 + (size_t)rows_in + rows_out + num_pages, compact = 64 + 3 * (size_t)num_pages;
    return fork > compact ? fork : compact;
}

hipError_t launch_kv4_fork(const PagesArgs& a, int num_cus, hipStream_t stream)
{
    (void)num_cus;
    hipLaunchKernelGGL(fork_plan, dim3(1), dim3(PLAN_THREADS), 0, stream, a);
    const dim3 grid((unsigned)(a.rows_in > a.rows_out ? a.rows_in : a.rows_out), (unsigned)(2 + a.layers));
    hipLaunchKernelGGL(fork_apply, grid, dim3(APPLY_THREADS), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_kv4_compact(const PagesArgs& a, int num_cus, hipStream_t stream)
{
    hipLaunchKernelGGL(compact_plan, dim3(1), dim3(PLAN_THREADS), 0, stream, a);
    hipLaunchKernelGGL(compact_apply, dim3((unsigned)num_cus * 8), dim3(APPLY_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
