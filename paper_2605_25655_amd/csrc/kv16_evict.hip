// Requests of the fp16 cache brought back to a number of positions: which stay, fresh pages for them, and the move.  Memory-bound: kept keys and values are read and
// written once, the accumulated weights read a few times, the later ones from the caches.
#include "kv16.h"

namespace thi {

namespace {

// ---- workspace (words) -----------------------------------------------------------------------------------------------
struct Space {
    int *kept, *begin, *fresh, *index;      // per row: positions kept (0: left as it is), its first fresh page's place in `fresh`; fresh pages; kept positions
};
__host__ __device__ inline Space space_of(const Kv16EvictArgs& a)
{
    Space s;
    s.kept = a.ws;
    s.begin = s.kept + a.rows;
    s.fresh = s.begin + a.rows;
    s.index = s.fresh + a.num_pages;        // [layers][rows][Hkv][64 max_pages]
    return s;
}

__device__ __forceinline__ int length_of(const Kv16EvictArgs& a, int b)
{
    const int n = a.lens_in[b], most = a.max_pages * KV16_PAGE;
    return n < 0 ? 0 : n > most ? most : n;
}
__device__ __forceinline__ bool is_page(const Kv16EvictArgs& a, int e) { return e >= 0 && e < a.num_pages; }
__device__ __forceinline__ int pages_for(const Kv16EvictArgs& a, int kept)
{
    const long n = ((long)kept + a.headroom + KV16_PAGE - 1) / KV16_PAGE;
    return n < a.max_pages ? (int)n : a.max_pages;
}

// Positions of a row that have a page, by one wave.
__device__ __forceinline__ int live_positions(const Kv16EvictArgs& a, int b, int n, int lane)
{
    int count = 0;
    for (int j = lane; j * KV16_PAGE < n; j += 64)
        if (is_page(a, a.table_in[(size_t)b * a.max_pages + j])) count += n - j * KV16_PAGE < KV16_PAGE ? n - j * KV16_PAGE : KV16_PAGE;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) count += __shfl_xor(count, sh);
    return count;
}

// Exclusive sum over the workgroup's threads, and the total.
template <int THREADS>
__device__ __forceinline__ int scan(int x, int* s_wave, int& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int y = x;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
        const int z = __shfl_up(y, sh);
        if (lane >= sh) y += z;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = y;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? s_wave[w] : 0;
        total += s_wave[w];
    }
    return before + y - x;
}

// Who is evicted, which pages they get, and the tables and counts that follow: one workgroup.
constexpr int KE_PLAN = 1024;
__global__ __launch_bounds__(KE_PLAN) void kv16_evict_plan(Kv16EvictArgs a)
{
    __shared__ int s_wave[KE_PLAN / 64];
    const Space ws = space_of(a);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int b = wave; b < a.rows; b += KE_PLAN / 64) {
        const int n = length_of(a, b);
        int kept = 0;
        if (n > a.budget) {
            kept = live_positions(a, b, n, lane);
            kept = kept < a.budget ? kept : a.budget;
        }
        if (lane == 0) ws.kept[b] = n > a.budget ? kept : -1;
    }
    __syncthreads();
    // pages that they ask for, one row behind the other
    long asked = 0;
    for (int b0 = 0; b0 < a.rows; b0 += KE_PLAN) {
        const int b = b0 + tid, kept = b < a.rows ? ws.kept[b] : -1;
        int total;
        const int before = scan<KE_PLAN>(kept >= 0 ? pages_for(a, kept) : 0, s_wave, total);
        const long at = asked + before;
        if (b < a.rows) ws.begin[b] = at > a.num_pages ? a.num_pages : (int)at;      // (further than any free page)
        asked += total;
    }
    // the lowest free pages
    int free_pages = 0;
    for (int p0 = 0; p0 < a.num_pages; p0 += KE_PLAN) {
        const int p = p0 + tid, refs = p < a.num_pages ? a.refs_in[p] : 1;
        int total;
        const int before = scan<KE_PLAN>(refs == 0 ? 1 : 0, s_wave, total);
        if (refs == 0) ws.fresh[free_pages + before] = p;
        if (p < a.num_pages) a.refs_out[p] = refs;
        free_pages += total;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the counts have to be where atomic operations find them)
    __syncthreads();
    // Rows whose pages are there: the lengths, tables and counts that they leave with.  (counts by atomic operations on integers: the same in any order)
    int done = 0, left = 0;
    for (int b = wave; b < a.rows; b += KE_PLAN / 64) {
        const int kept = ws.kept[b], n = length_of(a, b), need = kept >= 0 ? pages_for(a, kept) : 0, begin = ws.begin[b];
        const bool moves = kept >= 0 && (long)begin + need <= free_pages;
        if (lane == 0) {
            a.lens_out[b] = moves ? kept : n;
            done += moves;
            left += kept >= 0 && !moves;
        }
        for (int j = lane; j < a.max_pages; j += 64) {
            const size_t at = (size_t)b * a.max_pages + j;
            const int e = a.table_in[at];
            int f = e;
            if (moves) {
                f = j < need ? ws.fresh[begin + j] : -1;
                if (is_page(a, e)) atomicSub(&a.refs_out[e], 1);
                if (j < need) atomicAdd(&a.refs_out[f], 1);
            }
            a.table_out[at] = f;
        }
        if (lane == 0 && !moves) ws.kept[b] = -1;
    }
    if (!a.info) return;
    __shared__ int s_info[2];
    if (tid < 2) s_info[tid] = 0;
    __syncthreads();
    if (lane == 0 && done) atomicAdd(&s_info[0], done);
    if (lane == 0 && left) atomicAdd(&s_info[1], left);
    __syncthreads();
    if (tid < 2) a.info[tid] = s_info[tid];
}

// A weight's place in the order: larger numbers for larger weights, NaN the lowest.
__device__ __forceinline__ unsigned order_of(float w)
{
    if (w != w) return 0u;
    const unsigned u = __builtin_bit_cast(unsigned, w + 0.0f);      // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which positions of a row a cache head of a layer keeps, in their order: a workgroup each.  The k-th largest weight by its bits, eight at a time from the top.
constexpr int KE_SELECT = 1024;
__global__ __launch_bounds__(KE_SELECT) void kv16_evict_select(Kv16EvictArgs a)
{
    __shared__ int s_wave[KE_SELECT / 64];
    __shared__ int s_count[256];
    __shared__ unsigned s_prefix;
    __shared__ int s_left;
    const Space ws = space_of(a);
    const int tid = threadIdx.x, lane = tid & 63, g = blockIdx.x, b = blockIdx.y, layer = blockIdx.z;
    const int kept = ws.kept[b];
    if (kept < 0) return;
    const int n = length_of(a, b);
    const size_t at = (((size_t)layer * a.rows + b) * a.Hkv + g) * a.max_pages * KV16_PAGE;
    const float* const weights = a.weights_in + at;
    int* const index = ws.index + at;
    const int* const table = a.table_in + (size_t)b * a.max_pages;
    auto live = [&](int p) { return p < n && is_page(a, table[p / KV16_PAGE]); };
    auto guarded = [&](int p) { return p < a.sinks || p >= n - a.recent; };
    // what is left of the budget for the others
    int mine = 0;
    for (int p = tid; p < n; p += KE_SELECT) mine += live(p) && guarded(p) ? 1 : 0;
    int sure;
    scan<KE_SELECT>(mine, s_wave, sure);
    int want = kept - sure;                      // >= 0: no more than the budget is guarded
    unsigned prefix = 0, mask = 0;               // weights above the prefix are kept, of those equal to it (in the end) `want`
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) s_count[tid] = 0;
        __syncthreads();
        for (int p = tid; p < n; p += KE_SELECT) {
            const unsigned u = order_of(weights[p]);
            if (live(p) && !guarded(p) && (u & mask) == prefix) atomicAdd(&s_count[u >> shift & 255u], 1);
        }
        __syncthreads();
        if (tid < 64) {                          // from the top: lane 0 the four highest
            int c[4], all = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) all += c[k] = s_count[255 - (lane * 4 + k)];
            int upto = all;
#pragma unroll
            for (int sh = 1; sh < 64; sh <<= 1) {
                const int z = __shfl_up(upto, sh);
                if (lane >= sh) upto += z;
            }
            int above = upto - all;
            const unsigned long long who = __builtin_amdgcn_ballot_w64(upto >= want);
            const int first = who ? __builtin_ctzll(who) : 63;      // (want is at most the number of candidates)
            if (lane == first) {
                int k = 0;
                while (k < 3 && above + c[k] < want) above += c[k++];
                s_prefix = prefix | (unsigned)(255 - (lane * 4 + k)) << shift;
                s_left = want - above;
            }
        }
        __syncthreads();
        prefix = s_prefix;
        want = s_left;
        mask |= 255u << shift;
        __syncthreads();
    }
    int placed = 0, equal = 0;
    for (int p0 = 0; p0 < n; p0 += KE_SELECT) {
        const int p = p0 + tid;
        const bool there = p < n && live(p), guard = guarded(p);
        const unsigned u = there ? order_of(weights[p]) : 0u;
        const bool even = there && !guard && u == prefix;
        int total;
        const int rank = scan<KE_SELECT>(even ? 1 : 0, s_wave, total) + equal;
        equal += total;
        const bool keep = there && (guard || u > prefix || (even && rank < want));
        const int to = scan<KE_SELECT>(keep ? 1 : 0, s_wave, total) + placed;
        placed += total;
        if (keep) index[to] = p;
    }
}

// The move: a workgroup takes one fresh page of one cache head of a layer, 64 kept positions from wherever they were.
constexpr int KE_MOVE = 256;
template <int D>
__global__ __launch_bounds__(KE_MOVE) void kv16_evict_move(Kv16EvictArgs a)
{
    __shared__ long s_from[KV16_PAGE];           // where the head's block of the position's page begins
    __shared__ int s_pos[KV16_PAGE];
    const Space ws = space_of(a);
    const int tid = threadIdx.x, g = blockIdx.y, b = blockIdx.z % a.rows, layer = blockIdx.z / a.rows;
    const int kept = ws.kept[b];
    const size_t at = (((size_t)layer * a.rows + b) * a.Hkv + g) * a.max_pages * KV16_PAGE;
    if (kept < 0) {                              // left as it is
        const int n = length_of(a, b);
        for (int p = blockIdx.x * KE_MOVE + tid; p < n; p += gridDim.x * KE_MOVE) a.weights_out[at + p] = a.weights_in[at + p];
        return;
    }
    const int p0 = blockIdx.x * KV16_PAGE, count = kept - p0 < KV16_PAGE ? kept - p0 : KV16_PAGE;
    if (count <= 0) return;
    uint16_t* const pool = a.pages + (size_t)layer * a.layer_values;
    const size_t page_values = (size_t)a.Hkv * kv16_head_values(D);
    if (tid < KV16_PAGE) {
        const int p = tid < count ? ws.index[at + p0 + tid] : -1;
        s_pos[tid] = p & (KV16_PAGE - 1);
        s_from[tid] = p < 0 ? 0 : (long)((size_t)a.table_in[(size_t)b * a.max_pages + p / KV16_PAGE] * page_values + (size_t)g * kv16_head_values(D));
        if (p >= 0) a.weights_out[at + p0 + tid] = a.weights_in[at + p];
    }
    __syncthreads();
    uint16_t* const to = pool + (size_t)ws.fresh[ws.begin[b] + blockIdx.x] * page_values + (size_t)g * kv16_head_values(D);
#pragma unroll 4
    for (int i = tid; i < KV16_PAGE * D / 8; i += KE_MOVE) {
        const int p = i & (KV16_PAGE - 1), part = i / KV16_PAGE;
        if (p < count) *reinterpret_cast<uintx4*>(to + kv16_key_at(p, part, D)) = ld_stream(pool + s_from[p] + kv16_key_at(s_pos[p], part, D));
    }
    // eight positions of a column are 16 bytes
#pragma unroll 2
    for (int i = tid; i < KV16_PAGE / 8 * D; i += KE_MOVE) {
        const int col = i % D, oct = i / D, first = (oct >> 2) * 32 + (oct & 3) * 4;      // positions first + 0 .. 3 and first + 16 + 0 .. 3
        uint16_t x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int p = first + (k >> 2) * 16 + (k & 3);
            x[k] = p < count ? pool[s_from[p] + kv16_value_at(s_pos[p], col, D)] : 0;
        }
        uint16_t* const put = to + kv16_value_at(first, col, D);
        if (first + 19 < count) {
            uintx4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = x[2 * k] | (unsigned)x[2 * k + 1] << 16;
            *reinterpret_cast<uintx4*>(put) = y;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (first + (k >> 2) * 16 + (k & 3) < count) put[k] = x[k];
        }
    }
}

}  // namespace

size_t kv16_evict_words(int layers, int rows, int Hkv, int max_pages, int num_pages)
{
    return 2 * (size_t)rows + num_pages + (size_t)layers * rows * Hkv * max_pages * KV16_PAGE;
}

hipError_t launch_kv16_evict(const Kv16EvictArgs& a, int num_cus, hipStream_t stream)
{
    (void)num_cus;
    hipLaunchKernelGGL(kv16_evict_plan, dim3(1), dim3(KE_PLAN), 0, stream, a);
    hipLaunchKernelGGL(kv16_evict_select, dim3((unsigned)a.Hkv, (unsigned)a.rows, (unsigned)a.layers), dim3(KE_SELECT), 0, stream, a);
    const long most = (long)a.max_pages * KV16_PAGE < a.budget ? (long)a.max_pages * KV16_PAGE : a.budget;
    const dim3 grid((unsigned)((most + KV16_PAGE - 1) / KV16_PAGE), (unsigned)a.Hkv, (unsigned)(a.rows * a.layers));
    if (a.D == 128) hipLaunchKernelGGL((kv16_evict_move<128>), grid, dim3(KE_MOVE), 0, stream, a);
    else hipLaunchKernelGGL((kv16_evict_move<64>), grid, dim3(KE_MOVE), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
