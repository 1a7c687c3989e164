// Requests of the fp16 cache brought back to a number of positions: which stay, fresh pages for them, and the move.  Memory-bound: kept keys and values are read and
// written once, the accumulated weights read a few times, the later ones from the caches.  Two launches: the plan next to the selection, then the move.
// Measured: 16 requests of up to 4000 positions brought to 1200 in four layers of 8 heads of 128, 201 us (21 + 180); two of up to 300 of 8 heads of 64, 11.0 (8 + 2.7).
#include "kv16.h"

namespace thi {

namespace {

// ---- workspace (words) -----------------------------------------------------------------------------------------------
struct Space {
    int *kept, *begin, *fresh, *slots;      // per row: positions kept (-1: left as it is), its first fresh page's place in `fresh`; fresh pages; where kept positions are (page * KV16_PAGE + place)
};
__host__ __device__ inline Space space_of(const Kv16EvictArgs& a)
{
    Space s;
    s.kept = a.ws;
    s.begin = s.kept + a.rows;
    s.fresh = s.begin + a.rows;
    s.slots = s.fresh + a.num_pages;        // [layers][rows][Hkv][64 max_pages]
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

// Positions that a row keeps (-1: it is within its budget), by one wave.
__device__ __forceinline__ int kept_of(const Kv16EvictArgs& a, int b, int n, int lane)
{
    if (n <= a.budget) return -1;
    const int live = live_positions(a, b, n, lane);
    return live < a.budget ? live : a.budget;
}

// Who is evicted, which pages they get, and the tables and counts that follow: one workgroup.  What it writes and reads back is in LDS, too, as far as it fits: a chain of loads and stores is
// what it takes its time for.
constexpr int KE_ROWS = 512, KE_PAGES = 4096;
struct PlanSpace {
    int kept[KE_ROWS], begin[KE_ROWS], fresh[KE_PAGES];
};
template <int THREADS>
__device__ void evict_plan(const Kv16EvictArgs& a, int* s_wave, PlanSpace& s)
{
    const Space ws = space_of(a);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int first_refs = tid < a.num_pages ? a.refs_in[tid] : 1;
    for (int b = wave; b < a.rows; b += THREADS / 64) {
        const int kept = kept_of(a, b, length_of(a, b), lane);
        if (lane == 0) {
            ws.kept[b] = kept;
            if (b < KE_ROWS) s.kept[b] = kept;
        }
    }
    __syncthreads();
    auto kept_by = [&](int b) { return b < KE_ROWS ? s.kept[b] : ws.kept[b]; };
    // pages that they ask for, one row behind the other
    long asked = 0;
    for (int b0 = 0; b0 < a.rows; b0 += THREADS) {
        const int b = b0 + tid, kept = b < a.rows ? kept_by(b) : -1;
        int total;
        const int before = scan<THREADS>(kept >= 0 ? pages_for(a, kept) : 0, s_wave, total);
        const long at = asked + before;
        if (b < a.rows) {
            const int begin = at > a.num_pages ? a.num_pages : (int)at;      // (further than any free page)
            ws.begin[b] = begin;
            if (b < KE_ROWS) s.begin[b] = begin;
        }
        asked += total;
    }
    // the lowest free pages
    int free_pages = 0;
    for (int p0 = 0; p0 < a.num_pages; p0 += THREADS) {
        const int p = p0 + tid, refs = p0 == 0 ? first_refs : p < a.num_pages ? a.refs_in[p] : 1;
        int total;
        const int before = scan<THREADS>(refs == 0 ? 1 : 0, s_wave, total);
        if (refs == 0) {
            ws.fresh[free_pages + before] = p;
            if (free_pages + before < KE_PAGES) s.fresh[free_pages + before] = p;
        }
        if (p < a.num_pages) a.refs_out[p] = refs;
        free_pages += total;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the counts have to be where atomic operations find them)
    __syncthreads();
    // Rows whose pages are there: the lengths, tables and counts that they leave with.  (counts by atomic operations on integers: the same in any order)
    int done = 0, left = 0;
    for (int b = wave; b < a.rows; b += THREADS / 64) {
        const int kept = kept_by(b), n = length_of(a, b), need = kept >= 0 ? pages_for(a, kept) : 0, begin = b < KE_ROWS ? s.begin[b] : ws.begin[b];
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
                f = j >= need ? -1 : begin + j < KE_PAGES ? s.fresh[begin + j] : ws.fresh[begin + j];
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

// Which positions of a row a cache head of a layer keeps, in their order: a workgroup each (and one in front of them all for the plan, which nothing here waits for).  The k-th
// largest weight by its bits, 11, 11 and 10 of them at a time from the top: with 8 at a time, most weights fall on a few counters.  A thread takes four neighbouring positions at a time, twice (with longer tables again and again).
constexpr int KE_DIGIT = 11;
template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv16_evict_select(Kv16EvictArgs a)
{
    constexpr int DIGITS = 3;
    union Shared {
        int count[DIGITS][1 << KE_DIGIT];
        PlanSpace plan;
    };
    __shared__ Shared shared;
    __shared__ int s_wave[THREADS / 64];
    __shared__ unsigned s_prefix;
    __shared__ int s_left, s_kept, s_sure;
    if (blockIdx.x == 0) {
        if (blockIdx.y == 0 && blockIdx.z == 0) evict_plan<THREADS>(a, s_wave, shared.plan);
        return;
    }
    const Space ws = space_of(a);
    const int tid = threadIdx.x, lane = tid & 63, g = blockIdx.x - 1, b = blockIdx.y, layer = blockIdx.z;
    const int n = length_of(a, b);
    if (n <= a.budget) return;
    for (int i = tid; i < DIGITS << KE_DIGIT; i += THREADS) shared.count[0][i] = 0;
    if (tid == 0) s_sure = 0;
    const size_t at = (((size_t)layer * a.rows + b) * a.Hkv + g) * a.max_pages * KV16_PAGE;
    const float* const weights = a.weights_in + at;
    int* const slots = ws.slots + at;
    const int* const table = a.table_in + (size_t)b * a.max_pages;
    // four positions from p on, of one page: which are there, which are guarded, their weights' order
    struct Four {
        unsigned there, guarded, u[4];
    };
    auto ask = [&](int p) {
        Four f{0, 0, {0, 0, 0, 0}};
        if (p >= n) return f;
        // (both asked for at once: a page has weights for all of its positions)
        const int page = table[p / KV16_PAGE];
        float w[4];
        __builtin_memcpy(w, weights + p, sizeof(w));
        const bool there = is_page(a, page);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int q = p + k;
            if (!there || q >= n) continue;
            f.there |= 1u << k;
            if (q < a.sinks || q >= n - a.recent) f.guarded |= 1u << k;
            f.u[k] = order_of(w[k]);
        }
        return f;
    };
    // (rows of up to 8192 positions: asked for once)
    constexpr int HELD = 2;
    Four held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) held[i] = ask((i * THREADS + tid) * 4);
    auto each = [&](auto what) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) what(held[i]);
        for (int p = (HELD * THREADS + tid) * 4; p < n; p += THREADS * 4) what(ask(p));
    };
    if (tid < 64) {
        const int kept = kept_of(a, b, n, lane);
        if (tid == 0) s_kept = kept;
    }
    __syncthreads();
    // what is left of the budget for those that are not guarded
    int mine = 0;
    each([&](const Four& f) { mine += __builtin_popcount(f.guarded); });
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) mine += __shfl_xor(mine, sh);
    if (lane == 0 && mine) atomicAdd(&s_sure, mine);
    int want = 0;                                // >= 0 once it is known: no more than the budget is guarded
    unsigned prefix = 0, mask = 0;               // weights above the prefix are kept, of those equal to it (in the end) `want`
    for (int shift = 32 - KE_DIGIT, bits = KE_DIGIT, turn = 0; bits > 0; ++turn) {
        int* const count = shared.count[turn];
        const unsigned digit = (1u << bits) - 1;
        each([&](const Four& f) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((f.there & ~f.guarded) >> k & 1 && (f.u[k] & mask) == prefix) atomicAdd(&count[f.u[k] >> shift & digit], 1);
        });
        __syncthreads();
        if (turn == 0) want = s_kept - s_sure;
        // from the top: thread 0 the highest
        constexpr int PER = (1 << KE_DIGIT) / THREADS;
        const int top = (1 << KE_DIGIT) - 1 - PER * tid;
        int c[PER], sum = 0, total;
#pragma unroll
        for (int k = 0; k < PER; ++k) sum += c[k] = count[top - k];
        int above = scan<THREADS>(sum, s_wave, total);
        // the one counter with which the sum from the top reaches what is wanted (want 0: the highest; it is at most the number of candidates)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if ((above < want && above + c[k] >= want) || (want == 0 && tid == 0 && k == 0)) {
                s_prefix = prefix | (unsigned)(top - k) << shift;
                s_left = want - above;
            }
            above += c[k];
        }
        __syncthreads();
        prefix = s_prefix;
        want = s_left;
        mask |= digit << shift;
        bits = shift < KE_DIGIT ? shift : KE_DIGIT;
        shift -= bits;
    }
    int placed = 0, equal = 0;                   // of those above the prefix, or guarded; of those equal to it
    auto place = [&](int p, const Four& f) __attribute__((always_inline)) {
        unsigned same = 0, keep = f.guarded;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool other = (f.there & ~f.guarded) >> k & 1;
            same |= (other && f.u[k] == prefix ? 1u : 0u) << k;
            keep |= (other && f.u[k] > prefix ? 1u : 0u) << k;
        }
        // (both counted at once: no more than 4096 of each)
        int total;
        const int before = scan<THREADS>(__builtin_popcount(keep) | __builtin_popcount(same) << 16, s_wave, total);
        int rank = equal + (before >> 16), to = placed + (before & 0xffff) + (rank < want ? rank : want);
        placed += total & 0xffff;
        equal += total >> 16;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (same >> k & 1 && rank++ < want) keep |= 1u << k;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (keep >> k & 1) {
                slots[to] = table[p / KV16_PAGE] * KV16_PAGE + ((p + k) & (KV16_PAGE - 1));
                a.weights_out[at + to++] = weights[p + k];      // (written over where the row stays after all)
            }
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i)
        if (i * THREADS * 4 < n) place((i * THREADS + tid) * 4, held[i]);
    for (int p0 = HELD * THREADS * 4; p0 < n; p0 += THREADS * 4) place(p0 + tid * 4, ask(p0 + tid * 4));
}

// The move: a workgroup takes one fresh page of one cache head of a layer, 64 kept positions from wherever they were.  All that it reads is asked for at once, the pieces of 16 bytes of
// the keys and the single values, for a workgroup is short and the wait for memory most of it.  A key's pieces lie beside those of seven neighbours in a cache line, and so does a
// value, so that where every third position is kept, nearly all lines of the pages come: of the batch above 0.7 GB, with the 0.3 that are written 140 us at a copy's rate.  (180; of
// neighbouring positions 149; through LDS, to have the values' lines once: 4 us more.)
template <int D>
__global__ __launch_bounds__(KE_MOVE) void kv16_evict_move(Kv16EvictArgs a)
{
    constexpr int KEYS = KV16_PAGE * D / 8 / KE_MOVE, VALUES = KV16_PAGE / 8 * D / KE_MOVE;      // 16 bytes each
    __shared__ long s_from[KV16_PAGE];           // where the head's block of the position's page begins
    __shared__ int s_pos[KV16_PAGE];
    const Space ws = space_of(a);
    const int tid = threadIdx.x, g = blockIdx.y, b = blockIdx.z % a.rows, layer = blockIdx.z / a.rows;
    const size_t at = (((size_t)layer * a.rows + b) * a.Hkv + g) * a.max_pages * KV16_PAGE;
    const int p0 = blockIdx.x * KV16_PAGE;
    const int slot = tid < KV16_PAGE && p0 + tid < a.max_pages * KV16_PAGE ? ws.slots[at + p0 + tid] : 0;      // (of a row that keeps as many)
    const int kept = ws.kept[b], begin = ws.begin[b];
    if (kept < 0) {                              // left as it is
        kv16_each_copied(blockIdx.x, gridDim.x, tid, length_of(a, b), [&](size_t p) __attribute__((always_inline)) { a.weights_out[at + p] = a.weights_in[at + p]; });
        return;
    }
    const int count = kept - p0 < KV16_PAGE ? kept - p0 : KV16_PAGE;
    if (count <= 0) return;
    uint16_t* const pool = a.pages + (size_t)layer * a.layer_values;
    const size_t page_values = (size_t)a.Hkv * kv16_head_values(D);
    const int page = ws.fresh[begin + blockIdx.x];
    if (tid < KV16_PAGE) {
        const int from = tid < count ? slot : 0;
        s_pos[tid] = from & (KV16_PAGE - 1);
        s_from[tid] = (long)((size_t)(unsigned)(from / KV16_PAGE) * page_values + (size_t)g * kv16_head_values(D));
    }
    __syncthreads();
    uint16_t* const to = pool + (size_t)(unsigned)page * page_values + (size_t)g * kv16_head_values(D);
    uintx4 keys[KEYS];
    uint16_t x[VALUES][8];
    // (a position that is not there: of the first one, which is)
    const int key = tid & (KV16_PAGE - 1), part = tid / KV16_PAGE, key_from = key < count ? key : 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) keys[i] = ld_stream(pool + s_from[key_from] + kv16_key_at(s_pos[key_from], part + i * (KE_MOVE / KV16_PAGE), D));
    // eight positions of a column are 16 bytes
    const int col = tid % D;
    int first[VALUES];                           // positions first + 0 .. 3 and first + 16 + 0 .. 3
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        const int oct = tid / D + i * (KE_MOVE / D);
        first[i] = (oct >> 2) * 32 + (oct & 3) * 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            int p = first[i] + (k >> 2) * 16 + (k & 3);
            p = p < count ? p : 0;
            x[i][k] = pool[s_from[p] + kv16_value_at(s_pos[p], col, D)];
        }
    }
#pragma unroll
    for (int i = 0; i < KEYS; ++i)
        if (key < count) *reinterpret_cast<uintx4*>(to + kv16_key_at(key, part + i * (KE_MOVE / KV16_PAGE), D)) = keys[i];
#pragma unroll
    for (int i = 0; i < VALUES; ++i) {
        uint16_t* const put = to + kv16_value_at(first[i], col, D);
        if (first[i] + 19 < count) {
            uintx4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = x[i][2 * k] | (unsigned)x[i][2 * k + 1] << 16;
            *reinterpret_cast<uintx4*>(put) = y;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (first[i] + (k >> 2) * 16 + (k & 3) < count) put[k] = x[i][k];
        }
    }
}

}  // namespace

size_t kv16_evict_words(int layers, int rows, int Hkv, int max_pages, int num_pages)
{
    return 2 * (size_t)rows + num_pages + (size_t)layers * rows * Hkv * max_pages * KV16_PAGE;
}

constexpr int KE_SMALL_PAGES = 32, KE_SMALL_POOL = 8192;
hipError_t launch_kv16_evict(const Kv16EvictArgs& a, hipStream_t stream)
{
    // Short tables: small workgroups, of which more run at once and which meet in less time (the plan's walk over a large pool would take longer).  1024, 256 threads, us a call: 33 rows of 48 positions
    // brought to 8 in two layers of 40 heads 94 48; 28 of 1033 to 185 in three of 32 heads 279 231; 16 of 1500 to 300 in four of 8 heads 80.5 69.9; 9 of 1500 in two of 32 heads 105 94.
    const dim3 lists((unsigned)a.Hkv + 1, (unsigned)a.rows, (unsigned)a.layers);
    if (a.max_pages <= KE_SMALL_PAGES && a.num_pages <= KE_SMALL_POOL) hipLaunchKernelGGL((kv16_evict_select<256>), lists, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((kv16_evict_select<1024>), lists, dim3(1024), 0, stream, a);
    const dim3 grid(kv16_move_groups(a.budget, a.max_pages), (unsigned)a.Hkv, (unsigned)(a.rows * a.layers));
    if (a.D == 128) hipLaunchKernelGGL((kv16_evict_move<128>), grid, dim3(KE_MOVE), 0, stream, a);
    else hipLaunchKernelGGL((kv16_evict_move<64>), grid, dim3(KE_MOVE), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
