// Attention over the paged fp16 cache.  out = softmax(scale q K^T) V per head, K and V in pages; row i of a request's n new tokens stands at position
// length - n + i and sees the positions up to its own whose page exists: all of them, or with a window the last `window` and the first `sinks`.
#include "kv16.h"

#include <mutex>
#include <type_traits>

namespace thi {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
#define GLOBAL __attribute__((address_space(1)))

// What a request's rows are -- [first, first + n) of q, the last n of `len` positions -- and which pages any of them sees: the `lead` first ones (sinks), then those from
// `skip` pages further on.  Whatever the arrays hold stays within the buffers.
struct Request {
    int first, n, len;
    int lead, skip, pages;           // the v-th page to look at, v < pages, is page v of the request, or v + skip from v = lead on
};
__device__ __forceinline__ Request find_request(const Kv16AttnArgs& a, int b)
{
    Request r{b, 1, a.seq_lens[b], 0, 0, 0};
    const long most = (long)a.max_pages * KV16_PAGE;
    r.len = r.len < 0 ? 0 : r.len > most ? (int)most : r.len;
    if (a.q_offsets) {
        int o0 = a.q_offsets[b], o1 = a.q_offsets[b + 1];
        o0 = o0 < 0 ? 0 : o0 > a.T ? a.T : o0;
        o1 = o1 < o0 ? o0 : o1 > a.T ? a.T : o1;
        r.first = o0;
        r.n = o1 - o0 < a.max_q ? o1 - o0 : a.max_q;
        // rows past max_q, which are not written, and the positions that only they see (fewer positions than that: the others see nothing, as with none)
        const int left = o1 - o0 - r.n;
        r.len = r.len > left ? r.len - left : 0;
    }
    r.pages = (r.len + KV16_PAGE - 1) / KV16_PAGE;
    if (a.window > 0) {
        const int before = r.len - r.n + 1;                                   // positions up to the first row's own
        const int from = before > a.window ? (before - a.window) / KV16_PAGE : 0;
        const int sinks = a.sinks / KV16_PAGE + (a.sinks % KV16_PAGE != 0);
        r.lead = sinks < from ? sinks : from;
        r.skip = from - r.lead;
        r.pages -= r.skip;
    }
    return r;
}
// Is it this launch's?
__device__ __forceinline__ bool ours(const Kv16AttnArgs& a, const Request& r) { return a.whose == Kv16AttnArgs::EVERYONES || (r.n * a.group <= KV16_FEW_ROWS) == (a.whose == Kv16AttnArgs::THOSE_OF_FEW_ROWS); }
__device__ __forceinline__ int page_number(const Request& r, int v) { return v < r.lead ? v : v + r.skip; }

// What a row sees: positions below `end`, from `from` on or below the sinks.
struct Sight {
    int from, end;
};
__device__ __forceinline__ Sight sight_of(const Kv16AttnArgs& a, const Request& rq, int token)
{
    const int end = rq.len - rq.n + token + 1;
    return Sight{a.window > 0 && end > a.window ? end - a.window : 0, end};
}
__device__ __forceinline__ bool sees(const Sight& s, int sinks, int pos) { return pos < s.end && (pos >= s.from || pos < sinks); }

// Pages per chunk of a request that looks at `pages` of them: a function of its own length and of how many workgroups the call has (by its B, max_q and max_pages), so that in
// calls of the same extents a request's chunk borders, and with them the bits of its result, do not depend on the other requests.
__device__ __forceinline__ int chunk_pages(const Kv16AttnArgs& a, int pages)
{
    const int size = a.nsplit == 1 ? pages : (pages + a.nsplit - 1) / a.nsplit;
    return size > a.min_chunk ? size : a.min_chunk;
}

// Where a request's r-th row of a cache head with `group` query heads lies among the partial results and statistics: by request and token, so that they
// take what the largest request asks for and not what all tokens of the call do.
__device__ __forceinline__ size_t part_row(const Kv16AttnArgs& a, int b, int r, int g, int group)
{
    return ((size_t)b * a.part_q + r / group) * a.Hq + (size_t)g * group + r % group;
}

// The same by cache head, for what kv16_attn_weights and kv16_attn_weigh read.
__device__ __forceinline__ size_t stats_row(const Kv16AttnArgs& a, int b, int g, int r) { return ((size_t)b * a.Hkv + g) * a.tiles * KV16_TILE_ROWS + r; }

// over the lanes of the same lo (the four hi)
__device__ __forceinline__ float max_over_hi(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < __builtin_inff(); }

// The sum of weights times values for one row, from the definition: only positions that it sees, each weight above zero.  For rows whose result is not finite in some
// column: matrix products multiply a weight of zero with a value that the row does not see, and a NaN there must not come through; and a weight that underflows
// turns an infinity into a NaN.  Called by all THREADS threads of a workgroup; thread d < D returns column d, and the sum of the weights.
template <int D, int THREADS>
__device__ __forceinline__ float slow_row(const Kv16AttnArgs& a, const Request& rq, int b, int g, size_t head_row, int token, int v0, int v1, float m, float* s_w, float& total)
{
    const int tid = threadIdx.x;
    const Sight sight = sight_of(a, rq, token);
    const uint16_t* const q = a.q + head_row * D;
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    const float ms = m == -__builtin_inff() ? 0.f : m;
    float sum = 0.f;
    total = 0.f;
    for (int v = v0; v < v1; ++v) {
        const int number = page_number(rq, v), page = table[number];
        if (page < 0 || page >= a.num_pages) continue;                        // (uniform)
        const uint16_t* const head = a.pages + ((size_t)(unsigned)page * a.Hkv + g) * kv16_head_values(D);
        __syncthreads();
        if (tid < KV16_PAGE) {
            float t = 0.f;
            for (int part = 0; part < D / 8; ++part) {
                const half8 k = __builtin_bit_cast(half8, ld_cached(head + kv16_key_at(tid, part, D))), x = __builtin_bit_cast(half8, ld_cached(q + part * 8));
#pragma unroll
                for (int e = 0; e < 8; ++e) t = __builtin_fmaf((float)k[e], (float)x[e], t);
            }
            const float w = __builtin_amdgcn_exp2f(t * a.scale2 - ms);
            s_w[tid] = !sees(sight, a.sinks, number * KV16_PAGE + tid) ? -1.f : w < 1e-37f && t * a.scale2 > -__builtin_inff() ? 1e-37f : w;
        }
        __syncthreads();
        if (tid < D)
            for (int p = 0; p < KV16_PAGE; ++p) {
                const float w = s_w[p];
                if (w != -1.f) {
                    sum += w * half_bits_to_float(head[kv16_value_at(p, tid, D)]);
                    total += w;
                }
            }
    }
    __syncthreads();
    return sum;
}

// ---- one token per request, or a few: up to 16 rows of a cache head, cut along the positions ------------------------
//
// What bounds it is the pages' way from memory, 4 D bytes a position and cache head.  A workgroup (four waves, or eight) takes a chunk of the pages that one request looks at, for one cache head; a
// wave takes half of every second page (or fourth), 32 positions, straight from memory into registers, its next half in flight behind it.  (Whole pages, every fourth, leave waves of short chunks without
// work: 32 requests of up to 2048 positions, 32/32 heads of 128, 116 us, like this 110.)  Rows are (new token, query head of the group) pairs, the columns of two matrix products
// (v_mfma_f32_16x16x32_f16):
//   S = K Q^T     : 16 positions x 16 rows;
//   O^T = V^T P^T : a lane has the weights of positions 16 i + 4 hi + r of its row, which is the B operand as it stands, for the page holds the values in that order.
// So nothing but the rows' maxima crosses lanes, and those only when a weight leaves fp16's range.  Weights are multiplied as two fp16 summands (2^-21 of a weight
// off at most down to 2^-12 of the largest, 2^-33 of that below, where one alone is off by 2^-11 and as much as the result's own rounding).
// Measured, us a pass with kv16_attn_combine: those 32 requests 107 with eight waves (6.4 TB/s; a copy of 128 MiB 7.1), 3 of 131000 and less on 64/8 heads 86 (6.2 TB/s), 16 of 32000 and less with a window
// of 4096 48 (5.3), two of 468 and less with 8 heads of 64 columns 5.9, which is a launch and four loads one behind the other.
template <int D, int WAVES> constexpr int KD_LDS = WAVES * 16 * (D + 4) * 4;
constexpr float WEIGHT_LOG2 = 9.0f;              // weights are held as 2^9 p of a maximum that may lag by 2^6 (fp16 ends at 2^16)

// The n-th request by length, the longest first, of up to 64.  Workgroups that follow each other by as many as there are compute units share one, so with chunks in this order, every second one backwards,
// each has long and short ones: 24 requests of up to 5000 positions, 64/8 heads of 128, 50 -> 46 us, with weights 64 -> 57; 64 of 6000 160 -> 146.
__device__ __forceinline__ int request_in_order(const Kv16AttnArgs& a, int n)
{
    const int lane = threadIdx.x & 63, len = lane < a.B ? a.seq_lens[lane] : 0;
    int before = 0;
    for (int i = 0; i < a.B; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        before += other > len || (other == len && i < lane);
    }
    return __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.B && before == n));      // (the places are a permutation, so some lane has this one)
}

// Two fp16 summands of four weights (the large one truncated, so that the small one is not negative).
__device__ __forceinline__ void split_weights(const float (&w)[4], half4& large, half4& small)
{
    const half2v h0 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[0], w[1])), h1 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[2], w[3]));
    large = half4{h0[0], h0[1], h1[0], h1[1]};
    const half2v first = {(_Float16)-1.0f, (_Float16)0.0f}, second = {(_Float16)0.0f, (_Float16)-1.0f};
    const float r[4] = {__builtin_amdgcn_fdot2(h0, first, w[0], false), __builtin_amdgcn_fdot2(h0, second, w[1], false), __builtin_amdgcn_fdot2(h1, first, w[2], false),
                        __builtin_amdgcn_fdot2(h1, second, w[3], false)};      // w - large, without conversions
    const half2v s0 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(r[0], r[1])), s1 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(r[2], r[3]));
    small = half4{s0[0], s0[1], s1[0], s1[1]};
}
__device__ __forceinline__ half8 join(half4 a, half4 b) { return half8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// SCORES: they are left for kv16_attn_weigh, 4 bytes a row and position: 24 requests of up to 5000 positions, 64/8 heads, 46 us without weights, 57 with them: 8 for the stores, 3 for the sums.
template <int D, int WAVES, bool SCORES>
__global__ __launch_bounds__(64 * WAVES, 2) void kv16_attn_decode(Kv16AttnArgs a)
{
    constexpr int NB = D / 32, NT = D / 16;      // blocks of a key, tiles of a value's columns
    constexpr int HALF = 32;                     // positions of half a page
    extern __shared__ uintx4 kd_smem[];
    float (*const s_o)[16][D + 4] = reinterpret_cast<float (*)[16][D + 4]>(kd_smem);      // of each wave
    __shared__ float s_m[WAVES][16], s_l[WAVES][16], s_w[KV16_PAGE];
    __shared__ unsigned s_odd;

    const int tid = threadIdx.x, lane = tid & 63, lo = lane & 15, hi = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = a.group;
    const int g = blockIdx.x, chunk = blockIdx.z, b = a.sorted ? request_in_order(a, chunk & 1 ? a.B - 1 - (int)blockIdx.y : (int)blockIdx.y) : (int)blockIdx.y;
    const Request rq = find_request(a, b);
    const int rows = rq.n * group;               // at most 16: row r is token r / group, head r % group
    if (rows <= 0 || !ours(a, rq)) return;
    const int size = chunk_pages(a, rq.pages);
    const int c0 = chunk * size, c1 = c0 + size < rq.pages ? c0 + size : rq.pages;
    if (chunk > 0 && c0 >= rq.pages) return;
    const bool whole = rq.pages <= size;
    if (tid == 0) s_odd = 0;

    auto row_of_column = [&](int r) { return (size_t)(rq.first + r / group) * a.Hq + (size_t)g * group + r % group; };      // (token, head) row of q and out
    const int col = lo < rows ? lo : rows - 1;
    half8 queries[NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) queries[k] = __builtin_bit_cast(half8, ld_cached(a.q + row_of_column(col) * D + k * 32 + hi * 8));
    if (a.queries && chunk == 0 && wv == 0)      // as operands, for kv16_attn_weights
#pragma unroll
        for (int k = 0; k < NB; ++k) *reinterpret_cast<half8*>(a.queries + (stats_row(a, b, g, 0) / 16 * NB + k) * 512 + lane * 8) = queries[k];
    const Sight mine = sight_of(a, rq, col / group);
    const Sight low = sight_of(a, rq, 0), high = sight_of(a, rq, rq.n - 1);

    // This wave's half of pages c0 + wv / 2, then every WAVES / 2-th; an entry that is no page: -1.  Loads are unconditional (a page that is not there: page 0), so that nothing
    // waits for a load but what uses it.
    const int half = wv & 1, v0 = c0 + (wv >> 1), n_it = (c1 - v0 + WAVES / 2 - 1) / (WAVES / 2);
    int entries = -1;                            // of the 64 pages from iteration `it` & ~63 on, one per lane
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    auto page_at = [&](int it) {                 // asked for in order
        if ((it & 63) == 0) {
            const int v = v0 + (it + lane) * (WAVES / 2);
            entries = v < c1 ? table[page_number(rq, v)] : -1;
            asm volatile("" : "+v"(entries));    // waited for here, and not in every iteration behind whatever else is in flight
        }
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e >= 0 && e < a.num_pages ? e : -1;
    };
    const uint16_t* const heads = a.pages + (size_t)g * kv16_head_values(D) + half * HALF * D;
    const size_t page_values = (size_t)a.Hkv * kv16_head_values(D);
    auto head = [&](int page) { return heads + (size_t)(unsigned)(page < 0 ? 0 : page) * page_values; };
    uintx4 kx[2 * NB], vx[NT];                   // keys of two tiles of positions, values
    auto ask_keys = [&](int page) __attribute__((always_inline)) {
        const uint16_t* const from = head(page);
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) kx[i] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(from + i * 512 + lane * 8));
    };
    auto ask_values = [&](int page, int t) __attribute__((always_inline)) {
        const uint16_t* const from = head(page) + kv16_values(D);
        vx[t] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(from + t * 512 + lane * 8));
    };
    int page = n_it > 0 ? page_at(0) : -1;
    ask_keys(page);
#pragma unroll
    for (int t = 0; t < NT; ++t) ask_values(page, t);

    // m: the maximum that the row's weights refer to; start: WEIGHT_LOG2 - m, so that a weight is 2^(score + start); l: the weights' sum, as a product with ones
    // (every element is the lane's row's)
    float m = -__builtin_inff(), start = 0.f;
    bool fresh = true;                           // some row has no maximum yet
    floatx4 l = {0.f, 0.f, 0.f, 0.f};
    const half8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
    floatx4 o[NT];                               // O^T: column 16 t + 4 hi + i of the lane's row
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};

    for (int it = 0; it < n_it; ++it) {
        const int number = page_number(rq, v0 + it * (WAVES / 2));
        const int next = it + 1 < n_it ? page_at(it + 1) : -1;
        const bool there = page >= 0;
        const int base = number * KV16_PAGE + half * HALF;
        floatx4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, kx[i * NB + k]), queries[k], s[i], 0, 0, 0);
        ask_keys(next);
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = __builtin_fmaf(s[i >> 2][i & 3], a.scale2, start);
        if (!there || base + HALF > low.end || (base < high.from && base + HALF > a.sinks)) {      // some row does not see all of it
            unsigned keep[4] = {0, 0, 0, 0};     // of the values' dwords: what any row of the tile sees
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int pos = base + 16 * (i >> 2) + 4 * hi + (i & 3);
                if (!there || !sees(mine, a.sinks, pos)) t[i] = -__builtin_inff();
                if (there && sees(Sight{low.from, high.end}, a.sinks, pos)) keep[i >> 1] |= 0xffffu << (16 * (i & 1));
            }
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) vx[k][i] &= keep[i];
        }
        floatx4 score[2];                        // stored behind the values' loads: those of the next half are waited for in order, and a store takes longer
        if (SCORES)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) score[i][r] = t[4 * i + r] == -__builtin_inff() ? t[4 * i + r] : s[i][r] * a.scale2;
        half8 pl, ps;
        auto weights = [&]() __attribute__((always_inline)) {
            half4 large[2], small[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(t[4 * i + r]);
                split_weights(w, large[i], small[i]);
            }
            pl = join(large[0], large[1]);
            ps = join(small[0], small[1]);
        };
        weights();
        // Is a weight past 2^15?  Its fp16 exponent is 30 or 31 then, and 0x0800 more carries into the sign.  No maximum crosses lanes unless one is.
        half2v top = {0, 0};
#pragma unroll
        for (int r = 0; r < 8; r += 2) top = __builtin_elementwise_maximum(top, half2v{pl[r], pl[r + 1]});
        if (fresh || __builtin_amdgcn_ballot_w64(((__builtin_bit_cast(unsigned, top) + 0x08000800u) & 0x80008000u) != 0) != 0ull) {
            float mb = t[0];                     // (a NaN comes through; its row is not a number anyway)
#pragma unroll
            for (int i = 1; i < 8; ++i) mb = __builtin_elementwise_maximum(mb, t[i]);
            const float mn = __builtin_elementwise_maximum(m, max_over_hi(mb) - start);
            const bool none = mn == -__builtin_inff();
            const float corr = __builtin_amdgcn_exp2f(m - (none ? 0.f : mn)), now = none ? 0.f : WEIGHT_LOG2 - mn;
            fresh = __builtin_amdgcn_ballot_w64(none) != 0ull;
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = t[i] - start + now;
            m = mn;
            start = now;
            l *= corr;
#pragma unroll
            for (int k = 0; k < NT; ++k) o[k] *= corr;
            weights();
        }
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pl, l, 0, 0, 0);
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, ps, l, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            const half8 v = __builtin_bit_cast(half8, vx[k]);
            o[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, o[k], 0, 0, 0);
            o[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ps, o[k], 0, 0, 0);
            ask_values(next, k);
        }
        if (SCORES && lo < rows) {
            float* const to = a.scores + (((size_t)b * a.Hkv + g) * a.max_q * group + lo) * a.max_pages * KV16_PAGE + base + 4 * hi;
#pragma unroll
            for (int i = 0; i < 2; ++i) *reinterpret_cast<floatx4*>(to + 16 * i) = score[i];
        }
        page = next;
    }

#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<floatx4*>(&s_o[wv][lo][16 * t + 4 * hi]) = o[t];
    if (hi == 0) { s_m[wv][lo] = m; s_l[wv][lo] = l[0]; }
    __syncthreads();
    auto finish = [&](int c, int d, float of, float lf, float mn) {
        const size_t row = row_of_column(c), pr = part_row(a, b, c, g, group);
        if (whole) {
            a.out[row * D + d] = lf == 0.f ? 0 : to_half_bits(of / lf);
            if (d == 0 && a.stats) {
                float* const to = a.stats + 2 * stats_row(a, b, g, c);
                to[0] = mn == -__builtin_inff() ? 0.f : mn;
                to[1] = lf == 0.f ? 0.f : 1.0f / lf;
            }
        } else {
            float* const po = a.part + (pr * a.nsplit + chunk) * kv16_part(D);
            po[d] = of;
            if (d == 0) { po[D] = mn; po[D + 1] = po[D + 2] = lf; }
        }
    };
    auto merge = [&](int c, float (&cw)[WAVES], float& lf) {      // fixed order: waves 0 .. WAVES - 1
        // (a maximum that is not a number stays one: a wave has it from a score of infinity or NaN, and behind one of the others' slow_row would make a sum of infinity of it, one over which is zero)
        float mn = s_m[0][c];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) mn = __builtin_elementwise_maximum(mn, s_m[w][c]);
        const float ms = mn == -__builtin_inff() ? 0.f : mn;
        lf = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            cw[w] = __builtin_amdgcn_exp2f(s_m[w][c] - ms);
            lf += s_l[w][c] * cw[w];
        }
        return mn;
    };
    for (int idx = tid; idx < rows * D; idx += 64 * WAVES) {
        const int c = idx / D, d = idx % D;
        float cw[WAVES], lf, of = 0.f;
        const float mn = merge(c, cw, lf);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) of += s_o[w][c][d] * cw[w];
        // (weights are 2^WEIGHT_LOG2 times what they stand for, all of them)
        if (finite(of)) finish(c, d, of, lf, mn);
        else atomicOr(&s_odd, 1u << c);
    }
    __syncthreads();
    const unsigned odd = s_odd;
    for (int c = 0; c < rows; ++c) {
        if (!(odd >> c & 1)) continue;           // (uniform)
        float cw[WAVES], lf;
        const float mn = merge(c, cw, lf);
        const float of = slow_row<D, 64 * WAVES>(a, rq, b, g, row_of_column(c), c / group, c0, c1, mn, s_w, lf);
        if (tid < D) finish(c, tid, of * 512.0f, lf * 512.0f, mn);
    }
}

// The chunks' (sum, maximum, weight) triples of a request's rows, (token, head) pairs in the order of q.  A group of D threads has a row of up to eight chunks to itself, or any where there are many rows; else all
// groups take every GROUPS-th chunk each, eight loads in flight, and meet in LDS: a fixed order.  The loads come before anything is known of the request (what lies behind its last
// chunk is the workspace's, and not used).  16 requests of 64 heads and six chunks: 4.6 us (a row for a workgroup: 5.2).
constexpr int KC_THREADS = 512, KC_AHEAD = 8, KC_ROWS = 4096;
template <int D> __host__ __device__ bool combine_alone(const Kv16AttnArgs& a) { return a.nsplit <= KC_AHEAD || (long)a.B * a.Hq * a.part_q >= KC_ROWS; }
template <int D> __host__ __device__ int combine_blocks(const Kv16AttnArgs& a)
{
    const int rows = a.Hq * a.part_q, each = combine_alone<D>(a) ? KC_THREADS / D : 1;
    return a.nsplit > 1 ? (rows + each - 1) / each : 0;
}
template <int D>
__device__ __forceinline__ void combine_rows(const Kv16AttnArgs& a, int block, int b)
{
    constexpr int GROUPS = KC_THREADS / D;
    __shared__ float s_o[GROUPS][D], s_w[GROUPS][KV16_MAX_SPLIT];
    const int lane = threadIdx.x & 63, d = threadIdx.x % D, grp = threadIdx.x / D;
    const bool alone = combine_alone<D>(a);
    if (block >= combine_blocks<D>(a)) return;
    const int row = alone ? block * GROUPS + grp : block, chunk = alone ? 0 : grp, stride = alone ? 1 : GROUPS, own = alone ? grp : 0;
    const bool exists = row < a.part_q * a.Hq;
    const int i = row / a.Hq;
    const float* const first = a.part + ((size_t)b * a.part_q * a.Hq + (exists ? row : 0)) * a.nsplit * kv16_part(D);
    float m = lane < a.nsplit ? first[(size_t)lane * kv16_part(D) + D] : 0.f;
    float w = lane < a.nsplit ? first[(size_t)lane * kv16_part(D) + D + 1] : 0.f;
    float v[KC_AHEAD];
#pragma unroll
    for (int k = 0; k < KC_AHEAD; ++k) v[k] = chunk + k * stride < a.nsplit ? first[(size_t)(chunk + k * stride) * kv16_part(D) + d] : 0.f;
    const Request rq = find_request(a, b);
    const int size = chunk_pages(a, rq.pages), live = (rq.pages + size - 1) / size;
    const bool cut = exists && i < rq.n && rq.pages > size && ours(a, rq);      // (one chunk: the first pass has written this output)
    m = lane < live ? m : -__builtin_inff();
    w = lane < live ? w : 0.f;
    float top = m;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, sh));
    const float c = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.f : top));
    float l = w * c;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) l += __shfl_xor(l, sh);
    if (alone || grp == 0) s_w[own][lane] = __builtin_fmaxf(c, 1e-37f);      // (an infinity in a chunk whose weights underflow stays one; a group's waves write the same)
    __syncthreads();
    float sum = 0.f;
    for (int k0 = chunk;;) {
#pragma unroll
        for (int k = 0; k < KC_AHEAD; ++k)
            if (k0 + k * stride < live) sum += v[k] * s_w[own][k0 + k * stride];
        k0 += KC_AHEAD * stride;
        if (k0 >= live) break;
#pragma unroll
        for (int k = 0; k < KC_AHEAD; ++k) v[k] = k0 + k * stride < live ? first[(size_t)(k0 + k * stride) * kv16_part(D) + d] : 0.f;
    }
    if (!alone) {
        s_o[grp][d] = sum;
        __syncthreads();
        sum = s_o[0][d];
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) sum += s_o[k][d];
    }
    if (!cut || (!alone && grp > 0)) return;
    a.out[((size_t)rq.first * a.Hq + row) * D + d] = l == 0.f ? 0 : to_half_bits(sum / l);
    if (d == 0 && a.stats && !a.scores) {
        float exact = 0.f;
        for (int k = 0; k < live; ++k) exact += first[(size_t)k * kv16_part(D) + D + 2] * s_w[own][k];
        const int h = row - i * a.Hq, g = h / a.group;
        float* const to = a.stats + 2 * stats_row(a, b, g, i * a.group + h - g * a.group);
        to[0] = top == -__builtin_inff() ? 0.f : top;
        to[1] = exact == 0.f ? 0.f : 1.0f / exact;
    }
}
template <int D>
__global__ __launch_bounds__(KC_THREADS) void kv16_attn_combine(Kv16AttnArgs a)
{
    combine_rows<D>(a, blockIdx.x, blockIdx.y);
}

// ---- many rows of a cache head: prompts and chunks of them ----------------------------------------------------------
//
// A workgroup takes 128 rows of one cache head, 32 a wave, and walks the pages that any of them sees.  Pages come straight into LDS as they lie in memory (two buffers for keys, two for
// values, 64 KB where D is 128: two workgroups a compute unit), which is the order in which the operands of v_mfma_f32_16x16x32_f16 are read: 1 KB in a row for a wave, no bank conflicts.
// The products are those of kv16_attn_decode, with two tiles of 16 rows, so that each operand from LDS is multiplied twice.
//
// What bounds it are the matrix products, 4 D FLOP a position and row, and the exponentials, one a position and row, in whose time the SIMD's matrix core rests.  So a wave has
// the exponentials of a page between the products of the next page's scores, and its scaling and maxima between those of the values, and the two workgroups of a compute unit fill what is
// left.  Weights are one fp16 each, cut (see weigh); a maximum may lag behind by 2^6, so that accumulators are hardly ever scaled.
// Measured: a prompt of 4096 tokens, 40/40 heads of 128, 190 to 195 us from card to card (880 to 910 TFLOP/s of what it sees; a matrix product of 8192^3 reaches 1387 here); chunks of up to 777 tokens on up to 8029
// positions, window 2000, 64/8 heads, 126 us, where the 616 tiles of equal work are two or three to a compute unit, 20 percent more than their mean.  256 rows in one workgroup a compute unit:
// 267 and 197 us.  Exponentials between products, or by themselves: 209 and 129, 211 and 141; products of 16x16x32 instead of 32x32x16, which read half the
// operands but take more power, so that the clock goes down: 197 and 129 instead of 209 and 129.  The weights' sum as a product with ones instead of 32 instructions a page: 200.6 -> 196.7 on one card; operands of
// both products asked for in one stream, over what a turn begins with: -> 194, and 129 -> 125.  Cut into chunks wherever that fills compute units that have one
// workgroup: 5 chunks of 128 tokens, window 4096, 126 -> 111 us, but one of 800 on 4000 99 -> 126, for partial results are 4 D bytes a row: so only where chunks_worth() says (kv16_api.hip).
constexpr int KP_WAVES = 4, KP_AHEAD = 4, KP_BUFS = 2;
template <int D, int WAVES> constexpr int KP_LDS = 2 * KP_BUFS * 64 * D * 2 + WAVES * 2048;

// 64 x 16 bytes from `base` + 16 * lane to LDS
__device__ __forceinline__ void kp_bring(const uint16_t* base, unsigned lane_bytes, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_bytes), "s"(base), "s"(lds) : "memory");
}
__device__ __forceinline__ void kp_barrier()      // (loads into LDS stay in flight; kp_wait is for them)
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
template <int N> __device__ __forceinline__ void kp_wait() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// What a workgroup of WAVES waves works on: 32 WAVES rows of a cache head from row r0 on, and of the pages its request looks at c0 .. c1 - 1.
struct Tile {
    Request rq;
    int g, b, chunk, r0, all_rows, c0, c1;
    bool whole;
    __device__ __forceinline__ size_t row(const Kv16AttnArgs& a, int r) const { return (size_t)(rq.first + r / a.group) * a.Hq + (size_t)g * a.group + r % a.group; }      // of q and out
};
template <int WAVES> __device__ __forceinline__ Tile find_tile(const Kv16AttnArgs& a)
{
    Tile t;
    // the last rows first: they see the most
    const int number = blockIdx.x / (unsigned)a.Hkv;
    t.g = blockIdx.x - number * a.Hkv;
    t.r0 = (a.tiles - 1 - number) * 32 * WAVES;
    t.b = blockIdx.y;
    t.chunk = blockIdx.z;
    t.rq = find_request(a, t.b);
    t.all_rows = t.rq.n * a.group;
    const int size = chunk_pages(a, t.rq.pages);
    t.whole = t.rq.pages <= size;
    t.c0 = t.chunk * size;
    t.c1 = t.c0 + size < t.rq.pages ? t.c0 + size : t.rq.pages;
    return t;
}
// The arguments, read again: kept over the loop, they would take the scalar registers that it needs.
__device__ __forceinline__ const Kv16AttnArgs& arguments_again()
{
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Kv16AttnArgs*)(const void*)p;
}

// The result is divided by the sum of the weights as they were multiplied, rounded to fp16; STATS: the sum of the weights themselves, too, for kv16_attn_weights.
template <int D, int WAVES, bool STATS>
__global__ __launch_bounds__(64 * WAVES, 2) void kv16_attn_prompt(Kv16AttnArgs a)
{
    constexpr int NB = D / 32, NT = D / 16;      // steps of 32 columns of the scores' product, tiles of 16 columns of the result
    constexpr int PART = 64 * D * 2;             // bytes of a page's keys, or values, of a head
    constexpr int MINE = PART / 1024 / WAVES; // loads of each that a wave makes
    extern __shared__ uintx4 kp_smem[];
    __shared__ unsigned s_odd[WAVES];
    __shared__ Tile s_tile;
    __shared__ float s_m[32 * WAVES], s_exact[32 * WAVES], s_w[KV16_PAGE];

    const int tid = threadIdx.x, lane = tid & 63, lo = lane & 15, hi = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Tile tile = find_tile<WAVES>(a);
    const Request& rq = tile.rq;
    const int r0 = tile.r0, all_rows = tile.all_rows, c0 = tile.c0, c1 = tile.c1;
    if (r0 >= all_rows || !ours(a, rq) || (tile.chunk > 0 && c0 >= rq.pages)) return;
    if (tid == 0) s_tile = tile;                 // (for the end)

    // The lane's two rows, w0 + lo and 16 further on (rows that are not there: the last one), and what they see.
    const int w0 = r0 + wv * 32, first_token = r0 / a.group, first_head = r0 - first_token * a.group;
    size_t row[2];                               // of q and out
    int token[2];
    Sight mine[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int r = w0 + 16 * c + lo < all_rows ? w0 + 16 * c + lo : all_rows - 1, n = (r - r0 + first_head) / a.group;
        token[c] = first_token + n;
        row[c] = (size_t)(rq.first + token[c]) * a.Hq + (size_t)tile.g * a.group + (r - r0 + first_head - n * a.group);
        mine[c] = sight_of(a, rq, token[c]);
    }
    const Sight low = sight_of(a, rq, __builtin_amdgcn_readfirstlane(token[0])), high = sight_of(a, rq, __builtin_amdgcn_readlane(token[1], 15));
    const int last_row = r0 + 32 * WAVES - 1 < all_rows ? r0 + 32 * WAVES - 1 : all_rows - 1;
    const int tile_from = sight_of(a, rq, first_token).from, tile_end = sight_of(a, rq, first_token + (last_row - r0 + first_head) / a.group).end;
    const bool rows_here = w0 < all_rows;

    // The pages of this chunk that some row of the tile sees: of the sinks, then from the first row's window to the last row's own
    int first = tile_from / KV16_PAGE - rq.skip, past = (tile_end + KV16_PAGE - 1) / KV16_PAGE - rq.skip;
    int lead = a.sinks / KV16_PAGE + (a.sinks % KV16_PAGE != 0);      // (more than the request's where an earlier tile's window begins among them: nothing is skipped then)
    lead = lead < first ? lead : first;
    lead = lead < c1 ? lead : c1;
    first = first > c0 ? first : c0;
    past = past < c1 ? past : c1;
    const int n_lead = lead > c0 ? lead - c0 : 0, n_it = n_lead + (past > first ? past - first : 0);
    // (what the loop needs of it, in few scalar registers: the position at which turn `it`'s page begins)
    const int from_lead = c0 * KV16_PAGE, from_window = (first - n_lead + rq.skip) * KV16_PAGE;
    auto base_of = [&](int it) { return it * KV16_PAGE + (it < n_lead ? from_lead : from_window); };
    int entries = -1;
    const int* const table = a.page_table + (size_t)tile.b * a.max_pages;
    auto list = [&](int it) {                    // the table's entries of turns it .. it + 63, one a lane
        const int at = it + lane < n_it ? it + lane : n_it - 1;      // (no branch, here and in scrub: a loop with one that lanes take apart is put together anew, and accumulators are copied)
        const int e = table[at < 0 ? 0 : base_of(at) / KV16_PAGE];
        entries = it + lane < n_it ? e : -1;
    };
    auto listed = [&]() { asm volatile("" : "+v"(entries)); };      // waited for here
    auto page_at = [&](int it) __attribute__((always_inline)) {      // -1: not there
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e < a.num_pages ? e : -1;
    };

    list(0);
    half8 queries[2][NB];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b) queries[c][b] = __builtin_bit_cast(half8, ld_cached(a.q + row[c] * D + b * 32 + hi * 8));

    const unsigned smem_at = (unsigned)(size_t)(__attribute__((address_space(3))) void*)kp_smem, lane16 = lane * 16;
    const uint16_t* const heads = a.pages + (size_t)tile.g * kv16_head_values(D);
    const size_t page_values = (size_t)a.Hkv * kv16_head_values(D);
    // where a page's keys begin (a page that is not there: page 0, for nobody), and the j-th load of this wave's share of its keys or values
    auto head = [&](int page) __attribute__((always_inline)) { return heads + (size_t)(unsigned)(page < 0 ? 0 : page) * page_values; };
    const unsigned lds_at = smem_at + wv * 1024;
    auto bring_keys = [&](const uint16_t* from, unsigned buf, int j) __attribute__((always_inline)) {
        kp_bring(from + (wv + j * WAVES) * 512, lane16, lds_at + buf + j * WAVES * 1024);
    };
    auto bring_values = [&](const uint16_t* from, unsigned buf, int j) __attribute__((always_inline)) {
        kp_bring(from + kv16_values(D) + (wv + j * WAVES) * 512, lane16, lds_at + KP_BUFS * PART + buf + j * WAVES * 1024);
    };

    float m[2] = {-__builtin_inff(), -__builtin_inff()}, start[2] = {0.f, 0.f}, exact[2] = {0.f, 0.f};      // exact: of this lane's positions only
    floatx4 l[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};      // the weights' sum, as a product with ones (every element is the lane's row's)
    const half8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
    bool fresh = true;
    floatx4 o[2][NT], s[2][4];
    half8 pw[2][2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int t = 0; t < NT; ++t) o[c][t] = floatx4{0.f, 0.f, 0.f, 0.f};

    // A turn's operands, each for two products, in the order in which they are multiplied: 4 NB of the next page's keys, 2 NT of this page's values.  They are asked for KP_AHEAD ahead, in this
    // order, or the compiler would ask for each where it is needed and wait; the first ones in front of what the turn begins with.  `between` puts vector work into the time that the
    // i-th takes.
    constexpr int KEYS = 4 * NB, VALUES = 2 * NT;
    half8 f[KP_AHEAD];
    auto key = [&](unsigned buf, int i) __attribute__((always_inline)) { return __builtin_bit_cast(half8, kp_smem[buf / 16 + lane + ((i & 3) * NB + (i >> 2)) * 64]); };
    auto value = [&](unsigned buf, int i) __attribute__((always_inline)) { return __builtin_bit_cast(half8, kp_smem[(KP_BUFS * PART + buf) / 16 + lane + i * 64]); };
    auto ask_keys = [&](unsigned buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < KP_AHEAD; ++i) f[i] = key(buf, i);
        __builtin_amdgcn_sched_barrier(0);
    };
    // the scores of a page, into s; then values of another one are asked for
    auto multiply_keys = [&](unsigned buf, unsigned values, auto between) __attribute__((always_inline)) {
        const floatx4 none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
#pragma unroll
            for (int c = 0; c < 2; ++c) s[c][i & 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[i % KP_AHEAD], queries[c][i >> 2], i < 4 ? none : s[c][i & 3], 0, 0, 0);
            f[i % KP_AHEAD] = i + KP_AHEAD < KEYS ? key(buf, i + KP_AHEAD) : value(values, i + KP_AHEAD - KEYS);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // a page's weights times its values
    auto multiply_values = [&](unsigned buf, auto between) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
#pragma unroll
            for (int c = 0; c < 2; ++c) o[c][i % NT] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[(KEYS + i) % KP_AHEAD], pw[c][i / NT], o[c][i % NT], 0, 0, 0);
            if (i + KP_AHEAD < VALUES) f[(KEYS + i) % KP_AHEAD] = value(buf, i + KP_AHEAD);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // t: what the exponentials of a page are of, 16 positions for each of the lane's rows; largest: the largest of them
    float t[32], largest[2] = {-__builtin_inff(), -__builtin_inff()};
    auto scale = [&](int i) __attribute__((always_inline)) { t[i] = __builtin_fmaf(s[i >> 4][(i >> 2) & 3][i & 3], a.scale2, start[i >> 4]); };
    auto look = [&](int i) __attribute__((always_inline)) {      // (a NaN does not show, but its row's sums are not numbers)
        largest[i >> 3] = __builtin_fmaxf(__builtin_fmaxf(largest[i >> 3], t[2 * i]), t[2 * i + 1]);
    };
    // The i-th pair of weights.  They are cut to fp16's bits, not rounded to the nearest: their sum is one of cut weights too, so that what all are too small by cancels, and what is left is
    // half a step of each as with the other rounding; that one's conversion, of two values to the nearest, keeps matrix products of the SIMD's other wave from running for half of its time,
    // this one's does not.  (So do exponentials, for all of theirs.)
    auto weigh = [&](int i) __attribute__((always_inline)) {
        const int c = i >> 3, k = (i >> 2) & 1, e = 2 * (i & 3);
        const float w0 = __builtin_amdgcn_exp2f(t[2 * i]), w1 = __builtin_amdgcn_exp2f(t[2 * i + 1]);
        if (STATS) exact[c] += w0 + w1;
        const half2v w = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w0, w1));
        pw[c][k][e] = w[0];
        pw[c][k][e + 1] = w[1];
    };
    // What a row does not see of the page, and a maximum that weights refer to if there is none or a weight would be past 2^15.
    auto settle = [&](int base) __attribute__((always_inline)) {
        bool masked = false;
        if (base + KV16_PAGE > low.end) {        // some row's end is in front of the page's
            masked = true;
#pragma unroll
            for (int i = 0; i < 32; ++i) t[i] = mine[i >> 4].end - base - 4 * hi > 16 * ((i >> 2) & 3) + (i & 3) ? t[i] : -__builtin_inff();
        }
        if (base < high.from && base + KV16_PAGE > a.sinks) {      // some row's window begins behind the page's first position, and not all of them are sinks
            masked = true;
            const int hidden = a.sinks - base - 4 * hi;
            const int span[2] = {mine[0].from > a.sinks ? mine[0].from - a.sinks : 0, mine[1].from > a.sinks ? mine[1].from - a.sinks : 0};
#pragma unroll
            for (int i = 0; i < 32; ++i) t[i] = (unsigned)(16 * ((i >> 2) & 3) + (i & 3) - hidden) < (unsigned)span[i >> 4] ? -__builtin_inff() : t[i];
        }
        if (masked) {
            largest[0] = largest[1] = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) look(i);
        }
        if (fresh || __builtin_amdgcn_ballot_w64(__builtin_fmaxf(largest[0], largest[1]) > 15.0f) != 0ull) {
            fresh = false;
            bool some = false;                   // (else all sums are zeros)
            float corr[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float mn = __builtin_fmaxf(m[c], max_over_hi(largest[c]) - start[c]);
                const bool none = mn == -__builtin_inff();
                corr[c] = __builtin_amdgcn_exp2f(m[c] - (none ? 0.f : mn));
                const float now = none ? 0.f : WEIGHT_LOG2 - mn;
                fresh = fresh || __builtin_amdgcn_ballot_w64(none) != 0ull;
                some = some || __builtin_amdgcn_ballot_w64(m[c] != -__builtin_inff()) != 0ull;
#pragma unroll
                for (int i = 0; i < 16; ++i) t[16 * c + i] = t[16 * c + i] - start[c] + now;
                m[c] = mn;
                start[c] = now;
                l[c] *= corr[c];
                if (STATS) exact[c] *= corr[c];
            }
            // By way of LDS, some at a time: the compiler gives products of the accumulators registers of their own, and copies all of them to and fro on the other path (64 moves
            // of pairs a page, each a time in which no matrix product runs).
            if (some) {
                uintx4* const own = kp_smem + 2 * KP_BUFS * PART / 16 + wv * 128 + lane;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) own[c * 64] = __builtin_bit_cast(uintx4, o[c][n] * corr[c]);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                    for (int c = 0; c < 2; ++c) o[c][n] = __builtin_bit_cast(floatx4, own[c * 64]);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            }
        }
        largest[0] = largest[1] = -__builtin_inff();
    };
    // Values that nobody may read -- behind the request's last position, or of a page that is not there -- become zeros: a weight of zero times a NaN is one.
    auto scrub = [&](int base, bool there, unsigned buf) {
        char* const values = reinterpret_cast<char*>(kp_smem) + KP_BUFS * PART + buf;
        asm volatile("" : "+s"(base));           // (what depends on it stays here, under the caller's condition)
#pragma unroll
        for (int j = 0; j < PART / 16 / (64 * WAVES); ++j) {
            const int i = j * 64 * WAVES + tid;
            const int first_pos = base + i / (PART / 32) * 32 + (i / 16 & 3) * 4;
            uintx4 x = reinterpret_cast<uintx4*>(values)[i];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!there || first_pos + 16 * (e >> 2) + (e & 3) >= rq.len) x[e >> 1] &= ~(0xffffu << (16 * (e & 1)));
            reinterpret_cast<uintx4*>(values)[i] = x;
        }
    };

    // A wave's work is a chain: the scores of page 0, and then a turn for every page: it settles the weights' exponents, takes the exponentials between the products of the next page's scores, and
    // multiplies the weights with its values.  The waves meet at a turn's end; in turn `it` they read the values of page it and the keys of page it + 1, and what comes in meanwhile are
    // values of page it + 1 and keys of page it + 2, into the buffers that were read in the turn before.
    // (A wave works on all pages up to its last row's own; behind the last one it multiplies keys of whatever is there, for nobody: accumulators under a condition are copied.)
    const int here_end = rows_here ? high.end : 0;
    auto turns_to = [&](int end, int from, int most) { const int n = (end - from + KV16_PAGE - 1) / KV16_PAGE; return end <= from ? 0 : n < most ? n : most; };
    const int lead_turns = turns_to(here_end, from_lead, n_lead);
    const int n_wave = lead_turns < n_lead ? lead_turns : n_it > n_lead ? n_lead + turns_to(here_end, from_window + n_lead * KV16_PAGE, n_it - n_lead) : n_lead;
    listed();
    int page = page_at(0), page1 = page_at(1), page2 = page_at(2);      // of pages it, it + 1, it + 2
    const uint16_t *from1 = head(page1), *from2 = head(page2);
#pragma unroll
    for (int j = 0; j < MINE; ++j) {
        bring_keys(head(page), 0, j);
        bring_values(head(page), 0, j);
        bring_keys(from1, PART, j);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int b = 0; b < NB; ++b) asm volatile("" : "+v"(queries[c][b]));      // waited for here, and not in every turn behind what is on its way into LDS
    if (STATS && tile.chunk == 0 && rows_here)      // as operands, for kv16_attn_weights
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int b = 0; b < NB; ++b)
                *reinterpret_cast<half8*>(a.queries + (stats_row(a, tile.b, tile.g, w0 + 16 * c) / 16 * NB + b) * 512 + lane * 8) = queries[c][b];
    kp_wait<0>();
    kp_barrier();
    ask_keys(0u);
    multiply_keys(0u, 0u, [](int) {});
#pragma unroll
    for (int i = 0; i < 32; ++i) scale(i);
#pragma unroll
    for (int i = 0; i < 16; ++i) look(i);
    kp_barrier();
    unsigned b0 = 0, b1 = PART;                  // buffers of pages it and it + 1
    auto bring = [&](int j) __attribute__((always_inline)) {
        if (j < MINE) bring_keys(from2, b0, j);
        else if (j < 2 * MINE) bring_values(from1, b1, j - MINE);
    };
    auto begin = [&](int it) __attribute__((always_inline)) {
        if (page < 0 || base_of(it) + KV16_PAGE > rq.len) {
            scrub(base_of(it), page >= 0, b0);
            kp_barrier();
        }
        if (((it + 3) & 63) == 0) {
            list(it + 3);
            listed();
        }
    };
    auto end = [&](int it) __attribute__((always_inline)) {
        page = page1;
        page1 = page2;
        page2 = page_at(it + 3);
        from1 = from2;
        from2 = head(page2);
        const unsigned b = b0;
        b0 = b1;
        b1 = b;
        kp_wait<0>();
        kp_barrier();
    };
    // (tested at its end: a loop that is left at its head has the accumulators live in two places, and copies them)
    if (n_wave > 0) {
        int it = 0;
        do {
            ask_keys(b1);
            settle(page < 0 ? 0x7fffff00 : base_of(it));      // (nothing of a page that is not there is seen)
            begin(it);
            multiply_keys(b1, b0, [&](int i) __attribute__((always_inline)) {
                weigh(i * (16 / KEYS));
                if (KEYS == 8) weigh(2 * i + 1);
                bring(i);
            });
            // (the sum of the weights: by products, or each weight would be a vector instruction more)
            multiply_values(b0, [&](int i) __attribute__((always_inline)) {
                constexpr int BEGIN = 4, EACH = 16 / VALUES;      // of the next scores, 4 EACH at a time
                if (i < BEGIN) l[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pw[i & 1][i >> 1], l[i & 1], 0, 0, 0);
                else if (i < BEGIN + 16 / (2 * EACH)) {
#pragma unroll
                    for (int k = 0; k < 4 * EACH; ++k) scale(4 * EACH * (i - BEGIN) + k);
#pragma unroll
                    for (int k = 0; k < 2 * EACH; ++k) look(2 * EACH * (i - BEGIN) + k);
                }
            });
            end(it);
        } while (++it < n_wave);
    }
    for (int it = n_wave; it < n_it; ++it) {
        begin(it);
#pragma unroll
        for (int j = 0; j < 2 * MINE; ++j) bring(j);
        end(it);
    }
    kp_wait<0>();                                // (nothing may be on its way into LDS that is no longer this workgroup's)

    const Kv16AttnArgs& e = arguments_again();
    const Tile& at = s_tile;
    unsigned odd_rows = 0;                       // of the wave's 32
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        if (STATS) {
            exact[c] += __shfl_xor(exact[c], 16);
            exact[c] += __shfl_xor(exact[c], 32);
        }
        bool odd = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd = odd || !finite(o[c][t][i]);
        unsigned long long lanes = __builtin_amdgcn_ballot_w64(odd);
        lanes |= lanes >> 32;
        odd_rows |= ((unsigned)(lanes | lanes >> 16) & 0xffffu) << (16 * c);
    }
    const int here = at.all_rows - at.r0 - wv * 32;          // rows of this wave
    if (here < 32) odd_rows &= here <= 0 ? 0u : (1u << here) - 1u;
    if (lane == 0) s_odd[wv] = odd_rows;
    auto put_stats = [&](int r, float mm, float ll) {
        float* const to = e.stats + 2 * stats_row(e, at.b, at.g, r);
        to[0] = mm == -__builtin_inff() ? 0.f : mm;
        to[1] = ll == 0.f ? 0.f : 1.0f / ll;
    };
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int own = 16 * c + lo, r = at.r0 + wv * 32 + own;
        if (hi == 0) { s_m[wv * 32 + own] = m[c]; s_exact[wv * 32 + own] = exact[c]; }
        if (own >= here || (odd_rows >> own & 1)) continue;
        if (at.whole) {
            const float inv = l[c][0] == 0.f ? 0.f : 1.0f / l[c][0];
            uint16_t* const out = e.out + row[c] * D;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const half4 y = {(_Float16)(o[c][t][0] * inv), (_Float16)(o[c][t][1] * inv), (_Float16)(o[c][t][2] * inv), (_Float16)(o[c][t][3] * inv)};
                *reinterpret_cast<half4*>(out + 16 * t + 4 * hi) = y;
            }
            if (STATS && hi == 0) put_stats(r, m[c], exact[c]);
        } else {
            float* const po = e.part + (part_row(e, at.b, r, at.g, e.group) * e.nsplit + at.chunk) * kv16_part(D);
#pragma unroll
            for (int t = 0; t < NT; ++t) *reinterpret_cast<floatx4*>(po + 16 * t + 4 * hi) = o[c][t];
            if (hi == 0) { po[D] = m[c]; po[D + 1] = l[c][0]; po[D + 2] = exact[c]; }
        }
    }
    __syncthreads();
    for (int w = 0; w < WAVES; ++w) {
        unsigned rows = __builtin_amdgcn_readfirstlane(s_odd[w]);
        while (rows) {
            const int c = w * 32 + __builtin_ctz(rows), r = at.r0 + c;
            rows &= rows - 1;
            const float mm = s_m[c];
            float ll;
            const float of = slow_row<D, 64 * WAVES>(e, at.rq, at.b, at.g, at.row(e, r), r / e.group, at.c0, at.c1, mm, s_w, ll) * 512.0f;
            ll *= 512.0f;
            if (at.whole) {
                if (tid < D) e.out[at.row(e, r) * D + tid] = ll == 0.f ? 0 : to_half_bits(of / ll);
                if (STATS && tid == 0) put_stats(r, mm, s_exact[c]);
            } else {
                float* const po = e.part + (part_row(e, at.b, r, at.g, e.group) * e.nsplit + at.chunk) * kv16_part(D);
                if (tid < D) po[tid] = of;
                if (tid == 0) { po[D] = mm; po[D + 1] = ll; po[D + 2] = s_exact[c]; }
            }
        }
    }
}

// ---- what each position got of the rows' attention -------------------------------------------------------------------
//
// Up to 16 rows of a cache head: the few-rows kernel leaves its scores (4 bytes a row and position next to the 4 D that it reads); here they become weights with the rows' maxima and sums,
// and are added up over the rows.  A thread takes four positions.  Where requests are cut, the last workgroups put the rows' chunks together (combine_rows), and the others find the
// maxima and sums of their rows by themselves, so that neither waits for the other.
template <int D>
__global__ __launch_bounds__(KC_THREADS) void kv16_attn_weigh(Kv16AttnArgs a, int weighing)
{
    const int block = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    if (block >= weighing) {
        combine_rows<D>(a, (block - weighing) * a.Hkv + g, b);
        return;
    }
    __shared__ float s_m[KV16_FEW_ROWS], s_inv[KV16_FEW_ROWS];
    const int p0 = (block * KC_THREADS + threadIdx.x) * 4, wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const Request rq = find_request(a, b);
    if (block * KC_THREADS * 4 >= rq.len) return;
    const int number = p0 / KV16_PAGE, rows = rq.n * a.group, before = rq.len - rq.n;
    const size_t at = ((size_t)b * a.Hkv + g) * a.max_pages * KV16_PAGE + p0;
    const size_t stride = (size_t)a.max_pages * KV16_PAGE;
    const float* const scores = a.scores + ((size_t)b * a.Hkv + g) * a.max_q * a.group * stride + p0;
    const bool looked = p0 < rq.len && (number < rq.lead || number >= rq.lead + rq.skip);
    floatx4 s[8];
    auto ask = [&](int from) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 8; ++r) s[r] = looked && from + r < rows ? *reinterpret_cast<const floatx4*>(scores + (from + r) * stride) : floatx4{0.f, 0.f, 0.f, 0.f};
    };
    ask(0);
    const int size = chunk_pages(a, rq.pages), live = (rq.pages + size - 1) / size;
    for (int r = wv; r < rows; r += KC_THREADS / 64) {
        const size_t pr = part_row(a, b, r, g, a.group);
        float m, inv;
        if (live <= 1) {
            const float* const mine = a.stats + 2 * stats_row(a, b, g, r);
            m = mine[0];
            inv = mine[1];
        } else {
            const float* const mine = a.part + (pr * a.nsplit + lane) * kv16_part(D) + D;
            const float x = lane < live ? mine[0] : -__builtin_inff();
            float sum = lane < live ? mine[2] : 0.f;
            m = x;
#pragma unroll
            for (int sh = 1; sh < 64; sh <<= 1) m = __builtin_fmaxf(m, __shfl_xor(m, sh));
            m = m == -__builtin_inff() ? 0.f : m;
            sum *= __builtin_amdgcn_exp2f(x - m);
#pragma unroll
            for (int sh = 1; sh < 64; sh <<= 1) sum += __shfl_xor(sum, sh);
            inv = sum == 0.f ? 0.f : 1.0f / sum;
        }
        if (lane == 0) {
            s_m[r] = m;
            s_inv[r] = inv * 512.0f;             // (sums are of 2^WEIGHT_LOG2 times the weights)
        }
    }
    __syncthreads();
    if (p0 >= rq.len) return;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int from = 0;;) {
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if (!looked || from + r >= rows) continue;
            const float m = s_m[from + r], inv = s_inv[from + r];
            if (!finite(inv)) {                  // (the same for all threads) a sum that is not a number: what the row sees becomes one, and that only, for zero times it is one, too
                const int page = a.page_table[(size_t)b * a.max_pages + number];
                const Sight mine = sight_of(a, rq, (from + r) / a.group);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (page >= 0 && page < a.num_pages && sees(mine, a.sinks, p0 + k)) sum[k] = inv;
                continue;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] = __builtin_fmaf(inv == 0.f ? 0.f : __builtin_amdgcn_exp2f(s[r][k] - m), inv, sum[k]);
        }
        from += 8;
        if (from >= rows) break;
        ask(from);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (p0 + k < rq.len) a.weights_out[at + k] = (a.weights_in && p0 + k < before ? a.weights_in[at + k] : 0.f) + sum[k];
}

// More rows: the scores are made again.  A workgroup takes a page of a cache head, whose keys stay in its waves' registers (the A operand); the rows that see any of it come by, 16
// at a time, every WAVES-th 16 in a wave.  Weights in fp32, added up per lane (a lane has one row of each 16), then over lanes and waves: a fixed order.  Where the rows are in parts (plan_weights),
// one more launch adds their sums.
// For each 16 rows and 64 positions 262 kFLOP of matrix products (D = 128), 1024 exponentials and 4 KB of queries; the last is what bounds it.  So kv16_attn_prompt leaves the queries as operands, a
// KB at a time: from where they stand, 16 rows a load, the rows of 32 heads 8 KB apart fall on one channel of the cache (2001 tokens of 32/32 heads of 128, all of the call: 102 us, like this 87; 80 to 85 with the attention as it is now).
// Two pages in a workgroup, which halve the queries' way, leave too few of them (2001 tokens of 64/8 heads 317 us against 212); products of the next rows between the weights of the last: no gain
// (89); four pages in a workgroup, a page a wave, queries by way of LDS and rows in parts of 512 whose sums one more launch adds: less for them (161 as against 169), more for 32/32 heads (97).  Eight waves instead of four where the workgroups are few: 2001 tokens of 64/8 heads 188 -> 170 us; where they are not, it is the other way round (of 32/32: 87 -> 93).
constexpr int KW_PER_CU = 2;                     // up to so many workgroups for a compute unit: of eight waves instead of four
template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void kv16_attn_weights(Kv16AttnArgs a)
{
    constexpr int NB = D / 32, TILES = 4, SPAN = KV16_PAGE;      // tiles of 16 positions
    __shared__ float s_sum[WAVES][4 * TILES][64];
    const int tid = threadIdx.x, lane = tid & 63, lo = lane & 15, hi = lane >> 4, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int number = blockIdx.x / (unsigned)a.Hkv, g = blockIdx.x - number * a.Hkv, b = blockIdx.y, part = blockIdx.z;      // the first pages first: the most rows see them
    const Request rq = find_request(a, b);
    const int p0 = number * KV16_PAGE, group = a.group, before = rq.len - rq.n;
    if (p0 >= rq.len) return;
    const int page = a.page_table[(size_t)b * a.max_pages + number];
    const bool there = page >= 0 && page < a.num_pages;
    const uint16_t* const from = a.pages + ((size_t)(unsigned)(there ? page : 0) * a.Hkv + g) * kv16_head_values(D);
    half8 keys[TILES][NB];
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int k = 0; k < NB; ++k) keys[i][k] = __builtin_bit_cast(half8, ld_cached(from + (i * NB + k) * 512 + lane * 8));
    float sum[4 * TILES];
#pragma unroll
    for (int i = 0; i < 4 * TILES; ++i) sum[i] = 0.f;
    // the tokens that see any of it: from the one at its first position on, to the last that has its last position in the window
    const int first = p0 > before ? p0 - before : 0;
    int last = rq.n;
    if (a.window > 0 && p0 >= a.sinks) {
        const long most = (long)p0 + SPAN - 1 + a.window - before;      // token i sees from before + i + 1 - window on
        last = most < last ? (most < 0 ? 0 : (int)most) : last;
    }
    // rows of (token, head) pairs, 16 at a time as the attention left them
    const int tile_first = first * group / 16, tile_last = (last * group + 15) / 16, part_first = part * a.part_tiles, part_last = part_first + a.part_tiles;
    const int tile0 = (tile_first > part_first ? tile_first : part_first) + wv, tile_end = tile_last < part_last ? tile_last : part_last;
    int token = (tile0 * 16 + lo) / group, rest = (tile0 * 16 + lo) % group;
    const int token_step = 16 * WAVES / group, rest_step = 16 * WAVES - token_step * group;
    const size_t row0 = stats_row(a, b, g, 0) + tile0 * 16;
    const uint16_t* q = a.queries + row0 * D + lane * 8;
    const float* stats = a.stats + 2 * (row0 + lo);
    struct Rows {
        half8 q[NB];
        float2 stats;
        int token;
    };
    int left = tile_end - tile0;                 // (the last ones are asked for again, for nobody)
    auto ask = [&](Rows& x) __attribute__((always_inline)) {
        x.token = left > 0 ? token : last;      // (behind the last tile: of nobody)
#pragma unroll
        for (int k = 0; k < NB; ++k) x.q[k] = __builtin_bit_cast(half8, ld_cached(q + k * 512));
        x.stats = *reinterpret_cast<const float2*>(stats);
        left -= WAVES;
        token += token_step;
        rest += rest_step;
        if (rest >= group) {
            rest -= group;
            ++token;
        }
        if (left > 0) {
            q += 16 * WAVES * D;
            stats += 2 * 16 * WAVES;
        }
    };
    auto weigh = [&](const Rows& x) __attribute__((always_inline)) {
        const Sight mine = sight_of(a, rq, x.token), low = sight_of(a, rq, __builtin_amdgcn_readfirstlane(x.token)), high = sight_of(a, rq, __builtin_amdgcn_readlane(x.token, 15));
        floatx4 s[TILES];
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
            for (int i = 0; i < TILES; ++i) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(keys[i][k], x.q[k], k == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : s[i], 0, 0, 0);
        // (a sum that is not a number: a maximum that is not one, so that what the row sees becomes one, and that only)
        const bool number = finite(x.stats.y);
        const float m = number ? x.stats.x : __builtin_nanf(""), inv = x.token >= last ? 0.f : number ? x.stats.y * 512.0f : 1.0f;
        float w[4 * TILES];
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) w[i] = __builtin_fmaf(s[i >> 2][i & 3], a.scale2, -m);
        const bool none = inv == 0.f;            // a row that is not there, or sees nothing
        if (__builtin_amdgcn_ballot_w64(none) != 0ull || p0 + SPAN > low.end) {
            int seen = (none ? 0 : mine.end) - p0 - 4 * hi;
            asm volatile("" : "+v"(seen));      // (here, under the condition, and what depends on it)
#pragma unroll
            for (int i = 0; i < 4 * TILES; ++i) w[i] = seen > 16 * (i >> 2) + (i & 3) ? w[i] : -__builtin_inff();
        }
        if (p0 < high.from && p0 + SPAN > a.sinks) {
            const int span = mine.from > a.sinks ? mine.from - a.sinks : 0;
            int hidden = a.sinks - p0 - 4 * hi;
            asm volatile("" : "+v"(hidden));
#pragma unroll
            for (int i = 0; i < 4 * TILES; ++i) w[i] = (unsigned)(16 * (i >> 2) + (i & 3) - hidden) < (unsigned)span ? -__builtin_inff() : w[i];
        }
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) sum[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(w[i]), inv, sum[i]);
#pragma unroll
        for (int i = 0; i < 4 * TILES; ++i) asm volatile("" : "+v"(sum[i]));      // (now: next to the following products)
    };
    const int turns = there && first < last && tile0 < tile_end ? (tile_end - tile0 + WAVES - 1) / WAVES : 0;
    if (turns > 0) {
        Rows one, other;
        ask(one);
        int it = 0;
        do {                                     // (two turns: no copies from one to the other, each of which would wait for the load)
            ask(other);
            weigh(one);
            ask(one);
            weigh(other);                        // (of rows behind the last, in the end)
            __builtin_amdgcn_sched_barrier(0);
        } while ((it += 2) < turns);
    }
#pragma unroll
    for (int i = 0; i < 4 * TILES; ++i) s_sum[wv][i][lane] = sum[i];
    __syncthreads();
    if (tid >= SPAN) return;
    const int i = 4 * (tid >> 4) + (tid & 3), h = (tid >> 2) & 3;
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
        for (int k = 0; k < 16; ++k) total += s_sum[w][i][16 * h + ((k + tid) & 15)];      // (each thread in an order of its own, the same every time; no two of a bank at once)
    const int pos = p0 + tid;
    if (pos >= rq.len) return;
    const size_t at = ((size_t)b * a.Hkv + g) * a.max_pages * KV16_PAGE + pos;
    if (a.parts > 1) a.part[(size_t)part * a.B * a.Hkv * a.max_pages * KV16_PAGE + at] = total;
    else a.weights_out[at] = (a.weights_in && pos < before ? a.weights_in[at] : 0.f) + total;
}

// The sums of the parts of the rows.
constexpr int KA_THREADS = 256;
__global__ __launch_bounds__(KA_THREADS) void kv16_attn_add(Kv16AttnArgs a)
{
    const int p0 = (blockIdx.x * KA_THREADS + threadIdx.x) * 4, g = blockIdx.y, b = blockIdx.z;
    const size_t each = (size_t)a.B * a.Hkv * a.max_pages * KV16_PAGE, at = ((size_t)b * a.Hkv + g) * a.max_pages * KV16_PAGE + p0;
    const Request rq = find_request(a, b);
    if (p0 >= rq.len) return;
    floatx4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int part = 0; part < a.parts; ++part) sum += *reinterpret_cast<const floatx4*>(a.part + part * each + at);
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (p0 + k < rq.len) a.weights_out[at + k] = (a.weights_in && p0 + k < rq.len - rq.n ? a.weights_in[at + k] : 0.f) + sum[k];
}

template <int D, bool STATS>
void launch_prompt(const Kv16AttnArgs& a, dim3 grid, hipStream_t stream)
{
    static std::once_flag attr_once;
    std::call_once(attr_once, [] {
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&kv16_attn_prompt<D, KP_WAVES, STATS>), hipFuncAttributeMaxDynamicSharedMemorySize, KP_LDS<D, KP_WAVES>);
    });
    hipLaunchKernelGGL((kv16_attn_prompt<D, KP_WAVES, STATS>), grid, dim3(64 * KP_WAVES), (KP_LDS<D, KP_WAVES>), stream, a);
}

template <int D, int WAVES>
void launch_few(const Kv16AttnArgs& a, hipStream_t stream)
{
    static std::once_flag attr_once;
    std::call_once(attr_once, [] {
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&kv16_attn_decode<D, WAVES, false>), hipFuncAttributeMaxDynamicSharedMemorySize, KD_LDS<D, WAVES>);
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&kv16_attn_decode<D, WAVES, true>), hipFuncAttributeMaxDynamicSharedMemorySize, KD_LDS<D, WAVES>);
    });
    const dim3 grid((unsigned)a.Hkv, (unsigned)a.B, (unsigned)a.nsplit);
    const int combining = combine_blocks<D>(a), weighing = (a.max_pages * (KV16_PAGE / 4) + KC_THREADS - 1) / KC_THREADS;
    if (a.scores) {
        hipLaunchKernelGGL((kv16_attn_decode<D, WAVES, true>), grid, dim3(64 * WAVES), (KD_LDS<D, WAVES>), stream, a);
        hipLaunchKernelGGL((kv16_attn_weigh<D>), dim3((unsigned)(weighing + (combining + a.Hkv - 1) / a.Hkv), (unsigned)a.Hkv, (unsigned)a.B), dim3(KC_THREADS), 0, stream, a, weighing);
        return;
    }
    hipLaunchKernelGGL((kv16_attn_decode<D, WAVES, false>), grid, dim3(64 * WAVES), (KD_LDS<D, WAVES>), stream, a);
    if (combining) hipLaunchKernelGGL((kv16_attn_combine<D>), dim3((unsigned)combining, (unsigned)a.B), dim3(KC_THREADS), 0, stream, a);
}

template <int D>
void launch_many(const Kv16AttnArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.Hkv * a.tiles), (unsigned)a.B, (unsigned)a.nsplit);
    const int combining = combine_blocks<D>(a);
    if (a.weights_out) launch_prompt<D, true>(a, grid, stream);
    else launch_prompt<D, false>(a, grid, stream);
    if (combining) hipLaunchKernelGGL((kv16_attn_combine<D>), dim3((unsigned)combining, (unsigned)a.B), dim3(KC_THREADS), 0, stream, a);
}

template <int D>
hipError_t launch(const Kv16AttnArgs* few, const Kv16AttnArgs* many, hipStream_t stream)
{
    if (few && few->wide) launch_few<D, 8>(*few, stream);
    else if (few) launch_few<D, 4>(*few, stream);
    if (many) launch_many<D>(*many, stream);
    if (many && many->weights_out) {
        const dim3 pages((unsigned)(many->max_pages * many->Hkv), (unsigned)many->B, (unsigned)many->parts);
        if ((long)many->max_pages * many->Hkv * many->B * many->parts <= KW_PER_CU * many->num_cus) hipLaunchKernelGGL((kv16_attn_weights<D, 8>), pages, dim3(512), 0, stream, *many);
        else hipLaunchKernelGGL((kv16_attn_weights<D, 4>), pages, dim3(256), 0, stream, *many);
        if (many->parts > 1)
            hipLaunchKernelGGL(kv16_attn_add, dim3((unsigned)((many->max_pages * (KV16_PAGE / 4) + KA_THREADS - 1) / KA_THREADS), (unsigned)many->Hkv, (unsigned)many->B), dim3(KA_THREADS), 0, stream, *many);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv16_attention(const Kv16AttnArgs* few, const Kv16AttnArgs* many, hipStream_t stream)
{
    return (few ? few : many)->D == 128 ? launch<128>(few, many, stream) : launch<64>(few, many, stream);
}

}  // namespace thi
