// Attention over the 4-bit cache.  out = softmax(scale q K^T) V per head, K and V in pages; row i of a request's n new tokens sees the
// positions 0 .. length - n + i whose page exists.
#include "kv4.h"

#include <mutex>
#include <type_traits>

namespace thi {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// What a request's rows are: [first, first + n) of q, the last n of `len` positions.  Whatever the arrays hold stays within the buffers.
struct Request {
    int first, n, len;
};
__device__ __forceinline__ Request find_request(const Kv4AttnArgs& a, int b)
{
    Request r{b, 1, a.seq_lens[b]};
    const long most = (long)a.max_pages * KV4_PAGE;
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
    return r;
}

// ---- one token per request, or a few: 16 rows of a cache head at a time, cut along the positions --------------------
//
// A workgroup (4 waves) takes a chunk of one request's pages for one cache head; a wave takes a page at a time, straight from memory into
// registers, the next one in flight behind it.  Rows are (new token, query head of the group) pairs, 16 of them the columns of a
// matrix product:
//   S = K Q^T : v_mfma_f32_16x16x32_f16, 16 positions x 16 rows; a lane converts what it loaded of a key's row (v_cvt_scalef32_pk_f16_fp4, the
//               block's scale with it), the queries stay in registers in the same order of columns;
//   O^T = V^T P^T : a lane has the weights of positions 16 i + 4 hi + r of its row, which is the B operand of the next product as
//               it stands if the product's inner index runs over the positions in that order; the page holds the values so that a
//               lane's 16 bytes are these positions of two neighbouring columns (even and odd columns are tiles of their own).
// So nothing but the rows' maxima crosses lanes, and those only when a weight leaves fp16's range.  Weights are multiplied as two fp16 summands (2^-21 of a weight
// off at most down to 2^-12 of the largest, 2^-33 of that below, where one alone is off by 2^-11 and as much as the result's own rounding).
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
template <int D> struct PageRegs {
    uintx4 k[4];
    unsigned ks;
    uintx4 v[D / 32], vs[D / 32];
};

constexpr int KD_THREADS = 256, KD_WAVES = 4;
constexpr float WEIGHT_LOG2 = 9.0f;              // weights are held as 2^9 p of a maximum that may lag by 2^6 (fp16 ends at 2^16)

// byte i of w as the exponent of a float; the conversions take nothing else of it
__device__ __forceinline__ float scale_of(unsigned w, int i)
{
    return __builtin_bit_cast(float, i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1);
}
template <int I> __device__ __forceinline__ unsigned pair_of(unsigned codes, float s) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, I)); }

// Scores of 16 positions x 16 rows, in powers of two.
//
// The keys' codes are a matrix operand as they stand (v_mfma_scale_f32_16x16x128_f8f6f4: a lane's 16 bytes are one block of 32, the scales of the
// four tiles of a page one dword).  The queries, times the softmax scale and log2 e, are the other: each block of 32 as the sum of four e2m3
// numbers with scales of their own, 2^-4 apart.  Each takes four bits more; what is left is 2^-16 of the first scale at most, and the block's largest is more than
// 3.75 times that scale: 2^-17.9 of it.  The instruction runs at four times fp16's rate, so the four products cost what fp16's would; nothing has to be
// converted, nor, where the keys come from LDS, read in four times the bytes.  With D = 64 two of the four blocks are empty (the lanes hi >= 2: zeros on the queries' side).
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef float floatx32 __attribute__((ext_vector_type(32)));
typedef unsigned uintx6 __attribute__((ext_vector_type(6)));

struct Queries {
    intx8 f[4];
    unsigned scales;
};

struct QueryRow {
    uintx4 x[4];
};
// the lane's block of a row as it stands
template <int D> __device__ __forceinline__ QueryRow ask_queries(const uint16_t* row, int hi)
{
    QueryRow q;
#pragma unroll
    for (int s = 0; s < 4; ++s) q.x[s] = ld_cached(row + (hi < D / 32 ? hi : 0) * 32 + s * 8);
    return q;
}
template <int D> __device__ __forceinline__ void take_queries(const QueryRow& row, int hi, float scale2, Queries& q)
{
    const bool any = hi < D / 32;
    floatx16 even, odd;                          // columns of the block, then what the summands so far leave of them
    unsigned high = 0, low = 0;                  // the largest magnitudes' bits of the odd and even columns, in the upper half
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const uintx4 x = row.x[s];
        const half8 h = __builtin_bit_cast(half8, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            even[4 * s + e] = any ? (float)h[2 * e] * scale2 : 0.f;
            odd[4 * s + e] = any ? (float)h[2 * e + 1] * scale2 : 0.f;
            const unsigned u = x[e] & 0x7fff0000u, v = (x[e] << 16) & 0x7fff0000u;
            high = u > high ? u : high;
            low = v > low ? v : low;
        }
    }
    const unsigned top16 = any ? (high > low ? high : low) >> 16 : 0u;
    const unsigned top = __builtin_bit_cast(unsigned, half_bits_to_float((uint16_t)top16) * __builtin_fabsf(scale2));
    // the smallest 2^e that keeps the largest within 7.5; the summands' scales go down to e - 12
    int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x700000u ? 1 : 0);
    e = e < 13 ? 13 : e;
    q.scales = 0;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const float scale = __builtin_bit_cast(float, (unsigned)(e - 4 * s) << 23);
        // The conversions write their registers while they still read, and the compiler does not know: an operand that is needed no more may be given
        // some of the result's (a scale was, and the last summand was wrong that way).  Each is needed until behind its conversion.
        const uintx6 codes = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
        asm volatile("" : "+v"(even), "+v"(odd) : "v"(scale), "v"(codes));
        if (s < 3) {
            const floatx32 part = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(codes, scale);
            asm volatile("" : : "v"(scale), "v"(codes), "v"(part));
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                even[k] -= part[2 * k];
                odd[k] -= part[2 * k + 1];
            }
        }
#pragma unroll
        for (int k = 0; k < 6; ++k) q.f[s][k] = (int)codes[k];
        q.f[s][6] = q.f[s][7] = 0;
        q.scales |= (unsigned)(e - 4 * s) << (8 * s);
    }
    if (top16 >= 0x7c00u || top >= 0x7f800000u) q.scales = 0xffffffffu;      // infinities and NaN: the row is not a number
}
// where the lane's share of a page's keys lies; its scales, but for the lanes whose queries are empty, which must not meet a NaN
template <int D> __device__ __forceinline__ int key_offset(int lo, int hi) { return lo * (D / 2) + (hi & (D / 32 - 1)) * 16; }
template <int D> __device__ __forceinline__ int key_scale_offset(int lo, int hi) { return kv4_key_scales(D) + ((hi & (D / 32 - 1)) * 16 + lo) * 4; }
template <int D> __device__ __forceinline__ unsigned lane_scales(unsigned scales, int hi) { return D == 128 || hi < D / 32 ? scales : 0x7f7f7f7fu; }

// One of the four products of a tile (the smallest summand first).  A product that waits for the one in front of it takes twice as long: they go over
// several tiles before the next step.
template <int TILE, int STEP> __device__ __forceinline__ floatx4 score_step(uintx4 keys, unsigned scales, const Queries& q, floatx4 acc)
{
    const intx8 k = {(int)keys[0], (int)keys[1], (int)keys[2], (int)keys[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, q.f[3 - STEP], acc, 4, 2, TILE, (int)scales, 3 - STEP, (int)q.scales);
}
// Scores of a page's four tiles of 16 positions with CT tiles of rows, plus `from` of the lane's row.
template <int CT> __device__ __forceinline__ void score_page(const uintx4 (&keys)[4], unsigned scales, const Queries (&q)[CT], const floatx4 (&from)[CT], floatx4 (&acc)[CT][4])
{
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[ct][i] = from[ct];
    auto step = [&](auto s) __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            acc[ct][0] = score_step<0, decltype(s)::value>(keys[0], scales, q[ct], acc[ct][0]);
            acc[ct][1] = score_step<1, decltype(s)::value>(keys[1], scales, q[ct], acc[ct][1]);
            acc[ct][2] = score_step<2, decltype(s)::value>(keys[2], scales, q[ct], acc[ct][2]);
            acc[ct][3] = score_step<3, decltype(s)::value>(keys[3], scales, q[ct], acc[ct][3]);
        }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
}

// over the lanes of the same lo (the four hi)
__device__ __forceinline__ float max_over_hi(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
// The uniform part of an address, which stays in scalar registers this way.
#define GLOBAL __attribute__((address_space(1)))
__device__ __forceinline__ const GLOBAL unsigned char* uniform(const unsigned char* p)
{
    unsigned long long u = reinterpret_cast<unsigned long long>(p);
    asm volatile("" : "+s"(u));
    return reinterpret_cast<const GLOBAL unsigned char*>(u);
}

// Pages per chunk of a request with `pages` of them: a function of its own length and of how many workgroups the call has, so that a
// request's chunk borders, and with them the bits of its result, do not depend on its neighbours.
__device__ __forceinline__ int chunk_pages(const Kv4AttnArgs& a, int pages)
{
    const int size = (pages + a.nsplit - 1) / a.nsplit;
    return size > a.min_chunk ? size : a.min_chunk;
}

// Where a request's r-th row of a cache head with `group` query heads lies among the partial results: by request and token, so that they
// take what the largest request asks for and not what all tokens of the call do.
__device__ __forceinline__ size_t part_row(const Kv4AttnArgs& a, int b, int r, int g, int group)
{
    return ((size_t)b * a.max_q + r / group) * a.Hq + (size_t)g * group + r % group;
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

// MULTI: the rows of a tile may be of several new tokens, which see different positions.
template <int D, bool MULTI>
__global__ __launch_bounds__(KD_THREADS, MULTI ? 2 : 3) void kv4_attn_decode(Kv4AttnArgs a)
{
    constexpr int NB = D / 32;                   // blocks of a row
    __shared__ float s_o[KD_WAVES][16][D + 4];
    __shared__ float s_m[KD_WAVES][16], s_l[KD_WAVES][16];

    const int tid = threadIdx.x, lane = tid & 63, lo = lane & 15, hi = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = a.Hq / a.Hkv;
    const int g = blockIdx.x / a.tiles, r0 = (blockIdx.x % a.tiles) * 16;      // first row of this tile: row r is token r / group, head r % group
    const int b = blockIdx.y, chunk = blockIdx.z;
    const Request rq = find_request(a, b);
    const int rows = rq.n * group - r0 < 16 ? rq.n * group - r0 : 16;
    if (rows <= 0) return;
    const int pages = (rq.len + KV4_PAGE - 1) / KV4_PAGE, size = chunk_pages(a, pages);
    const int c0 = chunk * size, c1 = c0 + size < pages ? c0 + size : pages;
    if (chunk > 0 && c0 >= pages) return;
    const bool whole = pages <= size;

    const int n_it = (c1 - c0 - wv + KD_WAVES - 1) / KD_WAVES;      // this wave's pages: c0 + wv, c0 + wv + 4, ...
    auto row_of_column = [&](int c) {            // (token, head) row of q and out
        const int r = r0 + c;
        return (size_t)(rq.first + r / group) * a.Hq + (size_t)g * group + r % group;
    };
    const int col = lo < rows ? lo : rows - 1;
    const QueryRow query_row = ask_queries<D>(a.q + row_of_column(col) * D, hi);      // (in front of the page: it is waited for first)
    int entries = -1;                            // of the 64 pages from iteration `it` & ~63 on, one per lane
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    auto page_at = [&](int it) {                 // asked for in order
        if ((it & 63) == 0) {
            const int j = c0 + wv + (it + lane) * KD_WAVES;
            entries = j < c1 ? table[j] : -1;
            asm volatile("" : "+v"(entries));    // waited for here, and not in every iteration behind whatever else is in flight
        }
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e >= 0 && e < a.num_pages ? e : -1;
    };
    // One page's registers: the next page's keys are asked for when the scores are made, the next page's values block by block as they are multiplied.
    // Unconditionally (a page that is not there: page 0), so that nothing waits for a load but what uses it.
    PageRegs<D> x;
    const unsigned char* const heads = a.pages + (size_t)g * kv4_head_bytes(D);
    const size_t page_bytes = (size_t)a.Hkv * kv4_head_bytes(D);
    auto head = [&](int page) { return heads + (size_t)(unsigned)(page < 0 ? 0 : page) * page_bytes; };
    unsigned k_off = key_offset<D>(lo, hi), ks_off = key_scale_offset<D>(lo, hi) - kv4_key_scales(D), v_off = lane * 16, vs_off = hi * 16;
    auto ask_keys = [&](int page) __attribute__((always_inline)) {
        const unsigned char* from = head(page);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.k[i] = __builtin_nontemporal_load(reinterpret_cast<const GLOBAL uintx4*>(uniform(from) + k_off + i * 8 * D));
        x.ks = *reinterpret_cast<const GLOBAL unsigned*>(uniform(from + kv4_key_scales(D)) + ks_off);
    };
    auto ask_values = [&](int page, int t) __attribute__((always_inline)) {
        const unsigned char* const from = head(page);
        x.vs[t] = *reinterpret_cast<const GLOBAL uintx4*>(uniform(from + kv4_value_scales(D) + t * 64) + vs_off);
        x.v[t] = __builtin_nontemporal_load(reinterpret_cast<const GLOBAL uintx4*>(uniform(from + kv4_values(D) + t * 1024) + v_off));
    };
    int page = n_it > 0 ? page_at(0) : -1;
    ask_keys(page);
#pragma unroll
    for (int t = 0; t < NB; ++t) ask_values(page, t);

    Queries queries[1];
    take_queries<D>(query_row, hi, a.scale2, queries[0]);
    // positions this lane's row sees, and what every row of the tile sees
    const int seen = rq.len - rq.n + (MULTI ? (r0 + col) / group : 0) + 1;
    const int all_see = rq.len - rq.n + (MULTI ? r0 / group : 0) + 1;

    // m: the maximum that the row's weights refer to; start: what its scores start from (WEIGHT_LOG2 - m, so that a weight is 2^score); l: the weights'
    // sum, as a product with ones (every element is the lane's row's)
    float m = -__builtin_inff(), start = 0.f;
    bool fresh = true;                           // some row has no maximum yet
    floatx4 l = {0.f, 0.f, 0.f, 0.f};
    const half8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
    floatx4 o[2 * NB];                           // O^T: column 32 t + 2 (4 hi + i) of the lane's row in o[2 t], its right neighbour in o[2 t + 1]
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};

    for (int it = 0; it < n_it; ++it) {
        const int next = it + 1 < n_it ? page_at(it + 1) : -1;
        asm volatile("" : "+v"(k_off), "+v"(ks_off), "+v"(v_off), "+v"(vs_off));      // (not to be added to addresses in front of the loop, 64 bits wide)
        const bool there = page >= 0;
        const int base = there ? (c0 + wv + it * KD_WAVES) * KV4_PAGE : 0x7fffff00;      // (nothing of a page that is not there is seen)
        const bool masked = base + KV4_PAGE > all_see;
        floatx4 scores[1][4];
        {
            const floatx4 from[1] = {floatx4{start, start, start, start}};
            score_page<1>(x.k, lane_scales<D>(x.ks, hi), queries, from, scores);
        }
        ask_keys(next);
        float t[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = scores[0][i >> 2][i & 3];
        int first[NB];                               // the first position of a block that is not a number, where rows see different positions
        bool told = false;
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) t[i] = base + 16 * (i >> 2) + 4 * hi + (i & 3) < seen ? t[i] : -__builtin_inff();
            // Weights are zero where a row does not see a position, but 0 * NaN must not come through: scales of positions that no row sees become 0, and
            // where rows see different ones a NaN's scale too; the rows that do see it are told afterwards.
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int live = there ? rq.len - (base + 16 * i + 4 * hi) : 0;      // of the four bytes
                const unsigned keep = live >= 4 ? 0xffffffffu : live <= 0 ? 0u : (1u << (8 * live)) - 1u;
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    x.vs[k][i] &= keep;
                    const unsigned w = ~x.vs[k][i];                      // a byte of zero: a scale byte of 255
                    odd = odd || ((w - 0x01010101u) & ~w & 0x80808080u) != 0;
                }
            }
            if (MULTI && __builtin_amdgcn_ballot_w64(odd) != 0ull) {
                told = true;
#pragma unroll
                for (int k = 0; k < NB; ++k) {
                    first[k] = 0x7fffffff;
#pragma unroll
                    for (int i = 15; i >= 0; --i)
                        if ((x.vs[k][i >> 2] >> (8 * (i & 3)) & 255u) == 255u) {
                            first[k] = base + 16 * (i >> 2) + 4 * hi + (i & 3);
                            x.vs[k][i >> 2] &= ~(255u << (8 * (i & 3)));
                        }
#pragma unroll
                    for (int sh = 16; sh < 64; sh <<= 1) {
                        const int other = __shfl_xor(first[k], sh);
                        first[k] = other < first[k] ? other : first[k];
                    }
                }
            }
        }
        half8 pl[2], ps[2];
        auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                half4 large[2], small[2];
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    float w[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(t[8 * k + 4 * i2 + r]);
                    split_weights(w, large[i2], small[i2]);
                }
                pl[k] = join(large[0], large[1]);
                ps[k] = join(small[0], small[1]);
            }
        };
        weights();
        // Is a weight past 2^15?  Its fp16 exponent is 30 or 31 then, and 0x0800 more carries into the sign.  No maximum crosses lanes unless one is.
        half2v top = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 8; r += 2) top = __builtin_elementwise_maximum(top, half2v{pl[k][r], pl[k][r + 1]});
        if (fresh || __builtin_amdgcn_ballot_w64(((__builtin_bit_cast(unsigned, top) + 0x08000800u) & 0x80008000u) != 0) != 0ull) {
            float mb = t[0];                         // (a NaN comes through; its row is not a number anyway)
#pragma unroll
            for (int i = 1; i < 16; ++i) mb = __builtin_elementwise_maximum(mb, t[i]);
            const float mn = __builtin_elementwise_maximum(m, max_over_hi(mb) - start);
            const bool none = mn == -__builtin_inff();
            const float corr = __builtin_amdgcn_exp2f(m - (none ? 0.f : mn)), now = none ? 0.f : WEIGHT_LOG2 - mn;
            fresh = __builtin_amdgcn_ballot_w64(none) != 0ull;
#pragma unroll
            for (int i = 0; i < 16; ++i) t[i] += now - start;
            m = mn;
            start = now;
            l *= corr;
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k) o[k] *= corr;
            weights();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pl[k], l, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < 2; ++k) l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, ps[k], l, 0, 0, 0);
#pragma unroll
        for (int b4 = 0; b4 < NB; ++b4) {
            half8 ev[2], od[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uintx4 e, d;
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    const unsigned c = x.v[b4][2 * k + i2], w = x.vs[b4][2 * k + i2];
                    const unsigned y0 = pair_of<0>(c, scale_of(w, 0)), y1 = pair_of<1>(c, scale_of(w, 1)), y2 = pair_of<2>(c, scale_of(w, 2)), y3 = pair_of<3>(c, scale_of(w, 3));
                    e[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
                    e[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x05040100u);
                    d[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
                    d[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x07060302u);
                }
                ev[k] = __builtin_bit_cast(half8, e);
                od[k] = __builtin_bit_cast(half8, d);
            }
            ask_values(next, b4);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                o[2 * b4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ev[k], pl[k], o[2 * b4], 0, 0, 0);
                o[2 * b4 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(od[k], pl[k], o[2 * b4 + 1], 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                o[2 * b4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ev[k], ps[k], o[2 * b4], 0, 0, 0);
                o[2 * b4 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(od[k], ps[k], o[2 * b4 + 1], 0, 0, 0);
            }
        }
        if (MULTI && told) {
#pragma unroll
            for (int k = 0; k < NB; ++k)
                if (first[k] < seen) o[2 * k] = o[2 * k + 1] = floatx4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
        }
        page = next;
    }

#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s_o[wv][lo][32 * t + 8 * hi + 2 * i] = o[2 * t][i];
            s_o[wv][lo][32 * t + 8 * hi + 2 * i + 1] = o[2 * t + 1][i];
        }
    if (hi == 0) { s_m[wv][lo] = m; s_l[wv][lo] = l[0]; }
    __syncthreads();
    for (int idx = tid; idx < rows * D; idx += KD_THREADS) {
        const int c = idx / D, d = idx % D;
        float mn = s_m[0][c];
#pragma unroll
        for (int w = 1; w < KD_WAVES; ++w) mn = __builtin_fmaxf(mn, s_m[w][c]);
        const float ms = mn == -__builtin_inff() ? 0.f : mn;
        float lf = 0.f, of = 0.f;
#pragma unroll
        for (int w = 0; w < KD_WAVES; ++w) {      // fixed order: waves 0..3
            const float cw = __builtin_amdgcn_exp2f(s_m[w][c] - ms);
            lf += s_l[w][c] * cw;
            of += s_o[w][c][d] * cw;
        }
        const size_t row = row_of_column(c);
        if (whole) a.out[row * D + d] = lf == 0.f ? 0 : to_half_bits(of / lf);
        else {
            float* const po = a.part + (part_row(a, b, r0 + c, g, group) * a.nsplit + chunk) * (D + 2);
            po[d] = of;
            if (d == 0) { po[D] = mn; po[D + 1] = lf; }
        }
    }
}

// The chunks' (sum, maximum, weight) triples of a row.  Groups of D threads take every KC_GROUPS-th chunk each, eight loads in flight, and meet in LDS:
// a fixed order.  (One thread per column over all chunks: 14.6 us with 48 of them, 256 rows.)
constexpr int KC_THREADS = 512;
template <int D>
__global__ __launch_bounds__(KC_THREADS) void kv4_attn_combine(Kv4AttnArgs a)
{
    constexpr int GROUPS = KC_THREADS / D;
    __shared__ float s_o[GROUPS][D], s_w[KV4_MAX_SPLIT];
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, d = threadIdx.x % D, grp = threadIdx.x / D;
    const Request rq = find_request(a, b);
    if (i >= rq.n) return;
    const int pages = (rq.len + KV4_PAGE - 1) / KV4_PAGE, size = chunk_pages(a, pages);
    if (pages <= size) return;                  // one chunk: the first pass has written this output
    const int live = (pages + size - 1) / size;
    const size_t row = (size_t)(rq.first + i) * a.Hq + h;
    const float* const first = a.part + part_row(a, b, i, h, 1) * a.nsplit * (D + 2);
    const float m = lane < live ? first[(size_t)lane * (D + 2) + D] : -__builtin_inff();
    const float w = lane < live ? first[(size_t)lane * (D + 2) + D + 1] : 0.f;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = grp + k * GROUPS < live ? first[(size_t)(grp + k * GROUPS) * (D + 2) + d] : 0.f;
    float top = m;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, sh));
    const float c = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.f : top));
    float l = w * c;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) l += __shfl_xor(l, sh);
    if (threadIdx.x < 64) s_w[lane] = c;
    __syncthreads();
    float o = 0.f;
    for (int k0 = 0;;) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (grp + (k0 + k) * GROUPS < live) o += v[k] * s_w[grp + (k0 + k) * GROUPS];
        k0 += 8;
        if (k0 * GROUPS >= live) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = grp + (k0 + k) * GROUPS < live ? first[(size_t)(grp + (k0 + k) * GROUPS) * (D + 2) + d] : 0.f;
    }
    s_o[grp][d] = o;
    __syncthreads();
    if (threadIdx.x >= D) return;
    float sum = s_o[0][d];
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) sum += s_o[k][d];
    a.out[row * D + d] = l == 0.f ? 0 : to_half_bits(sum / l);
}

template <int D>
hipError_t launch_decode(const Kv4AttnArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.Hkv * a.tiles), (unsigned)a.B, (unsigned)a.nsplit);
    if (a.max_q > 1) hipLaunchKernelGGL((kv4_attn_decode<D, true>), grid, dim3(KD_THREADS), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attn_decode<D, false>), grid, dim3(KD_THREADS), 0, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_attn_combine<D>), dim3((unsigned)a.Hq, (unsigned)a.max_q, (unsigned)a.B), dim3(KC_THREADS), 0, stream, a);
    return hipGetLastError();
}


// ---- many rows of a cache head: prompts and chunks of them ----------------------------------------------------------
//
// A workgroup takes KP_WAVES * 16 * CT rows of one cache head and walks the pages that any of them sees.  Its waves bring a page in once
// between them, convert it to fp16 and leave it in LDS in the order in which the matrix operands are read (a lane's 16 bytes behind
// its neighbour's: no bank conflicts, no address arithmetic); two such buffers, and the codes of the page behind in registers.  Products and
// the lanes' order of positions are the few-rows kernel's; a wave holds CT tiles of 16 rows, each operand read from LDS feeds CT products.
// Bound by neither the matrix cores (busy 35 % of a prompt of 4096 tokens, 40 heads: some 223 us) nor the vector ALU (41 %; an exponential costs a wave 16 cycles, 16 of them and some 50 plain
// instructions against 32 products of 16 cycles per page and tile): a page takes a SIMD some 5100 cycles, of which its two waves' products are 2180 and their vector work about as many, so that the
// turns hardly overlap.  Causal tiles add an eighth (640 tiles of 4 to 64 pages end after 99 pages on the busiest unit, 87.5 on the mean one).  At heads of 128 six registers spill (28 bytes of scratch).
//
// A weight is one fp16 number here, as the sums that divide the result take it (error against 64 bits 2.4e-4 to 2.5e-4, of which the result's own rounding is 2.1e-4; a
// second summand would take 36 products more to the 68 of a page and wave): 2^9 p of a maximum that may lag by 2^6, so that weights down
// to 2^-23 are normal numbers.  The sums are rescaled when some row's maximum has grown by more, which costs as much as the rest of a page's vector work, and all
// waves wait for the one: with 2^11 and a lag of 2^4 that was most iterations.
constexpr int KP_WAVES = 8, KP_AHEAD = 2;
template <int D> constexpr int KP_BUF = 4096 + 256 + 128 * D;      // a page in LDS: key codes, key scales, values in fp16

__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");      // (loads into registers stay in flight)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, int CT>
__global__ __launch_bounds__(512, 2) void kv4_attn_prompt(Kv4AttnArgs a)
{
    constexpr int NB = D / 32, ROWS = KP_WAVES * 16 * CT;
    constexpr int BUF = KP_BUF<D>, V_AT = 4096 + 256;       // bytes of a buffer: key codes and scales as loaded (a lane's behind each other), values in fp16
    extern __shared__ uintx4 kp_smem[];
    __shared__ int s_nan[4][NB][2];              // of a page that not every row sees whole: the first position that is not a number in half a block
    char* const smem = reinterpret_cast<char*>(kp_smem);

    const int tid = threadIdx.x, lane = tid & 63, lo = lane & 15, hi = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = a.Hq / a.Hkv;
    const int b = blockIdx.y, chunk = blockIdx.z;
    const Request rq = find_request(a, b);
    const int all_rows = rq.n * group;
    // the cache head varies fastest: workgroups are dealt to the XCDs in turn, and those of a head share what they read; the last rows, which see the
    // most, come first
    const int g = blockIdx.x % a.Hkv, tiles = (all_rows + ROWS - 1) / ROWS, tile = tiles - 1 - (int)(blockIdx.x / a.Hkv);
    if (tile < 0) return;
    const int r0 = tile * ROWS, rows = all_rows - r0 < ROWS ? all_rows - r0 : ROWS;
    const int pages = (rq.len + KV4_PAGE - 1) / KV4_PAGE, size = chunk_pages(a, pages);
    if (chunk > 0 && chunk * size >= pages) return;
    const bool whole = pages <= size;
    const int before = rq.len - rq.n;            // positions in front of the new tokens (negative: the first rows see nothing)
    const int tile_sees = before + (r0 + rows - 1) / group + 1;                  // by its last row
    const int tile_all = before + r0 / group + 1;                                // by every row
    int c0 = chunk * size, c1 = c0 + size < pages ? c0 + size : pages;
    const int last = (tile_sees + KV4_PAGE - 1) / KV4_PAGE;
    c1 = c1 < last ? c1 : last;

    const int w0 = r0 + wv * 16 * CT;            // this wave's first row
    auto row_index = [&](int ct) { const int r = w0 + ct * 16 + lo; return r < all_rows ? r : all_rows - 1; };
    Queries queries[CT];
    int seen[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int r = row_index(ct), token = r / group;
        seen[ct] = before + token + 1;
        take_queries<D>(ask_queries<D>(a.q + ((size_t)(rq.first + token) * a.Hq + (size_t)g * group + r % group) * D, hi), hi, a.scale2, queries[ct]);
    }
    const int wave_all = before + (w0 < all_rows ? w0 : all_rows - 1) / group + 1;
    const int wave_last = w0 + 16 * CT - 1 < all_rows ? w0 + 16 * CT - 1 : all_rows - 1;
    const int wave_sees = w0 < all_rows ? before + wave_last / group + 1 : -0x7fffffff;      // (no rows: nothing)

    // m: the maximum that a row's weights refer to; from: what its scores start from (WEIGHT_LOG2 - m, so that a weight is 2^score); l: the
    // weights' sums, as a product with ones (every element is the lane's row's)
    float m[CT];
    floatx4 from[CT], l[CT], o[CT][2 * NB];
    bool fresh = true;                           // some row has no maximum yet
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -__builtin_inff();
        from[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
        l[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < 2 * NB; ++t) o[ct][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    int entries = -1;
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    auto page_at = [&](int it) {                 // page c0 + it, asked for in order
        if ((it & 63) == 0) {
            const int j = c0 + it + lane;
            entries = j < c1 ? table[j] : -1;
            // waited for here, and not in every iteration behind whatever else is in flight
            asm volatile("" : "+v"(entries));
        }
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e >= 0 && e < a.num_pages ? e : -1;
    };
    // What a wave brings in of a page: half a tile of 16 positions of the keys, as it is, and half a block of 32 columns of the values, converted (D = 64: a
    // quarter, by every other wave).  Loads are unconditional (a page that is not there: page 0), so that nothing waits for them but what uses them.
    const int k_tile = wv >> 1, k_half = wv & 1, block = wv & (NB - 1), half = (wv >> 2) & 1;
    const bool brings_values = D == 128 || (wv & 2) == 0;
    uintx2 raw_k, raw_v, raw_vs;
    unsigned raw_ks;
    const unsigned char* const heads = a.pages + (size_t)g * kv4_head_bytes(D);
    const size_t page_bytes = (size_t)a.Hkv * kv4_head_bytes(D);
    const unsigned k_off = k_tile * 8 * D + key_offset<D>(lo, hi) + k_half * 8, ks_off = key_scale_offset<D>(lo, hi);
    const unsigned v_off = kv4_values(D) + block * 1024 + lane * 16 + half * 8, vs_off = kv4_value_scales(D) + block * 64 + hi * 16 + half * 8;
    auto head = [&](int page) { return heads + (size_t)(unsigned)(page < 0 ? 0 : page) * page_bytes; };
    // (an offset that the compiler may not add to the uniform part of the address outside the loop: that is an addition of 64 bits per load)
    auto lane_part = [](unsigned off) __attribute__((always_inline)) { asm volatile("" : "+v"(off)); return off; };
    auto issue_keys = [&](int page) __attribute__((always_inline)) {
        raw_k = *reinterpret_cast<const uintx2*>(head(page) + lane_part(k_off));
        raw_ks = *reinterpret_cast<const unsigned*>(head(page) + lane_part(ks_off));
    };
    auto issue_values = [&](int page) __attribute__((always_inline)) {
        raw_v = *reinterpret_cast<const uintx2*>(head(page) + lane_part(v_off));
        raw_vs = *reinterpret_cast<const uintx2*>(head(page) + lane_part(vs_off));
    };
    auto put_keys = [&](int it) __attribute__((always_inline)) {
        char* const buf = smem + (it & 1) * BUF;
        *reinterpret_cast<uintx2*>(buf + (k_tile * 64 + lane) * 16 + k_half * 8) = raw_k;
        reinterpret_cast<unsigned*>(buf + 4096)[lane] = lane_scales<D>(raw_ks, hi);      // (the same by every wave)
    };
    // Values about to be put of which some row does not see everything: as in the few-rows kernel.
    auto scrub = [&](int it, bool there) __attribute__((always_inline)) {
        const int base = (c0 + it) * KV4_PAGE;
        if (base + KV4_PAGE <= tile_all && there) return;
        int first = 0x7fffffff;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            const int pos = base + 32 * half + 16 * (i >> 2) + 4 * hi + (i & 3);
            const bool dead = pos >= rq.len || !there, odd = (raw_vs[i >> 2] >> (8 * (i & 3)) & 255u) == 255u;
            if (odd && !dead) first = pos;
            if (odd || dead) raw_vs[i >> 2] &= ~(255u << (8 * (i & 3)));
        }
#pragma unroll
        for (int sh = 16; sh < 64; sh <<= 1) {
            const int other = __shfl_xor(first, sh);
            first = other < first ? other : first;
        }
        if (brings_values && lane == 0) s_nan[it & 3][block][half] = first;
    };
    // The conversion in steps of two or three instructions, to stand between products: 0 .. 3 and 4 .. 7 the positions of a tile each, 8 the store.
    struct Converted {
        unsigned y[4];
        uintx4 even, odd;
    };
    auto convert = [&](int step, int it, Converted& x) __attribute__((always_inline)) {
        const int i = step >> 2;
        if (step < 8) {
            const unsigned c = raw_v[i], w = raw_vs[i];
            if ((step & 3) == 0) x.y[0] = pair_of<0>(c, scale_of(w, 0));
            if ((step & 3) == 1) {
                x.y[1] = pair_of<1>(c, scale_of(w, 1));
                x.even[2 * i] = __builtin_amdgcn_perm(x.y[1], x.y[0], 0x05040100u);
                x.odd[2 * i] = __builtin_amdgcn_perm(x.y[1], x.y[0], 0x07060302u);
            }
            if ((step & 3) == 2) x.y[2] = pair_of<2>(c, scale_of(w, 2));
            if ((step & 3) == 3) {
                x.y[3] = pair_of<3>(c, scale_of(w, 3));
                x.even[2 * i + 1] = __builtin_amdgcn_perm(x.y[3], x.y[2], 0x05040100u);
                x.odd[2 * i + 1] = __builtin_amdgcn_perm(x.y[3], x.y[2], 0x07060302u);
            }
        } else if (step == 8 && brings_values) {
            uintx4* const vb = reinterpret_cast<uintx4*>(smem + (it & 1) * BUF + V_AT);
            vb[(block * 4 + half) * 64 + lane] = x.even;
            vb[(block * 4 + 2 + half) * 64 + lane] = x.odd;
        }
    };

    half8 pw[CT][2];
    const half8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
    struct Keys {
        uintx4 k[4];
        unsigned scales;
    };
    auto fetch_keys = [&](int it, Keys& keys) __attribute__((always_inline)) {
        const char* const buf = smem + (it & 1) * BUF;
        keys.scales = reinterpret_cast<const unsigned*>(buf + 4096)[lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) keys.k[i] = reinterpret_cast<const uintx4*>(buf)[i * 64 + lane];
    };
    // Weights times values of iteration `it`, whose weights are in pw.  The operands of two blocks of columns are asked for ahead, in this order, or the
    // compiler would ask for each where it is needed and wait; the next page's keys behind them.
    auto weigh = [&](int it, Keys& keys, auto between) __attribute__((always_inline)) {
        const int buf = it & 1, base = (c0 + it) * KV4_PAGE;
        const uintx4* const vb = reinterpret_cast<const uintx4*>(smem + buf * BUF + V_AT) + lane;
        half8 f[KP_AHEAD + 1][4];
        auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[t % (KP_AHEAD + 1)][i] = __builtin_bit_cast(half8, vb[(t * 4 + i) * 64]);
        };
#pragma unroll
        for (int t = 0; t < KP_AHEAD && t < NB; ++t) fetch(t);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            if (t + KP_AHEAD < NB) fetch(t + KP_AHEAD);
            else if (t + KP_AHEAD == NB) fetch_keys(it + 1, keys);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    if (t == 0) l[ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pw[ct][k], l[ct], 0, 0, 0);
                    o[ct][2 * t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t % (KP_AHEAD + 1)][k], pw[ct][k], o[ct][2 * t], 0, 0, 0);
                    o[ct][2 * t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[t % (KP_AHEAD + 1)][2 + k], pw[ct][k], o[ct][2 * t + 1], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    between((t * 2 + k) * CT + ct);      // vector work for the time that the products take
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (base + KV4_PAGE > tile_all) {
#pragma unroll
            for (int t = 0; t < NB; ++t) {
                const int u = s_nan[it & 3][t][0], v = s_nan[it & 3][t][1], first = u < v ? u : v;
                if (first != 0x7fffffff) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        if (first < seen[ct]) o[ct][2 * t] = o[ct][2 * t + 1] = floatx4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
                }
            }
        }
    };
    auto soften = [&](int it, bool there, floatx4 (&acc)[CT][4]) __attribute__((always_inline)) {
        const int base = there ? (c0 + it) * KV4_PAGE : 0x7fffff00;      // (nothing of a page that is not there is seen)
        if (base + KV4_PAGE > wave_all) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (base + 16 * (i >> 2) + 4 * hi + (i & 3) >= seen[ct]) acc[ct][i >> 2][i & 3] = -__builtin_inff();
        }
        auto weights = [&](int ct) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 8; ++r) pw[ct][k][r] = (_Float16)__builtin_amdgcn_exp2f(acc[ct][2 * k + (r >> 2)][r & 3]);
        };
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) weights(ct);
        // Is a weight past 2^15?  Its fp16 exponent is 30 or 31 then, and 0x0800 more carries into the sign.  No maximum crosses
        // lanes unless one is.
        const bool again = fresh || it == 1 || it == 3 || it == 7;       // (all waves together, while maxima still grow)
        bool grown[CT], any = again;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            half2v top = {0, 0};
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int r = 0; r < 8; r += 2) top = __builtin_elementwise_maximum(top, half2v{pw[ct][k][r], pw[ct][k][r + 1]});
            grown[ct] = again || __builtin_amdgcn_ballot_w64(((__builtin_bit_cast(unsigned, top) + 0x08000800u) & 0x80008000u) != 0) != 0ull;
            any = any || grown[ct];
        }
        if (!any) return;
        fresh = false;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (!grown[ct]) continue;
            float mb = acc[ct][0][0];            // (a NaN comes through; its row is not a number anyway)
#pragma unroll
            for (int i = 1; i < 16; ++i) mb = __builtin_elementwise_maximum(mb, acc[ct][i >> 2][i & 3]);
            const float mn = __builtin_elementwise_maximum(m[ct], max_over_hi(mb) - from[ct][0]);
            const bool none = mn == -__builtin_inff();
            const float corr = __builtin_amdgcn_exp2f(m[ct] - (none ? 0.f : mn)), start = none ? 0.f : WEIGHT_LOG2 - mn, more = start - from[ct][0];
            fresh = fresh || __builtin_amdgcn_ballot_w64(none) != 0ull;
            m[ct] = mn;
            from[ct] = floatx4{start, start, start, start};
            l[ct] *= corr;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[ct][i] += more;
#pragma unroll
            for (int t = 0; t < 2 * NB; ++t) o[ct][t] *= corr;
            weights(ct);
        }
    };

    // The two halves of the waves (one of each on every SIMD) take turns: while one multiplies, the other has its exponentials.  In slot 2 p the first half
    // multiplies (the weights of page p - 1 with their values, then the scores of page p), in slot 2 p + 1 the second half.  Between its products a wave puts
    // its part of the values of page p and of the keys of page p + 1 into LDS: before slot 2 p + 2 all of that is there, and what it
    // replaces, two pages before, was read in slot 2 p - 1 for the last time.
    const int n_it = c1 - c0 > 0 ? c1 - c0 : 0;
    const int sees = wave_sees - c0 * KV4_PAGE, n_wave = wave_sees <= c0 * KV4_PAGE ? 0 : (sees + KV4_PAGE - 1) / KV4_PAGE < n_it ? (sees + KV4_PAGE - 1) / KV4_PAGE : n_it;
    int page[4];                                 // of iterations it .. it + 3
#pragma unroll
    for (int i = 0; i < 4; ++i) page[i] = i < n_it ? page_at(i) : -1;
    issue_keys(page[0]);
    issue_values(page[0]);
    put_keys(0);
    issue_keys(page[1]);
    lds_barrier();
    if (wv >= 4) lds_barrier();
    floatx4 acc[CT][4];
    Keys keys;
    auto pin = [&]() __attribute__((always_inline)) {      // (products may be moved past a barrier, which concerns memory only; here they are what the turns are about)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(acc[ct][i]));
    };
    // everything that comes in for iteration `it`, page[0] being its page (pages past the last one: of page 0, for nobody)
    auto bring = [&](int it) __attribute__((always_inline)) {
        Converted x;
#pragma unroll
        for (int i = 0; i < 9; ++i) convert(i, it, x);
        put_keys(it + 1);
        issue_values(page[1]);
        issue_keys(page[2]);
    };
    auto advance = [&](int it) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 3; ++i) page[i] = page[i + 1];
        page[3] = it + 4 < n_it ? page_at(it + 4) : -1;
    };
    if (n_wave > 0) {
        fetch_keys(0, keys);
        score_page<CT>(keys.k, keys.scales, queries, from, acc);
        pin();
    }
    scrub(0, page[0] >= 0);
    bring(0);
    lds_barrier();
    for (int it = 0; it < n_wave; ++it) {
        soften(it, page[0] >= 0, acc);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) asm volatile("" : "+v"(pw[ct][0]), "+v"(pw[ct][1]));
        advance(it);
        scrub(it + 1, page[0] >= 0);
        lds_barrier();
        Converted x;
        weigh(it, keys, [&](int step) __attribute__((always_inline)) {
            constexpr int LAST = 4 * NB * CT / 2 - 1;                // of the steps (D = 64: seven, so two at a time)
            if constexpr (LAST >= 13) {
                convert(step, it + 1, x);
                if (step == 9) put_keys(it + 2);
                if (step == 11) issue_values(page[1]);
                if (step == 13) issue_keys(page[2]);
            } else {
                convert(2 * step, it + 1, x);
                convert(2 * step + 1, it + 1, x);
                if (step == 5) put_keys(it + 2);
                if (step == 6) issue_values(page[1]);
                if (step == 7) issue_keys(page[2]);
            }
        });
        score_page<CT>(keys.k, keys.scales, queries, from, acc);      // (behind the last page: of whatever is there, for nobody)
        pin();
        lds_barrier();
    }
    for (int it = n_wave; it < n_it; ++it) {
        advance(it);
        scrub(it + 1, page[0] >= 0);
        lds_barrier();
        bring(it + 1);
        lds_barrier();
    }
    if (wv < 4) lds_barrier();

#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int r = w0 + ct * 16 + lo;
        const float lf = l[ct][0];               // (summed by the matrix product over all lanes)
        if (r >= all_rows) continue;
        const size_t row = (size_t)(rq.first + r / group) * a.Hq + (size_t)g * group + r % group;
        if (whole) {
            const float inv = lf == 0.f ? 0.f : 1.0f / lf;
#pragma unroll
            for (int t = 0; t < NB; ++t) {
                half8 y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[2 * i] = (_Float16)(o[ct][2 * t][i] * inv);
                    y[2 * i + 1] = (_Float16)(o[ct][2 * t + 1][i] * inv);
                }
                *reinterpret_cast<uintx4*>(a.out + row * D + 32 * t + 8 * hi) = __builtin_bit_cast(uintx4, y);
            }
        } else {
            float* const po = a.part + (part_row(a, b, r, g, group) * a.nsplit + chunk) * (D + 2);
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    po[32 * t + 8 * hi + 2 * i] = o[ct][2 * t][i];
                    po[32 * t + 8 * hi + 2 * i + 1] = o[ct][2 * t + 1][i];
                }
            if (hi == 0) { po[D] = m[ct]; po[D + 1] = lf; }
        }
    }
}

template <int D, int CT>
hipError_t launch_prompt(const Kv4AttnArgs& a, hipStream_t stream)
{
    constexpr int LDS = 2 * KP_BUF<D>;
    static std::once_flag attr_once;
    std::call_once(attr_once, [] {
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_attn_prompt<D, CT>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    });
    const long rows = (long)a.max_q * (a.Hq / a.Hkv), per = KP_WAVES * 16 * CT;
    const dim3 grid((unsigned)((rows + per - 1) / per * a.Hkv), (unsigned)a.B, (unsigned)a.nsplit);
    hipLaunchKernelGGL((kv4_attn_prompt<D, CT>), grid, dim3(64 * KP_WAVES), LDS, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_attn_combine<D>), dim3((unsigned)a.Hq, (unsigned)a.max_q, (unsigned)a.B), dim3(KC_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t stream)
{
    if (a.split_rows) return a.D == 128 ? launch_decode<128>(a, stream) : launch_decode<64>(a, stream);
    return a.D == 128 ? launch_prompt<128, 2>(a, stream) : launch_prompt<64, 2>(a, stream);
}

}  // namespace thi
