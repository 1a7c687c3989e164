// Attention over the 4-bit cache.  out = softmax(scale q K^T) V per head, K and V in pages; row i of a request's n new tokens sees the
// positions 0 .. length - n + i whose page exists.
#include "kv4.h"

#include <mutex>

namespace thi {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

// What a request's rows are: [first, first + n) of q, on `len` positions.  Whatever the arrays hold stays within the buffers.
struct Request {
    int first, n, len;
};
__device__ __forceinline__ Request find_request(const Kv4AttnArgs& a, int b)
{
    Request r{b, 1, a.seq_lens[b]};
    if (a.q_offsets) {
        int o0 = a.q_offsets[b], o1 = a.q_offsets[b + 1];
        o0 = o0 < 0 ? 0 : o0 > a.T ? a.T : o0;
        o1 = o1 < o0 ? o0 : o1 > a.T ? a.T : o1;
        r.first = o0;
        r.n = o1 - o0 < a.max_q ? o1 - o0 : a.max_q;
    }
    const long most = (long)a.max_pages * KV4_PAGE;
    r.len = r.len < 0 ? 0 : r.len > most ? (int)most : r.len;
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
// So nothing but the rows' maxima crosses lanes.  Weights are multiplied as two fp16 summands of 2^15 p (2^-22 of a weight off at most down to 2^-17, where
// one alone is off by 2^-11 and as much as the result's own rounding).
struct PageRegs128 { uintx4 k[4]; unsigned ks; uintx4 v[4], vs[4]; };
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
struct PageRegs64 { uintx2 k[4]; unsigned ks; uintx4 v[2], vs[2]; };
template <int D> struct PageRegsOf { typedef PageRegs128 type; };
template <> struct PageRegsOf<64> { typedef PageRegs64 type; };

constexpr int KD_THREADS = 256, KD_WAVES = 4;
constexpr float KD_WEIGHT_LOG2 = 15.0f;          // weights are held as 2^15 p

// byte i of w as the exponent of a float; the conversions take nothing else of it
__device__ __forceinline__ float scale_of(unsigned w, int i)
{
    return __builtin_bit_cast(float, i == 0 ? w << 23 : i == 1 ? w << 15 : i == 2 ? w << 7 : w >> 1);
}
template <int I> __device__ __forceinline__ unsigned pair_of(unsigned codes, float s) { return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, I)); }
__device__ __forceinline__ half8 row_values(unsigned codes, float s)
{
    const uintx4 o = {pair_of<0>(codes, s), pair_of<1>(codes, s), pair_of<2>(codes, s), pair_of<3>(codes, s)};
    return __builtin_bit_cast(half8, o);
}

// over the lanes of the same lo (the four hi)
__device__ __forceinline__ float max_over_hi(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_fmaxf(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ float sum_over_hi(float x)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    x = __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_bit_cast(float, (unsigned)b[0]) + __builtin_bit_cast(float, (unsigned)b[1]);
}

// Pages per chunk of a request with `pages` of them: a function of its own length and of how many workgroups the call has, so that a
// request's chunk borders, and with them the bits of its result, do not depend on its neighbours.
__device__ __forceinline__ int chunk_pages(const Kv4AttnArgs& a, int pages)
{
    const int size = (pages + a.nsplit - 1) / a.nsplit;
    return size > a.min_chunk ? size : a.min_chunk;
}

// Two fp16 summands of four weights.
__device__ __forceinline__ void split_weights(const float (&w)[4], half4& large, half4& small)
{
    const half2v h0 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[0], w[1])), h1 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[2], w[3]));
    large = half4{h0[0], h0[1], h1[0], h1[1]};
    const half2v s0 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[0] - (float)h0[0], w[1] - (float)h0[1]));
    const half2v s1 = __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_pkrtz(w[2] - (float)h1[0], w[3] - (float)h1[1]));
    small = half4{s0[0], s0[1], s1[0], s1[1]};
}

__device__ __forceinline__ half8 join(half4 a, half4 b) { return half8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// MULTI: the rows of a tile may be of several new tokens, which see different positions.
template <int D, bool MULTI>
__global__ __launch_bounds__(KD_THREADS, 2) void kv4_attn_decode(Kv4AttnArgs a)
{
    constexpr int NB = D / 32, KS = D / 32;      // blocks of a row; matrix steps of a score
    typedef typename PageRegsOf<D>::type Regs;
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

    auto row_of_column = [&](int c) {            // (token, head) row of q and out
        const int r = r0 + c;
        return (size_t)(rq.first + r / group) * a.Hq + (size_t)g * group + r % group;
    };
    const int col = lo < rows ? lo : rows - 1;
    half8 qf[KS];
    {
        const uint16_t* const qrow = a.q + row_of_column(col) * D + hi * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(half8, ld_cached(qrow + s * 8));
    }
    // positions this lane's row sees, and what every row of the tile sees
    const int seen = rq.len - rq.n + (MULTI ? (r0 + col) / group : 0) + 1;
    const int all_see = rq.len - rq.n + (MULTI ? r0 / group : 0) + 1;

    float m = -__builtin_inff(), l = 0.f;
    floatx4 o[2 * NB];                           // O^T: column 32 t + 2 (4 hi + i) of the lane's row in o[2 t], its right neighbour in o[2 t + 1]
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};

    const int n_it = (c1 - c0 - wv + KD_WAVES - 1) / KD_WAVES;      // this wave's pages: c0 + wv, c0 + wv + 4, ...
    int entries = -1;                            // of the 64 pages from iteration `it` & ~63 on, one per lane
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    auto page_at = [&](int it) {
        if ((it & 63) == 0) {
            const int j = c0 + wv + (it + lane) * KD_WAVES;
            entries = j < c1 ? table[j] : -1;
        }
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e >= 0 && e < a.num_pages ? e : -1;
    };
    auto issue = [&](int page, Regs& x) __attribute__((always_inline)) {
        if (page < 0) return;
        const unsigned char* const base = a.pages + ((size_t)page * a.Hkv + g) * kv4_head_bytes(D);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            typedef __typeof__(x.k[0]) K;
            x.k[i] = __builtin_nontemporal_load(reinterpret_cast<const K*>(base + i * 8 * D + lo * (D / 2) + hi * (D / 8)));
        }
        x.ks = *reinterpret_cast<const unsigned*>(base + kv4_key_scales(D) + ((D == 128 ? hi : hi >> 1) * 16 + lo) * 4);
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            x.v[t] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(base + kv4_values(D) + t * 1024 + lane * 16));
            x.vs[t] = *reinterpret_cast<const uintx4*>(base + kv4_value_scales(D) + t * 64 + hi * 16);
        }
    };
    auto multiply = [&](const Regs& x, const uintx4 (&vs)[NB], const half8 (&pl)[2], const half8 (&ps)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            half8 ev[2], od[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uintx4 e, d;
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    const unsigned c = x.v[t][2 * k + i2], w = vs[t][2 * k + i2];
                    const unsigned y0 = pair_of<0>(c, scale_of(w, 0)), y1 = pair_of<1>(c, scale_of(w, 1)), y2 = pair_of<2>(c, scale_of(w, 2)), y3 = pair_of<3>(c, scale_of(w, 3));
                    e[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
                    e[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x05040100u);
                    d[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
                    d[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x07060302u);
                }
                ev[k] = __builtin_bit_cast(half8, e);
                od[k] = __builtin_bit_cast(half8, d);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                o[2 * t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ev[k], pl[k], o[2 * t], 0, 0, 0);
                o[2 * t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(od[k], pl[k], o[2 * t + 1], 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                o[2 * t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ev[k], ps[k], o[2 * t], 0, 0, 0);
                o[2 * t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(od[k], ps[k], o[2 * t + 1], 0, 0, 0);
            }
        }
    };
    auto compute = [&](int page, int it, Regs& x) __attribute__((always_inline)) {
        if (page < 0) return;
        const int base = (c0 + wv + it * KD_WAVES) * KV4_PAGE;
        const bool masked = base + KV4_PAGE > all_see;
        float t[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = scale_of(x.ks, i);
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KS; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(row_values(x.k[i][k], s), qf[k], acc, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) t[4 * i + r] = acc[r] * a.scale2;
        }
        if (masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) t[i] = base + 16 * (i >> 2) + 4 * hi + (i & 3) < seen ? t[i] : -__builtin_inff();
        }
        float mb = t[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mb = __builtin_fmaxf(mb, t[i]);
        const float mn = __builtin_fmaxf(m, max_over_hi(mb));
        const float ms = mn == -__builtin_inff() ? 0.f : mn;
        const float corr = __builtin_amdgcn_exp2f(m - ms);
        float sum = 0.f;
        half8 pl[2], ps[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            half4 large[2], small[2];
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
                float w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    w[r] = __builtin_amdgcn_exp2f(t[8 * k + 4 * i2 + r] - (ms - KD_WEIGHT_LOG2));
                    sum += w[r];
                }
                split_weights(w, large[i2], small[i2]);
            }
            pl[k] = join(large[0], large[1]);
            ps[k] = join(small[0], small[1]);
        }
        l = l * corr + sum;
        m = mn;
        if (__builtin_amdgcn_ballot_w64(corr != 1.0f) != 0ull) {
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k) o[k] *= corr;
        }
        if (!masked) {
            multiply(x, x.vs, pl, ps);
            return;
        }
        // Weights are zero where a row does not see a position, but 0 * NaN must not come through: scales of positions that no row sees become 0, and where
        // rows see different ones a NaN's scale too; the rows that do see it are told afterwards.
        uintx4 vs[NB];
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int live = rq.len - (base + 16 * i + 4 * hi);          // of the four bytes
            const unsigned keep = live >= 4 ? 0xffffffffu : live <= 0 ? 0u : (1u << (8 * live)) - 1u;
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                vs[k][i] = x.vs[k][i] & keep;
                const unsigned w = ~vs[k][i];                            // a byte of zero: a scale byte of 255
                odd = odd || ((w - 0x01010101u) & ~w & 0x80808080u) != 0;
            }
        }
        if (MULTI && __builtin_amdgcn_ballot_w64(odd) != 0ull) {
            int first[NB];                                               // the first position of a block that is not a number
#pragma unroll
            for (int k = 0; k < NB; ++k) {
                first[k] = 0x7fffffff;
#pragma unroll
                for (int i = 15; i >= 0; --i)
                    if ((vs[k][i >> 2] >> (8 * (i & 3)) & 255u) == 255u) {
                        first[k] = base + 16 * (i >> 2) + 4 * hi + (i & 3);
                        vs[k][i >> 2] &= ~(255u << (8 * (i & 3)));
                    }
            }
            multiply(x, vs, pl, ps);
#pragma unroll
            for (int k = 0; k < NB; ++k) {
#pragma unroll
                for (int sh = 16; sh < 64; sh <<= 1) {
                    const int other = __shfl_xor(first[k], sh);
                    first[k] = other < first[k] ? other : first[k];
                }
                if (first[k] < seen) o[2 * k] = o[2 * k + 1] = floatx4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
            }
            return;
        }
        multiply(x, vs, pl, ps);
    };

    Regs x0, x1;
    int p0 = n_it > 0 ? page_at(0) : -1, p1;
    issue(p0, x0);
    for (int it = 0; it < n_it; it += 2) {
        p1 = it + 1 < n_it ? page_at(it + 1) : -1;
        issue(p1, x1);
        compute(p0, it, x0);
        p0 = it + 2 < n_it ? page_at(it + 2) : -1;
        issue(p0, x0);
        compute(p1, it + 1, x1);
    }

    l = sum_over_hi(l);
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s_o[wv][lo][32 * t + 8 * hi + 2 * i] = o[2 * t][i];
            s_o[wv][lo][32 * t + 8 * hi + 2 * i + 1] = o[2 * t + 1][i];
        }
    if (hi == 0) { s_m[wv][lo] = m; s_l[wv][lo] = l; }
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
            float* const po = a.part + (row * a.nsplit + chunk) * (D + 2);
            po[d] = of;
            if (d == 0) { po[D] = mn; po[D + 1] = lf; }
        }
    }
}

// The chunks' (sum, maximum, weight) triples of a row, in chunk order.
template <int D>
__global__ __launch_bounds__(D) void kv4_attn_combine(Kv4AttnArgs a)
{
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, d = threadIdx.x, lane = threadIdx.x & 63;
    const Request rq = find_request(a, b);
    if (i >= rq.n) return;
    const int pages = (rq.len + KV4_PAGE - 1) / KV4_PAGE, size = chunk_pages(a, pages);
    if (pages <= size) return;                  // one chunk: the first pass has written this output
    const int live = (pages + size - 1) / size;
    const size_t row = (size_t)(rq.first + i) * a.Hq + h;
    const float* const first = a.part + row * a.nsplit * (D + 2);
    const float mine = lane < live ? first[(size_t)lane * (D + 2) + D] : -__builtin_inff();
    float top = mine;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, sh));
    const float ms = top == -__builtin_inff() ? 0.f : top;
    float l = 0.f, o = 0.f;
    for (int s = 0; s < live; ++s) {
        const float c = __builtin_amdgcn_exp2f(first[(size_t)s * (D + 2) + D] - ms);
        l += first[(size_t)s * (D + 2) + D + 1] * c;
        o += first[(size_t)s * (D + 2) + d] * c;
    }
    a.out[row * D + d] = l == 0.f ? 0 : to_half_bits(o / l);
}

template <int D>
hipError_t launch_decode(const Kv4AttnArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.Hkv * a.tiles), (unsigned)a.B, (unsigned)a.nsplit);
    if (a.max_q > 1) hipLaunchKernelGGL((kv4_attn_decode<D, true>), grid, dim3(KD_THREADS), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attn_decode<D, false>), grid, dim3(KD_THREADS), 0, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_attn_combine<D>), dim3((unsigned)a.Hq, (unsigned)a.max_q, (unsigned)a.B), dim3(D), 0, stream, a);
    return hipGetLastError();
}


// ---- many rows of a cache head: prompts and chunks of them ----------------------------------------------------------
//
// A workgroup takes KP_WAVES * 16 * CT rows of one cache head and walks the pages that any of them sees.  Its waves bring a page in once
// between them, convert it to fp16 and leave it in LDS in the order in which the matrix operands are read (a lane's 16 bytes behind
// its neighbour's: no bank conflicts, no address arithmetic); two such buffers, and the codes of the page behind in registers.  Products and
// the lanes' order of positions are the few-rows kernel's; a wave holds CT tiles of 16 rows, each operand read from LDS feeds CT products.
// Bound by the matrix cores and the vector ALU together (an exponential costs a wave 16 cycles, 16 of them and some 50 plain instructions against 32 products of
// 16 cycles per page and tile).
//
// A weight is one fp16 number here (off by as much as the result is by its own rounding), 2^11 p of a maximum that may lag by 2^4 (so that weights down to 2^-25 are normal numbers):
// the sums are rescaled only when some row's maximum has grown by more than that.
constexpr float KP_WEIGHT_LOG2 = 11.0f, KP_LAG = 4.0f;

__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");      // (loads into registers stay in flight)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, int CT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES / 4) void kv4_attn_prompt(Kv4AttnArgs a)
{
    constexpr int NB = D / 32, KS = D / 32, ROWS = WAVES * 16 * CT;
    constexpr int K_UNITS = 4 * KS * 64, V_UNITS = 4 * NB * 64, BUF = K_UNITS + V_UNITS;      // 16-byte units
    extern __shared__ uintx4 kp_smem[];
    __shared__ int s_nan[2][NB];                 // of a buffer that not every row sees whole: a block's first position that is not a number

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
    const bool flip = a.scale2 < 0.f;
    const float scale2 = __builtin_fabsf(a.scale2);
    half8 qf[CT][KS];
    int seen[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int r = row_index(ct), token = r / group;
        seen[ct] = before + token + 1;
        const uint16_t* const qrow = a.q + ((size_t)(rq.first + token) * a.Hq + (size_t)g * group + r % group) * D + hi * (D / 4);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            uintx4 x = ld_cached(qrow + s * 8);
            if (flip) x ^= 0x80008000u;
            qf[ct][s] = __builtin_bit_cast(half8, x);
        }
    }
    const int wave_all = before + (w0 < all_rows ? w0 : all_rows - 1) / group + 1;
    const int wave_last = w0 + 16 * CT - 1 < all_rows ? w0 + 16 * CT - 1 : all_rows - 1;
    const int wave_sees = w0 < all_rows ? before + wave_last / group + 1 : -0x7fffffff;      // (no rows: nothing)

    float m[CT], l[CT];
    floatx4 o[CT][2 * NB];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -__builtin_inff();
        l[ct] = 0.f;
#pragma unroll
        for (int t = 0; t < 2 * NB; ++t) o[ct][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    int entries = -1;
    const int* const table = a.page_table + (size_t)b * a.max_pages;
    auto page_at = [&](int it) {                 // page c0 + it, asked for in order
        if ((it & 63) == 0) {
            const int j = c0 + it + lane;
            entries = j < c1 ? table[j] : -1;
        }
        const int e = __builtin_amdgcn_readlane(entries, it & 63);
        return e >= 0 && e < a.num_pages ? e : -1;
    };
    // A wave's share of a page: KU tiles of 16 positions of the keys and VU blocks of 32 columns of the values.
    constexpr int KU = WAVES >= 8 ? 1 : 4 / WAVES, VU = WAVES >= 8 ? 1 : (NB + WAVES - 1) / WAVES;
    const int k_first = WAVES >= 8 ? wv : wv * KU, v_first = WAVES >= 8 ? wv - 4 : wv * VU;
    typedef __typeof__(typename PageRegsOf<D>::type{}.k[0]) KPiece;
    KPiece rk[KU];
    unsigned rks = 0;
    uintx4 rv[VU], rvs[VU];
    auto issue = [&](int page) __attribute__((always_inline)) {
        if (page < 0) return;
        const unsigned char* const base = a.pages + ((size_t)page * a.Hkv + g) * kv4_head_bytes(D);
        if (k_first < 4) {
#pragma unroll
            for (int u = 0; u < KU; ++u) rk[u] = *reinterpret_cast<const KPiece*>(base + (k_first + u) * 8 * D + lo * (D / 2) + hi * (D / 8));
            rks = *reinterpret_cast<const unsigned*>(base + kv4_key_scales(D) + ((D == 128 ? hi : hi >> 1) * 16 + lo) * 4);
        }
#pragma unroll
        for (int u = 0; u < VU; ++u)
            if (v_first + u >= 0 && v_first + u < NB) {
                rv[u] = *reinterpret_cast<const uintx4*>(base + kv4_values(D) + (v_first + u) * 1024 + lane * 16);
                rvs[u] = *reinterpret_cast<const uintx4*>(base + kv4_value_scales(D) + (v_first + u) * 64 + hi * 16);
            }
    };
    auto convert = [&](int it, int buf) __attribute__((always_inline)) {
        uintx4* const kb = kp_smem + buf * BUF;
        uintx4* const vb = kb + K_UNITS;
        const int base = (c0 + it) * KV4_PAGE;
        if (k_first < 4) {
#pragma unroll
            for (int u = 0; u < KU; ++u) {
                const float s = __builtin_bit_cast(float, (rks >> (8 * (k_first + u)) & 255u) << 23);
#pragma unroll
                for (int k = 0; k < KS; ++k) kb[((k_first + u) * KS + k) * 64 + lane] = __builtin_bit_cast(uintx4, row_values(rk[u][k], s));
            }
        }
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int t = v_first + u;
            if (t < 0 || t >= NB) continue;
            if (base + KV4_PAGE > tile_all) {    // some row does not see all of it: as in the few-rows kernel
                int first = 0x7fffffff;
#pragma unroll
                for (int i = 15; i >= 0; --i) {
                    const int pos = base + 16 * (i >> 2) + 4 * hi + (i & 3);
                    const bool dead = pos >= rq.len, odd = (rvs[u][i >> 2] >> (8 * (i & 3)) & 255u) == 255u;
                    if (odd && !dead) first = pos;
                    if (odd || dead) rvs[u][i >> 2] &= ~(255u << (8 * (i & 3)));
                }
#pragma unroll
                for (int sh = 16; sh < 64; sh <<= 1) {
                    const int other = __shfl_xor(first, sh);
                    first = other < first ? other : first;
                }
                if (lane == 0) s_nan[buf][t] = first;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uintx4 e, d;
#pragma unroll
                for (int i2 = 0; i2 < 2; ++i2) {
                    const unsigned c = rv[u][2 * k + i2], w = rvs[u][2 * k + i2];
                    const unsigned y0 = pair_of<0>(c, scale_of(w, 0)), y1 = pair_of<1>(c, scale_of(w, 1)), y2 = pair_of<2>(c, scale_of(w, 2)), y3 = pair_of<3>(c, scale_of(w, 3));
                    e[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
                    e[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x05040100u);
                    d[2 * i2] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
                    d[2 * i2 + 1] = __builtin_amdgcn_perm(y3, y2, 0x07060302u);
                }
                vb[(t * 4 + k) * 64 + lane] = e;
                vb[(t * 4 + 2 + k) * 64 + lane] = d;
            }
        }
    };

    const int n_it = c1 - c0;
    int page = n_it > 0 ? page_at(0) : -1, next = -1;
    issue(page);
    if (page >= 0) convert(0, 0);
    next = 1 < n_it ? page_at(1) : -1;
    issue(next);
    lds_barrier();
    for (int it = 0; it < n_it; ++it) {
        const int buf = it & 1, base = (c0 + it) * KV4_PAGE;
        const bool active = page >= 0 && base < wave_sees;
        const uintx4* const kb = kp_smem + buf * BUF;
        const uintx4* const vb = kb + K_UNITS;
        floatx4 acc[CT][4];
        if (active) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) acc[ct][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const half8 kf = __builtin_bit_cast(half8, kb[(i * KS + k) * 64 + lane]);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) acc[ct][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[ct][k], acc[ct][i], 0, 0, 0);
                }
            }
        }
        if (next >= 0) convert(it + 1, buf ^ 1);
        const int behind = it + 2 < n_it ? page_at(it + 2) : -1;
        issue(behind);
        if (active) {
            const bool masked = base + KV4_PAGE > wave_all;
            half8 pw[CT][2];
            float top[CT];
            if (masked) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (base + 16 * (i >> 2) + 4 * hi + (i & 3) >= seen[ct]) acc[ct][i >> 2][i & 3] = -__builtin_inff();
            }
            bool grown = false;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                float mb = acc[ct][0][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mb = __builtin_fmaxf(mb, acc[ct][i >> 2][i & 3]);
                top[ct] = max_over_hi(mb) * scale2;
                grown = grown || top[ct] - m[ct] > KP_LAG;
            }
            if (__builtin_amdgcn_ballot_w64(grown) != 0ull) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    const float mn = __builtin_fmaxf(m[ct], top[ct]);
                    const float corr = __builtin_amdgcn_exp2f(m[ct] - (mn == -__builtin_inff() ? 0.f : mn));
                    m[ct] = mn;
                    l[ct] *= corr;
#pragma unroll
                    for (int t = 0; t < 2 * NB; ++t) o[ct][t] *= corr;
                }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float off = KP_WEIGHT_LOG2 - (m[ct] == -__builtin_inff() ? 0.f : m[ct]);
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float w[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        w[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[ct][2 * k + (r >> 2)][r & 3], scale2, off));
                        sum += w[r];
                    }
#pragma unroll
                    for (int r = 0; r < 8; ++r) pw[ct][k][r] = (_Float16)w[r];
                }
                l[ct] += sum;
            }
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const half8 ev = __builtin_bit_cast(half8, vb[(t * 4 + k) * 64 + lane]), od = __builtin_bit_cast(half8, vb[(t * 4 + 2 + k) * 64 + lane]);
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        o[ct][2 * t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ev, pw[ct][k], o[ct][2 * t], 0, 0, 0);
                        o[ct][2 * t + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(od, pw[ct][k], o[ct][2 * t + 1], 0, 0, 0);
                    }
                }
            if (base + KV4_PAGE > tile_all) {
#pragma unroll
                for (int t = 0; t < NB; ++t) {
                    const int first = s_nan[buf][t];
                    if (first != 0x7fffffff) {
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct)
                            if (first < seen[ct]) o[ct][2 * t] = o[ct][2 * t + 1] = floatx4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
                    }
                }
            }
        }
        lds_barrier();
        page = next;
        next = behind;
    }

#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        const int r = w0 + ct * 16 + lo;
        const float lf = sum_over_hi(l[ct]);
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
            float* const po = a.part + (row * a.nsplit + chunk) * (D + 2);
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

template <int D, int CT, int WAVES>
hipError_t launch_prompt(const Kv4AttnArgs& a, hipStream_t stream)
{
    constexpr int LDS = 2 * (4 * (D / 32) + 4 * (D / 32)) * 64 * 16;
    static std::once_flag attr_once;
    std::call_once(attr_once, [] {
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&kv4_attn_prompt<D, CT, WAVES>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    });
    const long rows = (long)a.max_q * (a.Hq / a.Hkv), per = WAVES * 16 * CT;
    const dim3 grid((unsigned)((rows + per - 1) / per * a.Hkv), (unsigned)a.B, (unsigned)a.nsplit);
    hipLaunchKernelGGL((kv4_attn_prompt<D, CT, WAVES>), grid, dim3(64 * WAVES), LDS, stream, a);
    if (a.nsplit > 1) hipLaunchKernelGGL((kv4_attn_combine<D>), dim3((unsigned)a.Hq, (unsigned)a.max_q, (unsigned)a.B), dim3(D), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t stream)
{
    if (a.split_rows) return a.D == 128 ? launch_decode<128>(a, stream) : launch_decode<64>(a, stream);
    return a.D == 128 ? launch_prompt<128, 2, 8>(a, stream) : launch_prompt<64, 2, 8>(a, stream);
}

}  // namespace thi
