// Into the fp16 cache: RMSNorm of each head's query and key, rotary embedding, and the store of keys and values.  Memory-bound: a token's row of the QKV
// projection is read once, its rotated queries, keys and values are written once.
//
// Norm and rotation in fp32 (some 2^-22 of a row's largest pair, a thousandth of the rounding to fp16 at the end); angles are made and reduced in 64 bits, for a
// far position times its frequency has no more than a few bits left in 32.
#include "kv16.h"

namespace thi {

namespace {

constexpr int KV16_THREADS = 256;
constexpr int LANE_VALUES = 8;       // a lane's share of a head: 16 bytes

// Sine and cosine of x: x less the nearest multiple k of pi/2 (in two summands of 53 bits, each product fused), in 64 bits; then, in 32, the Taylor series up to
// r^11 and r^12 (|r| <= pi/4: what is left out is below 7e-12).  Beyond 2^30, where k pi/2 would need more, the library's.
__device__ __forceinline__ void turn_of(double x, float& sn, float& cs)
{
    if (!(__builtin_fabs(x) < 1073741824.0)) {
        double s, c;
        sincos(x, &s, &c);
        sn = (float)s;
        cs = (float)c;
        return;
    }
    const double k = __builtin_rint(x * 0.63661977236758134308);
    const float r = (float)__builtin_fma(-k, 6.123233995736766036e-17, __builtin_fma(-k, 1.5707963267948965580, x)), z = r * r;
    float s = -1.0f / 39916800.0f, c = 1.0f / 479001600.0f;
    s = __builtin_fmaf(s, z, 1.0f / 362880.0f);
    s = __builtin_fmaf(s, z, -1.0f / 5040.0f);
    s = __builtin_fmaf(s, z, 1.0f / 120.0f);
    s = __builtin_fmaf(s, z, -1.0f / 6.0f);
    s = __builtin_fmaf(s * z, r, r);
    c = __builtin_fmaf(c, z, -1.0f / 3628800.0f);
    c = __builtin_fmaf(c, z, 1.0f / 40320.0f);
    c = __builtin_fmaf(c, z, -1.0f / 720.0f);
    c = __builtin_fmaf(c, z, 1.0f / 24.0f);
    c = __builtin_fmaf(c, z, -0.5f);
    c = __builtin_fmaf(c, z, 1.0f);
    const int q = (int)k & 3;
    const float u = q & 1 ? c : s, v = q & 1 ? s : c;
    sn = q & 2 ? -u : u;
    cs = (q + 1) & 2 ? -v : v;
}

// Few tokens: a workgroup takes one, and of its heads every gridDim.y-th group of ROWS.  MANY: 2 ROWS tokens, and every gridDim.y-th head.  A row of LPH lanes has one head of one
// token at a time, or of two tokens 16 apart, eight neighbouring columns a lane, whose angles it makes once.
//
// A key's eight columns are 16 bytes of the page as they are.  A value's lie 16 bytes apart, beside those of seven more positions: four neighbouring ones and the four that are 16 further on
// (kv16.h).  MANY: where four rows' slots are such runs, they exchange dwords within their wave, and a lane stores eight positions of two columns, 32 bytes in a row; where only one
// token of its two belongs to a run, 8 bytes of each column; elsewhere each value by itself.  4001 tokens of 40+40+40 heads: without the values' stores 48 us, with 8 bytes a store 65 to 70.
template <int D, bool MANY>
__global__ __launch_bounds__(KV16_THREADS) void kv16_append(Kv16AppendArgs a)
{
    constexpr int LPH = D / LANE_VALUES, ROWS = KV16_THREADS / LPH, HH = MANY ? 1 : ROWS, N = MANY ? 2 : 1;      // N tokens a lane
    const int tid = threadIdx.x, part = tid % LPH, row = tid / LPH;
    // workgroups go round the eight XCDs: the four that follow each other on one take neighbouring tokens
    int window = blockIdx.x;
    if (MANY && window < (int)(gridDim.x & ~31u)) window = (window & ~31) + (window & 7) * 4 + (window >> 3 & 3);
    // (counted from a token whose half page begins with it, if the first one's does)
    const int t0 = MANY ? window * 2 * ROWS + (row & 15) + 32 * (row >> 4) - (a.slots[0] & 31) : window;
    int t[N], slot[N];
    bool token[N], stored[N];
    uint16_t* home[N];
    const uint16_t* from[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        t[n] = t0 + 16 * n;
        token[n] = t[n] >= 0 && t[n] < a.T;
        slot[n] = token[n] ? a.slots[t[n]] : -1;
        stored[n] = slot[n] >= 0 && slot[n] < a.num_pages * KV16_PAGE;
        home[n] = a.pages + (size_t)(unsigned)(stored[n] ? slot[n] / KV16_PAGE : 0) * a.Hkv * kv16_head_values(D);
        from[n] = a.qkv + (size_t)(token[n] ? t[n] : 0) * a.ld + part * LANE_VALUES;
    }
    const int H = a.Hq + 2 * a.Hkv, step = gridDim.y * HH;
    constexpr int AHEAD = MANY ? 2 : 3;
    uintx4 rows[AHEAD][N];
    auto ask = [&](int h0, uintx4 (&x)[N]) __attribute__((always_inline)) {
        const int h = h0 + (MANY ? 0 : row);
#pragma unroll
        for (int n = 0; n < N; ++n) x[n] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(from[n] + (size_t)(h < H ? h : 0) * D));
    };
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ask(blockIdx.y * HH + k * step, rows[k]);
    half8 gammas[2] = {};                          // the queries' and the keys'
    if (a.q_gamma) gammas[0] = __builtin_bit_cast(half8, ld_cached(a.q_gamma + part * LANE_VALUES));
    if (a.k_gamma) gammas[1] = __builtin_bit_cast(half8, ld_cached(a.k_gamma + part * LANE_VALUES));
    float cs[N][LANE_VALUES / 2], sn[N][LANE_VALUES / 2];
    if (a.theta) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const double at = token[n] ? (double)a.positions[t[n]] : 0.0;
#pragma unroll
            for (int e = 0; e < LANE_VALUES / 2; ++e) turn_of(at * (double)a.theta[part * 4 + e], sn[n][e], cs[n][e]);
        }
    }
    // MANY: are these four rows' tokens the four positions of a run, and the second four 16 further on in the same half page?
    const int r = row & 3;
    bool run[N], both = false;
    if (MANY) {
        const int lane = tid & 63, first = lane & ~(4 * LPH - 1);
        const unsigned long long four = (LPH == 16 ? ~0ull : 0xffffffffull << first);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int s0 = __shfl(stored[n] ? slot[n] : -1, first);
            run[n] = (__builtin_amdgcn_ballot_w64(s0 >= 0 && (s0 & 3) == 0 && stored[n] && slot[n] == s0 + r) & four) == four;
        }
        both = run[0] && run[N - 1] && slot[N - 1] == slot[0] + 16 && (slot[0] & 16) == 0;
    }
    typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
    for (int h0 = blockIdx.y * HH; h0 < H; h0 += step) {
        const int h = h0 + (MANY ? 0 : row);
        uintx4 raw[N];
#pragma unroll
        for (int n = 0; n < N; ++n) raw[n] = rows[0][n];
#pragma unroll
        for (int k = 0; k + 1 < AHEAD; ++k)
#pragma unroll
            for (int n = 0; n < N; ++n) rows[k][n] = rows[k + 1][n];
        ask(h0 + AHEAD * step, rows[AHEAD - 1]);
        if (h >= a.Hq + a.Hkv) {                   // a value
            const size_t head = (size_t)(h - a.Hq - a.Hkv) * kv16_head_values(D);
            uintx2 even[N], odd[N];                // four positions of columns 8 part + 2 r and of the next one
            if (MANY) {                            // (h is the same in all lanes)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    // dword r of the four rows: rows r and r ^ 1 exchange one of each pair, then rows r and r ^ 2
                    const uintx4 x = raw[n];
                    const bool second = r & 1, high = r & 2;
                    const unsigned g0 = (unsigned)__shfl_xor((int)(second ? x[0] : x[1]), LPH), g1 = (unsigned)__shfl_xor((int)(second ? x[2] : x[3]), LPH);
                    const unsigned x0 = second ? g0 : x[0], x1 = second ? x[1] : g0;      // dword r & 1, of the even and the odd row
                    const unsigned y0 = second ? g1 : x[2], y1 = second ? x[3] : g1;      // dword 2 + (r & 1)
                    const unsigned p0 = (unsigned)__shfl_xor((int)(high ? x0 : y0), 2 * LPH), p1 = (unsigned)__shfl_xor((int)(high ? x1 : y1), 2 * LPH);
                    const unsigned w0 = high ? p0 : x0, w1 = high ? p1 : x1, w2 = high ? y0 : p0, w3 = high ? y1 : p1;
                    even[n] = uintx2{__builtin_amdgcn_perm(w1, w0, 0x05040100u), __builtin_amdgcn_perm(w3, w2, 0x05040100u)};
                    odd[n] = uintx2{__builtin_amdgcn_perm(w1, w0, 0x07060302u), __builtin_amdgcn_perm(w3, w2, 0x07060302u)};
                }
            }
            if (MANY && both) {
                uint16_t* const at = home[0] + head + kv16_value_at(slot[0] & (KV16_PAGE - 4), part * LANE_VALUES + 2 * r, D);
                *reinterpret_cast<uintx4*>(at) = uintx4{even[0][0], even[0][1], even[N - 1][0], even[N - 1][1]};
                *reinterpret_cast<uintx4*>(at + 8) = uintx4{odd[0][0], odd[0][1], odd[N - 1][0], odd[N - 1][1]};
                continue;
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (MANY && run[n]) {
                    uint16_t* const at = home[n] + head + kv16_value_at(slot[n] & (KV16_PAGE - 4), part * LANE_VALUES + 2 * r, D);
                    *reinterpret_cast<uintx2*>(at) = even[n];
                    *reinterpret_cast<uintx2*>(at + 8) = odd[n];
                } else if (stored[n] && h < H) {
                    uint16_t* const at = home[n] + head + kv16_value_at(slot[n] & (KV16_PAGE - 1), part * LANE_VALUES, D);
#pragma unroll
                    for (int e = 0; e < LANE_VALUES; ++e) at[e * 8] = (uint16_t)(raw[n][e >> 1] >> (16 * (e & 1)));
                }
            }
            continue;
        }
        const bool query = h < a.Hq;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const half8 x = __builtin_bit_cast(half8, raw[n]);
            float y[LANE_VALUES];
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) y[e] = (float)x[e];
            if (query ? a.q_gamma != nullptr : a.k_gamma != nullptr) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
#pragma unroll
                for (int sh = 1; sh < LPH; sh <<= 1) ss += __shfl_xor(ss, sh);
                const float inv = 1.0f / __builtin_sqrtf(ss * (1.0f / D) + a.eps);
                const half8 gm = query ? gammas[0] : gammas[1];
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) y[e] = y[e] * inv * (float)gm[e];
            }
            if (a.theta) {
#pragma unroll
                for (int e = 0; e < LANE_VALUES; e += 2) {
                    const float u = y[e], v = y[e + 1];
                    y[e] = u * cs[n][e / 2] - v * sn[n][e / 2];
                    y[e + 1] = v * cs[n][e / 2] + u * sn[n][e / 2];
                }
            }
            half8 o;
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) o[e] = (_Float16)y[e];
            if (query) {
                if (token[n]) *reinterpret_cast<uintx4*>(a.q_out + ((size_t)t[n] * a.Hq + h) * D + part * LANE_VALUES) = __builtin_bit_cast(uintx4, o);
            } else if (stored[n])
                *reinterpret_cast<uintx4*>(home[n] + (size_t)(h - a.Hq) * kv16_head_values(D) + kv16_key_at(slot[n] & (KV16_PAGE - 1), part, D)) = __builtin_bit_cast(uintx4, o);
        }
    }
}

template <int D>
void append(const Kv16AppendArgs& a, int num_cus, hipStream_t stream)
{
    constexpr int ROWS = KV16_THREADS / (D / LANE_VALUES);
    const int H = a.Hq + 2 * a.Hkv;
    // Rows of up to 2.2 MB: a token for a workgroup.  One token / many, 32 + 32 + 32 heads of 128: 1.6 MB of scattered slots 6.8 / 8.4 us, 2.4 MB scattered 8.0 / 9.7, of one run 7.8 / 6.8, 3.7 MB
    // 10.3 / 11.6, 9.8 / 6.7, 7.4 MB 17.7 / 18.8, 16.9 / 8.4, 24.6 MB 53 / 53, 47 / 18; 64 + 8 + 8: 2 MB 6.5 / 7.6, 6.5 / 6.4, 6.1 MB 9.6 / 10.7, 8.8 / 8.0; 8 + 8 + 8 of 64: 1.5 MB 6.9 / 8.0,
    // 6.7 / 6.4, 3.1 MB 8.6 / 10.2, 8.2 / 6.4.
    if ((double)a.T * H * D * 2 <= 2.2e6) {
        hipLaunchKernelGGL((kv16_append<D, false>), dim3((unsigned)a.T, (unsigned)((H + ROWS - 1) / ROWS)), dim3(KV16_THREADS), 0, stream, a);
        return;
    }
    const int windows = (a.T + 31 + 2 * ROWS - 1) / (2 * ROWS);      // (up to 31 tokens' room in front of the first)
    // two workgroups for every compute unit (4001 tokens of 40 + 40 + 40 heads of 128: one 61 us, two 57, four 62, eight 66), of a head each at least
    int split = windows > 2 * num_cus ? 1 : 2 * num_cus / windows;
    split = split > H ? H : split;
    hipLaunchKernelGGL((kv16_append<D, true>), dim3((unsigned)windows, (unsigned)split), dim3(KV16_THREADS), 0, stream, a);
}

}  // namespace

hipError_t launch_kv16_append(const Kv16AppendArgs& a, int num_cus, hipStream_t stream)
{
    if (a.D == 128) append<128>(a, num_cus, stream);
    else append<64>(a, num_cus, stream);
    return hipGetLastError();
}

}  // namespace thi
