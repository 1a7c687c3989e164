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

// A workgroup takes TT tokens (1 or ROWS) and, of the heads, every (gridDim.y * ROWS / TT)-th group of ROWS / TT; a row of LPH lanes one head of one token at a time,
// eight neighbouring columns a lane, whose four angles it makes once.
//
// A key's eight columns are 16 bytes of the page as they are.  A value's lie 16 bytes apart, four neighbouring positions beside each other (kv16.h): with ROWS
// tokens, four rows whose slots are such a run exchange dwords within their wave, and a lane stores four positions of two columns; elsewhere each value by itself.
template <int D, int TT>
__global__ __launch_bounds__(KV16_THREADS) void kv16_append(Kv16AppendArgs a)
{
    constexpr int LPH = D / LANE_VALUES, ROWS = KV16_THREADS / LPH, HH = ROWS / TT;
    const int tid = threadIdx.x, part = tid % LPH, row = tid / LPH, tt = row / HH;
    // workgroups go round the eight XCDs: the four that follow each other on one take neighbouring tokens, whose values share lines of the page
    int window = blockIdx.x;
    if (TT > 1 && window < (int)(gridDim.x & ~31u)) window = (window & ~31) + (window & 7) * 4 + (window >> 3 & 3);
    // (counted from a token whose run of four in the page begins with it, if the first one's does)
    const int t = window * TT + tt - (TT > 1 ? a.slots[0] & 3 : 0);
    const bool token = t >= 0 && t < a.T;
    const int slot = token ? a.slots[t] : -1;
    const bool stored = slot >= 0 && slot < a.num_pages * KV16_PAGE;
    const int pos = slot & (KV16_PAGE - 1);
    uint16_t* const home = a.pages + (size_t)(unsigned)(stored ? slot / KV16_PAGE : 0) * a.Hkv * kv16_head_values(D);
    const int H = a.Hq + 2 * a.Hkv, step = gridDim.y * HH;
    const uint16_t* const from = a.qkv + (size_t)(token ? t : 0) * a.ld + part * LANE_VALUES;
    auto ask = [&](int h0) {
        const int h = h0 + row % HH;
        return __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(from + (size_t)(h < H ? h : 0) * D));
    };
    constexpr int AHEAD = 3;
    uintx4 rows[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) rows[k] = ask(blockIdx.y * HH + k * step);
    half8 gammas[2] = {};                          // the queries' and the keys'
    if (a.q_gamma) gammas[0] = __builtin_bit_cast(half8, ld_cached(a.q_gamma + part * LANE_VALUES));
    if (a.k_gamma) gammas[1] = __builtin_bit_cast(half8, ld_cached(a.k_gamma + part * LANE_VALUES));
    float cs[LANE_VALUES / 2], sn[LANE_VALUES / 2];
    if (a.theta) {
        const double at = token ? (double)a.positions[t] : 0.0;
#pragma unroll
        for (int e = 0; e < LANE_VALUES / 2; ++e) turn_of(at * (double)a.theta[part * 4 + e], sn[e], cs[e]);
    }
    // TT > 1: are these four rows the four positions of a run?
    const int r = row & 3;
    bool run = false;
    if (TT > 1) {
        const int lane = tid & 63, first = lane & ~(4 * LPH - 1), s0 = __shfl(stored ? slot : -1, first);
        const unsigned long long four = (LPH == 16 ? ~0ull : 0xffffffffull << first);
        const unsigned long long fit = __builtin_amdgcn_ballot_w64(s0 >= 0 && (s0 & 3) == 0 && stored && slot == s0 + r);
        run = (fit & four) == four;
    }
    for (int h0 = blockIdx.y * HH; h0 < H; h0 += step) {
        const int h = h0 + row % HH;
        const uintx4 raw = rows[0];
#pragma unroll
        for (int k = 0; k + 1 < AHEAD; ++k) rows[k] = rows[k + 1];
        rows[AHEAD - 1] = ask(h0 + AHEAD * step);
        if (h >= a.Hq + a.Hkv) {                   // a value
            uint16_t* const to = home + (size_t)(h - a.Hq - a.Hkv) * kv16_head_values(D);
            if (TT > 1 && run) {                   // (h is the same in all lanes)
                // dword r of the four rows: rows r and r ^ 1 exchange one of each pair, then rows r and r ^ 2
                const bool odd = r & 1, high = r & 2;
                const unsigned g0 = (unsigned)__shfl_xor((int)(odd ? raw[0] : raw[1]), LPH), g1 = (unsigned)__shfl_xor((int)(odd ? raw[2] : raw[3]), LPH);
                const unsigned x0 = odd ? g0 : raw[0], x1 = odd ? raw[1] : g0;      // dword r & 1, of the even and the odd row
                const unsigned y0 = odd ? g1 : raw[2], y1 = odd ? raw[3] : g1;      // dword 2 + (r & 1)
                const unsigned p0 = (unsigned)__shfl_xor((int)(high ? x0 : y0), 2 * LPH), p1 = (unsigned)__shfl_xor((int)(high ? x1 : y1), 2 * LPH);
                const unsigned w0 = high ? p0 : x0, w1 = high ? p1 : x1, w2 = high ? y0 : p0, w3 = high ? y1 : p1;
                typedef unsigned uintx2 __attribute__((ext_vector_type(2)));
                const uintx2 even = {__builtin_amdgcn_perm(w1, w0, 0x05040100u), __builtin_amdgcn_perm(w3, w2, 0x05040100u)};
                const uintx2 second = {__builtin_amdgcn_perm(w1, w0, 0x07060302u), __builtin_amdgcn_perm(w3, w2, 0x07060302u)};
                uint16_t* const at = to + kv16_value_at(pos & ~3, part * LANE_VALUES + 2 * r, D);
                *reinterpret_cast<uintx2*>(at) = even;
                *reinterpret_cast<uintx2*>(at + 8) = second;
            } else if (stored && h < H) {
                uint16_t* const at = to + kv16_value_at(pos, part * LANE_VALUES, D);
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) at[e * 8] = (uint16_t)(raw[e >> 1] >> (16 * (e & 1)));
            }
            continue;
        }
        const bool query = h < a.Hq;
        const half8 x = __builtin_bit_cast(half8, raw);
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
                y[e] = u * cs[e / 2] - v * sn[e / 2];
                y[e + 1] = v * cs[e / 2] + u * sn[e / 2];
            }
        }
        half8 o;
#pragma unroll
        for (int e = 0; e < LANE_VALUES; ++e) o[e] = (_Float16)y[e];
        if (query) {
            if (token) *reinterpret_cast<uintx4*>(a.q_out + ((size_t)t * a.Hq + h) * D + part * LANE_VALUES) = __builtin_bit_cast(uintx4, o);
        } else if (stored)
            *reinterpret_cast<uintx4*>(home + (size_t)(h - a.Hq) * kv16_head_values(D) + kv16_key_at(pos, part, D)) = __builtin_bit_cast(uintx4, o);
    }
}

template <int D>
void append(const Kv16AppendArgs& a, int num_cus, hipStream_t stream)
{
    constexpr int ROWS = KV16_THREADS / (D / LANE_VALUES);
    const int H = a.Hq + 2 * a.Hkv;
    if ((double)a.T * H * D * 2 <= 8.0e6) {
        hipLaunchKernelGGL((kv16_append<D, 1>), dim3((unsigned)a.T, (unsigned)((H + ROWS - 1) / ROWS)), dim3(KV16_THREADS), 0, stream, a);
        return;
    }
    const int windows = (a.T + 3 + ROWS - 1) / ROWS;      // (up to three rows in front of the first token)
    int split = windows > 8 * num_cus ? 1 : 8 * num_cus / windows;
    split = split > (H + 7) / 8 ? (H + 7) / 8 : split;
    hipLaunchKernelGGL((kv16_append<D, ROWS>), dim3((unsigned)windows, (unsigned)split), dim3(KV16_THREADS), 0, stream, a);
}

}  // namespace

hipError_t launch_kv16_append(const Kv16AppendArgs& a, int num_cus, hipStream_t stream)
{
    if (a.D == 128) append<128>(a, num_cus, stream);
    else append<64>(a, num_cus, stream);
    return hipGetLastError();
}

}  // namespace thi
