// Into and out of the 4-bit cache: RMSNorm of each head's query and key, rotary embedding, the store of keys and values, and
// the read-back.  Memory-bound: a token's row of the QKV projection is read once, its rotated queries and 4.25 bits a key and value written.
//
// Arithmetic in 64 bits up to the one rounding: neighbouring codes are up to a third of a value apart, so what a 32-bit sum's
// order leaves in the last bit must not decide between them, and a far position times its frequency needs them anyway.
#include "kv4.h"

namespace thi {

namespace {

constexpr int KV4_THREADS = 256;
constexpr int LANE_VALUES = 8;       // a lane's share of a head: 16 bytes

// x rounded to 32 bits so that no border between codes or scales, and no middle between two fp16 numbers, is met that x itself is not on: towards zero, the last bit set
// if anything was dropped (not finite: not finite).  What is rounded to a code or to fp16 from there is rounded once.  Cut to 24 bits first, so that the conversion is
// exact; what lies below fp32's normal numbers is far below half the smallest code.
__device__ __forceinline__ float to_float_sticky(double x)
{
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    const unsigned low = (unsigned)u, dropped = low & 0x1fffffffu;
    const float f = (float)__builtin_bit_cast(double, (u & 0xffffffff00000000ull) | (low & 0xe0000000u));
    return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, f) | (dropped ? 1u : 0u));
}

// 1 / sqrt(x): the instruction's estimate and two steps of Newton's method (each squares the error: 2^-52 and better).  Of an infinity (a head with one among its
// values) it is 0, and a step would make infinity times 0 of it.
__device__ __forceinline__ double inverse_sqrt(double x)
{
    const double estimate = __builtin_amdgcn_rsq(x);
    double r = estimate;
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(0.5 * r, __builtin_fma(-x * r, r, 1.0), r);
    return estimate == 0.0 ? 0.0 : r;
}

// The scale byte of a block whose largest magnitude has these bits: the smallest exponent e with max <= 7 2^e (7 is where the rounding to 6 would turn
// to the next value), 255 where it is not finite.
__device__ __forceinline__ unsigned scale_byte(unsigned max_bits)
{
    if (max_bits >= 0x7f800000u) return 255u;
    int e = (int)(max_bits >> 23) - 127 - 2 + ((max_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < KV4_MIN_EXP ? KV4_MIN_EXP : e > KV4_MAX_EXP ? KV4_MAX_EXP : e;
    return (unsigned)(e + 127);
}

// Eight values' codes, and the scale byte of their block (four neighbouring lanes).
__device__ __forceinline__ unsigned quantise(const float (&y)[LANE_VALUES], unsigned& byte)
{
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < LANE_VALUES; ++e) {
        const unsigned bits = __builtin_bit_cast(unsigned, y[e]) & 0x7fffffffu;
        m = bits > m ? bits : m;
    }
#pragma unroll
    for (int sh = 1; sh < 4; sh <<= 1) {
        const unsigned o = (unsigned)__shfl_xor((int)m, sh);
        m = o > m ? o : m;
    }
    byte = scale_byte(m);
    if (byte == 255u) return 0u;
    const float s = __builtin_bit_cast(float, byte << 23);
    unsigned c = 0;                        // to nearest, ties to the even code, at most 6 (the instruction takes the scale's exponent only)
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], s, 3);
    return c;
}

// Sine and cosine of x, to within 2^-52: x less the nearest multiple k of pi/2 (in two summands of 53 bits, each product fused), then the Taylor series up to
// r^15 and r^16 (|r| <= pi/4: what is left out is below 5e-17).  Beyond 2^30, where k pi/2 would need more, the library's.
__device__ __forceinline__ void sine_cosine(double x, double& sn, double& cs)
{
    if (!(__builtin_fabs(x) < 1073741824.0)) {
        sincos(x, &sn, &cs);
        return;
    }
    const double k = __builtin_rint(x * 0.63661977236758134308);
    const double r = __builtin_fma(-k, 6.123233995736766036e-17, __builtin_fma(-k, 1.5707963267948965580, x)), z = r * r;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
    s = __builtin_fma(s, z, 1.0 / 6227020800.0);
    s = __builtin_fma(s, z, -1.0 / 39916800.0);
    s = __builtin_fma(s, z, 1.0 / 362880.0);
    s = __builtin_fma(s, z, -1.0 / 5040.0);
    s = __builtin_fma(s, z, 1.0 / 120.0);
    s = __builtin_fma(s, z, -1.0 / 6.0);
    s = __builtin_fma(s * z, r, r);
    c = __builtin_fma(c, z, -1.0 / 87178291200.0);
    c = __builtin_fma(c, z, 1.0 / 479001600.0);
    c = __builtin_fma(c, z, -1.0 / 3628800.0);
    c = __builtin_fma(c, z, 1.0 / 40320.0);
    c = __builtin_fma(c, z, -1.0 / 720.0);
    c = __builtin_fma(c, z, 1.0 / 24.0);
    c = __builtin_fma(c, z, -0.5);
    c = __builtin_fma(c, z, 1.0);
    const int q = (int)k & 3;
    const double u = q & 1 ? c : s, v = q & 1 ? s : c;
    sn = q & 2 ? -u : u;
    cs = (q + 1) & 2 ? -v : v;
}

// A workgroup takes TT tokens (1 or ROWS) and, of the heads, every (gridDim.y * ROWS / TT)-th group of ROWS / TT; a row of LPH lanes one head of one token at a time,
// eight neighbouring values a lane, whose four angles it makes once.
//
// The values' codes lie in the page so that four neighbouring positions' bytes of a pair of columns are a dword (kv4.h); stored by
// themselves, 4001 tokens of 40 heads made 10 million byte stores, and the call took 83 us.  With ROWS tokens a workgroup stores dwords: where all its rows are runs of
// four that begin a dword, four rows exchange bytes within their wave; elsewhere it collects them in LDS, with two barriers a head, and stores dwords where a run allows it.
// 4001 tokens of 40+40+40 heads (186 MB): 58 us through LDS, 50 within waves (3.7 TB/s).  Four workgroups a compute unit: at 130 registers three fitted, and the rest
// of the grid was a second round (with the read-back 93 us instead of 77).
template <int D, int TT>
__global__ __launch_bounds__(KV4_THREADS, 4) void kv4_append(Kv4AppendArgs a)
{
    constexpr int LPH = D / LANE_VALUES, ROWS = KV4_THREADS / LPH, HH = ROWS / TT;
    __shared__ unsigned s_code[TT > 1 ? TT : 1][LPH];
    __shared__ unsigned char s_byte[TT > 1 ? TT : 1][D / 32];
    __shared__ long s_slot[TT];
    const int tid = threadIdx.x, part = tid % LPH, row = tid / LPH, tt = row / HH;
    // workgroups go round the eight XCDs: the four that follow each other on one take neighbouring tokens, whose bytes share lines of the page
    int window = blockIdx.x;
    if (TT > 1 && window < (int)(gridDim.x & ~31u)) window = (window & ~31) + (window & 7) * 4 + (window >> 3 & 3);
    // (counted from a token whose dword of the page begins with it, if the first one's does, so that a run of slots is the same groups of four throughout)
    const int t = window * TT + tt - (TT > 1 ? a.slots[0] & 3 : 0);
    const bool token = t >= 0 && t < a.T;
    const long limit = (long)a.num_pages * KV4_PAGE;
    const long slot = token ? a.slots[t] : -1;
    const bool stored = slot >= 0 && slot < limit;
    const int pos = (int)(slot & (KV4_PAGE - 1));
    if (TT > 1 && part == 0) s_slot[tt] = stored ? slot : -1;
    // the rows of the heads in front, three steps ahead of the arithmetic (4001 tokens of 120 heads: 83 us without, 52 with two or four; the waits are for all but the latest
    // loads and stores, so that three let a store of the step before run on), and the gammas once
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
    if (a.q_gamma) gammas[0] = __builtin_bit_cast(half8, *reinterpret_cast<const uintx4*>(a.q_gamma + part * LANE_VALUES));
    if (a.k_gamma) gammas[1] = __builtin_bit_cast(half8, *reinterpret_cast<const uintx4*>(a.k_gamma + part * LANE_VALUES));
    double cs[LANE_VALUES / 2], sn[LANE_VALUES / 2];
    if (a.theta) {
        const double at = token ? (double)a.positions[t] : 0.0;
        if (TT == 1) {                            // one token's angles, each once
            __shared__ double s_turn[D / 2][2];
            if (tid < D / 2) sine_cosine(at * (double)a.theta[tid], s_turn[tid][0], s_turn[tid][1]);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < LANE_VALUES / 2; ++e) {
                sn[e] = s_turn[part * 4 + e][0];
                cs[e] = s_turn[part * 4 + e][1];
            }
        } else {
#pragma unroll
            for (int e = 0; e < LANE_VALUES / 2; ++e) sine_cosine(at * (double)a.theta[part * 4 + e], sn[e], cs[e]);
        }
    }
    // TT > 1: this thread's four tokens when values are stored: a group that begins where a dword of the page does, counted round the TT tokens
    int lead = 0, pair_of_part = 0;
    bool run = false, whole = false;
    if (TT > 1) {
        __syncthreads();
        const long s4 = s_slot[tt & ~3];
        whole = __syncthreads_and(s4 >= 0 && (s4 & 3) == 0 && s_slot[tt] == s4 + (tt & 3)) != 0;      // every four rows are the four positions of a dword
        const int ahead = (int)(-s_slot[0] & 3);
        lead = (ahead + (tid / LPH) % (TT / 4) * 4) % TT;
        pair_of_part = tid / (LPH * (TT / 4));
        const long s0 = s_slot[lead];
        run = s0 >= 0 && (s0 & 3) == 0 && lead + 3 < TT;
        for (int k = 1; k < 4 && run; ++k) run = s_slot[lead + k] == s0 + k;
    }
    for (int h0 = blockIdx.y * HH; h0 < H; h0 += step) {
        const int h = h0 + row % HH;
        const bool there = token && h < H;
        const half8 x = __builtin_bit_cast(half8, rows[0]);
#pragma unroll
        for (int k = 0; k + 1 < AHEAD; ++k) rows[k] = rows[k + 1];
        rows[AHEAD - 1] = ask(h0 + AHEAD * step);
        float f[LANE_VALUES];
        if (h >= a.Hq + a.Hkv) {                   // a value: stored as it is
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) f[e] = (float)x[e];
        } else {
            double y[LANE_VALUES];
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) y[e] = (double)(float)x[e];
            if (h < a.Hq ? a.q_gamma != nullptr : a.k_gamma != nullptr) {
                double ss = 0.0;
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) ss = __builtin_fma(y[e], y[e], ss);
#pragma unroll
                for (int sh = 1; sh < LPH; sh <<= 1) ss += __shfl_xor(ss, sh);
                const double r = inverse_sqrt(ss * (1.0 / D) + (double)a.eps);
                const half8 gm = h < a.Hq ? gammas[0] : gammas[1];
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) y[e] *= r * (double)(float)gm[e];
            }
            if (a.theta) {
#pragma unroll
                for (int e = 0; e < LANE_VALUES; e += 2) {
                    const double u = y[e], v = y[e + 1];
                    y[e] = u * cs[e / 2] - v * sn[e / 2];
                    y[e + 1] = v * cs[e / 2] + u * sn[e / 2];
                }
            }
            // Queries are rounded to nearest on the way, but for those that a middle between two fp16 numbers might have come of: 12 zeros at the end, one value in 4096.
            // 4001 tokens of 118 + 1 + 1 heads with the read-back: 65 us without a look at that, 69 so, 73 with all of them the other way; of 64 + 8 + 8 50, 52, 54.
            unsigned end = 0;
            if (h < a.Hq) {
                end = 0xfffu;
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) {
                    f[e] = (float)y[e];
                    asm("" : "+v"(f[e]));          // (or the compiler makes one conversion of the two, some 40 instructions a value)
                    const unsigned bits = __builtin_bit_cast(unsigned, f[e]) & 0xfffu;
                    end = bits < end ? bits : end;
                }
            }
            if (end == 0) {
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) f[e] = to_float_sticky(y[e]);
            }
            if (h < a.Hq) {
                half8 o;
#pragma unroll
                for (int e = 0; e < LANE_VALUES; ++e) o[e] = (_Float16)f[e];
                if (there) *reinterpret_cast<uintx4*>(a.q_out + ((size_t)t * a.Hq + h) * D + part * LANE_VALUES) = __builtin_bit_cast(uintx4, o);
                continue;
            }
        }
        unsigned byte;
        const unsigned c = quantise(f, byte);
        const bool value = h >= a.Hq + a.Hkv;
        if (TT > 1 && value && whole) {            // four rows lie in one wave: bytes change places between them
            const int r = tt & 3;
            unsigned char* const base = a.pages + ((size_t)(slot >> 6) * a.Hkv + (h - a.Hq - a.Hkv)) * kv4_head_bytes(D);
            unsigned x = __builtin_amdgcn_perm((unsigned)__shfl_xor((int)c, 2 * LPH), c, r & 2 ? 0x03020706u : 0x05040100u);
            x = __builtin_amdgcn_perm((unsigned)__shfl_xor((int)x, LPH), x, r & 1 ? 0x03070105u : 0x06020400u);
            *reinterpret_cast<unsigned*>(base + kv4_values(D) + kv4_value_at(pos & ~3, part * 4 + r)) = x;      // the r-th pair of the four positions
            unsigned e = byte << (8 * r);
            e |= (unsigned)__shfl_xor((int)e, LPH);
            e |= (unsigned)__shfl_xor((int)e, 2 * LPH);
            if (r == 0 && part % 4 == 0) *reinterpret_cast<unsigned*>(base + kv4_value_scales(D) + kv4_value_scale_at(pos & ~3, part / 4)) = e;
            continue;
        }
        if (TT > 1 && value) {                     // (HH = 1: the same head for all rows)
            s_code[tt][part] = c;
            if (part % 4 == 0) s_byte[tt][part / 4] = (unsigned char)byte;
            __syncthreads();
            unsigned codes = 0, bytes = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                codes |= (s_code[(lead + k) % TT][part] >> (8 * pair_of_part) & 255u) << (8 * k);
                bytes |= (unsigned)s_byte[(lead + k) % TT][part / 4] << (8 * k);
            }
            const int hv = h - a.Hq - a.Hkv;
            auto head = [&](long s) { return a.pages + ((size_t)(s >> 6) * a.Hkv + hv) * kv4_head_bytes(D); };
            const bool scales = pair_of_part == 0 && part % 4 == 0;
            if (run) {
                unsigned char* const base = head(s_slot[lead]);
                const int p = (int)(s_slot[lead] & (KV4_PAGE - 1));
                *reinterpret_cast<unsigned*>(base + kv4_values(D) + kv4_value_at(p, part * 4 + pair_of_part)) = codes;
                if (scales) *reinterpret_cast<unsigned*>(base + kv4_value_scales(D) + kv4_value_scale_at(p, part / 4)) = bytes;
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const long s = s_slot[(lead + k) % TT];
                    if (s < 0) continue;
                    unsigned char* const base = head(s);
                    const int p = (int)(s & (KV4_PAGE - 1));
                    base[kv4_values(D) + kv4_value_at(p, part * 4 + pair_of_part)] = (unsigned char)(codes >> (8 * k));
                    if (scales) base[kv4_value_scales(D) + kv4_value_scale_at(p, part / 4)] = (unsigned char)(bytes >> (8 * k));
                }
            }
            __syncthreads();                       // read before the next head's codes come
            continue;
        }
        if (!there || !stored) continue;
        unsigned char* const base = a.pages + ((size_t)(slot >> 6) * a.Hkv + (value ? h - a.Hq - a.Hkv : h - a.Hq)) * kv4_head_bytes(D);
        if (value) {
#pragma unroll
            for (int e = 0; e < 4; ++e) base[kv4_values(D) + kv4_value_at(pos, part * 4 + e)] = (unsigned char)(c >> (8 * e));
            if (part % 4 == 0) base[kv4_value_scales(D) + kv4_value_scale_at(pos, part / 4)] = (unsigned char)byte;
        } else {
            *reinterpret_cast<unsigned*>(base + pos * (D / 2) + part * 4) = c;
            if (part % 4 == 0) base[kv4_key_scales(D) + kv4_key_scale_at(pos, part / 4)] = (unsigned char)byte;
        }
    }
}

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uintx4 values_of(unsigned c, unsigned byte)
{
    const float s = __builtin_bit_cast(float, byte << 23);
    uintx4 o;
    o[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 0));
    o[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 1));
    o[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 2));
    o[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 3));
    return o;
}

// TT tokens (1 or 4) of a head by LPH lanes.  Four neighbouring slots' value bytes are read as the dwords that hold them (one, or two where the run does not begin with
// one); other slots byte by byte.
template <int D, int TT>
__global__ __launch_bounds__(KV4_THREADS) void kv4_read(Kv4ReadArgs a)
{
    constexpr int LPH = D / LANE_VALUES;
    const size_t item = ((size_t)blockIdx.x * KV4_THREADS + threadIdx.x) / LPH;      // (tokens, head)
    const int part = threadIdx.x % LPH;
    const int t0 = (int)(item / a.Hkv) * TT, h = (int)(item % a.Hkv);
    if (t0 >= a.T) return;
    const long limit = (long)a.num_pages * KV4_PAGE;
    long slot[TT];
#pragma unroll
    for (int k = 0; k < TT; ++k) {
        slot[k] = t0 + k < a.T ? a.slots[t0 + k] : -1;
        if (slot[k] >= limit) slot[k] = -1;
    }
    auto head = [&](long s) { return a.pages + ((size_t)(s >> 6) * a.Hkv + h) * kv4_head_bytes(D); };
    auto out = [&](uint16_t* to, int k) { return reinterpret_cast<uintx4*>(to + ((size_t)(t0 + k) * a.Hkv + h) * D + part * LANE_VALUES); };
    const uintx4 none = {0u, 0u, 0u, 0u};
    if (a.k_out) {
        unsigned c[TT], e[TT];
#pragma unroll
        for (int k = 0; k < TT; ++k) {
            const long s = slot[k] < 0 ? 0 : slot[k];
            const int pos = (int)(s & (KV4_PAGE - 1));
            c[k] = *reinterpret_cast<const unsigned*>(head(s) + pos * (D / 2) + part * 4);
            e[k] = head(s)[kv4_key_scales(D) + kv4_key_scale_at(pos, part / 4)];
        }
#pragma unroll
        for (int k = 0; k < TT; ++k)
            if (t0 + k < a.T) *out(a.k_out, k) = slot[k] < 0 ? none : values_of(c[k], e[k]);
    }
    if (!a.v_out) return;
    // a token's four pairs and scale are bytes k of c[0 .. 3] and of e
    unsigned c[4] = {0, 0, 0, 0}, e = 0;
    bool run = TT == 4 && slot[0] >= 0;
#pragma unroll
    for (int k = 1; k < TT; ++k) run = run && slot[k] == slot[0] + k;
    if (run) {
        const long s0 = slot[0] & ~3l, s1 = (slot[0] + 3) & ~3l;
        const unsigned char *b0 = head(s0) + kv4_values(D), *b1 = head(s1) + kv4_values(D);
        const int p0 = (int)(s0 & (KV4_PAGE - 1)), p1 = (int)(s1 & (KV4_PAGE - 1));
        const unsigned shift = (unsigned)(slot[0] & 3);
        auto both = [&](int at0, int at1) { return __builtin_amdgcn_alignbyte(*reinterpret_cast<const unsigned*>(b1 + at1), *reinterpret_cast<const unsigned*>(b0 + at0), shift); };
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = both(kv4_value_at(p0, part * 4 + i), kv4_value_at(p1, part * 4 + i));
        e = both(32 * D + kv4_value_scale_at(p0, part / 4), 32 * D + kv4_value_scale_at(p1, part / 4));
    } else {
#pragma unroll
        for (int k = 0; k < TT; ++k) {
            const long s = slot[k] < 0 ? 0 : slot[k];
            const int pos = (int)(s & (KV4_PAGE - 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] |= (unsigned)head(s)[kv4_values(D) + kv4_value_at(pos, part * 4 + i)] << (8 * k);
            e |= (unsigned)head(s)[kv4_value_scales(D) + kv4_value_scale_at(pos, part / 4)] << (8 * k);
        }
    }
#pragma unroll
    for (int k = 0; k < TT; ++k) {
        unsigned codes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) codes |= (c[i] >> (8 * k) & 255u) << (8 * i);
        if (t0 + k < a.T) *out(a.v_out, k) = slot[k] < 0 ? none : values_of(codes, e >> (8 * k) & 255u);
    }
}

}  // namespace

template <int D>
static void append(const Kv4AppendArgs& a, int num_cus, hipStream_t stream)
{
    constexpr int ROWS = KV4_THREADS / (D / LANE_VALUES);
    const int H = a.Hq + 2 * a.Hkv;
    // Rows of up to 8 MB: the heads of one token in a workgroup, or several, which have every compute unit busy at once; beyond, many tokens for a workgroup, whose angles are made
    // once for its heads and whose values are stored as dwords.  One token / many, 64 + 8 + 8 heads of 128: 4 MB of scattered tokens 6.1 / 11.6 us, 8 MB 10.9 / 13.7, 16 MB 19.9 / 18.5, of one run
    // 5.7 / 10.7, 10.0 / 12.4, 18.7 / 16.7; 40 + 40 + 40 scattered 8.8 / 14.0, 15.3 / 17.0, 26.3 / 26.0, one run 7.7 / 11.0, 12.9 / 12.2, 22.1 / 15.0; 8 + 8 + 8 of 64 scattered 8.6 / 13.7, 14.9 / 16.7,
    // 27.7 / 25.2, one run 7.4 / 11.2, 12.3 / 11.4, 22.8 / 14.7.
    if ((double)a.T * H * D * 2 <= 8.0e6) {
        hipLaunchKernelGGL((kv4_append<D, 1>), dim3((unsigned)a.T, (unsigned)((H + ROWS - 1) / ROWS)), dim3(KV4_THREADS), 0, stream, a);
        return;
    }
    // one round of four workgroups a compute unit, while a workgroup has eight heads or more (its angles cost it as much as some heads)
    const int windows = (a.T + 3 + ROWS - 1) / ROWS;      // (up to three rows in front of the first token)
    int split = windows > 4 * num_cus ? 1 : 4 * num_cus / windows;
    split = split > (H + 7) / 8 ? (H + 7) / 8 : split;
    hipLaunchKernelGGL((kv4_append<D, ROWS>), dim3((unsigned)windows, (unsigned)split), dim3(KV4_THREADS), 0, stream, a);
}

hipError_t launch_kv4_append(const Kv4AppendArgs& a, int num_cus, hipStream_t stream)
{
    if (a.D == 128) append<128>(a, num_cus, stream);
    else append<64>(a, num_cus, stream);
    return hipGetLastError();
}

template <int D, int TT>
static void read(const Kv4ReadArgs& a, hipStream_t stream)
{
    const size_t items = (size_t)((a.T + TT - 1) / TT) * a.Hkv, per = KV4_THREADS / (D / LANE_VALUES);
    hipLaunchKernelGGL((kv4_read<D, TT>), dim3((unsigned)((items + per - 1) / per)), dim3(KV4_THREADS), 0, stream, a);
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream)
{
    // Up to 4 MB of keys: a token for a thread, beyond four.  One / four, 32 heads of 128, scattered slots 1 MB 4.0 / 5.9 us, 4 MB 7.2 / 8.3, 8 MB 12.4 / 13.1, one run 3.6 / 4.9,
    // 5.7 / 5.2, 8.8 / 7.5; 8 heads of 64, scattered 4 MB 7.4 / 8.3, 8 MB 13.1 / 13.6, one run 5.4 / 5.5, 8.7 / 7.6.
    const bool few = (double)a.T * a.Hkv * a.D * 2 <= 4.0e6;
    if (a.D == 128) few ? read<128, 1>(a, stream) : read<128, 4>(a, stream);
    else few ? read<64, 1>(a, stream) : read<64, 4>(a, stream);
    return hipGetLastError();
}

}  // namespace thi
