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

// x rounded to 32 bits so that no border between codes or scales is met that x itself is not on: towards zero, the last bit set if
// anything was dropped (|x| past the range: the largest finite value; not finite: not finite).
__device__ __forceinline__ float to_float_sticky(double x)
{
    const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
    const unsigned hi = (unsigned)(b >> 32), lo = (unsigned)b, power = (hi >> 20) & 0x7ff;
    unsigned f = ((hi & 0x7fffffffu) << 3 | lo >> 29) - (896u << 23);
    f |= (lo & 0x1fffffffu) != 0 ? 1u : 0u;
    if (power < 897) f = 0;
    if (power > 1150) f = power == 2047 ? 0x7fc00000u : 0x7f7fffffu;
    return __builtin_bit_cast(float, f | (hi & 0x80000000u));
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

template <int D>
__global__ __launch_bounds__(KV4_THREADS) void kv4_append(Kv4AppendArgs a)
{
    constexpr int LPH = D / LANE_VALUES, HEADS = KV4_THREADS / LPH;
    __shared__ double s_turn[D / 2][2];
    const int t = blockIdx.x, tid = threadIdx.x;
    if (a.theta) {
        if (tid < D / 2) {
            double sn, cs;
            sincos((double)a.positions[t] * (double)a.theta[tid], &sn, &cs);
            s_turn[tid][0] = cs;
            s_turn[tid][1] = sn;
        }
        __syncthreads();
    }
    const int part = tid % LPH;
    const long slot = a.slots[t];
    const bool stored = slot >= 0 && slot < (long)a.num_pages * KV4_PAGE;
    const int pos = (int)(slot & (KV4_PAGE - 1));
    const int H = a.Hq + 2 * a.Hkv;
    for (int h = blockIdx.y * HEADS + tid / LPH; h < H; h += gridDim.y * HEADS) {
        const uintx4 raw = *reinterpret_cast<const uintx4*>(a.qkv + (size_t)t * a.ld + (size_t)h * D + part * LANE_VALUES);
        const half8 x = __builtin_bit_cast(half8, raw);
        unsigned byte;
        if (h >= a.Hq + a.Hkv) {                   // a value: stored as it is
            float y[LANE_VALUES];
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) y[e] = (float)x[e];
            const unsigned c = quantise(y, byte);
            if (stored) {
                unsigned char* const base = a.pages + ((size_t)(slot >> 6) * a.Hkv + (h - a.Hq - a.Hkv)) * kv4_head_bytes(D);
#pragma unroll
                for (int e = 0; e < 4; ++e) base[kv4_values(D) + kv4_value_at(pos, part * 4 + e)] = (unsigned char)(c >> (8 * e));
                if (part % 4 == 0) base[kv4_value_scales(D) + kv4_value_scale_at(pos, part / 4)] = (unsigned char)byte;
            }
            continue;
        }
        double y[LANE_VALUES];
#pragma unroll
        for (int e = 0; e < LANE_VALUES; ++e) y[e] = (double)(float)x[e];
        const uint16_t* const gamma = h < a.Hq ? a.q_gamma : a.k_gamma;
        if (gamma) {
            double ss = 0.0;
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) ss += y[e] * y[e];
#pragma unroll
            for (int sh = 1; sh < LPH; sh <<= 1) ss += __shfl_xor(ss, sh);
            const double r = 1.0 / sqrt(ss / D + (double)a.eps);
            const half8 gm = __builtin_bit_cast(half8, *reinterpret_cast<const uintx4*>(gamma + part * LANE_VALUES));
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) y[e] *= r * (double)(float)gm[e];
        }
        if (a.theta) {
#pragma unroll
            for (int e = 0; e < LANE_VALUES; e += 2) {
                const double cs = s_turn[part * 4 + e / 2][0], sn = s_turn[part * 4 + e / 2][1], u = y[e], v = y[e + 1];
                y[e] = u * cs - v * sn;
                y[e + 1] = v * cs + u * sn;
            }
        }
        if (h < a.Hq) {
            half8 o;
#pragma unroll
            for (int e = 0; e < LANE_VALUES; ++e) o[e] = (_Float16)(float)y[e];
            *reinterpret_cast<uintx4*>(a.q_out + ((size_t)t * a.Hq + h) * D + part * LANE_VALUES) = __builtin_bit_cast(uintx4, o);
            continue;
        }
        float f[LANE_VALUES];
#pragma unroll
        for (int e = 0; e < LANE_VALUES; ++e) f[e] = to_float_sticky(y[e]);
        const unsigned c = quantise(f, byte);
        if (stored) {
            unsigned char* const base = a.pages + ((size_t)(slot >> 6) * a.Hkv + (h - a.Hq)) * kv4_head_bytes(D);
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

template <int D>
__global__ __launch_bounds__(KV4_THREADS) void kv4_read(Kv4ReadArgs a)
{
    constexpr int LPH = D / LANE_VALUES;
    const size_t item = ((size_t)blockIdx.x * KV4_THREADS + threadIdx.x) / LPH;      // (token, head)
    const int part = threadIdx.x % LPH;
    if (item >= (size_t)a.T * a.Hkv) return;
    const int t = (int)(item / a.Hkv), h = (int)(item % a.Hkv);
    const long slot = a.slots[t];
    const bool stored = slot >= 0 && slot < (long)a.num_pages * KV4_PAGE;
    const int pos = (int)(slot & (KV4_PAGE - 1));
    const unsigned char* const base = a.pages + ((size_t)(stored ? slot >> 6 : 0) * a.Hkv + h) * kv4_head_bytes(D);
    const uintx4 none = {0u, 0u, 0u, 0u};
    if (a.k_out) {
        const unsigned c = *reinterpret_cast<const unsigned*>(base + pos * (D / 2) + part * 4);
        const uintx4 o = values_of(c, base[kv4_key_scales(D) + kv4_key_scale_at(pos, part / 4)]);
        *reinterpret_cast<uintx4*>(a.k_out + item * D + part * LANE_VALUES) = stored ? o : none;
    }
    if (a.v_out) {
        unsigned c = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) c |= (unsigned)base[kv4_values(D) + kv4_value_at(pos, part * 4 + e)] << (8 * e);
        const uintx4 o = values_of(c, base[kv4_value_scales(D) + kv4_value_scale_at(pos, part / 4)]);
        *reinterpret_cast<uintx4*>(a.v_out + item * D + part * LANE_VALUES) = stored ? o : none;
    }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4AppendArgs& a, int num_cus, hipStream_t stream)
{
    const int heads = KV4_THREADS / (a.D / LANE_VALUES), groups = (a.Hq + 2 * a.Hkv + heads - 1) / heads;
    // few tokens: the heads of a token in workgroups of their own; many: one workgroup a token, which makes the rotation's angles once
    const int split = a.T >= 4 * num_cus ? 1 : groups;
    const dim3 grid((unsigned)a.T, (unsigned)split);
    if (a.D == 128) hipLaunchKernelGGL((kv4_append<128>), grid, dim3(KV4_THREADS), 0, stream, a);
    else hipLaunchKernelGGL((kv4_append<64>), grid, dim3(KV4_THREADS), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream)
{
    const size_t items = (size_t)a.T * a.Hkv, per = KV4_THREADS / (a.D / LANE_VALUES);
    const dim3 grid((unsigned)((items + per - 1) / per));
    if (a.D == 128) hipLaunchKernelGGL((kv4_read<128>), grid, dim3(KV4_THREADS), 0, stream, a);
    else hipLaunchKernelGGL((kv4_read<64>), grid, dim3(KV4_THREADS), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
