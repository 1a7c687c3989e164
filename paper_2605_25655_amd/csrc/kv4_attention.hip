// Attention over the 4-bit cache.  out = softmax(scale q K^T) V per head, K and V in pages; row i of a request's n new tokens sees the
// positions 0 .. length - n + i whose page exists.
#include "kv4.h"

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

// One wave per row and head; a lane takes a position of a page for the scores, then columns of the output.
template <int D>
__global__ __launch_bounds__(64) void kv4_attn_simple(Kv4AttnArgs a)
{
    __shared__ float s_q[D], s_p[64];
    const int h = blockIdx.x % a.Hq, i = blockIdx.x / a.Hq, b = blockIdx.y, lane = threadIdx.x;
    const Request rq = find_request(a, b);
    if (i >= rq.n) return;
    const size_t row = ((size_t)(rq.first + i) * a.Hq + h) * D;
    for (int d = lane; d < D; d += 64) s_q[d] = half_bits_to_float(a.q[row + d]) * a.scale2;
    __syncthreads();
    const int last = rq.len - rq.n + i, g = h / (a.Hq / a.Hkv);
    float m = -__builtin_inff(), l = 0.f, o[D / 64] = {};
    for (int pg = 0; pg * KV4_PAGE <= last; ++pg) {
        const int page = a.page_table[(size_t)b * a.max_pages + pg];
        if (page < 0 || page >= a.num_pages) continue;
        const unsigned char* const base = a.pages + ((size_t)page * a.Hkv + g) * kv4_head_bytes(D);
        const bool live = pg * KV4_PAGE + lane <= last;
        float t = 0.f;
        for (int blk = 0; blk < D / 32; ++blk) {
            const float s = __builtin_bit_cast(float, (unsigned)base[kv4_key_scales(D) + kv4_key_scale_at(lane, blk)] << 23);
            for (int e = 0; e < 16; ++e) {
                const half2v x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4((unsigned)base[lane * (D / 2) + blk * 16 + e], s, 0);
                t += (float)x[0] * s_q[blk * 32 + 2 * e] + (float)x[1] * s_q[blk * 32 + 2 * e + 1];
            }
        }
        t = live ? t : -__builtin_inff();
        float mx = t;
        for (int sh = 1; sh < 64; sh <<= 1) mx = __builtin_fmaxf(mx, __shfl_xor(mx, sh));
        const float mn = __builtin_fmaxf(m, mx), ms = mn == -__builtin_inff() ? 0.f : mn;
        const float corr = __builtin_amdgcn_exp2f(m - ms), p = __builtin_amdgcn_exp2f(t - ms);
        m = mn;
        l = l * corr + p;
        s_p[lane] = p;
        __syncthreads();
        for (int c = 0; c < D / 64; ++c) {
            const int d = lane + 64 * c;
            float acc = o[c] * corr;
            for (int pos = 0; pos < KV4_PAGE && pg * KV4_PAGE + pos <= last; ++pos) {
                const float s = __builtin_bit_cast(float, (unsigned)base[kv4_value_scales(D) + kv4_value_scale_at(pos, d / 32)] << 23);
                const half2v x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4((unsigned)base[kv4_values(D) + kv4_value_at(pos, d / 2)], s, 0);
                acc += s_p[pos] * (float)x[d & 1];
            }
            o[c] = acc;
        }
        __syncthreads();
    }
    for (int sh = 1; sh < 64; sh <<= 1) l += __shfl_xor(l, sh);
    for (int c = 0; c < D / 64; ++c) a.out[row + lane + 64 * c] = l == 0.f && m == -__builtin_inff() ? 0 : to_half_bits(o[c] / l);
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)a.max_q * (unsigned)a.Hq, (unsigned)a.B);
    if (a.D == 128) hipLaunchKernelGGL((kv4_attn_simple<128>), grid, dim3(64), 0, stream, a);
    else hipLaunchKernelGGL((kv4_attn_simple<64>), grid, dim3(64), 0, stream, a);
    return hipGetLastError();
}

}  // namespace thi
