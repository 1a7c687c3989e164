// The key/value cache in 4 bits: page layout, argument blocks and launchers of kv4.hip, kv4_attention.hip and pages.hip.
#pragma once

#include "thi_internal.h"

namespace thi {

// A page holds KV4_PAGE positions of all cache heads of one layer, 68 D bytes per head: key codes, key scales, value codes,
// value scales.  A value is an e2m1 code times 2^(byte - 127), a byte for 32 neighbouring values of a row.  The order of the bytes is
// the one in which the attention kernels' lanes take them (lane = 16 hi + lo of a matrix operand):
//   key codes    : a position's row, D/2 bytes; lane (lo, hi) takes the hi-th quarter of row lo of a tile of 16 positions, which
//                  for D = 128 is one block of 32;
//   key scales   : [block][position % 16][tile]: the lane's scales of the page's four tiles are one dword;
//   value codes  : [block][hi][pair of columns][tile][r] for position 16 tile + 4 hi + r: lane (pair, hi) takes in one 16-byte load the 16
//                  positions whose weights the scores' product leaves in the lanes of the same hi, so nothing crosses lanes;
//   value scales : [block][hi][tile][r], the 16 bytes that go with them.
constexpr int KV4_PAGE = 64;
constexpr int KV4_MIN_EXP = -23, KV4_MAX_EXP = 13;      // every stored value is an fp16 number
constexpr int kv4_head_bytes(int D) { return 68 * D; }
constexpr int kv4_key_scales(int D) { return 32 * D; }
constexpr int kv4_values(int D) { return 34 * D; }
constexpr int kv4_value_scales(int D) { return 66 * D; }
__host__ __device__ constexpr int kv4_key_scale_at(int pos, int block) { return block * 64 + (pos & 15) * 4 + (pos >> 4); }
__host__ __device__ constexpr int kv4_value_at(int pos, int pair) { return (pair >> 4) * 1024 + ((pos >> 2) & 3) * 256 + (pair & 15) * 16 + (pos >> 4) * 4 + (pos & 3); }
__host__ __device__ constexpr int kv4_value_scale_at(int pos, int block) { return block * 64 + ((pos >> 2) & 3) * 16 + (pos >> 4) * 4 + (pos & 3); }

struct Kv4AppendArgs {
    const uint16_t* qkv;             // [T, ld]
    const uint16_t *q_gamma, *k_gamma;   // [D] or nullptr
    const int* positions;            // [T], with theta
    const float* theta;              // [D/2] or nullptr: no rotation
    const int* slots;                // [T] page * KV4_PAGE + position in it; outside the pool: not stored
    uint16_t* q_out;                 // [T,Hq,D]
    unsigned char* pages;
    float eps;
    int T, ld, Hq, Hkv, D, num_pages;
};
hipError_t launch_kv4_append(const Kv4AppendArgs& a, int num_cus, hipStream_t stream);

struct Kv4ReadArgs {
    const unsigned char* pages;
    const int* slots;
    uint16_t *k_out, *v_out;         // [T,Hkv,D], either may be nullptr
    int T, Hkv, D, num_pages;
};
hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream);

struct Kv4AttnArgs {
    const uint16_t* q;               // [T,Hq,D]
    const unsigned char* pages;
    const int* page_table;           // [B,max_pages]
    const int* seq_lens;             // [B]
    const int* q_offsets;            // [B+1] or nullptr: one token per request
    uint16_t* out;                   // [T,Hq,D]
    float scale2;                    // softmax scale times log2(e)
    int B, T, Hq, Hkv, D, max_q, num_pages, max_pages;
    // how the rows are dealt (kv4_plan)
    float* part;                     // [B][max_q][Hq][nsplit][D + 2]: a chunk's unnormalised output, maximum, sum
    bool split_rows;                 // 16 rows of a cache head at a time, cut along the positions
    int tiles;                       // tiles of 16 rows
    int nsplit, min_chunk;           // chunks per request at most, pages per chunk at least
};
constexpr int KV4_MAX_SPLIT = 64;
void kv4_plan(Kv4AttnArgs& a, int num_cus);
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t stream);

struct PagesArgs {
    const int *refs_in, *table_in, *lens_in, *parents, *headroom;
    int *refs_out, *table_out, *lens_out, *info;
    char* pages;
    size_t page_bytes, layer_bytes;
    int rows_in, rows_out, layers, num_pages, max_pages;
    int* ws;                         // pages_workspace_words()
};
size_t pages_workspace_words(int rows_in, int rows_out, int num_pages);
hipError_t launch_kv4_fork(const PagesArgs& a, int num_cus, hipStream_t stream);
hipError_t launch_kv4_compact(const PagesArgs& a, int num_cus, hipStream_t stream);

}  // namespace thi
