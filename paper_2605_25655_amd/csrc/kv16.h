// The paged key/value cache in fp16: page layout, argument blocks and launchers of kv16.hip, kv16_attention.hip and kv16_evict.hip.
#pragma once

#include "thi_internal.h"

namespace thi {

// A page holds KV16_PAGE positions of all cache heads of one layer, 128 D values per head: 64 D of keys, 64 D of values.  Their order is the one in which
// the attention kernels' lanes take them (lane = 16 hi + lo of a 16x16x32 matrix operand, eight values a lane), so that every operand is 1 KB of contiguous memory:
//   keys   : [tile of 16 positions][block of 32 columns][hi][lo = position % 16][column % 8]
//   values : [half page][tile of 16 columns][hi][lo = column % 16][i][r] for position 32 half + 16 i + 4 hi + r: a lane's eight positions are those whose weights the
//            scores' product leaves in the lanes of the same hi, so nothing crosses lanes between the two products.
constexpr int KV16_PAGE = 64;
constexpr int kv16_head_values(int D) { return 128 * D; }
constexpr int kv16_values(int D) { return 64 * D; }
__host__ __device__ constexpr int kv16_key_at(int pos, int part, int D) { return (pos >> 4) * 16 * D + part * 128 + (pos & 15) * 8; }      // columns 8 part ..
__host__ __device__ constexpr int kv16_value_at(int pos, int col, int D)
{
    return 64 * D + (pos >> 5) * 32 * D + (col >> 4) * 512 + ((pos >> 2) & 3) * 128 + (col & 15) * 8 + ((pos >> 4) & 1) * 4 + (pos & 3);
}

struct Kv16AppendArgs {
    const uint16_t* qkv;                 // [T, ld]
    const uint16_t *q_gamma, *k_gamma;   // [D] or nullptr
    const int* positions;                // [T], with theta
    const float* theta;                  // [D/2] or nullptr: no rotation
    const int* slots;                    // [T] page * KV16_PAGE + position in it; outside the pool: not stored
    uint16_t* q_out;                     // [T,Hq,D]
    uint16_t* pages;
    float eps;
    int T, ld, Hq, Hkv, D, num_pages;
};
hipError_t launch_kv16_append(const Kv16AppendArgs& a, int num_cus, hipStream_t stream);

struct Kv16AttnArgs {
    const uint16_t* q;               // [T,Hq,D]
    const uint16_t* pages;
    const int* page_table;           // [B,max_pages]
    const int* seq_lens;             // [B]
    const int* q_offsets;            // [B+1] or nullptr: one token per request
    uint16_t* out;                   // [T,Hq,D]
    const float* weights_in;         // [B,Hkv,64 max_pages] or nullptr: nothing so far
    float* weights_out;              // the same shape, or nullptr: not asked for
    float scale2;                    // softmax scale times log2(e)
    int window, sinks;               // window 0: everything in front of a token
    int B, T, Hq, Hkv, D, max_q, num_pages, max_pages;
    int group;                       // Hq / Hkv query heads per cache head
    // how the rows are dealt (kv16_plan)
    enum Whose { EVERYONES, THOSE_OF_FEW_ROWS, THOSE_OF_MORE } whose;      // requests of this launch
    int part_q;                      // the most tokens of one of them
    float* part;                     // [B][part_q][Hq][nsplit][kv16_part(D)]: a chunk's unnormalised output, maximum, sum of the weights as they were multiplied, and as they are
    float* stats;                    // [B][Hkv][tiles KV16_TILE_ROWS][2]: a row's maximum and one over its sum, with weights_out
    uint16_t* queries;               // [B][Hkv][tiles KV16_TILE_ROWS / 16][D / 32][64][8]: queries as matrix operands, with weights_out, unless there are scores
    float* scores;                   // [B][Hkv][max_q group][64 max_pages]: scores in powers of two, with weights_out, if nobody has more rows than few
    int tiles;                       // of KV16_TILE_ROWS rows
    int nsplit, min_chunk;           // chunks per request at most, pages per chunk at least
    int num_cus;
    int parts, part_tiles;           // of the rows, so many tiles of 16 each, whose weights are summed by themselves: [parts][B][Hkv][64 max_pages] in `part`, when that is done with
    bool wide, sorted;               // few rows: eight waves to a workgroup, not four; requests by their length
};
constexpr int KV16_MAX_SPLIT = 64;
constexpr int KV16_FEW_ROWS = 16, KV16_TILE_ROWS = 128;
constexpr int kv16_part(int D) { return D + 4; }
// few: requests of up to KV16_FEW_ROWS rows of a cache head, many: more; nullptr: nobody
hipError_t launch_kv16_attention(const Kv16AttnArgs* few, const Kv16AttnArgs* many, hipStream_t stream);

struct Kv16EvictArgs {
    const int *refs_in, *table_in, *lens_in;
    const float* weights_in;         // [layers][rows][Hkv][64 max_pages]
    int *refs_out, *table_out, *lens_out;
    float* weights_out;
    int* info;
    uint16_t* pages;
    size_t layer_values;             // from layer to layer
    int budget, sinks, recent, headroom, layers, rows, Hkv, D, num_pages, max_pages;
    int* ws;                         // kv16_evict_words()
};
// The move's workgroups of a cache head, a page of kept positions each, and which of a row's n weights thread `thread` of one copies where the row stays as it is: every
// step-th from its own place on, in 64 bits, for a step is up to 2^31 (a budget of 2^28) and a place up to as much more.
constexpr int KE_MOVE = 512;
__host__ __device__ constexpr unsigned kv16_move_groups(int budget, int max_pages)
{
    const long held = (long)max_pages * KV16_PAGE, most = held < budget ? held : budget;
    return (unsigned)((most + KV16_PAGE - 1) / KV16_PAGE);
}
template <class Copy> __host__ __device__ __forceinline__ void kv16_each_copied(unsigned group, unsigned groups, unsigned thread, int n, Copy copy)
{
    for (size_t p = (size_t)group * KE_MOVE + thread; p < (size_t)n; p += (size_t)groups * KE_MOVE) copy(p);
}
size_t kv16_evict_words(int layers, int rows, int Hkv, int max_pages, int num_pages);
hipError_t launch_kv16_evict(const Kv16EvictArgs& a, hipStream_t stream);

}  // namespace thi
