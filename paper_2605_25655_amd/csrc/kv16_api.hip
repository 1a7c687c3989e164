// C-ABI entry points of the fp16 cache's operators: argument validation and launches.  Declarations and contract: include/thi.h.
#include "../../include/thi.h"
#include "kv16.h"

namespace {

using namespace thi;

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

bool heads_ok(int Hq, int Hkv, int D) { return Hq >= 1 && Hkv >= 1 && Hq <= 65535 && Hkv <= 65535 && Hq % Hkv == 0 && (D == 64 || D == 128); }

// slots are int32: the pool's last position has to have one
bool pool_ok(int num_pages) { return num_pages >= 1 && num_pages <= 0x7fffffff / KV16_PAGE; }

constexpr int MAX_PAGES = 1 << 24;      // of a row of the page table: positions stay below 2^30
constexpr size_t MAX_TILES = 1 << 23;   // of a request's rows, times cache heads: a launch's threads stay below 2^32
constexpr int MAX_KEPT = 1 << 28, MAX_TOKENS = 1 << 28;      // positions of a row that has been evicted from; tokens of a store: the same
constexpr long MAX_WEIGHED = 1 << 23;   // pages of a row of the table times cache heads, with weights: the same

// Pages of a chunk at least, chunks' workgroups for every compute unit, tables times columns that are not cut, pages in sight from which on requests of few rows are dealt apart, and requests and
// pages from which on they are dealt by length (plan)
constexpr int CHUNK = 4, FEW_PER_CU = 3, MANY_PER_CU = 2, FEW_UNCUT = 1280, APART = 72, SORTED = 4, SORTED_PAGES = 32;

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

// The most rows of partial results that a call of up to B requests, max_q rows and max_pages pages has.  Where plan() cuts, the chunks are at most FEW_PER_CU (MANY_PER_CU)
// workgroups of KV16_FEW_ROWS (KV16_TILE_ROWS) rows for every compute unit, so no batch has more rows than these hold; and no more than its own times the chunks of the longest table.
size_t most_rows(int B, int Hq, int Hkv, int max_q, int max_pages, int num_cus)
{
    auto at_most = [&](long q, long held) {
        const long chunks = (max_pages + CHUNK - 1) / CHUNK, own = (long)B * q * Hq;
        const long rows = chunks < 2 ? 0 : own > held ? held : own * (chunks < KV16_MAX_SPLIT ? chunks : KV16_MAX_SPLIT);
        return rows < held ? rows : held;
    };
    const int group = Hq / Hkv, q_few = KV16_FEW_ROWS / group;
    const long few = at_most(max_q < q_few ? max_q : q_few, (long)KV16_FEW_ROWS * FEW_PER_CU * num_cus);
    const long many = (long)max_q * group <= KV16_FEW_ROWS ? 0 : at_most(max_q, (long)KV16_TILE_ROWS * MANY_PER_CU * num_cus);
    return (size_t)(few > many ? few : many);
}
size_t bytes_of_rows(size_t rows, int D) { return rows ? round_up(rows * kv16_part(D) * sizeof(float)) : 256; }
size_t tiles_of(int Hq, int Hkv, int max_q) { return ((size_t)max_q * (Hq / Hkv) + KV16_TILE_ROWS - 1) / KV16_TILE_ROWS; }
size_t bytes_of_stats(int B, int Hq, int Hkv, int max_q) { return tiles_of(Hq, Hkv, max_q) * B * Hkv * KV16_TILE_ROWS * 2 * sizeof(float); }
size_t bytes_of_queries(int B, int Hq, int Hkv, int D, int max_q)
{
    return (size_t)max_q * (Hq / Hkv) <= KV16_FEW_ROWS ? 0 : tiles_of(Hq, Hkv, max_q) * B * Hkv * KV16_TILE_ROWS * D * 2;
}
// of the most that a call of up to so many leaves of its scores
size_t bytes_of_scores(int B, int Hq, int Hkv, int max_q, int max_pages)
{
    const int group = Hq / Hkv, q = KV16_FEW_ROWS / group < max_q ? KV16_FEW_ROWS / group : max_q;
    return round_up((size_t)B * q * Hq * max_pages * KV16_PAGE * sizeof(float));
}

// The most pages that a request's rows look at
long pages_in_sight(const Kv16AttnArgs& a)
{
    const long seen = a.window ? ((long)a.window + a.sinks + a.max_q) / KV16_PAGE + 3 : a.max_pages;
    return seen < a.max_pages ? seen : a.max_pages;
}
// Into how many chunks, at most `most`, requests of more rows are cut, by what that takes in us: a page 1.4 where each workgroup has a compute unit to itself, 1.9 where some share one, and 1.2 for each of those that do
// where most share; for partial results a launch and their bytes (of one chunk: `bytes`), written and read.
int chunks_worth(long items, long pages, long bytes, int most, int num_cus)
{
    int best = 1;
    double least = 0;
    for (int n = 1; n <= most; ++n) {
        const double each = 1.2 * (double)(items * n) / num_cus, page = items * n <= num_cus ? 1.4 : each > 1.9 ? each : 1.9;
        const double time = (double)((pages + n - 1) / n) * page + (n > 1 ? 5.0 + n * (double)bytes / 5e6 : 0.0);
        if (n == 1 || time < least) {
            best = n;
            least = time;
        }
    }
    return best;
}

// How the rows are dealt: up to KV16_FEW_ROWS of a request and cache head to kv16_attn_decode, more, KV16_TILE_ROWS at a time, to kv16_attn_prompt; and where that gives fewer
// workgroups than the compute units hold, requests are cut into chunks of at least CHUNK pages, whose results one more launch puts together.
// Measured, us a pass (requests of up to that many positions each; 64/8: query heads / cache heads of 128 columns):
//   the second kernel from 8, 16, 32, 64 rows on: 16 rows of 64/8, 4 x 9000: 32.5 29.8 29.7 29.7; 24 rows: 33 33 42 42; 32 rows: 34 34 40 40; 64 rows: 40 40 40 64; 16 rows of 32/32, 5 x 1500:
//     28.0 25.9 25.9 25.9; 64 rows: 38 38 38 54; 30 rows of 2 heads of 64 columns, 8 x 2000: 17.3 17.3 15.9 15.9.  16 is also what one matrix tile holds.
//   two, three, four workgroups for a compute unit (which holds three): 64/8, 24 x 5000: 57.6 50.1 47.9; 3 x 131000: 85 86 123; 16 x 32000, 4096 seen: 46.9 48.0 49.0; 32/32, 5 x 1500: 22.1
//     22.8 20.8
//   more rows: up to one, two, three workgroups for a compute unit (it holds two): 300 tokens of 64/8 behind 7700: 161 113 119; 128 of 32/32 behind 1872: 30 29 29; 64 of 64/8, 3 x 6000: 85 56
//     60; 128 of 64/8, 5 x 20000, 4096 seen: 128 128 111, but 800 of 40/40 behind 3200: 99 99 126; 1000 of 32/32 behind 5000: 128 139 149
//   more rows, up to two for a compute unit, and as many as chunks_worth() says: 157 of 40/40, 2 x 353: 29.0 18.6; 94 of 64/8, 610 seen of 7020: 39.9 24.7; 700 of 32/32, a prompt: 43.3 23.9; 642 of 8
//     heads of 64 columns, 5 prompts: 27.6 17.3; those above: the same
//   chunks of 2, 4, 8 pages at least: 128 tokens of 32/32 behind 1872: 36.1 25.5 29.8; 300 of 64/8 behind 7700: 110 111 113; one of 64/8, 1 x 3000: 11.3 12.0 13.4; 10 rows of 8 heads of 64
//     columns, 8 x 2000: 14.3 12.5 12.3
//   not cut, cut: 2 x 468 of 8 heads of 64 columns: 6.8 9.9; 2 x 1200 of these: 9.1 10.0; 2 x 1500 of these (past FEW_UNCUT): 10.4 8.5; 4 x 600 of 32/32: 10.3 13.1; 2 x 600 of 64/8: 10.5 11.6;
//     2 x 760 of 64/8 (past it): 11.4 10.8
//   few rows, four, eight waves a workgroup, where there are more of them than the compute units hold: 32 x 2048 of 32/32: 110.5 107.0; 64 x 2000 of these 204 196; 96 x 3000 of 64/8: 117 105; 20 x 2000
//     of 40/40: 82.6 75.1; where there are not: 24 x 4000 of 32/32: 150 155; 16 x 4000 112 116; 24 x 5000 of 64/8: 50.0 53.3; and of short tables (not past FEW_UNCUT), 32 x 500 of 32/32: 32.0 34.9
//   in the order of the batch, by length: 24 x 5000 of 64/8: 50.1 45.7; 64 x 6000: 160 146; 30 x 8000: 104 102; 16 x 32000, 4096 seen: 47.6 48.4; 32 x 2048 of 32/32: 106.8 108.0; of fewer or shorter
//     ones, 3 x 131000: 86.0 86.1; 8 x 1000: 12.6 13.2.  (The rule looks at neither windows, behind which all see as many pages, nor how many workgroups share a compute unit: 1 to 2 percent lost in the two
//     cases above that it takes along.  Up to 64 requests, whose lengths one wave holds.)
void plan(Kv16AttnArgs& a, bool few, int num_cus)
{
    a.group = a.Hq / a.Hkv;
    a.tiles = (int)tiles_of(a.Hq, a.Hkv, a.max_q);
    a.part_q = few && KV16_FEW_ROWS / a.group < a.max_q ? KV16_FEW_ROWS / a.group : a.max_q;
    const long items = (long)a.B * a.Hkv * (few ? 1 : a.tiles), pages = pages_in_sight(a);
    const long most = few && pages * a.D <= FEW_UNCUT ? 1 : (pages + CHUNK - 1) / CHUNK;
    a.min_chunk = CHUNK;
    long n = (long)(few ? FEW_PER_CU : MANY_PER_CU) * num_cus / items;
    n = n < 1 ? 1 : n > KV16_MAX_SPLIT ? KV16_MAX_SPLIT : n;
    n = n > most ? most : n;
    a.nsplit = (int)(few ? n : chunks_worth(items, pages, (long)a.B * a.max_q * a.Hq * kv16_part(a.D) * 8, (int)n, num_cus));
    a.num_cus = num_cus;
    a.wide = few && items > (long)FEW_PER_CU * num_cus && (long)a.max_pages * a.D > FEW_UNCUT;
    a.sorted = few && a.B >= SORTED && a.B <= 64 && a.max_pages >= SORTED_PAGES;
}
size_t rows_of(const Kv16AttnArgs& a) { return a.nsplit > 1 ? (size_t)a.B * a.part_q * a.Hq * a.nsplit : 0; }
// Are requests of few rows in a call of more dealt as if they were alone?  Some has to be there, by the number of tokens, and what a row sees has to be APART pages at least, for a tile of
// one row walks them as one of 128 does.  With all dealt alike / apart, us a pass, 512 new tokens and single ones (64/8 heads of 128 where nothing is said): 8000 positions and 3 x 131000:
// 2232 / 408; 8000 and 3 x 30000: 563 / 223; 5 x 8000: 202 / 194; 33 x 8000: 524 / 331; 33 x 30000, 4000 seen: 308 / 190; 17 x 8000 of 32/32: 460 / 472; below APART 5 x 4000: 107 / 115;
// 17 x 4000 of 32/32: 235 / 249; 9 x 2000: 57 / 74; 9 x 2000 of 32/32: 65 / 104.
bool apart(const Kv16AttnArgs& a)
{
    const long q_few = KV16_FEW_ROWS / a.group;
    return q_few > 0 && a.T <= (a.B - 1L) * a.max_q + q_few && pages_in_sight(a) >= APART;
}

// Parts of the rows whose weights are summed by themselves: of at least WEIGHED_ROWS rows, and no more workgroups than WEIGHED_GROUPS for it, so that their sums, of a page each, stay small.
// In one, of at least 4096, 2048, 1024 rows, us a pass with weights: a prompt of 2001 of 64/8 heads 168 158 148 147; of 2696, 86 seen and one sink (whose page all rows look at) 192 113 101 104; of 800
// 65 56 51 51; more workgroups anyway, a prompt of 2001 of 32/32 86 86 87 91; of 4000 248 254 259 263; 6 of 4399, 57 seen 292 319 338 381.
constexpr long WEIGHED_ROWS = 2048, WEIGHED_GROUPS = 2048;
long parts_of(int Hq, int Hkv, int max_q) { return ((long)max_q * (Hq / Hkv) + WEIGHED_ROWS - 1) / WEIGHED_ROWS; }
size_t bytes_of_parts(int Hq, int Hkv, int max_q) { return parts_of(Hq, Hkv, max_q) < 2 ? 0 : WEIGHED_GROUPS * KV16_PAGE * sizeof(float); }
void plan_weights(Kv16AttnArgs& a)
{
    const long most = WEIGHED_GROUPS / ((long)a.B * a.Hkv * a.max_pages), n = parts_of(a.Hq, a.Hkv, a.max_q), parts = n < most ? n : most > 1 ? most : 1;
    const long tiles = ((long)a.max_q * a.group + 15) / 16;
    a.part_tiles = (int)((tiles + parts - 1) / parts);
    a.parts = (int)((tiles + a.part_tiles - 1) / a.part_tiles);
}

int finish(hipError_t e) { return e == hipSuccess ? THI_OK : THI_ERR_HIP; }

}  // namespace

extern "C" {

size_t thi_kv16_page_bytes(int Hkv, int D)
{
    return heads_ok(Hkv, Hkv, D) ? (size_t)Hkv * kv16_head_values(D) * 2 : 0;
}

int thi_qk_norm_rope_kv16(const void* qkv, int ld, const void* q_gamma, const void* k_gamma, float eps, const int* positions, const float* theta,
                          const int* slots, void* q_out, void* pages, int T, int Hq, int Hkv, int D, int num_pages, void* hip_stream)
{
    if (!qkv || !slots || !q_out || !pages || (theta && !positions)) return THI_ERR_NULL;
    if (T < 1 || T > MAX_TOKENS || !heads_ok(Hq, Hkv, D) || !pool_ok(num_pages)) return THI_ERR_SHAPE;
    if ((ld & 7) || ld < (long)(Hq + 2 * Hkv) * D) return THI_ERR_SHAPE;
    if (misaligned(qkv, 16) || misaligned(q_gamma, 16) || misaligned(k_gamma, 16) || misaligned(q_out, 16) || misaligned(pages, 16) ||
        misaligned(positions, 4) || misaligned(theta, 4) || misaligned(slots, 4))
        return THI_ERR_ALIGN;
    (void)hipGetLastError();      // an error another user of the runtime left behind is not ours to report
    Kv16AppendArgs a{};
    a.qkv = (const uint16_t*)qkv;
    a.q_gamma = (const uint16_t*)q_gamma;
    a.k_gamma = (const uint16_t*)k_gamma;
    a.positions = positions;
    a.theta = theta;
    a.slots = slots;
    a.q_out = (uint16_t*)q_out;
    a.pages = (uint16_t*)pages;
    a.eps = eps;
    a.T = T; a.ld = ld; a.Hq = Hq; a.Hkv = Hkv; a.D = D; a.num_pages = num_pages;
    return finish(launch_kv16_append(a, device_cu_count(), (hipStream_t)hip_stream));
}

size_t thi_kv16_attention_workspace_bytes(int B, int T, int Hq, int Hkv, int D, int max_q, int max_pages, int weights)
{
    if (B < 1 || B > 65535 || T < 1 || !heads_ok(Hq, Hkv, D) || max_q < 1 || max_q > T || max_q > 65535 || max_pages < 1 || max_pages > MAX_PAGES ||
        tiles_of(Hq, Hkv, max_q) * Hkv > MAX_TILES || (weights && (long)max_pages * Hkv > MAX_WEIGHED))
        return 0;
    const size_t part = bytes_of_rows(most_rows(B, Hq, Hkv, max_q, max_pages, device_cu_count()), D);
    if (!weights) return part;
    const size_t sums = bytes_of_parts(Hq, Hkv, max_q);
    return (sums > part ? sums : part) + bytes_of_stats(B, Hq, Hkv, max_q) + bytes_of_queries(B, Hq, Hkv, D, max_q) + bytes_of_scores(B, Hq, Hkv, max_q, max_pages);
}

int thi_kv16_attention(const void* q, const void* pages, const int* page_table, const int* seq_lens, const int* q_offsets, float scale, int window, int sinks,
                       void* out, const float* weights_in, float* weights_out, int B, int T, int Hq, int Hkv, int D, int max_q, int num_pages, int max_pages,
                       void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!q || !pages || !page_table || !seq_lens || !out || !workspace || (weights_in && !weights_out)) return THI_ERR_NULL;
    const size_t need = thi_kv16_attention_workspace_bytes(B, T, Hq, Hkv, D, max_q, max_pages, weights_out != nullptr);
    if (!need || !pool_ok(num_pages) || (!q_offsets && (T != B || max_q != 1))) return THI_ERR_SHAPE;
    if (window < 0 || sinks < 0) return THI_ERR_SHAPE;
    if (misaligned(q, 16) || misaligned(pages, 16) || misaligned(out, 16) || misaligned(page_table, 4) || misaligned(seq_lens, 4) ||
        misaligned(q_offsets, 4) || misaligned(weights_in, 4) || misaligned(weights_out, 4) || misaligned(workspace, 256))
        return THI_ERR_ALIGN;
    const bool few = (long)max_q * (Hq / Hkv) <= KV16_FEW_ROWS;
    const size_t stats = weights_out ? bytes_of_stats(B, Hq, Hkv, max_q) : 0, queries = weights_out ? bytes_of_queries(B, Hq, Hkv, D, max_q) : 0;
    const size_t scores = weights_out && few ? bytes_of_scores(B, Hq, Hkv, max_q, max_pages) : 0;
    Kv16AttnArgs a{};
    a.B = B; a.T = T; a.Hq = Hq; a.Hkv = Hkv; a.D = D; a.max_q = max_q; a.num_pages = num_pages; a.max_pages = max_pages;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.q = (const uint16_t*)q;
    a.pages = (const uint16_t*)pages;
    a.page_table = page_table;
    a.seq_lens = seq_lens;
    a.q_offsets = q_offsets;
    a.out = (uint16_t*)out;
    a.weights_in = weights_in;
    a.weights_out = weights_out;
    a.scale2 = scale * 1.44269504088896340736f;
    if (a.scale2 == 0.f) a.scale2 = 1e-30f;      // (all weights equal either way; a masked score of -inf stays what it is)
    a.stats = weights_out ? (float*)workspace : nullptr;
    a.queries = queries ? (uint16_t*)((char*)workspace + stats) : nullptr;
    a.scores = scores ? (float*)((char*)workspace + stats) : nullptr;
    a.part = (float*)((char*)workspace + stats + queries + scores);
    plan(a, few, device_cu_count());
    if (weights_out && !few) plan_weights(a);
    size_t rows = rows_of(a);
    Kv16AttnArgs other = a;                      // of requests of few rows in a call of more; their partial results are put together before the others' are there
    const bool both = !few && apart(a);
    if (both) {
        plan(other, true, a.num_cus);
        other.whose = Kv16AttnArgs::THOSE_OF_FEW_ROWS;
        a.whose = Kv16AttnArgs::THOSE_OF_MORE;
        rows = rows_of(other) > rows ? rows_of(other) : rows;
    }
    const size_t sums = a.parts > 1 ? (size_t)a.parts * B * Hkv * max_pages * KV16_PAGE * sizeof(float) : 0, part = bytes_of_rows(rows, D);
    if (workspace_bytes < need || workspace_bytes < stats + queries + scores + (sums > part ? sums : part)) return THI_ERR_WORKSPACE;
    (void)hipGetLastError();
    return finish(launch_kv16_attention(few ? &a : both ? &other : nullptr, few ? nullptr : &a, (hipStream_t)hip_stream));
}

size_t thi_kv16_evict_workspace_bytes(int layers, int rows, int Hkv, int max_pages, int num_pages)
{
    if (layers < 1 || rows < 1 || layers > 65535 || rows > 65535 || (long)layers * rows > 65535 || !heads_ok(Hkv, Hkv, 64) || max_pages < 1 || max_pages > MAX_PAGES ||
        (long)rows * max_pages > 0x7fffffff ||      // (the pages that all rows ask for are counted in 32 bits)
        !pool_ok(num_pages))
        return 0;
    return round_up(kv16_evict_words(layers, rows, Hkv, max_pages, num_pages) * 4);
}

int thi_kv16_evict(const int* refs_in, const int* table_in, const int* lens_in, const float* weights_in, int budget, int sinks, int recent, int headroom,
                   int* refs_out, int* table_out, int* lens_out, float* weights_out, int* info, void* pages, size_t layer_bytes, int layers, int rows,
                   int Hkv, int D, int num_pages, int max_pages, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!refs_in || !table_in || !lens_in || !weights_in || !refs_out || !table_out || !lens_out || !weights_out || !pages || !workspace) return THI_ERR_NULL;
    const size_t need = thi_kv16_evict_workspace_bytes(layers, rows, Hkv, max_pages, num_pages);
    if (!need || !heads_ok(Hkv, Hkv, D)) return THI_ERR_SHAPE;
    if (budget < 1 || sinks < 0 || recent < 0 || headroom < 0 || (long)sinks + recent > budget) return THI_ERR_SHAPE;
    if (budget > MAX_KEPT && max_pages > MAX_KEPT / KV16_PAGE) return THI_ERR_SHAPE;
    if (refs_out == refs_in || table_out == table_in || lens_out == lens_in || weights_out == weights_in) return THI_ERR_SHAPE;
    if ((layer_bytes & 15) || (layers > 1 && layer_bytes < thi_kv16_page_bytes(Hkv, D) * (size_t)num_pages)) return THI_ERR_SHAPE;
    const void* const words[] = {refs_in, table_in, lens_in, weights_in, refs_out, table_out, lens_out, weights_out, info};
    for (const void* p : words)
        if (misaligned(p, 4)) return THI_ERR_ALIGN;
    if (misaligned(pages, 16) || misaligned(workspace, 256)) return THI_ERR_ALIGN;
    if (workspace_bytes < need) return THI_ERR_WORKSPACE;
    (void)hipGetLastError();
    const Kv16EvictArgs a{refs_in, table_in, lens_in, weights_in, refs_out, table_out, lens_out, weights_out, info, (uint16_t*)pages, layer_bytes / 2,
                          budget, sinks, recent, headroom, layers, rows, Hkv, D, num_pages, max_pages, (int*)workspace};
    return finish(launch_kv16_evict(a, (hipStream_t)hip_stream));
}

}  // extern "C"
