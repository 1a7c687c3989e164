// C-ABI entry points of the 4-bit cache's operators: argument validation and launches.  Declarations and contract: include/thi.h.
#include "../../include/thi.h"
#include "kv4.h"

namespace {

using namespace thi;

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

bool heads_ok(int Hq, int Hkv, int D) { return Hq >= 1 && Hkv >= 1 && Hq <= 65535 && Hkv <= 65535 && Hq % Hkv == 0 && (D == 64 || D == 128); }

// slots are int32: the pool's last position has to have one
bool pool_ok(int num_pages) { return num_pages >= 1 && num_pages <= 0x7fffffff / KV4_PAGE; }

constexpr int FEW_ROWS = 64, FEW_CHUNK = 8, ONE_PER_CU = 3, FEW_PER_CU = 2, MANY_CHUNK = 16, MANY_PER_CU = 1;      // kv4_plan

// The most rows of partial results that a call of up to B requests, max_q rows and max_pages pages has.  Where kv4_plan cuts, the chunks are at most ONE_PER_CU (MANY_PER_CU)
// workgroups of 16 (256) rows for every compute unit, so no batch has more rows than these hold; and no more than its own times the chunks of the longest table.
size_t most_rows(int B, int Hq, int Hkv, int max_q, int max_pages, int num_cus)
{
    auto at_most = [&](long q, int chunk, long held) {
        const long chunks = (max_pages + chunk - 1) / chunk, own = (long)B * q * Hq;
        const long rows = chunks < 2 ? 0 : own > held ? held : own * (chunks < KV4_MAX_SPLIT ? chunks : KV4_MAX_SPLIT);
        return rows < held ? rows : held;
    };
    const int group = Hq / Hkv, q_few = FEW_ROWS / group < 1 ? 0 : FEW_ROWS / group;
    const long few = max_pages <= 16 ? 0 : at_most(max_q < q_few ? max_q : q_few, FEW_CHUNK, 16L * ONE_PER_CU * num_cus);
    const long many = (long)max_q * group <= FEW_ROWS ? 0 : at_most(max_q, MANY_CHUNK, 256L * MANY_PER_CU * num_cus);
    return (size_t)(few > many ? few : many);
}

size_t bytes_of_rows(size_t rows, int D) { return rows ? (rows * (D + 2) * sizeof(float) + 255) / 256 * 256 : 256; }

int finish(hipError_t e) { return e == hipSuccess ? THI_OK : THI_ERR_HIP; }

}  // namespace

// Up to 64 rows of a cache head the few-rows kernel, beyond the prompt kernel.  The one / the other, 4 requests of 2000 positions, 64 query on 8 cache heads of 128:
// 64 rows 21.5 / 37.9 us, 128 36.8 / 45.2, 192 43.5 / 58.4; one of 30000: 64 rows 34.2 / 37.2, 96 45.9 / 39.7; 16 requests of 2000, 32 on 32 heads: 32 rows 54.7 / 98.6, 64 109.9 / 105.2,
// 96 163.6 / 109.8; 8 on 8 heads of 64, one of 30000: 64 rows 22.4 / 32.3, 128 34.2 / 35.9.
//
// Few rows: 16 at a time, the requests cut until there are as many workgroups for every compute unit as fit (three with one token a request; two with several, which for heads of 64 would
// fit three times too), but not below 8 pages a chunk, two for each wave, and not at all up to 16 pages: a chunk more costs its start, its merge, and the second
// launch.  Measured with 1 / 2 / 3 / 4 chunks: 32 x 32 items of up to 32 pages 39.4 / 42.9 / 46.0 / 48.8 us, 64 x 8 of 16 pages 15.8 / 29.1 / 30.1 / 31.4; with 8 / 16 / 24 / 32: 6 x 8 items of
// up to 126 pages 19.1 / 18.7 / 22.8 / 23.3, 4 x 8 of 2047 87.4 / 87.3 / 89.1 / 89.5, 8 of 313 19.8 / 14.4 / 13.4 / 12.6 (48: 14.7); 2 x 8 of 15 pages with one chunk 6.9, with two 9.3.
// Several tokens a request, for one / two / three workgroups a unit: 4 of up to 50000, 4 tokens, 40 on 40 heads 192 / 124 / 127 us; 6 of up to 12000, 3 tokens, 64 on 8 heads 35.6 / 29.3 / 34.7; 8 of 8000, 2
// tokens 22.0 / 23.0 / 26.3; 4 of up to 50000, 4 tokens, 8 on 8 heads of 64 27.5 / 24.2 / 24.1, 32 of 2048 10.7 / 15.3 / 16.2.
//
// Many rows: whole requests where the row tiles fill the chip, else a workgroup, of which one fits, for every compute unit, and chunks of 16 pages or more.  For one / two / three: 700 tokens on 4096
// positions, 64 on 8 heads 125 / 235 / 239 us, 32 on 32 125 / 141 / 141; 5 requests of 80 on up to 3000, 40 on 40 heads 71 / 107 / 98; 3 of 150 on up to 6000, 32 on 32 128 / 123 / 118; a prompt of 3000, 8 on 8 heads
// of 64 110 / 98 / 98.  Chunks of 8 / 16 / 32 pages at least: 64 tokens on 8000 positions, 64 on 8 heads, one request 51 / 57 / 80 us, two 90 / 71 / 90; 128 tokens, 32 on 32 60 / 48 / 66;
// 3 of 91 on 3388, 8 on 8 of 64 27 / 36 / 53.
//
// Every request is dealt as one of max_q rows, for the host knows no others: single tokens with long contexts do better in a call of their own (a chunk of 512 tokens on 8000 positions with three of
// them on 131000, 64 on 8 heads: 2414 us in one call, 309 in two).
void thi::kv4_plan(Kv4AttnArgs& a, int num_cus)
{
    const int group = a.Hq / a.Hkv;
    a.tiles = (int)(((long)a.max_q * group + 15) / 16);
    a.split_rows = (long)a.max_q * group <= FEW_ROWS;
    long n;
    if (a.split_rows) {
        const long items = (long)a.B * a.Hkv * a.tiles;
        a.min_chunk = FEW_CHUNK;
        n = a.max_pages <= 16 ? 1 : (long)(a.max_q > 1 ? FEW_PER_CU : ONE_PER_CU) * num_cus / items;
    } else {
        const long items = (long)a.B * a.Hkv * ((a.tiles + 15) / 16);
        a.min_chunk = MANY_CHUNK;
        n = (long)MANY_PER_CU * num_cus / items;
    }
    const long most = (a.max_pages + a.min_chunk - 1) / a.min_chunk;
    n = n < 1 ? 1 : n > KV4_MAX_SPLIT ? KV4_MAX_SPLIT : n;
    a.nsplit = (int)(n > most ? most : n);
}

extern "C" {

size_t thi_kv4_page_bytes(int Hkv, int D)
{
    return heads_ok(Hkv, Hkv, D) ? (size_t)Hkv * kv4_head_bytes(D) : 0;
}

int thi_qk_norm_rope_kv4(const void* qkv, int ld, const void* q_gamma, const void* k_gamma, float eps, const int* positions, const float* theta,
                         const int* slots, void* q_out, void* pages, int T, int Hq, int Hkv, int D, int num_pages, void* hip_stream)
{
    if (!qkv || !slots || !q_out || !pages || (theta && !positions)) return THI_ERR_NULL;
    if (T < 1 || !heads_ok(Hq, Hkv, D) || !pool_ok(num_pages)) return THI_ERR_SHAPE;
    if ((ld & 7) || ld < (long)(Hq + 2 * Hkv) * D) return THI_ERR_SHAPE;
    if (misaligned(qkv, 16) || misaligned(q_gamma, 16) || misaligned(k_gamma, 16) || misaligned(q_out, 16) || misaligned(pages, 16) ||
        misaligned(positions, 4) || misaligned(theta, 4) || misaligned(slots, 4))
        return THI_ERR_ALIGN;
    (void)hipGetLastError();      // an error another user of the runtime left behind is not ours to report
    Kv4AppendArgs a{};
    a.qkv = (const uint16_t*)qkv;
    a.q_gamma = (const uint16_t*)q_gamma;
    a.k_gamma = (const uint16_t*)k_gamma;
    a.positions = positions;
    a.theta = theta;
    a.slots = slots;
    a.q_out = (uint16_t*)q_out;
    a.pages = (unsigned char*)pages;
    a.eps = eps;
    a.T = T; a.ld = ld; a.Hq = Hq; a.Hkv = Hkv; a.D = D; a.num_pages = num_pages;
    return finish(launch_kv4_append(a, device_cu_count(), (hipStream_t)hip_stream));
}

int thi_kv4_read(const void* pages, const int* slots, void* k_out, void* v_out, int T, int Hkv, int D, int num_pages, void* hip_stream)
{
    if (!pages || !slots || (!k_out && !v_out)) return THI_ERR_NULL;
    if (T < 1 || !heads_ok(Hkv, Hkv, D) || !pool_ok(num_pages)) return THI_ERR_SHAPE;
    if (misaligned(pages, 16) || misaligned(slots, 4) || misaligned(k_out, 16) || misaligned(v_out, 16)) return THI_ERR_ALIGN;
    (void)hipGetLastError();
    Kv4ReadArgs a{(const unsigned char*)pages, slots, (uint16_t*)k_out, (uint16_t*)v_out, T, Hkv, D, num_pages};
    return finish(launch_kv4_read(a, (hipStream_t)hip_stream));
}

size_t thi_kv4_attention_workspace_bytes(int B, int T, int Hq, int Hkv, int D, int max_q, int max_pages)
{
    if (B < 1 || B > 65535 || T < 1 || !heads_ok(Hq, Hkv, D) || max_q < 1 || max_q > T || max_pages < 1 || max_pages > 0x7fffffff / KV4_PAGE) return 0;
    return bytes_of_rows(most_rows(B, Hq, Hkv, max_q, max_pages, device_cu_count()), D);
}

int thi_kv4_attention(const void* q, const void* pages, const int* page_table, const int* seq_lens, const int* q_offsets, float scale, void* out,
                      int B, int T, int Hq, int Hkv, int D, int max_q, int num_pages, int max_pages,
                      void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!q || !pages || !page_table || !seq_lens || !out || !workspace) return THI_ERR_NULL;
    if (!thi_kv4_attention_workspace_bytes(B, T, Hq, Hkv, D, max_q, max_pages) || !pool_ok(num_pages) || (!q_offsets && (T != B || max_q != 1))) return THI_ERR_SHAPE;
    if (misaligned(q, 16) || misaligned(pages, 16) || misaligned(out, 16) || misaligned(page_table, 4) || misaligned(seq_lens, 4) ||
        misaligned(q_offsets, 4) || misaligned(workspace, 256))
        return THI_ERR_ALIGN;
    Kv4AttnArgs a{};
    a.B = B; a.T = T; a.Hq = Hq; a.Hkv = Hkv; a.D = D; a.max_q = max_q; a.num_pages = num_pages; a.max_pages = max_pages;
    kv4_plan(a, device_cu_count());
    if (workspace_bytes < bytes_of_rows(a.nsplit > 1 ? (size_t)B * max_q * Hq * a.nsplit : 0, D)) return THI_ERR_WORKSPACE;
    (void)hipGetLastError();
    a.q = (const uint16_t*)q;
    a.pages = (const unsigned char*)pages;
    a.page_table = page_table;
    a.seq_lens = seq_lens;
    a.q_offsets = q_offsets;
    a.out = (uint16_t*)out;
    a.scale2 = scale * 1.44269504088896340736f;
    if (a.scale2 == 0.f) a.scale2 = 1e-30f;      // (all weights equal either way; a masked score of -inf stays what it is)
    a.part = (float*)workspace;
    return finish(launch_kv4_attention(a, (hipStream_t)hip_stream));
}

size_t thi_kv4_pages_workspace_bytes(int rows_out, int rows_in, int max_pages, int num_pages)
{
    if (rows_in < 1 || rows_out < 1 || max_pages < 1 || max_pages > 0x7fffffff / KV4_PAGE || !pool_ok(num_pages)) return 0;
    return (pages_workspace_words(rows_in, rows_out, num_pages) * 4 + 255) / 256 * 256;
}

static int check_pages(const void* pages, size_t page_bytes, int layers, size_t layer_bytes, int num_pages)
{
    if (!page_bytes || (page_bytes & 15) || layers < 1 || layers > 65533 || (layer_bytes & 15)) return THI_ERR_SHAPE;
    if (page_bytes > ((size_t)1 << 62) / (size_t)num_pages || (layers > 1 && layer_bytes < page_bytes * (size_t)num_pages)) return THI_ERR_SHAPE;
    return misaligned(pages, 16) ? THI_ERR_ALIGN : THI_OK;
}

int thi_kv4_fork(const int* refs_in, const int* table_in, const int* lens_in, const int* parents, const int* headroom,
                 int* refs_out, int* table_out, int* lens_out, int* info, void* pages, size_t page_bytes, int layers, size_t layer_bytes,
                 int rows_in, int rows_out, int num_pages, int max_pages, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!refs_in || !table_in || !lens_in || !parents || !refs_out || !table_out || !lens_out || !pages || !workspace) return THI_ERR_NULL;
    const size_t need = thi_kv4_pages_workspace_bytes(rows_out, rows_in, max_pages, num_pages);
    if (!need || refs_out == refs_in || table_out == table_in || lens_out == lens_in) return THI_ERR_SHAPE;
    const int rc = check_pages(pages, page_bytes, layers, layer_bytes, num_pages);
    if (rc != THI_OK) return rc;
    const void* const words[] = {refs_in, table_in, lens_in, parents, headroom, refs_out, table_out, lens_out, info};
    for (const void* p : words)
        if (misaligned(p, 4)) return THI_ERR_ALIGN;
    if (misaligned(workspace, 256)) return THI_ERR_ALIGN;
    if (workspace_bytes < need) return THI_ERR_WORKSPACE;
    (void)hipGetLastError();
    const PagesArgs a{refs_in, table_in, lens_in, parents, headroom, refs_out, table_out, lens_out, info, (char*)pages, page_bytes, layer_bytes,
                      rows_in, rows_out, layers, num_pages, max_pages, (int*)workspace};
    return finish(launch_kv4_fork(a, device_cu_count(), (hipStream_t)hip_stream));
}

int thi_kv4_compact(const int* refs_in, const int* table_in, int* refs_out, int* table_out, int* info, void* pages, size_t page_bytes,
                    int layers, size_t layer_bytes, int rows, int num_pages, int max_pages, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!refs_in || !table_in || !refs_out || !table_out || !pages || !workspace) return THI_ERR_NULL;
    const size_t need = thi_kv4_pages_workspace_bytes(rows, rows, max_pages, num_pages);
    if (!need || refs_out == refs_in || table_out == table_in) return THI_ERR_SHAPE;
    const int rc = check_pages(pages, page_bytes, layers, layer_bytes, num_pages);
    if (rc != THI_OK) return rc;
    const void* const words[] = {refs_in, table_in, refs_out, table_out, info};
    for (const void* p : words)
        if (misaligned(p, 4)) return THI_ERR_ALIGN;
    if (misaligned(workspace, 256)) return THI_ERR_ALIGN;
    if (workspace_bytes < need) return THI_ERR_WORKSPACE;
    (void)hipGetLastError();
    const PagesArgs a{refs_in, table_in, nullptr, nullptr, nullptr, refs_out, table_out, nullptr, info, (char*)pages, page_bytes, layer_bytes,
                      rows, rows, layers, num_pages, max_pages, (int*)workspace};
    return finish(launch_kv4_compact(a, device_cu_count(), (hipStream_t)hip_stream));
}

}  // extern "C"
