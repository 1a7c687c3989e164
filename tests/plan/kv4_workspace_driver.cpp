// A workspace that is large enough for a batch is large enough for every smaller one (test infrastructure; no GPU: linked with kv4_api.hip, the launchers are
// stand-ins that check what the kernels put into it).  Prints the sizes asked for, and the first call that is refused.
#include "../../include/thi.h"
#include "../../paper_2605_25655_amd/csrc/kv4.h"

#include <cstdio>

namespace thi {
static size_t given = 0;
static long chunked = 0;
hipError_t launch_kv4_append(const Kv4AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_read(const Kv4ReadArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_fork(const PagesArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_compact(const PagesArgs&, int, hipStream_t) { return hipSuccess; }
size_t pages_workspace_words(int, int, int) { return 64; }
hipError_t launch_kv4_attention(const Kv4AttnArgs& a, hipStream_t)
{
    if (a.nsplit == 1) return hipSuccess;
    ++chunked;
    return (size_t)a.B * a.max_q * a.Hq * a.nsplit * (a.D + 2) * sizeof(float) <= given ? hipSuccess : hipErrorInvalidValue;
}
}  // namespace thi

int main()
{
    void* const p = (void*)0x7f0000000000ull;      // aligned, never used
    const int heads[][3] = {{8, 8, 64}, {32, 32, 128}, {64, 8, 128}, {64, 1, 128}, {34, 2, 64}};
    const int batches[] = {1, 2, 3, 4, 5, 7, 16, 33, 64, 100}, rows[] = {1, 2, 3, 8, 9, 33, 64, 65, 129, 700, 4096}, tables[] = {1, 16, 17, 40, 100, 2047};
    long calls = 0;
    for (const auto& h : heads)
        for (int B : batches)
            for (int q : rows)
                for (int mp : tables) {
                    thi::given = thi_kv4_attention_workspace_bytes(B, B * q, h[0], h[1], h[2], q, mp);
                    if (!thi::given || thi::given % 256) return 2;
                    if (thi::given > ((size_t)80 << 20)) return 3;          // a bounded share of the device's memory, whatever the batch
                    for (int b : batches)
                        for (int r : rows)
                            for (int m : tables) {
                                if (b > B || r > q || m > mp) continue;
                                ++calls;
                                const int rc = thi_kv4_attention(p, p, (int*)p, (int*)p, (int*)p, 0.1f, p, b, b * r, h[0], h[1], h[2], r, 7, m, p, thi::given, nullptr);
                                if (rc == THI_OK) continue;
                                std::printf("status %d: %zu bytes for %d requests of %d rows, tables of %d, do not do for %d of %d, %d (%d/%d heads of %d)\n", rc, thi::given, B, q, mp, b, r, m, h[0], h[1], h[2]);
                                return 1;
                            }
                }
    std::printf("ok %ld calls, %ld in chunks\n", calls, thi::chunked);
    return thi::chunked > 1000 ? 0 : 4;
}
