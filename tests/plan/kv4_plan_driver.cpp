// How attention over the 4-bit cache is dealt (test infrastructure; no GPU: linked with kv4_api.hip and stand-ins).  Input: lines "B Hq Hkv D max_q max_pages";
// output: "few tiles nsplit min_chunk" for 256 compute units.
#include "../../paper_2605_25655_amd/csrc/kv4.h"

#include <cstdio>

namespace thi {
hipError_t launch_kv4_append(const Kv4AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_read(const Kv4ReadArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_fork(const PagesArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_compact(const PagesArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_kv4_attention(const Kv4AttnArgs&, hipStream_t) { return hipSuccess; }
size_t pages_workspace_words(int, int, int) { return 64; }
}  // namespace thi

int main()
{
    thi::Kv4AttnArgs a{};
    while (std::scanf("%d %d %d %d %d %d", &a.B, &a.Hq, &a.Hkv, &a.D, &a.max_q, &a.max_pages) == 6) {
        thi::kv4_plan(a, 256);
        std::printf("%d %d %d %d\n", (int)a.split_rows, a.tiles, a.nsplit, a.min_chunk);
    }
    return 0;
}
