// Driver of the planner of attention calls over the 8-bit cache and of its launch, for the
// sanitizer build (as host_kv8_driver.cpp). Without arguments: a launch whose layout the
// kernels do not take is refused before anything is launched. With "layouts": reads calls
// from the standard input, a line each,
//     batch heads kv_heads head_dim window n_q chunk lengths..., c_0's first
// and prints for each the layout that the library chooses:
//     few n_tiles n_whole parts cut n_kblocks workspace-bytes
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <cstring>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "../../paper_2506_03099_amd/csrc/tm_api.cpp"

namespace {

int refused_launch() {
    // 257 split tiles of 32 rows, one more than the merge is made for; no pointer of it exists
    tmk::Kv8AttnArgs a{};
    a.few = 4;
    a.B = 257;
    a.H = a.Hk = a.group = 1;
    a.n_q = a.rows = a.n_tiles = 1;
    a.n_whole = 0;
    a.parts = 2;
    a.n_kblocks = 50;
    a.n_ranges = 1;
    a.range_keys[0] = 50 * 64;
    a.n_blocks = 50;
    const hipError_t e = tmk::launch_attn_kv8(a, 128, nullptr);
    if (e != hipErrorInvalidValue) {
        std::fprintf(stderr, "a launch of 257 split tiles: %s\n", hipGetErrorString(e));
        return 1;
    }
    std::printf("host kv8 layout driver: all checks passed\n");
    return 0;
}

int layouts() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        int32_t B = 0, H = 0, Hk = 0, D = 0, window = 0, n_q = 0, n = 0;
        std::vector<int32_t> lengths;
        in >> B >> H >> Hk >> D >> window >> n_q;
        while (in >> n) lengths.push_back(n);
        if (lengths.empty()) return 1;
        int32_t chunk = 1;
        for (size_t i = 1; i < lengths.size(); ++i) chunk = std::max(chunk, lengths[i]);
        tm_kv8_cache c{};
        c.book.desc.batch = B;
        c.book.desc.heads = H;
        c.book.desc.head_dim = D;
        c.book.desc.tokens_per_frame = 1;
        c.book.desc.chunk_frames = chunk;
        c.book.desc.ref_frames = lengths[0];
        c.book.desc.window = window;
        c.book.desc.dtype = TM_BF16;
        c.kv_heads = Hk;
        tm_kv_cache_reset(&c.book);
        c.book.ref_len = lengths[0];
        c.book.latest = int32_t(lengths.size()) - 1;
        for (int32_t t = 1; t <= c.book.latest; ++t) {
            c.book.slot_chunk[(t - 1) % (window + 1)] = t;
            c.book.slot_len[(t - 1) % (window + 1)] = lengths[size_t(t)];
        }
        Kv8Geo z;
        tmk::Kv8AttnArgs a{};
        if (check_cache8(&c, &z) != TM_OK || plan_attn8(&c, z, c.book.latest, n_q, &a) != TM_OK) {
            std::fprintf(stderr, "%s: %s\n", line.c_str(), tm_last_error());
            return 1;
        }
        std::printf("%d %d %d %d %d %d %zu\n", a.few, a.n_tiles, a.n_whole, a.parts, a.cut, a.n_kblocks,
                    tm_kv8_attn_workspace(&c, c.book.latest, n_q));
    }
    return 0;
}

}  // namespace

int main(int argc, char** argv) {
    return argc > 1 && std::strcmp(argv[1], "layouts") == 0 ? layouts() : refused_launch();
}
