// Driver of tests/test_host_fp4_guards.py: whatever kernel a call over 4-bit codes goes to, the positions that the kernel counts (steps or stages, and what it counts for a
// tile or a request beside them) are 32-bit numbers.  The stand-in for the HIP runtime is that of host_fp4.cpp.
#define main host_fp4_main
#include "host_fp4.cpp"
#undef main

int main()
{
    int seen[6] = {};                         // of the three divisions: taken, and not taken for the numbers' sake alone
    const int shapes[][5] = {{32, 8, 128, 512, 7}, {8, 2, 128, 4096, 20}, {6, 2, 64, 256, 3}, {1, 1, 128, 100000, 1}, {32, 1, 128, 1024, 60}};
    for (const auto &x : shapes) {
        const int hq = x[0], hkv = x[1], d = x[2], chunk = x[3], segs = x[4], g = hq / hkv;
        int64_t last = 0;
        for (double b = 4; b < 130e6; b *= 1.05) {
            const int blocks = (int)b;
            if (blocks == last) continue;
            last = blocks;
            tetri_ctx *h = handle(hq, hkv, d, chunk, blocks, segs);
            Args a;
            a.n = segs;
            tetri_set_option(h, "attn_variant", 3);
            CHECK(prefill(h, a) == TETRI_OK);
            const int64_t tiles = (int64_t)chunk * g / kPrefillFp4Cols + segs, steps = ((int64_t)blocks * 16 + 31) / 32 + (chunk + 31) / 32;
            const bool small = tiles * (steps + kPrefillFp4TileSteps) <= INT_MAX;
            if (g_kernel == "small") { CHECK(small); ++seen[0]; } else { ++seen[1]; }
            tetri_set_option(h, "attn_variant", 2);
            tetri_set_option(h, "stream_wgs", 2);
            CHECK(prefill(h, a) == TETRI_OK);
            if (g_attn.stream_wgs > 0) {
                const int64_t stages = ((int64_t)blocks * 16 + 127) / 128 + (chunk + 127) / 128;
                CHECK(g_attn.tiles * (stages + kFp4TileStages) * (g_attn.stream_wgs + 1) <= INT_MAX);
                ++seen[2];
            } else {
                ++seen[3];
            }
            tetri_set_option(h, "decode_ranges", 4);
            for (int n : {2, 100, 1000}) {
                a.n = n;
                a.max_ctx = std::min(16 * (blocks - 1), 100000);
                CHECK(decode(h, a) == TETRI_OK);
                const int64_t all = n * (((int64_t)blocks * 16 + 31) / 32 + kFp4RequestSteps);
                if (g_kernel == "ranges") { CHECK(all <= INT_MAX); ++seen[4]; } else { ++seen[5]; }
            }
            tetri_destroy(h);
        }
    }
    for (int n : seen) CHECK(n > 0);
    std::printf("guards: ok\n");
    return 0;
}
