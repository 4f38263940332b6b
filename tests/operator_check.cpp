// Host-side checks of the shared-prefix attention's plans, of what its workspace holds, and of what the launches of
// the cache reordering, the shared attention and the log probabilities refuse.  Built by tests/test_operators_cpu.py
// with the host compiler against libsdsat.so; no device is touched (only invalid argument sets are passed to a launch).
#include <algorithm>
#include <cstdio>
#include <vector>

#include "kernels.h"

using namespace sdsat;

static int failures = 0;
#define CHECK(cond, ...)                      \
    do {                                      \
        if (!(cond)) {                        \
            std::printf("FAIL: " __VA_ARGS__); \
            std::printf("\n");                \
            ++failures;                       \
        }                                     \
    } while (0)

int main() {
    struct Cfg { int maxB, H, Dh, maxQ, S; };
    const Cfg cfgs[] = {{4, 4, 64, 6, 128}, {8, 32, 128, 64, 1312}, {16, 40, 128, 1024, 16896}, {64, 2, 128, 11, 4096},
                        {24, 8, 64, 300, 608}, {2, 1, 64, 1, 32}, {65, 3, 64, 2, 96}};
    for (const Cfg& c : cfgs) {
        const size_t have = shared_partial_floats_most(c.maxB, c.H, c.maxQ, c.Dh);
        for (int dtype = 0; dtype < 2; ++dtype)
            for (int B = 2; B <= c.maxB; B += 1 + B / 7)
                for (int group = 2; group <= B; ++group) {
                    if (B % group || B / group > kMaxShareGroups) continue;
                    for (int most : {0, 1, 3, 4, 5, 31, 32, 33, 511, c.S / 32 - 1}) {
                        if (most >= c.S / 32) continue;
                        std::vector<int> pages(B / group);
                        for (size_t g = 0; g < pages.size(); ++g) pages[g] = std::max(0, most - 2 * (int)g);
                        const SharedPlan one = plan_shared(B, group, c.H, 1, dtype, pages.data(), c.S - 1, c.S);
                        for (int q = 1; q <= c.maxQ; q += q < 18 ? 1 : 23)
                            for (int len : {32 * most, 32 * most + 45, c.S - q}) {
                                if (len < 32 * most || len + q > c.S) continue;
                                const SharedPlan p = plan_shared(B, group, c.H, q, dtype, pages.data(), len, c.S);
                                const int rows = p.staged ? 64 : 16;
                                CHECK(p.whole == (q > kAttnSplitRows) && (dtype == 1 || !p.staged) && (p.staged || dtype == 0 || !p.whole),
                                      "kind of workgroup at q %d", q);
                                if (p.whole) {
                                    CHECK(p.grid == B * c.H * p.tiles && p.tiles == (q + rows - 1) / rows, "grid of a long block, q %d", q);
                                    continue;
                                }
                                CHECK(shared_partial_floats(p, B, q, c.H, c.Dh) <= have, "parts: B %d group %d q %d need %zu have %zu",
                                      B, group, q, shared_partial_floats(p, B, q, c.H, c.Dh), have);
                                // every page of every group, and every own page up to the length, has a part
                                const int least = *std::min_element(pages.begin(), pages.end());
                                CHECK(p.chunk * p.prefix_parts >= most && p.own_chunk >= 1 && p.own_parts >= 1 &&
                                          p.own_parts * p.own_chunk >= (len + q + 31) / 32 - least &&
                                          p.slots == p.prefix_parts + p.own_parts,
                                      "parts: %d x %d for %d pages", p.chunk, p.prefix_parts, most);
                                CHECK(p.tiles * rows >= group * q && p.prefix_grid % 8 == 0 &&
                                          p.prefix_grid * (p.staged ? 1 : 2) >= (int)pages.size() * c.H * p.prefix_parts * p.tiles &&
                                          p.grid == p.prefix_grid + B * c.H * ((q + 15) / 16) * p.own_parts,
                                      "grid: %d, %d tiles", p.grid, p.tiles);
                                // the key ranges do not follow the block's rows or the committed length
                                CHECK(p.chunk == one.chunk && p.own_chunk == one.own_chunk && p.prefix_parts == one.prefix_parts,
                                      "key ranges vary with the block: B %d q %d len %d", B, q, len);
                            }
                    }
                }
    }
    int dummy[256] = {};
    void* ptr = dummy;
    float* fp = reinterpret_cast<float*>(ptr);
    // shared attention
    {
        int pages[2] = {4, 3};
        auto args = [&](int q) {
            SharedArgs a{};
            a.at.qbuf = fp; a.at.kc = a.at.vc = ptr; a.at.cache_len = dummy; a.at.B = 4; a.at.q = q; a.at.H = 2; a.at.S_max = 256;
            a.at.out = ptr; a.at.out_f32 = 1; a.at.ldo = 128; a.at.out_rows = 4 * q; a.at.err = dummy;
            a.group = 2; a.pages[0] = 4; a.pages[1] = 3; a.part = fp;
            return a;
        };
        auto bad = [&](const char* what, int dtype, int dh, SharedArgs a, SharedPlan p) {
            CHECK(launch_attention_shared(dtype, dh, p, a, nullptr) == hipErrorInvalidValue, "shared attention accepted %s", what);
        };
        const SharedPlan p = plan_shared(4, 2, 2, 6, 1, pages, 140, 256);
        SharedArgs a = args(6);
        bad("heads of 96", 1, 96, a, p);
        a.group = 3; bad("a group that does not divide the batch", 1, 64, a, p);
        a = args(6); a.pages[1] = 9; bad("more pages than slots", 1, 64, a, p);
        a = args(6); a.pages[1] = -1; bad("negative pages", 1, 64, a, p);
        a = args(6); a.pages[0] = p.chunk * p.prefix_parts + 1; bad("pages without a part", 1, 64, a, p);
        a = args(6); a.part = nullptr; bad("no buffer for the parts", 1, 64, a, p);
        a = args(6); a.at.S_max = 250; bad("a cache of broken pages", 1, 64, a, p);
        a = args(6); a.at.S_max = 1 << 25; bad("4 GiB of keys of a head", 1, 64, a, p);
        a = args(6); a.at.ldo = 130; bad("an odd row stride", 1, 64, a, p);
        a = args(6); a.at.qbuf = nullptr; bad("no queries", 1, 64, a, p);
        a = args(65); bad("a decode plan for a long block", 1, 64, a, p);
        SharedPlan r = p; r.staged = true; bad("staged floats", 0, 64, args(6), r);
        const SharedPlan w = plan_shared(4, 2, 2, 65, 1, pages, 140, 256);
        a = args(65); a.at.mask = reinterpret_cast<const uint64_t*>(ptr); bad("masks of a long block", 1, 64, a, w);
        r = w; r.staged = false; bad("a long bf16 block that is not staged", 1, 64, args(65), r);
    }
    // reordering
    {
        auto bad = [&](const char* what, int esz, int batch, int all, int Dh, int S, int len, const int* src, int first) {
            CHECK(launch_reorder(esz, ptr, ptr, 1024, 1, batch, all, 2, Dh, S, dummy, len, src, first, dummy, dummy, nullptr) ==
                      hipErrorInvalidValue, "reordering accepted %s", what);
        };
        bad("no sequences", 2, 0, 4, 64, 128, 20, dummy, 0);
        bad("more sequences than there are", 2, 5, 4, 64, 128, 20, dummy, 0);
        bad("1025 sequences", 2, 5, kReorderMaxBatch + 1, 64, 128, 20, dummy, 0);
        bad("broken pages", 2, 4, 4, 64, 120, 20, dummy, 0);
        bad("a length past the slots", 2, 4, 4, 64, 128, 129, dummy, 0);
        bad("a negative slot", 2, 4, 4, 64, 128, 20, dummy, -1);
        bad("2^24 slots", 2, 4, 4, 64, 1 << 24, 20, dummy, 0);
        bad("no map", 2, 4, 4, 64, 128, 20, nullptr, 0);
        bad("rows of 8 bytes", 2, 4, 4, 4, 128, 20, dummy, 0);
    }
    // log probabilities
    {
        auto bad = [&](const char* what, int M, int V, const int* tok, float T, int n, float* lp, int* ids, float* top, void* part) {
            CHECK(launch_token_logprobs(fp, M, V, tok, T, n, lp, fp, ids, top, part, dummy, dummy, nullptr) == hipErrorInvalidValue,
                  "log probabilities accepted %s", what);
        };
        bad("no rows", 0, 100, dummy, 1.f, 2, fp, dummy, fp, ptr);
        bad("temperature 0", 1, 100, dummy, 0.f, 2, fp, dummy, fp, ptr);
        bad("33 alternatives", 1, 100, dummy, 1.f, kMaxTop + 1, fp, dummy, fp, ptr);
        bad("more alternatives than ids", 1, 3, dummy, 1.f, 4, fp, dummy, fp, ptr);
        bad("no tokens", 1, 100, nullptr, 1.f, 2, fp, dummy, fp, ptr);
        bad("no room for the alternatives", 1, 100, dummy, 1.f, 2, fp, nullptr, fp, ptr);
        bad("no room for the alternatives' values", 1, 100, dummy, 1.f, 2, fp, dummy, nullptr, ptr);
        bad("no room for the segments", 1, 100000, dummy, 1.f, 2, fp, dummy, fp, nullptr);
        CHECK(logprob_part_bytes(7, 100) == 0, "one segment needs no workspace");
        CHECK(logprob_part_bytes(7, 32016) > 0, "segment results");
    }
    std::printf("ok (%d failed)\n", failures);
    return failures != 0;
}
