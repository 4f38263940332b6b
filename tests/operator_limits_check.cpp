// Host-side checks of limits: what the launches of the cache reordering, the shared attention and the log probabilities
// take and refuse at the ends of their ranges, and how large their grids and workspaces get.  Built by
// tests/test_operator_limits_cpu.py with the host compiler against libsdsat.so; no device is touched (only invalid
// argument sets are passed to a launch).
#include <algorithm>
#include <cstdio>
#include <limits>
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
    int dummy[256] = {};
    void* ptr = dummy;
    float* fp = reinterpret_cast<float*>(ptr);
    // reordering: a launch holds fewer than 2^32 threads of 256-thread workgroups, one per 8 KiB of a moved row until then
    {
        struct Cache { int esz, L, H, Dh, S; };
        for (const Cache& c : {Cache{2, 32, 32, 128, 262112}, Cache{2, 32, 32, 128, 262144}, Cache{2, 32, 32, 128, 1 << 20},
                               Cache{4, 40, 40, 128, 1 << 19}, Cache{2, 1, 1, 64, (1 << 24) - 32}, Cache{2, 128, 127, 64, 1 << 21}}) {
            CHECK(reorder_supported(c.esz, 4, c.L, c.H, c.Dh, c.S), "a cache of %d slots is refused", c.S);
            for (int len : {c.S, c.S - 31, 1, 0})
                for (int first : {0, 32, 4096, c.S}) {
                    const size_t row = (size_t)std::max(0, (len + 31) / 32 * 32 - first / 32 * 32) * c.Dh * c.esz;
                    const size_t chunks = (row + 8191) / 8192 * 2 * c.H * c.L;
                    const long n = reorder_workgroups(c.esz, c.L, c.H, c.Dh, len, first);
                    CHECK(n >= 1 && (unsigned long)n * 256 < 1ul << 32, "%ld workgroups", n);
                    CHECK((size_t)n == std::max<size_t>(1, chunks) || chunks * 256 >= 1ul << 32, "%ld workgroups for %zu chunks", n, chunks);
                }
        }
    }
    // shared attention: what is left of a prefix behind its pages is less than a page
    {
        int pages[2] = {4, 3};
        const SharedPlan p = plan_shared(4, 2, 2, 6, 1, pages, 140, 256);
        for (int rest : {-1, 32, 1 << 20}) {
            SharedArgs a{};
            a.at.qbuf = fp; a.at.kc = a.at.vc = ptr; a.at.cache_len = dummy; a.at.B = 4; a.at.q = 6; a.at.H = 2; a.at.S_max = 256;
            a.at.out = ptr; a.at.out_f32 = 1; a.at.ldo = 128; a.at.out_rows = 24; a.at.err = dummy;
            a.group = 2; a.pages[0] = 4; a.pages[1] = 3; a.rest[1] = rest; a.part = fp;
            CHECK(launch_attention_shared(1, 64, p, a, nullptr) == hipErrorInvalidValue, "shared attention accepted %d slots left", rest);
        }
    }
    // the shapes of tests/test_gpu_attention_shared_parts.py cut own slots into several parts
    {
        struct Shape { int B, group, H, S, pages0, pages1, len, parts; };
        for (const Shape& s : {Shape{4, 2, 2, 2752, 2, 15, 2580, 3}, Shape{4, 2, 3, 2752, 2, 15, 2580, 3}, Shape{2, 2, 32, 3424, 10, 0, 3333, 3},
                               Shape{4, 4, 32, 3424, 10, 0, 3333, 3}, Shape{3, 3, 32, 3424, 10, 0, 3333, 3}, Shape{2, 2, 2, 2336, 2, 0, 2112, 3}}) {
            const int pages[2] = {s.pages0, s.pages1};
            const SharedPlan p = plan_shared(s.B, s.group, s.H, 1, 1, pages, s.len, s.S);
            CHECK(p.own_parts >= s.parts, "%d sequences of %d heads: %d own parts", s.B, s.H, p.own_parts);
        }
    }
    // the parts of every plan fit what a context of these sizes reserves
    {
        struct Cfg { int maxB, H, Dh, maxQ, S; };
        for (const Cfg& c : {Cfg{4, 4, 64, 6, 128}, Cfg{64, 4, 64, 64, 128}, Cfg{8, 32, 128, 64, 1312}, Cfg{16, 40, 128, 1024, 16896},
                             Cfg{64, 2, 128, 11, 4096}, Cfg{24, 8, 64, 300, 608}, Cfg{2, 1, 64, 1, 32}, Cfg{130, 3, 64, 2, 96}, Cfg{64, 32, 128, 64, 4096}}) {
            const size_t have = shared_partial_floats_most(c.maxB, c.H, c.maxQ, c.Dh, c.S);
            for (int B = 2; B <= c.maxB; ++B)
                for (int group = 2; group <= B; ++group) {
                    if (B % group || B / group > kMaxShareGroups) continue;
                    for (int most = 0; most < c.S / 32; most += 1 + most / 3)
                        for (int other : {0, most / 2, most}) {   // the pages of the other groups
                            std::vector<int> pages(B / group, other);
                            pages[0] = most;
                            for (int q : {1, std::min(c.maxQ, kAttnSplitRows)})
                                for (int len : {32 * most, c.S - q}) {
                                    if (len < 32 * most || len + q > c.S) continue;
                                    const SharedPlan p = plan_shared(B, group, c.H, q, 1, pages.data(), len, c.S);
                                    CHECK(shared_partial_floats(p, B, q, c.H, c.Dh) <= have, "B %d group %d q %d, %d pages: %zu of %zu",
                                          B, group, q, most, shared_partial_floats(p, B, q, c.H, c.Dh), have);
                                }
                        }
                }
        }
        CHECK(shared_partial_floats_most(1, 32, 64, 128, 4096) == 0, "one sequence shares nothing");
    }
    // log probabilities: temperatures by which the logits cannot be scaled
    const float inf = std::numeric_limits<float>::infinity();
    for (float t : {0.f, -0.f, -1.f, 1e-45f, 1e-39f, 3.0e-39f, 3.5e-39f, 4.2e-39f, inf, -inf, std::numeric_limits<float>::quiet_NaN()})
        CHECK(launch_token_logprobs(fp, 1, 100, dummy, t, 2, fp, fp, dummy, fp, ptr, dummy, dummy, nullptr) == hipErrorInvalidValue,
              "log probabilities accepted the temperature %g", t);
    for (float t : {4.25e-39f, 5.877471754e-39f, 1e-30f, 1.f, 3.402823466e38f})
        CHECK(logprob_temperature_ok(t), "the temperature %g is refused", t);
    std::printf("ok (%d failed)\n", failures);
    return failures != 0;
}
