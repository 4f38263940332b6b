// Host-side checks of the paged cache's plans, of what its workspace holds, and of what the launches of appending,
// attention and logit rules refuse.  Built by tests/test_paged_cpu.py with the host compiler against libsdsat.so; no
// device is touched (only invalid argument sets are passed to a launch).
#include <algorithm>
#include <cstdio>

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
#define REFUSED(call, what) CHECK((call) == hipErrorInvalidValue, "not refused: %s", what)

int main() {
    struct Cfg { int H, Hkv, Dh, B, rows, ctx; };
    const Cfg cfgs[] = {{32, 8, 128, 64, 64, 4001}, {32, 8, 128, 1, 1, 130001}, {4, 4, 64, 1, 6, 96}, {40, 40, 128, 6, 9000, 8500},
                        {8, 1, 64, 100, 8000, 1}, {28, 4, 128, 4096, 1 << 20, 1 << 24}, {1024, 1, 64, 3, 1000, 131072}, {7, 7, 128, 2, 64, 33}};
    for (const Cfg& c : cfgs) {
        const PagedPlan p = plan_paged(c.Hkv, c.B, c.ctx);
        const int group = c.H / c.Hkv;
        CHECK(p.part_shift >= 4 && p.max_parts >= 1 && p.max_parts <= kPagedMaxParts && ((long)p.max_parts * kPage << p.part_shift) >= c.ctx,
              "parts: %d of 2^%d pages for %d slots", p.max_parts, p.part_shift, c.ctx);
        size_t tile_at = 0;
        const size_t have = paged_part_floats(p, c.H, c.Hkv, c.Dh, c.B, c.rows, &tile_at);
        for (int B = 1; B <= c.B; B += 1 + B / 3)
            for (long max_q = 1; max_q <= std::min(c.rows, c.ctx); max_q += 1 + max_q / 2)
                for (long rows = max_q; rows <= c.rows; rows += 1 + rows) {
                    PagedPlan q = p;
                    plan_paged_call(q, c.H, c.Hkv, B, (int)rows, (int)max_q, c.ctx);
                    CHECK(q.part_shift == p.part_shift && q.max_parts == p.max_parts, "a call moves the handle's parts");
                    CHECK(q.few_wgs >= 1 && ((long)q.call_parts * kPage << q.part_shift) >= c.ctx && q.call_parts <= q.max_parts,
                          "short chunks: %d workgroups, %d parts", q.few_wgs, q.call_parts);
                    // tiles: every sequence may end in one that is not full
                    const bool tiles = max_q * group > kPagedFewRows;
                    CHECK(tiles == (q.tile_wgs > 0), "tiles for %ld rows of a group of %d", max_q, group);
                    if (tiles) {
                        const long most = std::max<long>((rows * group / kPagedTileRows + B) * c.Hkv, kPagedTileParts);
                        CHECK(q.tile_wgs >= most, "%d workgroups for %ld tiles", q.tile_wgs, most);
                        CHECK(have >= tile_at + (size_t)kPagedTileParts * kPagedTileRows * (c.Dh + 4), "no room for the tiles' parts");
                    }
                    if (q.call_parts > 1)
                        CHECK(have >= (size_t)B * c.Hkv * q.max_parts * kPagedFewRows * (c.Dh + 4) && tile_at >= (size_t)B * c.Hkv * q.max_parts * kPagedFewRows * (c.Dh + 4),
                              "no room for the short chunks' parts");
                }
    }

    int ints[8] = {0};
    alignas(16) static char mem[64];
    const PagedSeqs seqs{ints, ints, ints, 1, 2, 4, 4, 64, 3, ints};
    PagedAppendArgs ap{};
    ap.seq = seqs;
    ap.kp = ap.vp = ap.qout = mem;
    ap.x = mem;
    ap.H = 2; ap.Hkv = 1; ap.ldx = 256; ap.ldq = 128; ap.rot = 64;
    auto append = [&](const char* what, auto change) {
        PagedAppendArgs a = ap;
        int dh = 64;
        change(a, dh);
        REFUSED(launch_paged_append(1, 1, dh, a, nullptr), what);
    };
    append("append: head_dim 96", [](PagedAppendArgs&, int& dh) { dh = 96; });
    append("append: no K", [](PagedAppendArgs& a, int&) { a.kp = nullptr; });
    append("append: no x", [](PagedAppendArgs& a, int&) { a.x = nullptr; });
    append("append: no error flag", [](PagedAppendArgs& a, int&) { a.seq.err = nullptr; });
    append("append: H % Hkv", [](PagedAppendArgs& a, int&) { a.H = 3; a.Hkv = 2; });
    append("append: rot past the head", [](PagedAppendArgs& a, int&) { a.rot = 72; });
    append("append: rot % 8", [](PagedAppendArgs& a, int&) { a.rot = 12; });
    append("append: ldx % 8", [](PagedAppendArgs& a, int&) { a.ldx = 260; });
    append("append: max_len past the table", [](PagedAppendArgs& a, int&) { a.seq.max_len = 65; });
    append("append: no sequences", [](PagedAppendArgs& a, int&) { a.seq.B = 0; });

    PagedPlan plan = plan_paged(1, 1, 64);
    plan_paged_call(plan, 2, 1, 1, 4, 4, 64);
    PagedAttnArgs at{};
    at.seq = seqs;
    at.kp = at.vp = at.q = mem;
    at.out = mem;
    at.part = reinterpret_cast<float*>(mem);
    at.ldq = at.ldo = 128; at.H = 2; at.Hkv = 1; at.scale = 1.f;
    at.part_shift = plan.part_shift; at.max_parts = plan.max_parts; at.tile_wgs = plan.tile_wgs; at.few_wgs = plan.few_wgs;
    at.few_once = plan.few_once;
    auto attend = [&](const char* what, auto change) {
        PagedAttnArgs a = at;
        PagedPlan p = plan;
        int dh = 64;
        change(a, p, dh);
        REFUSED(launch_paged_attention(1, dh, p, a, nullptr), what);
    };
    using A = PagedAttnArgs&;
    using P = PagedPlan&;
    attend("attention: head_dim 96", [](A, P, int& dh) { dh = 96; });
    attend("attention: no V", [](A a, P, int&) { a.vp = nullptr; });
    attend("attention: no scratch", [](A a, P, int&) { a.part = nullptr; });
    attend("attention: scale 0", [](A a, P, int&) { a.scale = 0.f; });
    attend("attention: scale NaN", [](A a, P, int&) { a.scale = __builtin_nanf(""); });
    attend("attention: window below 0", [](A a, P, int&) { a.window = -1; });
    attend("attention: mask with a window", [](A a, P, int&) { static uint64_t m; a.mask = &m; a.window = 3; });
    attend("attention: mask of long chunks", [](A a, P, int&) { static uint64_t m; a.mask = &m; a.seq.max_q = 65; });
    attend("attention: H % Hkv", [](A a, P, int&) { a.H = 3; a.Hkv = 2; });
    attend("attention: another plan's parts", [](A a, P, int&) { a.part_shift += 1; });
    attend("attention: parts too short", [](A a, P p, int&) { a.part_shift = p.part_shift = 0; a.max_parts = p.max_parts = 1; });
    attend("attention: tiles that the plan lacks", [](A a, P, int&) { a.seq.max_q = a.seq.rows = 33; });
    attend("attention: ldq % 8", [](A a, P, int&) { a.ldq = 132; });

    LogitRuleArgs ru{};
    float z[4];
    ru.logits = z; ru.out = z; ru.B = 1; ru.q = 1; ru.V = 4; ru.err = ints;
    auto rules = [&](const char* what, auto change) {
        LogitRuleArgs a = ru;
        change(a);
        REFUSED(launch_logit_rules(a, nullptr), what);
    };
    rules("rules: no logits", [](LogitRuleArgs& a) { a.logits = nullptr; });
    rules("rules: no rows", [](LogitRuleArgs& a) { a.q = 0; });
    rules("rules: history without lengths", [&](LogitRuleArgs& a) { a.history = ints; a.history_ld = 3; });
    rules("rules: history of 2^24", [&](LogitRuleArgs& a) { a.history = a.history_len = ints; a.history_ld = 1 << 24; });
    rules("rules: tokens of 65 rows", [&](LogitRuleArgs& a) { a.tokens = ints; a.q = 65; });
    rules("rules: allowed words too few", [&](LogitRuleArgs& a) { static uint32_t w; a.allowed = &w; a.V = 33; a.allowed_ld = 1; });
    std::printf("%s (%d failed)\n", failures ? "FAILED" : "ok", failures);
    return failures != 0;
}
