// Host-side check of how a tile's pages are cut into parts: more parts than the scratch holds are never asked for, whatever
// number of tiles a call's sequences come to (starts that do not ascend count rows several times).  Built by
// tests/test_paged_bounds_cpu.py with the host compiler; no device is touched.
#include <algorithm>
#include <cstdint>
#include <cstdio>

#include "kernels.h"

using namespace sdsat;

int main() {
    int failures = 0;
    const int heads[] = {1, 2, 3, 8, 12, 40, 96, 128, 1000, 1024};
    auto check = [&](int64_t tiles, int kv) {
        const int64_t splits = paged_tile_splits((int)tiles, kv);
        if (splits < 1 || splits > kPagedMaxTileParts || (splits > 1 && tiles * kv * splits > kPagedTileParts) ||
            (splits < kPagedMaxTileParts && tiles * kv * (splits + 1) <= kPagedTileParts)) {
            std::printf("FAIL: %lld tiles of %d key heads in %lld parts\n", (long long)tiles, kv, (long long)splits);
            ++failures;
        }
    };
    // what count_pieces returns: up to 2^24 for each of 64 lanes
    for (int kv : heads) {
        for (int64_t tiles = 0; tiles < 3000; ++tiles) check(tiles, kv);
        for (int shift = 10; shift <= 30; ++shift)
            for (int64_t by = -3; by <= 3; ++by) check(std::min<int64_t>((1ll << shift) + by, 1 << 30), kv);
        for (int64_t product = 1ll << 31; product <= 1ll << 36; product *= 2)   // past an int, and round to nothing
            for (int64_t by = -1; by <= 2; ++by)
                if (product / kv + by <= 1 << 30) check(product / kv + by, kv);
    }
    std::printf("%s (%d failed)\n", failures ? "FAILED" : "ok", failures);
    return failures != 0;
}
