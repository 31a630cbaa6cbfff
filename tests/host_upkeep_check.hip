// Host-side check of the rules by which the upkeep of the bf16 cache is launched (no GPU call), at sizes where they were measured.  Built against
// the library and run by tests/test_host_upkeep_rules.py.
#include <cstdio>

#include "../paper_2601_11822_amd/csrc/kernels.h"

static int fails = 0;
#define CHECK(c, ...) do { if (!(c)) { if (fails++ < 10) { std::printf("FAIL %s:%d: ", __FILE__, __LINE__); std::printf(__VA_ARGS__); std::printf("\n"); } } } while (0)

// Rows go past the caches by their bytes, however many or few they are
static void store() {
    struct { int Hq, Hkv, hd, rows; bool past; } of[] = {
        {32, 8, 128, 2048, false}, {32, 8, 128, 2049, false}, {32, 8, 128, 4096, true}, {32, 8, 128, 16444, true}, {64, 8, 128, 2048, false}, {64, 8, 128, 4096, true},
        {8, 2, 128, 2049, false}, {8, 2, 128, 4096, false}, {8, 2, 128, 16384, true}, {32, 4, 64, 8192, false}, {32, 4, 64, 16384, true}, {16, 1, 128, 8192, false},
        {1, 1, 64, 33000000, true}, {32768, 2048, 128, 1000, true}, {8, 2, 128, 1, false}};
    for (auto &w : of) {
        KvStoreArgs a{};
        a.Hq = w.Hq, a.Hkv = w.Hkv, a.hd = w.hd, a.max_rows = w.rows;
        CHECK(kv_store_past(a) == w.past, "%d rows of %d/%d heads of %d", w.rows, w.Hq, w.Hkv, w.hd);
    }
}

int main() {
    store();
    std::printf(fails ? "%d failures\n" : "ok\n", fails);
    return fails != 0;
}
