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

// Long runs are shared by workgroups, up to the largest bound of rows there is
static void plan() {
    static int32_t up;
    struct { int B, max_rows; bool trees; int shares; } of[] = {
        {1, 0, false, 1}, {1, 4096, false, 1}, {1, 4097, false, 2}, {64, 16384, false, 4}, {65, 16384, false, 2}, {1, 300000, false, 64}, {1, 2147483647 - 4096, false, 64},
        {1, 2147483647 - 4094, false, 64}, {1, 2147483647, false, 64}, {64, 2147483647, true, 1}, {65535, 2147483647, false, 64}, {65535, 1000000, false, 1}};
    for (auto &w : of) {
        KvPlanArgs a{};
        a.B = w.B, a.max_rows = w.max_rows, a.parents = w.trees ? &up : nullptr;
        CHECK(kv_plan_shares(a) == w.shares, "%d requests, %d rows: %d shares", w.B, w.max_rows, kv_plan_shares(a));
    }
}

int main() {
    plan();
    store();
    std::printf(fails ? "%d failures\n" : "ok\n", fails);
    return fails != 0;
}
