// Host-side check of the rules by which launches over a 4-bit cache take their forms (no GPU call), at sizes where the forms were
// measured and at those that GPU tests are about.  Built against the library and run by tests/test_host_kv4_forms.py.
#include <cstdio>

#include "../paper_2601_11822_amd/csrc/kernels.h"

static int fails = 0;
#define CHECK(c, ...) do { if (!(c)) { if (fails++ < 10) { std::printf("FAIL %s:%d: ", __FILE__, __LINE__); std::printf(__VA_ARGS__); std::printf("\n"); } } } while (0)

// Decode: B rows of Hkv kv heads, contexts of up to max_ctx tokens
static void decode_forms() {
    struct { int B, Hkv, max_ctx; Kv4DecodeForm form; } of[] = {
        {1, 8, 901, KV4_WHOLE8}, {1, 8, 1536, KV4_WHOLE8}, {1, 8, 1665, KV4_SHARES}, {1, 8, 2048, KV4_SHARES}, {1, 4, 1800, KV4_SHARES}, {1, 1, 1700, KV4_SHARES},
        {2, 8, 1701, KV4_WHOLE8}, {8, 8, 2001, KV4_WHOLE8}, {8, 8, 2601, KV4_SHARES}, {16, 8, 2601, KV4_WHOLE8}, {16, 8, 6001, KV4_SHARES},
        {32, 8, 6001, KV4_WHOLE8}, {32, 8, 6145, KV4_SHARES}, {33, 8, 4097, KV4_WHOLE4}, {33, 8, 4609, KV4_SHARES}, {64, 8, 4097, KV4_WHOLE4},
        {32, 8, 32768, KV4_SHARES}, {203, 4, 1501, KV4_WHOLE4}, {1, 128, 2900, KV4_WHOLE8}, {1, 300, 4000, KV4_WHOLE4}, {65535, 8, 100, KV4_WHOLE4}};
    for (auto &w : of) CHECK(kv4_decode_form(w.B, w.Hkv, w.max_ctx) == w.form, "%d rows, %d heads, %d tokens: %d", w.B, w.Hkv, w.max_ctx, kv4_decode_form(w.B, w.Hkv, w.max_ctx));
}

int main() {
    decode_forms();
    if (fails) { std::printf("%d checks failed\n", fails); return 1; }
    std::printf("forms ok\n");
    return 0;
}
