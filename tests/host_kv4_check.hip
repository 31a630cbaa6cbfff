// Host-side check of the rules by which launches over a 4-bit cache take their forms (no GPU call), at sizes where the forms were
// measured and at those that GPU tests are about.  Built against the library and run by tests/test_host_kv4_forms.py.
#include <algorithm>
#include <cstdio>
#include <vector>

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

// The decode launches that GPU tests are about: the form, the pieces of the longest row (by the tokens of all rows) or the tiles of 32
// tokens that a wave takes at most (more than 32: block ids are asked for a second time).
static void tested_decode() {
    struct { int B, Hkv, max_ctx, tokens, longest; Kv4DecodeForm form; int least_pieces, least_tiles; } of[] = {
        {3, 2, 32768, 30007, 30001, KV4_SHARES, 9, 1}, {1, 4, 20001, 20001, 20001, KV4_SHARES, 9, 1},
        {70, 4, 4601, 6947, 4601, KV4_WHOLE4, 1, 33}, {70, 4, 4608, 6954, 4608, KV4_WHOLE4, 1, 33},
        {8, 16, 17101, 136108, 17101, KV4_SHARES, 2, 33}, {70, 4, 701, 24000, 701, KV4_WHOLE4, 1, 1},
        {2, 4, 1501, 1522, 1501, KV4_WHOLE8, 1, 1}, {65, 4, 1501, 2845, 1501, KV4_WHOLE4, 1, 1}, {2, 4, 9000, 5022, 5001, KV4_SHARES, 2, 1}, {1, 4, 9000, 301, 301, KV4_SHARES, 0, 1}};
    for (auto &w : of) {
        CHECK(kv4_decode_form(w.B, w.Hkv, w.max_ctx) == w.form, "%d rows of up to %d", w.B, w.max_ctx);
        const int units = (w.tokens + 127) / 128, wgs = std::max(1, std::min(512 / w.Hkv, units / kv4_least_share(w.max_ctx))), share = units / wgs;
        const int pieces = w.form == KV4_SHARES ? (w.longest + 127) / 128 / (share + 1) : 1, tiles = w.form == KV4_SHARES ? share : ((w.longest + 31) / 32 + 3) / 4;
        CHECK(pieces >= w.least_pieces && tiles >= w.least_tiles, "%d rows of up to %d: %d pieces, %d tiles a wave", w.B, w.max_ctx, pieces, tiles);
    }
}

// Prompts
static void prompt_forms() {
    struct { int Hq, Hkv, hd; std::vector<int> lens, starts; int cols, least_cut, most_cut; bool fold; } of[] = {
        {32, 8, 128, {19}, {6005}, 128, 9, 64, false}, {16, 4, 64, {7, 19}, {9000, 6005}, 128, 9, 64, false},
        {32, 8, 128, {2048}, {0}, 128, 1, 1, true}, {9, 3, 128, {2100, 1900}, {0, 0}, 128, 1, 1, true}, {12, 3, 64, {2100, 1900}, {0, 0}, 128, 1, 1, true},
        {128, 8, 128, {2041, 30}, {0, 3000}, 256, 1, 8, false}, {128, 8, 128, {2041}, {0}, 256, 1, 1, false},
        {8, 4, 64, {200}, {0}, 128, 1, 1, false}, {8, 4, 128, {200}, {0}, 128, 1, 1, false}, {8, 4, 64, {5, 3}, {5000, 40}, 128, 2, 64, false}, {8, 4, 128, {5, 3}, {5000, 40}, 128, 2, 64, false}};
    for (auto &w : of) {
        Kv4PromptArgs a{};
        a.Hq = w.Hq, a.Hkv = w.Hkv, a.hd = w.hd;
        a.seq.n_req = (int)w.lens.size();
        for (size_t r = 0; r < w.lens.size(); ++r) a.seq.cu[r + 1] = a.seq.cu[r] + w.lens[r], a.seq.start[r] = w.starts[r];
        const Kv4PromptPlan p = kv4_prompt_plan(a);
        int most = 0;
        for (size_t r = 0; r < w.lens.size(); ++r) most = std::max(most, a.cut[r]);
        CHECK(p.cols == w.cols && most >= w.least_cut && most <= w.most_cut && (a.fold > 0) == w.fold, "%d rows of %d/%d heads of %d: %d columns, cut in %d, fold %d, %d workgroups", a.seq.cu[a.seq.n_req], w.Hq, w.Hkv, w.hd, p.cols, most, a.fold, p.n * w.Hkv);
    }
}

int main() {
    decode_forms();
    tested_decode();
    prompt_forms();
    if (fails) { std::printf("%d checks failed\n", fails); return 1; }
    std::printf("forms ok\n");
    return 0;
}
