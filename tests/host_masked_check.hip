// Host-side check of the rules by which windowed and tree attention take their forms (no GPU call), at sizes where the forms were measured
// and at those that GPU tests are about.  Built against the library and run by tests/test_host_masked_forms.py.
#include <algorithm>
#include <cstdio>
#include <vector>

#include "../paper_2601_11822_amd/csrc/kernels.h"

static int fails = 0;
#define CHECK(c, ...) do { if (!(c)) { if (fails++ < 10) { std::printf("FAIL %s:%d: ", __FILE__, __LINE__); std::printf(__VA_ARGS__); std::printf("\n"); } } } while (0)

static MaskedAttnArgs heads(int Hq, int Hkv) {
    MaskedAttnArgs a{};
    a.Hq = Hq, a.Hkv = Hkv, a.hd = 128;
    return a;
}
static void check(const char *what, int i, MaskedAttnArgs &a, MaskedKind kind, int cut) {
    const MaskedForm f = masked_form(a);
    CHECK(f.kind == kind && a.cut == cut, "%s %d: form %d, %d pieces", what, i, f.kind, a.cut);
    const int64_t pieces = (int64_t)a.n_units * a.Hkv * a.cut;
    CHECK(a.cut == 1 || (pieces <= MASKED_PIECES && a.cut <= MASKED_MAX_CUT), "%s %d: %lld pieces", what, i, (long long)pieces);
    CHECK(a.unit_rows >= 1 && a.unit_rows * (a.Hq / a.Hkv) <= MASKED_COLS, "%s %d: units of %d rows", what, i, a.unit_rows);
    CHECK((kind == MASKED_FEW4 || kind == MASKED_FEW8) == (a.unit_rows == 32 / (a.Hq / a.Hkv)), "%s %d: units of %d rows", what, i, a.unit_rows);
}

static void decode_forms() {
    static int32_t lens;
    struct { int Hq, Hkv, B, max_ctx, window, sinks; MaskedKind kind; int cut; } of[] = {
        {32, 8, 1, 4096, 1024, 4, MASKED_FEW8, 8}, {32, 8, 1, 8193, 8192, 4, MASKED_FEW8, 16}, {32, 8, 1, 4097, 4096, 0, MASKED_FEW8, 16}, {32, 8, 1, 4001, 4096, 0, MASKED_FEW8, 8}, {32, 8, 64, 8193, 4096, 4, MASKED_FEW4, 1},
        {32, 8, 32, 8193, 4096, 4, MASKED_FEW8, 1}, {8, 2, 1, 100, 64, 0, MASKED_FEW8, 1}, {16, 1, 1, 1 << 30, 1 << 30, 0, MASKED_FEW8, 16},
        {16, 1, 65535, 2147483632, 2147483647, 2147483647, MASKED_FEW4, 1}, {16, 1, 1, 2147483632, 2147483647, 2147483647, MASKED_FEW8, 16}};
    for (auto &w : of) {
        MaskedAttnArgs a = heads(w.Hq, w.Hkv);
        a.ctx_lens = &lens, a.B = w.B, a.max_ctx = w.max_ctx, a.window = w.window, a.sinks = w.sinks;
        check("decode", int(&w - of), a, w.kind, w.cut);
        CHECK(a.n_units == w.B, "decode %d: %d units", int(&w - of), a.n_units);
    }
}

static void prompt_forms() {
    struct { int Hq, Hkv; std::vector<int> lens, starts; int window, sinks; MaskedKind kind; int cut; } of[] = {
        {32, 8, {100}, {3000}, 2048, 4, MASKED_FEW8, 2}, {32, 8, {512}, {3000}, 2048, 4, MASKED_TEAMS, 2}, {32, 8, {16384}, {0}, 4096, 4, MASKED_WIDE, 1},
        {32, 8, {1024}, {0}, 4096, 0, MASKED_TEAMS, 1}, {32, 8, {2048}, {0}, 4096, 0, MASKED_TEAMS, 1}, {32, 8, {2500}, {0}, 4096, 0, MASKED_WIDE, 1}, {32, 8, {2048}, {0}, 512, 0, MASKED_WIDE, 1},
        {32, 8, {2048}, {4000}, 8192, 0, MASKED_WIDE, 1}, {32, 8, {100, 1600}, {0, 0}, 8192, 0, MASKED_TEAMS, 1}, {64, 8, {1024}, {0}, 4096, 0, MASKED_WIDE, 1}, {32, 8, {300}, {0}, 4096, 0, MASKED_FEW4, 1},
        {32, 8, {37, 0, 1}, {5, 9, 0}, 50, 20, MASKED_FEW8, 1}, {8, 2, {0, 0}, {0, 0}, 50, 20, MASKED_FEW4, 1},
        // what GPU tests are about
        {32, 8, {100}, {3000}, 3000, 5, MASKED_TEAMS, 8}, {64, 16, {160}, {41000}, 2147483647, 0, MASKED_TEAMS, 3},
        {64, 16, {300}, {41000}, 2147483647, 0, MASKED_TEAMS, 1}, {64, 16, {600}, {41000}, 2147483647, 0, MASKED_WIDE, 1},
        {32, 8, {1300, 100}, {0, 20}, 2147483647, 0, MASKED_TEAMS, 1}, {32, 8, {1300, 100}, {0, 20}, 1250, 16, MASKED_TEAMS, 1},
        {32, 8, {600}, {41000}, 2147483647, 0, MASKED_TEAMS, 1}, {32, 8, {1200}, {41000}, 2147483647, 0, MASKED_WIDE, 1}};
    for (auto &w : of) {
        MaskedAttnArgs a = heads(w.Hq, w.Hkv);
        a.window = w.window, a.sinks = w.sinks, a.seq.n_req = (int)w.lens.size();
        for (size_t r = 0; r < w.lens.size(); ++r) a.seq.cu[r + 1] = a.seq.cu[r] + w.lens[r], a.seq.start[r] = w.starts[r];
        if (a.seq.cu[a.seq.n_req] == 0) {
            masked_form(a);
            CHECK(a.n_units == 0, "no rows: %d units", a.n_units);
        } else check("prompt", int(&w - of), a, w.kind, w.cut);
        std::vector<int> units(w.lens.size(), -1);   // each request once, with its units
        int n = 0;
        for (int i = 0; a.n_units && i < a.seq.n_req; ++i) {
            const MaskedRun &r = a.runs[i];
            CHECK(r.req >= 0 && r.req < a.seq.n_req && units[r.req] == -1, "prompt %d: run %d", int(&w - of), i);
            units[r.req] = r.units, n += r.units;
            CHECK(r.start == w.starts[r.req] && r.units == (w.lens[r.req] + a.unit_rows - 1) / a.unit_rows, "prompt %d: run %d", int(&w - of), i);
        }
        CHECK(n == a.n_units, "prompt %d: %d units of %d", int(&w - of), n, a.n_units);
    }
}

// The requests whose rows see least come last: they stand first
static void prompt_order() {
    MaskedAttnArgs a = heads(32, 8);
    const int lens[] = {1500, 100, 2000, 700, 64, 0}, starts[] = {0, 3000, 500, 2000, 9, 4000}, order[] = {4, 0, 2, 3, 1, 5};
    a.window = 4096, a.seq.n_req = 6;
    for (int r = 0; r < 6; ++r) a.seq.cu[r + 1] = a.seq.cu[r] + lens[r], a.seq.start[r] = starts[r];
    masked_form(a);
    for (int i = 0; i < 6; ++i) CHECK(a.runs[i].req == order[i], "place %d: request %d", i, a.runs[i].req);
}

static void tree_forms() {
    static int32_t lens, cu;
    struct { int Hq, Hkv, B, max_draft, max_ctx; MaskedKind kind; int cut; } of[] = {
        {32, 8, 1, 8, 2056, MASKED_FEW8, 8}, {32, 8, 1, 8, 8008, MASKED_FEW8, 16}, {32, 8, 32, 32, 4128, MASKED_TEAMS, 1}, {32, 8, 16, 32, 4128, MASKED_TEAMS, 2}, {32, 8, 4, 32, 4032, MASKED_TEAMS, 8},
        {32, 8, 64, 16, 4112, MASKED_WIDE, 1}, {32, 8, 8, 16, 916, MASKED_FEW8, 2}, {32, 8, 1, 60, 3560, MASKED_FEW8, 4},
        // what GPU tests are about
        {32, 8, 2, 40, 3640, MASKED_TEAMS, 8}, {64, 16, 5, 64, 41064, MASKED_TEAMS, 1}, {64, 16, 9, 64, 41064, MASKED_WIDE, 1},
        {32, 8, 10, 64, 41064, MASKED_TEAMS, 1}, {32, 8, 17, 64, 41064, MASKED_WIDE, 1}, {64, 16, 1, 64, 41064, MASKED_TEAMS, 8}};
    for (auto &w : of) {
        MaskedAttnArgs a = heads(w.Hq, w.Hkv);
        a.ctx_lens = &lens, a.cu_rows = &cu, a.B = w.B, a.max_ctx = w.max_ctx, a.max_draft = w.max_draft, a.max_rows = w.B * w.max_draft;
        check("tree", int(&w - of), a, w.kind, w.cut);
    }
    // the lists of nine short requests under a bound of 9600 tokens, once and ten times: two teams, and one
    for (int times : {1, 10})
        for (auto [Hq, Hkv] : {std::pair{4, 4}, {8, 2}, {9, 3}, {16, 1}, {32, 2}, {64, 4}})
            for (int draft : {33, 64}) {
                MaskedAttnArgs a = heads(Hq, Hkv);
                a.ctx_lens = &lens, a.cu_rows = &cu, a.B = 9 * times, a.max_ctx = 9600, a.max_draft = draft, a.max_rows = 9 * times * draft;
                const MaskedKind kind = masked_form(a).kind;
                CHECK(kind == (a.n_units * Hkv > MASKED_PIECES ? MASKED_WIDE : MASKED_TEAMS), "%d x nine, %d/%d heads, %d rows: form %d", times, Hq, Hkv, draft, kind);
                CHECK(times == 1 || draft == 33 || kind == MASKED_WIDE, "%d/%d heads", Hq, Hkv);
            }
}

int main() {
    decode_forms();
    prompt_forms();
    prompt_order();
    tree_forms();
    std::printf(fails ? "%d failures\n" : "ok\n", fails);
    return fails != 0;
}
