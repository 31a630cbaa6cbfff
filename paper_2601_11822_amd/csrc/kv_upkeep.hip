// The bf16 paged cache's upkeep on the GPU: block tables and slots of a step's new tokens from the requests' lengths (plan), the
// tokens' rotation and write (store), and the move of an accepted path behind the cached tokens (compact).
#include <algorithm>

#include "kernels.h"

namespace {

// ---------------------------------------------------------------------------------------------
// Plan.  With n_b new tokens of request b behind len_b cached ones and held_b blocks in its table:
//   need_b = max(0, ceil((len_b + n_b) / 16) - held_b),   cu = exclusive sums of n,   first = exclusive sums of need,
//   the k-th new block of all is free[n_free - 1 - k],    slot of token t of request b = 16 * table_b[t / 16] + t % 16.
// Every workgroup forms the sums over all requests itself, then writes what belongs to its requests (blockIdx.x) and, of long runs,
// to its share of their rows (blockIdx.y).  What a call reads and writes in place (held, n_free) the last workgroup to have read
// everything writes: a ticket counts them and is zero again behind the launch.
// Bound by latency: lengths, then the sums, then held blocks' ids.  64 trees of 16 rows 7.2 us, 1000 runs of up to 63 rows 6.2.
// ---------------------------------------------------------------------------------------------
constexpr int PLAN_REQS = 64, PLAN_WAVES = 16;   // requests and waves of a workgroup

// Sums that stop at 2^32 - 1: of terms of up to 2^31 - 1, a sum is right, or more than any bound.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false); }
// inclusive sums of a row of 16 lanes, by lane moves (1, 2, 4, 8 to the right, zeros from outside)
__device__ __forceinline__ uint32_t row_sums(uint32_t x) {
    x = add_sat(x, moved<0x111, 0xf>(x));
    x = add_sat(x, moved<0x112, 0xf>(x));
    x = add_sat(x, moved<0x114, 0xf>(x));
    return add_sat(x, moved<0x118, 0xf>(x));
}
// and of the wave: lane 15 of a row to the next one (rows 1 and 3), lane 31 to the upper half
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
    x = row_sums(x);
    x = add_sat(x, moved<0x142, 0xa>(x));
    return add_sat(x, moved<0x143, 0xc>(x));
}

__global__ __launch_bounds__(64 * PLAN_WAVES) void kv_plan_kernel(KvPlanArgs a) {
    constexpr int T = 64 * PLAN_WAVES, K = PLAN_REQS / PLAN_WAVES;
    __shared__ uint32_t s_n[PLAN_WAVES], s_need[PLAN_WAVES];
    __shared__ int s_row[PLAN_REQS], s_first[PLAN_REQS], s_len[PLAN_REQS], s_new[PLAN_REQS], s_held[PLAN_REQS], s_more[PLAN_REQS];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int r0 = blockIdx.x * PLAN_REQS, mine = min(PLAN_REQS, a.B - r0);
    const bool first_y = blockIdx.y == 0;
    if (tid == 0) s_bad = 0;
    const int given = *a.n_free, n_free = min(max(given, 0), a.free_cap);

    // sums over the requests, T at a time
    uint32_t tot_n = 0, tot_need = 0;
    int bad = 0, held_mine = 0, need_mine = 0;   // of request tid
    for (int b0 = 0; b0 < a.B; b0 += T) {
        const int b = b0 + tid;
        int n = 0, need = 0, len = -1, held = 0;
        if (b < a.B) {
            len = a.lens[b], held = a.held[b], n = a.n_new[b];
            const int64_t end = (int64_t)len + n;
            if (len == -1) n = 0;
            else if (len < 0 || n < 0 || held < 0 || (a.parents && n > a.parent_stride)) bad |= RS_FLAG_LENGTHS, n = 0;
            else if (held > a.max_blk || (int64_t)len > 16ll * held || end > 16ll * a.max_blk) bad |= 2, n = 0;
            else need = max((int)((end + 15) >> 4) - held, 0);
        }
        if (b0 == 0) held_mine = held, need_mine = need;
        const uint32_t x = wave_sums(n), y = wave_sums(need);
        if (b0 > 0) __syncthreads();   // the sums of those before have been read
        if (lane == 63) s_n[wave] = x, s_need[wave] = y;
        __syncthreads();
        const uint32_t xs = row_sums(s_n[lane & 15]), ys = row_sums(s_need[lane & 15]);   // of the waves
        const uint32_t xw = wave > 0 ? __builtin_amdgcn_readlane(xs, wave - 1) : 0, yw = wave > 0 ? __builtin_amdgcn_readlane(ys, wave - 1) : 0;
        const int i = b - r0;
        if (i >= 0 && i < mine) {
            s_row[i] = add_sat(tot_n, add_sat(xw, x)) - n, s_first[i] = add_sat(tot_need, add_sat(yw, y)) - need;   // (looked at only if the totals are right)
            s_len[i] = len, s_new[i] = n, s_held[i] = held, s_more[i] = need;
        }
        tot_n = add_sat(tot_n, __builtin_amdgcn_readlane(xs, 15));
        tot_need = add_sat(tot_need, __builtin_amdgcn_readlane(ys, 15));
    }
    if (bad) atomicOr(&s_bad, bad);
    asm volatile("" ::"v"(given));   // has been read
    __syncthreads();
    // this workgroup's sums are formed: once all have theirs, nobody reads held and n_free any more
    const int wgs = gridDim.x * gridDim.y;
    int arrived = 0;
    if (tid == 0 && wgs > 1) arrived = atomicAdd(a.ticket, 1);
    bad = s_bad;
    if (!bad && tot_n > (uint32_t)a.max_rows) bad = RS_FLAG_LENGTHS;
    if (!bad && tot_need > (uint32_t)n_free) bad = RS_FLAG_NO_BLOCKS;
    if (first_y) {
        for (int i = tid; i < mine; i += T) a.cu_rows[r0 + i] = bad ? 0 : s_row[i];
        if (r0 + mine == a.B && tid == 0) a.cu_rows[a.B] = bad ? 0 : (int)tot_n;
    }
    if (!bad) {
        auto source = [&](int i, int j) -> const int32_t * {   // where the id of a request's block j stands
            return j < s_held[i] ? a.tables + (size_t)(r0 + i) * a.max_blk + j : a.free_ids + n_free - 1 - (s_first[i] + j - s_held[i]);
        };
        auto slot_of = [&](int id, int token) {
            if ((unsigned)id < (unsigned)a.n_blocks) return 16 * id + (token & 15);
            atomicOr(a.err_flag, 2);
            return -1;
        };
        // A wave takes up to K requests, a lane a token of each, with everything asked for at once; where there are fewer requests than waves
        // several waves share one.
        const int sub = mine >= PLAN_WAVES ? 1 : PLAN_WAVES / mine, step = PLAN_WAVES / sub, part = wave % sub + sub * blockIdx.y, parts = sub * gridDim.y;
        int id[K], fresh[K], up[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = wave / sub + k * step, j = lane + 64 * part;
            id[k] = fresh[k] = 0, up[k] = -1;
            if (i >= mine) continue;
            if (j < s_new[i]) id[k] = *source(i, (s_len[i] + j) >> 4);
            if (j < s_more[i]) fresh[k] = *source(i, s_held[i] + j);
            if (a.parents && j < s_new[i]) up[k] = a.parents[(size_t)(r0 + i) * a.parent_stride + j];
        }
        // Trees: a lane's ancestors by doubling: after k steps `mask` holds 2^k of them and `up` is the one behind; the requests' steps in turn, so
        // that one's exchange is under way beside another's.
        uint64_t mask[K];
        if (a.parents) {
            bool some = false;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (up[k] < -1 || up[k] >= lane) {
                    atomicOr(a.err_flag, RS_FLAG_LENGTHS);
                    up[k] = -1;
                }
                mask[k] = 1ull << lane;
                some = some || up[k] >= 0;
            }
            while (__any(some)) {
                some = false;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const uint64_t m = __shfl(mask[k], up[k] & 63, 64);
                    const int u = __shfl(up[k], up[k] & 63, 64);
                    if (up[k] >= 0) mask[k] |= m, up[k] = u;
                    some = some || up[k] >= 0;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = wave / sub + k * step;
            if (i >= mine) continue;   // (uniform)
            const int n = s_new[i], row = s_row[i], len = s_len[i], held = s_held[i], more = s_more[i];
            int32_t *tab = a.tables + (size_t)(r0 + i) * a.max_blk + held;
            const int j0 = lane + 64 * part;
            if (j0 < more) tab[j0] = fresh[k];
            for (int j = j0 + 64 * parts; j < more; j += 64 * parts) tab[j] = *source(i, held + j);
            if (j0 < n) {
                a.positions[row + j0] = len + (a.parents ? __popcll(mask[k]) - 1 : j0);
                a.slots[row + j0] = slot_of(id[k], len + j0);
                if (a.masks) a.masks[row + j0] = mask[k];
            }
            for (int j = j0 + 64 * parts; j < n; j += 64 * parts) {   // (chains alone: a tree has no more than 64 tokens)
                a.positions[row + j] = len + j;
                a.slots[row + j] = slot_of(*source(i, (len + j) >> 4), len + j);
            }
        }
    }
    if (tid == 0) s_last = wgs == 1 || arrived == wgs - 1;
    __syncthreads();
    if (!s_last) return;
    if (tid < a.B) a.held_out[tid] = bad ? held_mine : held_mine + need_mine;
    for (int b = tid + T; b < a.B; b += T) {
        const int len = a.lens[b], held = a.held[b], n = a.n_new[b];
        a.held_out[b] = bad || len == -1 ? held : max((int)(((int64_t)len + n + 15) >> 4), held);
    }
    if (tid == 0) {
        *a.n_free_out = bad ? given : n_free - (int)tot_need;
        *a.ticket = 0;
        if (bad) atomicOr(a.err_flag, bad);
    }
}

// ---------------------------------------------------------------------------------------------
// Store.  Pair i (dims i and i + hd/2) of a query or key head turns by the angle position * base^(-2i/hd), the position being the row's on
// the pair's axis; cos and sin come from the table that was formed in float64.  Memory bound: q, k and v are read once and written once.
// Workgroups for kv heads (first, as they have the longer way), then for the query heads of 16 rows (rows x 8-dim chunks by lane, the angles in
// registers for all heads).  A token's key is 16-byte pieces of its block and its value single elements, so the rows that share a block are
// written together: the wave of the kv_rows rows among which a run of rows with the same block begins writes all of that run.
// 512 rows of the 8B heads in runs of 8: 7.5 us; 16444 rows of four prompts on three axes 86 us, 4.7 TB/s; a copy of 2 GiB reaches 4.9.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int pair_axis(const KvStoreArgs &a, int pair) { return (int)(a.axis[pair >> 5] >> (2 * (pair & 31)) & 3); }

struct Positions {   // of a row, on each axis
    int p[RS_AXES];
    __device__ __forceinline__ Positions at(int lane) const {
        Positions r;
#pragma unroll
        for (int x = 0; x < RS_AXES; ++x) r.p[x] = __shfl(p[x], lane, 64);
        return r;
    }
};
__device__ __forceinline__ Positions positions_of(const KvStoreArgs &a, int row) {
    Positions r;
#pragma unroll
    for (int x = 0; x < RS_AXES; ++x) r.p[x] = x < a.n_axes ? a.positions[(size_t)x * a.max_rows + row] : 0;
    return r;
}
__device__ __forceinline__ bool in_table(const KvStoreArgs &a, const Positions &r) {
    bool ok = true;
#pragma unroll
    for (int x = 0; x < RS_AXES; ++x) ok = ok && (unsigned)r.p[x] < (unsigned)a.max_pos;
    return ok;
}
// cos and sin of the 8 pairs from `pair` on
__device__ __forceinline__ void angles(const KvStoreArgs &a, const Positions &r, int pair, CosSin cs[8]) {
    const int half = a.hd >> 1;
    const CosSin *t = a.table + pair;
    if (a.n_axes == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) cs[i] = t[(size_t)r.p[0] * half + i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int x = pair_axis(a, pair + i);
        cs[i] = t[(size_t)(x == 0 ? r.p[0] : x == 1 ? r.p[1] : x == 2 ? r.p[2] : r.p[3]) * half + i];
    }
}
__device__ __forceinline__ void turn(const CosSin cs[8], bf16x8 &lo, bf16x8 &hi) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x0 = (float)lo[i], x1 = (float)hi[i];
        lo[i] = (bf16_t)(x0 * cs[i].c - x1 * cs[i].s);
        hi[i] = (bf16_t)(x1 * cs[i].c + x0 * cs[i].s);
    }
}

// Rows of a wave of the kv heads.  Of few rows four, so that short runs are not written one after the other by few waves; of many 16, as three waves in four would
// only look for the beginning of a run.  us with 4 / 16, 8B heads: 64 single rows 10.3 / 31.7, 512 rows in runs of 8 8.8 / 12.6, 2048 in runs of 8 21.0 / 18.9,
// in one run 20.0 / 11.6; 8/2 heads, 4096 rows in runs of 8 13.3 / 14.0, in one run 11.6 / 7.7.
constexpr int STORE_SHORT = 2048;

typedef uint32_t u32x4_s __attribute__((ext_vector_type(4)));
template <bool PAST> __device__ __forceinline__ bf16x8 ld_row(const bf16_t *p) { return PAST ? ld_bf16x8_stream(p) : ld_bf16x8(p); }
template <bool PAST> __device__ __forceinline__ void st_row(bf16_t *p, bf16x8 v) {
    if (PAST) __builtin_nontemporal_store(v, (bf16x8 *)p);
    else st_bf16x8(p, v);
}

// PAST: rows of so many bytes that they are read and written past the caches (16444 rows of the 8B heads, in us: 97; only the loads 97, only the
// stores 91, both 83; with the parts of a row in workgroups far apart, so that its angles are fetched again, 108).
template <int HD, bool PAST>
__global__ __launch_bounds__(256) void kv_store_kernel(KvStoreArgs a, int kv_groups, int kv_parts, int q_parts) {
    constexpr int C = HD / 16;   // 8-dim chunks of half a head
    constexpr int BLK = 16 * HD, PL = HD / 8;   // PL: places of a lane's V
    constexpr int ROUNDS = 16 * C / 64;   // of items (row, 8 pairs) of a key block
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int rows = a.n_rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
    const int kv_rows = rows > STORE_SHORT ? 16 : 4;   // (of the rows there are: the bound may be far above them)
    if ((int)blockIdx.x >= kv_groups * kv_parts) {
        // a thread: 8 pairs of a row, in every second one of 8 heads
        const int at = blockIdx.x - kv_groups * kv_parts, row0 = 16 * (at / q_parts), h0 = at % q_parts * 8;
        for (int it = tid; it < 16 * C * 2; it += 256) {
            const int c = it % C, row = row0 + it / C % 16, first = h0 + it / (16 * C);
            if (row >= rows) continue;
            const bf16_t *p = a.qkv + (size_t)row * a.row_stride + 8 * c;
            const Positions r = positions_of(a, row);
            bf16x8 lo[4], hi[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)   // all asked for before one is written (queries in place are the thread's own)
                if (first + 2 * k < a.Hq) lo[k] = ld_row<PAST>(p + (first + 2 * k) * HD), hi[k] = ld_row<PAST>(p + (first + 2 * k) * HD + HD / 2);
            if (!in_table(a, r)) {
                atomicOr(a.err_flag, 1);
                continue;
            }
            if (!a.q_out) continue;
            CosSin cs[8];
            angles(a, r, 8 * c, cs);
            bf16_t *q = a.q_out + (size_t)row * a.q_stride + 8 * c;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (first + 2 * k < a.Hq) {
                    turn(cs, lo[k], hi[k]);
                    st_row<PAST>(q + (first + 2 * k) * HD, lo[k]);
                    st_row<PAST>(q + (first + 2 * k) * HD + HD / 2, hi[k]);
                }
        }
        return;
    }
    const int row0 = kv_rows * ((int)blockIdx.x / kv_parts), kvh = (int)blockIdx.x % kv_parts * 4 + wave;
    if (row0 >= rows || kvh >= a.Hkv) return;
    // lane l: slot and positions of row row0 - 1 + l, and the slot's block, -1: not a row, or none
    auto block_at = [&](int slot) { return slot < 0 || (slot >> 4) >= a.n_blocks ? -1 : slot >> 4; };
    const int r_l = row0 - 1 + lane;
    const bool is_row = lane < kv_rows + 16 && r_l >= 0 && r_l < rows;
    const int sl = is_row ? a.slots[r_l] : -1, bl = block_at(sl);
    const Positions ps = positions_of(a, is_row ? r_l : row0);
    const bool mine = lane > 0 && lane <= kv_rows;
    if (mine && bl < 0 && sl != -1) atomicOr(a.err_flag, 2);
    const int prev = __shfl_up(bl, 1, 64);
    uint64_t starts = __ballot(mine && bl >= 0 && bl != prev);
    while (starts) {
        const int l0 = __ffsll((unsigned long long)starts) - 1;
        starts &= starts - 1;
        const int blk = __builtin_amdgcn_readlane(bl, l0);
        int first = row0 - 1 + l0;
        // lane l < 16: slot and positions of row first + l
        int my = __shfl(sl, (l0 + lane) & 63, 64);
        Positions pos = ps.at((l0 + lane) & 63);
        if (lane >= 16) my = -1;
        for (;;) {   // 16 rows at a time: a block has no more places, but slots may name one twice
            const uint64_t same = __ballot(block_at(my) == blk);
            const int n = __ffsll((unsigned long long)~same) - 1;   // rows of this block from `first` on
            if (n == 0) break;
            bf16_t *kd = a.k_pool + ((size_t)blk * a.Hkv + kvh) * BLK, *vd = a.v_pool + ((size_t)blk * a.Hkv + kvh) * BLK;
            const bf16_t *src = a.qkv + (size_t)first * a.row_stride + (size_t)(a.Hq + kvh) * HD;
            // whether the places are consecutive, and every position is in the table (a bad one is reported by the queries' workgroups)
            const int t0 = __builtin_amdgcn_readfirstlane(my) & 15, inside = in_table(a, pos);
            const bool plain = !__any(lane < n && (!inside || (my & 15) != t0 + lane));

            // V, where the places are consecutive: a lane has two dims of all rows (head_dim 64: a half-wave eight places)
            const int dp = lane % (HD / 2), u0 = lane / (HD / 2) * 8;
            uint32_t w[PL];
            if (plain) {
#pragma unroll
                for (int u = 0; u < PL; ++u) {
                    const int r = u0 + u - t0;
                    w[u] = r >= 0 && r < n ? *(const uint32_t *)(src + (size_t)r * a.row_stride + a.Hkv * HD + 2 * dp) : 0u;
                }
            }
            // K: items (row, 8 pairs), everything asked for at once
            {
                bf16x8 lo[ROUNDS], hi[ROUNDS];
                CosSin cs[ROUNDS][8];
                int place[ROUNDS];
#pragma unroll
                for (int k = 0; k < ROUNDS; ++k) {
                    const int it = 64 * k + lane, c = it % C, r = it / C;
                    const Positions at = pos.at(r);
                    const int slot = __shfl(my, r, 64), ok = __shfl(inside, r, 64);
                    place[k] = r < n && ok ? slot & 15 : -1;
                    if (place[k] >= 0) {
                        const bf16_t *p = src + (size_t)r * a.row_stride + 8 * c;
                        lo[k] = ld_row<PAST>(p), hi[k] = ld_row<PAST>(p + HD / 2);
                        angles(a, at, 8 * c, cs[k]);
                    }
                }
#pragma unroll
                for (int k = 0; k < ROUNDS; ++k) {
                    const int c = (64 * k + lane) % C;
                    if (place[k] < 0) continue;
                    turn(cs[k], lo[k], hi[k]);
                    st_bf16x8(kd + kpool_chunk_offset(place[k], 8 * c), lo[k]);
                    st_bf16x8(kd + kpool_chunk_offset(place[k], HD / 2 + 8 * c), hi[k]);
                }
            }
            if (plain) {
                uint32_t ev[PL / 2], od[PL / 2];
#pragma unroll
                for (int j = 0; j < PL / 2; ++j) {
                    ev[j] = (w[2 * j] & 0xffffu) | (w[2 * j + 1] << 16);
                    od[j] = (w[2 * j] >> 16) | (w[2 * j + 1] & 0xffff0000u);
                }
                bf16_t *dst = vd + 2 * dp * 16 + u0;
                if (n == 16) {
#pragma unroll
                    for (int j = 0; j < PL / 8; ++j) {
                        *(u32x4_s *)(dst + 8 * j) = u32x4_s{ev[4 * j], ev[4 * j + 1], ev[4 * j + 2], ev[4 * j + 3]};
                        *(u32x4_s *)(dst + 16 + 8 * j) = u32x4_s{od[4 * j], od[4 * j + 1], od[4 * j + 2], od[4 * j + 3]};
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < PL / 2; ++j) {   // pairs of places; at the ends one alone, so that others are not touched
                        const int lo = u0 + 2 * j - t0;
                        const bool has_lo = lo >= 0 && lo < n, has_hi = lo + 1 >= 0 && lo + 1 < n;
                        if (has_lo && has_hi) {
                            *(uint32_t *)(dst + 2 * j) = ev[j];
                            *(uint32_t *)(dst + 16 + 2 * j) = od[j];
                        } else if (has_lo || has_hi) {
                            const int at = 2 * j + (has_hi ? 1 : 0), shift = has_hi ? 16 : 0;
                            *(uint16_t *)(dst + at) = (uint16_t)(ev[j] >> shift);
                            *(uint16_t *)(dst + 16 + at) = (uint16_t)(od[j] >> shift);
                        }
                    }
                }
            } else {
                for (int i0 = 0; i0 < n * HD; i0 += 64) {   // rows in any order: element by element
                    const int it = i0 + lane, r = it % n, d = it / n, t = __shfl(my, r, 64) & 15, ok = __shfl(inside, r, 64);
                    if (it < n * HD && ok) vd[d * 16 + t] = src[(size_t)r * a.row_stride + a.Hkv * HD + d];
                }
            }
            if (n < 16) break;
            first += 16;
            my = lane < 16 && first + lane < rows ? a.slots[first + lane] : -1;
            pos = positions_of(a, min(first + lane, rows - 1));
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Compact.  Token ctx + keep[i] of a request takes the place of token ctx + i, in every layer.  keep ascends, so a token moves to a place
// before its own and before those of all that come later: a wave takes a (request, layer, kv head) for itself, eight tokens at a time, and has
// read all of them before it writes one.  Latency bound: lengths, indices, block ids, tokens.  32 layers of one request's path 3.2 us of the GPU, 16 layers
// of 64 requests' 8.3.
// ---------------------------------------------------------------------------------------------
template <int HD>
__global__ __launch_bounds__(256) void kv_compact_kernel(KvCompactArgs a) {
    constexpr int N = 8, KR = N * HD / 8 / 64, VR = N * HD / 64;   // tokens at a time; 16-byte pieces and single elements of a lane
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, b = blockIdx.y, layer = blockIdx.z;
    const int kvh = blockIdx.x * 4 + wave;
    if (kvh >= a.Hkv) return;
    const int ctx = a.ctx_lens[b], n = a.keep_lens[b];
    const int k = lane < a.keep_stride ? a.keep[(size_t)b * a.keep_stride + lane] : 0;
    if (ctx == -1 || n == 0) return;
    if (ctx < 0 || n < 0 || n > a.keep_stride) {
        if (lane == 0) atomicOr(a.err_flag, RS_FLAG_LENGTHS);
        return;
    }
    const int32_t *tab = a.tables + (size_t)b * a.max_blk;
    const int before = __shfl_up(k, 1, 64);
    const bool mine = lane < n;
    if (__any(mine && (k <= (lane > 0 ? before : -1) || k >= 64))) {
        if (lane == 0) atomicOr(a.err_flag, RS_FLAG_LENGTHS);
        return;
    }
    int src = -1, dst = -1;
    if (mine && (int64_t)ctx + k < 16ll * a.max_blk) src = tab[(ctx + k) >> 4], dst = tab[(ctx + lane) >> 4];
    if (__any(mine && ((unsigned)src >= (unsigned)a.n_blocks || (unsigned)dst >= (unsigned)a.n_blocks))) {
        if (lane == 0) atomicOr(a.err_flag, 2);
        return;
    }
    const int ps = (ctx + k) & 15, pd = (ctx + lane) & 15;
    const int stay = __ffsll((unsigned long long)__ballot(mine && k != lane)) - 1;   // the first that moves
    if (stay < 0) return;
    bf16_t *kp = a.k_pool + layer * a.layer_stride + (size_t)kvh * 16 * HD, *vp = a.v_pool + layer * a.layer_stride + (size_t)kvh * 16 * HD;
    const size_t blk = (size_t)a.Hkv * 16 * HD;
    for (int i0 = stay; i0 < n; i0 += N) {
        // item e of a lane: token i0 + e % N, so that neighbouring lanes have neighbouring places
        const int i = min(i0 + lane % N, n - 1);
        const bool there = i0 + lane % N < n;
        const size_t s0 = __shfl(src, i, 64) * blk, d0 = __shfl(dst, i, 64) * blk;
        const int s_at = __shfl(ps, i, 64), d_at = __shfl(pd, i, 64);
        bf16x8 kk[KR];
        bf16_t vv[VR];
#pragma unroll
        for (int e = 0; e < KR; ++e) kk[e] = ld_bf16x8(kp + s0 + kpool_chunk_offset(s_at, 8 * (8 * e + lane / N)));
#pragma unroll
        for (int e = 0; e < VR; ++e) vv[e] = vp[s0 + 16 * (8 * e + lane / N) + s_at];
        if (there) {
#pragma unroll
            for (int e = 0; e < KR; ++e) st_bf16x8(kp + d0 + kpool_chunk_offset(d_at, 8 * (8 * e + lane / N)), kk[e]);
#pragma unroll
            for (int e = 0; e < VR; ++e) vp[d0 + 16 * (8 * e + lane / N) + d_at] = vv[e];
        }
    }
}

}  // namespace

static int plan_groups(const KvPlanArgs &a) { return (a.B + PLAN_REQS - 1) / PLAN_REQS; }
// long runs: some 4096 rows for each workgroup
int kv_plan_shares(const KvPlanArgs &a) { return a.parents ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(((int64_t)a.max_rows / plan_groups(a) + 4095) / 4096, 64)); }

void launch_kv_plan(hipStream_t st, const KvPlanArgs &a) {
    hipLaunchKernelGGL(kv_plan_kernel, dim3(plan_groups(a), kv_plan_shares(a)), dim3(64 * PLAN_WAVES), 0, st, a);
}

// What is read and written, against the caches.  One run of rows / and attention under a window of 256 over the queries, in us through the caches and past
// them: 8B heads, 2048 rows (50 MB) 11.0 / 33.9 and 11.6 / 35.7, 4096 23.5 / 65.0 and 21.6 / 64.2, 16384 90 / 234 and 84 / 227; 64/8 heads, 2048 (84 MB)
// 18.4 / 59.8 and 19.5 / 60.7; 8/2 heads, 4096 (25 MB) 7.5 / 26.2 and 7.7 / 27.4, 16384 (101 MB) 26.9 / 70.3 and 23.0 / 68.6.
bool kv_store_past(const KvStoreArgs &a) { return (int64_t)a.max_rows * (a.Hq + 2 * a.Hkv) * a.hd * 4 > 80ll << 20; }

void launch_kv_store(hipStream_t st, const KvStoreArgs &a) {
    const int kv_groups = std::max((a.max_rows + 15) / 16, (std::min(a.max_rows, STORE_SHORT) + 3) / 4), kv_parts = (a.Hkv + 3) / 4, q_parts = (a.Hq + 7) / 8;
    const dim3 grid(kv_groups * kv_parts + (a.max_rows + 15) / 16 * q_parts);
    auto launch = [&](auto *kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, kv_groups, kv_parts, q_parts); };
    const bool past = kv_store_past(a);
    if (a.hd == 128) past ? launch(kv_store_kernel<128, true>) : launch(kv_store_kernel<128, false>);
    else past ? launch(kv_store_kernel<64, true>) : launch(kv_store_kernel<64, false>);
}

void launch_kv_compact(hipStream_t st, const KvCompactArgs &a) {
    const dim3 grid((a.Hkv + 3) / 4, a.B, a.n_layers);
    if (a.hd == 128) hipLaunchKernelGGL(kv_compact_kernel<128>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv_compact_kernel<64>, grid, dim3(256), 0, st, a);
}
