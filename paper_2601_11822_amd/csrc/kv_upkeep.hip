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
// Bound by latency: lengths, then the sums, then held blocks' ids.
// ---------------------------------------------------------------------------------------------
constexpr int PLAN_REQS = 64;   // requests of a workgroup

__global__ __launch_bounds__(256) void kv_plan_kernel(KvPlanArgs a) {
    __shared__ uint32_t s_n[4], s_need[4];
    __shared__ int s_row[PLAN_REQS], s_first[PLAN_REQS], s_len[PLAN_REQS], s_new[PLAN_REQS], s_held[PLAN_REQS], s_more[PLAN_REQS];
    __shared__ int64_t s_tot_n[4], s_tot_need[4];
    __shared__ int s_bad, s_last;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int r0 = blockIdx.x * PLAN_REQS, mine = min(PLAN_REQS, a.B - r0);
    const bool first_y = blockIdx.y == 0;
    if (tid == 0) s_bad = 0;
    const int n_free = min(max(*a.n_free, 0), a.free_cap);

    // sums over the requests, 256 at a time
    uint32_t carry_n = 0, carry_need = 0;
    int bad = 0;
    int64_t tot_n = 0, tot_need = 0;
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int b = b0 + tid;
        int n = 0, need = 0, len = -1, held = 0;
        if (b < a.B) {
            len = a.lens[b], held = a.held[b];
            if (len != -1) {
                n = a.n_new[b];
                const int64_t end = (int64_t)len + n;
                if (len < 0 || n < 0 || held < 0 || (a.parents && n > a.parent_stride)) bad |= RS_FLAG_LENGTHS, n = 0;
                else if (held > a.max_blk || (int64_t)len > 16ll * held || end > 16ll * a.max_blk) bad |= 2, n = 0;
                else need = max((int)((end + 15) >> 4) - held, 0);
            }
        }
        tot_n += n, tot_need += need;
        uint32_t x = n, y = need;   // inclusive sums of the wave
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t xo = __shfl_up(x, o, 64), yo = __shfl_up(y, o, 64);
            if (lane >= o) x += xo, y += yo;
        }
        __syncthreads();   // the sums of the 256 before have been read
        if (lane == 63) s_n[wave] = x, s_need[wave] = y;
        __syncthreads();
        uint32_t row = carry_n + x - n, first = carry_need + y - need;
        for (int w = 0; w < wave; ++w) row += s_n[w], first += s_need[w];
        for (int w = 0; w < 4; ++w) carry_n += s_n[w], carry_need += s_need[w];
        const int i = b - r0;
        if (i >= 0 && i < mine) s_row[i] = row, s_first[i] = first, s_len[i] = len, s_new[i] = n, s_held[i] = held, s_more[i] = need;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        tot_n += __shfl_xor(tot_n, o, 64);
        tot_need += __shfl_xor(tot_need, o, 64);
    }
    if (lane == 0) s_tot_n[wave] = tot_n, s_tot_need[wave] = tot_need;
    if (bad) atomicOr(&s_bad, bad);
    __syncthreads();
    tot_n = s_tot_n[0] + s_tot_n[1] + s_tot_n[2] + s_tot_n[3];
    tot_need = s_tot_need[0] + s_tot_need[1] + s_tot_need[2] + s_tot_need[3];
    bad = s_bad;
    if (!bad && tot_n > a.max_rows) bad = RS_FLAG_LENGTHS;
    if (!bad && tot_need > n_free) bad = RS_FLAG_NO_BLOCKS;
    if (tid == 0) {
        // the sums of this call have been formed by this workgroup: once all have, nobody reads held and n_free any more
        const int wgs = gridDim.x * gridDim.y;
        s_last = wgs == 1 || atomicAdd(a.ticket, 1) == wgs - 1;
    }
    __syncthreads();
    if (s_last) {
        for (int b = tid; b < a.B; b += 256) {
            const int len = a.lens[b], held = a.held[b];
            a.held_out[b] = bad || len == -1 ? held : max((int)(((int64_t)len + a.n_new[b] + 15) >> 4), held);
        }
        if (tid == 0) {
            *a.n_free_out = bad ? *a.n_free : n_free - (int)tot_need;
            *a.ticket = 0;
            if (bad) atomicOr(a.err_flag, bad);
        }
    }
    if (first_y) {
        for (int i = tid; i < mine; i += 256) a.cu_rows[r0 + i] = bad ? 0 : s_row[i];
        if (r0 + mine == a.B && tid == 0) a.cu_rows[a.B] = bad ? 0 : (int)tot_n;
    }
    if (bad) return;
    auto block_of = [&](int i, int j) { return j < s_held[i] ? a.tables[(size_t)(r0 + i) * a.max_blk + j] : a.free_ids[n_free - 1 - (s_first[i] + j - s_held[i])]; };
    auto slot_of = [&](int i, int token) {
        const int id = block_of(i, token >> 4);
        if ((unsigned)id < (unsigned)a.n_blocks) return 16 * id + (token & 15);
        atomicOr(a.err_flag, 2);
        return -1;
    };
    for (int i = wave; i < mine; i += 4) {
        if (first_y)
            for (int j = lane; j < s_more[i]; j += 64) a.tables[(size_t)(r0 + i) * a.max_blk + s_held[i] + j] = a.free_ids[n_free - 1 - (s_first[i] + j)];
        const int n = s_new[i], row = s_row[i], len = s_len[i];
        if (a.parents) {
            // a lane a token; ancestors by doubling: after k steps `mask` holds 2^k of them and `up` is the one behind
            if (!first_y || n == 0) continue;
            int up = lane < n ? a.parents[(size_t)(r0 + i) * a.parent_stride + lane] : -1;
            if (up < -1 || up >= lane) {
                atomicOr(a.err_flag, RS_FLAG_LENGTHS);
                up = -1;
            }
            uint64_t mask = 1ull << lane;
#pragma unroll
            for (int k = 0; k < 6; ++k) {
                const uint64_t m = __shfl(mask, up & 63, 64);
                const int u = __shfl(up, up & 63, 64);
                if (up >= 0) mask |= m, up = u;
            }
            if (lane < n) {
                a.positions[row + lane] = len + __popcll(mask) - 1;
                a.slots[row + lane] = slot_of(i, len + lane);
                if (a.masks) a.masks[row + lane] = mask;
            }
        } else {
            for (int j = lane + 64 * blockIdx.y; j < n; j += 64 * gridDim.y) {
                a.positions[row + j] = len + j;
                a.slots[row + j] = slot_of(i, len + j);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Store.  Pair i (dims i and i + hd/2) of a query or key head turns by the angle position * base^(-2i/hd), the position being the row's on
// the pair's axis; cos and sin come from the table that was formed in float64.  Memory bound: q, k and v are read once and written once.
// Workgroups: of 16 rows the query heads (rows x 8-dim chunks by lane, the angles in registers for all heads), then the kv heads.
// A token's key is 16-byte pieces of its block and its value single elements, so the rows that share a block are written together: the
// workgroup of the 16 rows among which a run of rows with the same block begins writes all of that run.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ int pair_axis(const KvStoreArgs &a, int pair) { return (int)(a.axis[pair >> 5] >> (2 * (pair & 31)) & 3); }

// cos and sin of the 8 pairs from `pair` on of a row; false: a position outside the table
__device__ __forceinline__ bool angles(const KvStoreArgs &a, int row, int pair, CosSin cs[8]) {
    const int half = a.hd >> 1;
    int pos[4];
    bool ok = true;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        pos[x] = x < a.n_axes ? a.positions[(size_t)x * a.max_rows + row] : 0;
        ok = ok && (unsigned)pos[x] < (unsigned)a.max_pos;
    }
    if (!ok) return false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int x = pair_axis(a, pair + i);
        cs[i] = a.table[(size_t)(x == 0 ? pos[0] : x == 1 ? pos[1] : x == 2 ? pos[2] : pos[3]) * half + pair + i];
    }
    return true;
}
__device__ __forceinline__ void turn(const CosSin cs[8], bf16x8 &lo, bf16x8 &hi) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x0 = (float)lo[i], x1 = (float)hi[i];
        lo[i] = (bf16_t)(x0 * cs[i].c - x1 * cs[i].s);
        hi[i] = (bf16_t)(x1 * cs[i].c + x0 * cs[i].s);
    }
}

template <int HD>
__global__ __launch_bounds__(256) void kv_store_kernel(KvStoreArgs a, int n_groups, int q_parts) {
    constexpr int C = HD / 16;   // 8-dim chunks of half a head
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int group = blockIdx.x % n_groups, part = blockIdx.x / n_groups;
    const int rows = a.n_rows ? min(max(*a.n_rows, 0), a.max_rows) : a.max_rows;
    const int row0 = 16 * group;
    if (row0 >= rows) return;
    if (part < q_parts) {
        const int h0 = part * 8, h1 = min(a.Hq, h0 + 8);
        for (int it = tid; it < 16 * C * 2; it += 256) {   // two threads a (row, chunk), every second head each
            const int c = it % C, row = row0 + it / C % 16, first = h0 + it / (16 * C);
            CosSin cs[8];
            if (row >= rows) continue;
            if (!angles(a, row, 8 * c, cs)) {
                atomicOr(a.err_flag, 1);
                continue;
            }
            if (!a.q_out) continue;
            for (int head = first; head < h1; head += 2) {
                const bf16_t *p = a.qkv + (size_t)row * a.row_stride + head * HD + 8 * c;
                bf16_t *q = a.q_out + (size_t)row * a.q_stride + head * HD + 8 * c;
                bf16x8 lo = ld_bf16x8(p), hi = ld_bf16x8(p + HD / 2);
                turn(cs, lo, hi);
                st_bf16x8(q, lo);
                st_bf16x8(q + HD / 2, hi);
            }
        }
        return;
    }
    const int kvh = (part - q_parts) * 4 + wave;
    if (kvh >= a.Hkv) return;
    // lane l < 17: the block of row row0 - 1 + l (-1: not a row, or none)
    auto slot_at = [&](int row) { return row >= 0 && row < rows ? a.slots[row] : -1; };
    auto block_at = [&](int slot) { return slot < 0 || (slot >> 4) >= a.n_blocks ? -1 : slot >> 4; };
    const int r_l = row0 - 1 + lane;
    const int sl = lane < 17 ? slot_at(r_l) : -1, bl = block_at(sl);
    if (lane > 0 && lane < 17 && r_l < rows && bl < 0 && sl != -1) atomicOr(a.err_flag, 2);
    const int prev = __shfl_up(bl, 1, 64);
    uint64_t starts = __ballot(lane > 0 && lane < 17 && bl >= 0 && bl != prev);
    while (starts) {
        const int l0 = __ffsll((unsigned long long)starts) - 1;
        starts &= starts - 1;
        int first = row0 - 1 + l0;
        const int blk = __builtin_amdgcn_readlane(bl, l0);
        for (;;) {   // 16 rows at a time: a block has no more places, but slots may name one twice
            const int my = lane < 16 ? slot_at(first + lane) : -1;
            const uint64_t same = __ballot(lane < 16 && block_at(my) == blk);
            const int n = __ffsll((unsigned long long)~same) - 1;   // rows of this block from `first` on
            if (n == 0) break;
            bf16_t *kd = a.k_pool + ((size_t)blk * a.Hkv + kvh) * 16 * HD, *vd = a.v_pool + ((size_t)blk * a.Hkv + kvh) * 16 * HD;
            for (int i0 = 0; i0 < n * C; i0 += 64) {
                const int it = i0 + lane, c = it % C, row = first + it / C, t = __shfl(my, it / C & 15, 64) & 15;
                CosSin cs[8];
                if (it >= n * C || !angles(a, row, 8 * c, cs)) continue;   // (a bad position is reported by the queries' workgroups)
                const bf16_t *p = a.qkv + (size_t)row * a.row_stride + (size_t)(a.Hq + kvh) * HD + 8 * c;
                bf16x8 lo = ld_bf16x8(p), hi = ld_bf16x8(p + HD / 2);
                turn(cs, lo, hi);
                st_bf16x8(kd + kpool_chunk_offset(t, 8 * c), lo);
                st_bf16x8(kd + kpool_chunk_offset(t, HD / 2 + 8 * c), hi);
            }
            for (int i0 = 0; i0 < n * HD; i0 += 64) {
                const int it = i0 + lane, r = it % n, d = it / n, row = first + r, t = __shfl(my, r, 64) & 15;
                bool ok = it < n * HD;
                for (int x = 0; x < a.n_axes; ++x) ok = ok && (unsigned)a.positions[(size_t)x * a.max_rows + row] < (unsigned)a.max_pos;
                if (ok) vd[d * 16 + t] = a.qkv[(size_t)row * a.row_stride + (size_t)(a.Hq + a.Hkv + kvh) * HD + d];
            }
            if (n < 16) break;
            first += 16;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Compact.  Token ctx + keep[i] of a request takes the place of token ctx + i, in every layer; keep ascends, so that a token moves to
// a place before its own, and all that move are read before one is written.  A workgroup per (request, kv head, layer).
// ---------------------------------------------------------------------------------------------
template <int HD>
__global__ __launch_bounds__(256) void kv_compact_kernel(KvCompactArgs a) {
    __shared__ bf16x8 s_k[64 * HD / 8];
    __shared__ bf16_t s_v[64 * HD];
    __shared__ int s_src[64], s_dst[64];   // 16 * block + place
    __shared__ int s_bad;
    const int tid = threadIdx.x, kvh = blockIdx.x, b = blockIdx.y, layer = blockIdx.z;
    const int ctx = a.ctx_lens[b], n = a.keep_lens[b];
    if (ctx == -1 || n == 0) return;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    if (ctx < 0 || n < 0 || n > a.keep_stride) {
        if (tid == 0) atomicOr(a.err_flag, RS_FLAG_LENGTHS);
        return;
    }
    const int32_t *keep = a.keep + (size_t)b * a.keep_stride, *tab = a.tables + (size_t)b * a.max_blk;
    if (tid < n) {
        const int k = keep[tid], before = tid > 0 ? keep[tid - 1] : -1;
        if (k <= before || k >= 64) atomicOr(&s_bad, RS_FLAG_LENGTHS);
        else if ((int64_t)ctx + k >= 16ll * a.max_blk) atomicOr(&s_bad, 2);
        else {
            const int src = tab[(ctx + k) >> 4], dst = tab[(ctx + tid) >> 4];
            if ((unsigned)src >= (unsigned)a.n_blocks || (unsigned)dst >= (unsigned)a.n_blocks) atomicOr(&s_bad, 2);
            s_src[tid] = 16 * src + ((ctx + k) & 15);
            s_dst[tid] = 16 * dst + ((ctx + tid) & 15);
        }
    }
    __syncthreads();
    if (s_bad) {
        if (tid == 0) atomicOr(a.err_flag, s_bad);
        return;
    }
    // the first tokens that stay where they are
    int stay = 0;
    while (stay < n && s_src[stay] == s_dst[stay]) ++stay;
    const int m = n - stay;
    if (m == 0) return;
    bf16_t *kp = a.k_pool + layer * a.layer_stride, *vp = a.v_pool + layer * a.layer_stride;
    auto head = [&](int slot) { return ((size_t)(slot >> 4) * a.Hkv + kvh) * 16 * HD; };
    for (int it = tid; it < m * (HD / 8); it += 256) {
        const int i = it % m, c = it / m, s = s_src[stay + i];
        s_k[it] = ld_bf16x8(kp + head(s) + kpool_chunk_offset(s & 15, 8 * c));
    }
    for (int it = tid; it < m * HD; it += 256) {
        const int i = it % m, d = it / m, s = s_src[stay + i];
        s_v[it] = vp[head(s) + 16 * d + (s & 15)];
    }
    __syncthreads();
    for (int it = tid; it < m * (HD / 8); it += 256) {
        const int i = it % m, c = it / m, s = s_dst[stay + i];
        st_bf16x8(kp + head(s) + kpool_chunk_offset(s & 15, 8 * c), s_k[it]);
    }
    for (int it = tid; it < m * HD; it += 256) {
        const int i = it % m, d = it / m, s = s_dst[stay + i];
        vp[head(s) + 16 * d + (s & 15)] = s_v[it];
    }
}

}  // namespace

void launch_kv_plan(hipStream_t st, const KvPlanArgs &a) {
    const int x = (a.B + PLAN_REQS - 1) / PLAN_REQS;
    // long runs: some 1024 rows for each workgroup
    const int y = a.parents ? 1 : std::max(1, std::min((a.max_rows / x + 1023) / 1024, 256));
    hipLaunchKernelGGL(kv_plan_kernel, dim3(x, y), dim3(256), 0, st, a);
}

void launch_kv_store(hipStream_t st, const KvStoreArgs &a) {
    const int groups = (a.max_rows + 15) / 16, q_parts = (a.Hq + 7) / 8, kv_parts = (a.Hkv + 3) / 4;
    const dim3 grid(groups * (q_parts + kv_parts));
    if (a.hd == 128) hipLaunchKernelGGL(kv_store_kernel<128>, grid, dim3(256), 0, st, a, groups, q_parts);
    else hipLaunchKernelGGL(kv_store_kernel<64>, grid, dim3(256), 0, st, a, groups, q_parts);
}

void launch_kv_compact(hipStream_t st, const KvCompactArgs &a) {
    const dim3 grid(a.Hkv, a.B, a.n_layers);
    if (a.hd == 128) hipLaunchKernelGGL(kv_compact_kernel<128>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv_compact_kernel<64>, grid, dim3(256), 0, st, a);
}
