// Attention over the bf16 paged cache for rows that do not see all that is before them: windows with sinks (decode rows and prompt
// rows), and the tokens of a drafted tree.
//
//   o(row) = sum_j w_j v_j / sum_j w_j,   w_j = exp(q k_j / sqrt(hd) - max),   over the keys j that the row sees:
//   window:  j <= p  and  (j > p - window  or  j < sinks),   p the row's position;
//   tree:    j < ctx, and ctx + t for every bit t of the row's ancestor mask.
// A row that sees nothing gets zero.  What a key holds that a row does not see, NaN included, does not reach that row.
// Scores, maxima, sums and joins are float32.  Weights go into the product with V as bf16, as over this cache everywhere: V is bf16 and the matrix unit takes
// both factors of one type, so more bits would be a second product.  It adds 0.0011 to 0.0015 to the 0.0016 that the output's own rounding leaves, in quadrature.
//
// A UNIT is as many rows of one request and one kv head as fit in 128 columns, or 32, a column being (row, query head of the group): the
// keys of a block are read once for all of them.  Where units are fewer than compute units, each one's keys are cut in pieces.  The blocks that any row of a unit sees are counted through (`Span`): those of the
// sinks, then those of the windows; blocks between are not looked at, nor are their table entries.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

#define NEG_INF (-__builtin_huge_valf())

namespace {

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

typedef uint32_t u32x4_m __attribute__((ext_vector_type(4)));

// What a unit's rows see.
struct Span {
    int row0 = 0, rows = 0;      // rows of q and out
    int req = 0;                 // row of the block tables
    int first = 0;               // window: position of the unit's first row; tree: cached tokens
    int i0 = 0, n = 0;           // tree: the unit's first row among the request's n
    int sink_blocks = 0, skip = 0, blocks = 0;   // counted block j is table entry j, from sink_blocks on j + skip
    bool dead = false;           // rows without a request, or with a length out of range: zero
};

template <bool TREE>
__device__ __forceinline__ Span unit_span(const MaskedAttnArgs &a, int u) {
    Span s;
    const int per = a.unit_rows;
    int end;   // keys before this position
    if (TREE) {
        s.req = u / a.units_per_req;
        s.i0 = u % a.units_per_req * per;
        const int r0 = a.cu_rows[s.req], r1 = a.cu_rows[s.req + 1];
        s.first = a.ctx_lens[s.req];
        if (r0 < 0 || r1 < r0 || r1 > a.max_rows || r1 - r0 > a.max_draft) {   // not a row is touched
            if (threadIdx.x == 0) atomicOr(a.err_flag, RS_FLAG_LENGTHS);
            return s;
        }
        s.n = r1 - r0;
        s.rows = min(per, s.n - s.i0);
        if (s.rows <= 0) return s;
        s.row0 = r0 + s.i0;
        if (s.first < 0 || s.first > a.max_ctx - s.n) {
            if (threadIdx.x == 0) atomicOr(a.err_flag, 8);
            s.dead = true;
            return s;
        }
        end = s.first + s.n;
    } else {
        if (a.ctx_lens) {
            s.req = s.row0 = u;
            s.rows = 1;
            s.first = a.ctx_lens[u];
            if (s.first < 0 || s.first >= a.max_ctx) {
                if (s.first != -1 && threadIdx.x == 0) atomicOr(a.err_flag, 8);
                s.dead = true;
                return s;
            }
        } else {
            u = a.n_units - 1 - u;   // the last rows of a prompt see most
            MaskedRun run = a.runs[0];
            for (int i = 1; i < a.seq.n_req && u >= run.units; ++i) u -= run.units, run = a.runs[i];
            s.req = run.req;
            s.row0 = a.seq.cu[s.req] + u * per;
            s.rows = min(per, a.seq.cu[s.req + 1] - s.row0);
            s.first = run.start + u * per;
        }
        end = s.first + s.rows;
        const int oldest = max(s.first - a.window + 1, 0), w0 = oldest >> 4;
        s.sink_blocks = min((min(a.sinks, end) + 15) >> 4, w0);
        s.skip = w0 - s.sink_blocks;
    }
    s.blocks = ((end + 15) >> 4) - s.skip;
    return s;
}

// What one row sees.
struct Sight {
    int lo, hi, sinks;       // window: keys lo .. hi and those below sinks (of them none above hi)
    int ctx;                 // tree: keys below, and the bits of
    uint64_t bits;
    // The 16 keys from pos on, a bit each.  (Without branches: of a chain of conditions on 16 score registers the compiler, clang 22 of ROCm 7.2,
    // made control flow that lost the first register's.)
    template <bool TREE>
    __device__ __forceinline__ uint32_t sees16(int pos) const {
        auto upto = [](int n) { return (1u << min(max(n, 0), 16)) - 1; };
        if (TREE) {
            const int d = ctx - pos;
            const uint64_t drafted = d > 0 ? bits << min(d, 63) : bits >> min(-d, 63);
            return upto(d) | ((d < 16 && d > -64 ? (uint32_t)drafted : 0u) & 0xffffu);
        }
        return upto(hi - pos + 1) & (~upto(lo - pos) | upto(sinks - pos));
    }
};
template <bool TREE>
__device__ __forceinline__ Sight row_sight(const MaskedAttnArgs &a, const Span &s, int r) {
    Sight v{};
    if (TREE) {
        v.ctx = s.first;
        const int i = s.i0 + r;
        v.bits = a.masks ? a.masks[s.row0 + r] : (2ull << i) - 1;
        if (s.n < 64) v.bits &= (1ull << s.n) - 1;   // places behind the request's rows hold nothing
    } else {
        v.hi = s.first + r;
        v.lo = max(v.hi - a.window + 1, 0);
        v.sinks = a.sinks;
    }
    return v;
}
// What any of the unit's rows sees.  The other values of a block are cleared before they are multiplied: a weight of zero times what a place behind the
// last token holds, or one before the window, may be NaN, and pools need not be zeroed.  (Values that some of the rows see are left to careful_unit.)
template <bool TREE>
__device__ __forceinline__ Sight unit_sight(const MaskedAttnArgs &a, const Span &s) {
    Sight v{};
    if (TREE) {
        v.ctx = s.first + s.n;
    } else {
        v.hi = s.first + s.rows - 1;
        v.lo = max(s.first - a.window + 1, 0);
        v.sinks = a.sinks;
    }
    return v;
}
// Two values of the tokens 2j and 2j + 1 of a bit each in `seen`: which bits of them stay.
__device__ __forceinline__ uint32_t keep_pair(uint32_t seen, int j) { return (seen >> 2 * j & 1 ? 0x0000ffffu : 0u) | (seen >> 2 * j & 2 ? 0xffff0000u : 0u); }

// Weights of a block: the half-waves (same column) hold tokens 4h..4h+3 and 8+4h..8+4h+3 and trade their middle pieces; h = 0 then has tokens
// 0-7, h = 1 tokens 8-15, the contraction slices of V's own layout.
__device__ __forceinline__ bf16x8 by_tokens(bf16x8 p) {
    u32x4_m w = __builtin_bit_cast(u32x4_m, p);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const auto sw = __builtin_amdgcn_permlane32_swap(w[u], w[u + 2], false, false);
        w[u] = sw[0];
        w[u + 2] = sw[1];
    }
    return __builtin_bit_cast(bf16x8, w);
}

__device__ __forceinline__ bf16_t *out_at(const MaskedAttnArgs &a, const Span &s, int col, int hk, int G) {
    return a.out + (size_t)(s.row0 + col / G) * a.out_stride + (size_t)(hk * G + col % G) * a.hd;
}

// A unit's keys may be cut in pieces, which leave their sums in part_o [piece][column][hd] and part_ml (maximum of raw scores, sum of weights).
struct Piece {
    int unit, piece, cut;   // of `cut` pieces (1: the whole unit)
    int first, cols;        // place of the unit's first piece, columns of a place
    int ticket;
    __device__ __forceinline__ size_t at(int p, int col) const { return (size_t)(first + p) * cols + col; }
};
// The idx-th (unit, piece) of a kv head: the first pieces of all units, then the second ones, ...
__device__ __forceinline__ Piece piece_of(const MaskedAttnArgs &a, int idx, int hk, int cols) {
    const int u = idx % a.n_units, t = u * a.Hkv + hk;
    return {u, idx / a.n_units, a.cut, t * a.cut, cols, t};
}

// Four dims of each of K columns, their pieces taken in order (eight asked for together): get(k, i, &ml, &v).
template <int K, class Get>
__device__ __forceinline__ void join_columns(const MaskedAttnArgs &a, int cut, Get get, bf16x4 (&out)[K]) {
    constexpr int N = 8;
    float top[K], l[K];   // over the pieces so far
    f32x4 acc[K];
#pragma unroll
    for (int k = 0; k < K; ++k) top[k] = NEG_INF, l[k] = 0.f, acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < cut; i0 += N) {
        float2 ml[K][N];
        f32x4 x[K][N];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) get(k, min(i0 + i, cut - 1), ml[k][i], x[k][i]);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float m = top[k];
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i0 + i < cut) m = fmaxf(m, ml[k][i].x);
            const float ref = m == NEG_INF ? 0.f : m, keep = exp2f((top[k] - ref) * a.scale_log2);
            top[k] = m;
            l[k] *= keep;
            acc[k] = acc[k] * keep;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i0 + i >= cut || ml[k][i].y == 0.f) continue;   // (a sum of nothing: a piece none of whose keys the row sees)
                const float e = exp2f((ml[k][i].x - ref) * a.scale_log2);
                l[k] += ml[k][i].y * e;
                acc[k] += x[k][i] * e;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[k][i] = (bf16_t)(l[k] == 0.f ? 0.f : acc[k][i] / l[k]);
}

// Units of few columns: the last workgroup of a (unit, kv head) to arrive brings the pieces together, in their order, so that results do not
// depend on which one that is.  The sums are written and read at the device's scope, which passes the XCDs' own L2 caches by; a workgroup's have
// arrived when its waves have waited for them, in front of the ticket.  (A fence at that scope writes back and invalidates whole caches
// instead.)  Units of many columns are joined by a launch of their own: 64 KB a piece are too much for one workgroup.
struct Far {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    static constexpr int DEVICE = 16;   // cache policy: sc1
    __amdgpu_buffer_rsrc_t o, ml;
    __device__ __forceinline__ explicit Far(const MaskedAttnArgs &a)
        : o(__builtin_amdgcn_make_buffer_rsrc(a.part_o, 0, MASKED_PIECES * MASKED_COLS * a.hd * 4, 0x00020000)),
          ml(__builtin_amdgcn_make_buffer_rsrc(a.part_ml, 0, MASKED_PIECES * MASKED_COLS * 2 * 4, 0x00020000)) {}
    __device__ __forceinline__ void put_o(size_t i, f32x4 v) const { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), o, (int)(4 * i), 0, DEVICE); }
    __device__ __forceinline__ void put_ml(size_t i, float2 v) const { __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), ml, (int)(8 * i), 0, DEVICE); }
    __device__ __forceinline__ f32x4 get_o(size_t i) const { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(o, (int)(4 * i), 0, DEVICE)); }
    __device__ __forceinline__ float2 get_ml(size_t i) const { return __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(ml, (int)(8 * i), 0, DEVICE)); }
};
template <int HD, int T>
__device__ __forceinline__ void join_pieces(const MaskedAttnArgs &a, const Span &s, int hk, const Piece &pc) {
    __shared__ int last;
    const int G = a.Hq / a.Hkv, cols = s.rows * G;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's sums have arrived
    __syncthreads();
    if (threadIdx.x == 0) {
        int32_t *ticket = a.tickets + pc.ticket;
        last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pc.cut - 1;
        if (last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!last) return;
    const Far far(a);
    const int d = threadIdx.x % (HD / 4) * 4, col0 = threadIdx.x / (HD / 4);
    auto join = [&](auto items) {   // a thread's: four dims of a column, those of the columns T / (HD / 4) behind it
        constexpr int K = items;
        if (col0 >= cols) return;
        bf16x4 v[K];
        join_columns<K>(a, pc.cut, [&](int k, int i, float2 &ml, f32x4 &x) {
            const size_t at = pc.at(i, min(col0 + k * (4 * T / HD), cols - 1));
            ml = far.get_ml(at);
            x = far.get_o(at * HD + d);
        }, v);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int col = col0 + k * (4 * T / HD);
            if (col < cols) *(bf16x4 *)(out_at(a, s, col, hk, G) + d) = v[k];
        }
    };
    if (cols <= 4 * T / HD) join(std::integral_constant<int, 1>());
    else join(std::integral_constant<int, 32 * HD / (4 * T)>());
}

// The same sums one key after the other in float32, without the matrix unit: for units whose result is not finite.  There a weight
// of zero times a value that is infinite or NaN may have reached rows that do not see that value; here it cannot.  Slow (some ms for
// 4096 keys), and only taken where a key or value that some row of the unit sees is not finite: what no row sees is cleared.
template <int HD, bool TREE>
__device__ __forceinline__ void careful_unit(const MaskedAttnArgs &a, const Span &s, int hk, int b0, int b1, const Piece &pc, int threads) {
    constexpr int D = 32;   // dims of a thread
    const int G = a.Hq / a.Hkv, parts = HD / D;
    const int32_t *tab = a.tables + (size_t)s.req * a.max_blk;
    for (int item = threadIdx.x; item < s.rows * G * parts; item += threads) {
        const int col = item / parts, d0 = item % parts * D;
        const Sight see = row_sight<TREE>(a, s, col / G);
        const bf16_t *q = a.q + (size_t)(s.row0 + col / G) * a.q_stride + (size_t)(hk * G + col % G) * HD;
        float m = NEG_INF, l = 0.f, o[D];
        for (int i = 0; i < D; ++i) o[i] = 0.f;
        for (int j = b0; j < b1; ++j) {
            const int e = j < s.sink_blocks ? j : j + s.skip, blk = tab[e];
            if ((unsigned)blk >= (unsigned)a.n_blocks) continue;
            const size_t head = ((size_t)blk * a.Hkv + hk) * 16 * HD;
            const uint32_t seen = see.sees16<TREE>(16 * e);
#pragma unroll 1
            for (int t = 0; t < 16; ++t) {
                if (!(seen >> t & 1)) continue;
                float dot = 0.f;
#pragma unroll 1
                for (int d = 0; d < HD; d += 8) {
                    const bf16x8 x = ld_bf16x8(q + d), y = ld_bf16x8(a.k_pool + head + kpool_chunk_offset(t, d));
                    for (int i = 0; i < 8; ++i) dot = fmaf((float)x[i], (float)y[i], dot);
                }
                const float top = fmaxf(m, dot), ref = top == NEG_INF ? 0.f : top;
                const float keep = exp2f((m - ref) * a.scale_log2), w = exp2f((dot - ref) * a.scale_log2);
                l = l * keep + w;
                for (int i = 0; i < D; ++i) o[i] = o[i] * keep + w * (float)a.v_pool[head + (size_t)(d0 + i) * 16 + t];
                m = top;
            }
        }
        if (pc.cut > 1) {
            const size_t at = pc.at(pc.piece, col);
            const Far far(a);   // (whoever joins them)
            for (int i = 0; i < D; i += 4) far.put_o(at * HD + d0 + i, f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]});
            if (d0 == 0) far.put_ml(at, float2{m, l});
        } else {
            bf16_t *p = out_at(a, s, col, hk, G) + d0;
            for (int i = 0; i < D; ++i) p[i] = (bf16_t)(l == 0.f ? 0.f : o[i] / l);
        }
    }
}

// Into how many pieces a tree's unit is cut follows from its length, in steps of 64 keys, and all units' together, which no host knows: none is
// to have much more than an equal share of the launch's pieces.
__device__ __forceinline__ int tree_cut(const MaskedAttnArgs &a, int steps) {
    __shared__ int64_t sums[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int64_t sum = 0;   // (whole numbers: the same for every workgroup)
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int n = (int)((uint32_t)a.cu_rows[b + 1] - (uint32_t)a.cu_rows[b]), ctx = a.ctx_lens[b];
        if (n > 0 && n <= a.max_draft && ctx >= 0 && ctx <= a.max_ctx - n) sum += (int64_t)((n + a.unit_rows - 1) / a.unit_rows) * ((ctx + n + 63) >> 6);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int w = 0; w < waves; ++w) sum += sums[w];
    const float share = fmaxf(1.125f * (float)sum * a.Hkv / MASKED_PIECES, 4.f);
    return __builtin_amdgcn_readfirstlane(min(max((int)ceilf(steps / share), 1), a.cut));
}

// Units of up to 128 columns, or one of the `cut` pieces of a unit's keys, by KH teams of four waves.  A wave owns 32 columns, and of a step's keys
// (64, four blocks, for each team) those of its team.  Keys come by LDS-DMA into two buffers of K and two of V, a step ahead; all waves of a
// team use them.  (Four buffers of half as many keys, in us with them / so: a prompt of 1024 rows 29.5 / 26.1, sixteen trees of 32 rows behind 500
// to 4096 tokens 57.8 / 56.0, 32 of them 79.8 / 80.9.)  S^T = K Q^T and O^T = V^T P^T, so that a lane owns one column; the teams' sums are
// brought together at the end.
// What runs beside the matrix unit is written out: the products of the next step's scores alternate with most of this one's exponentials, the
// products with V with the rest of them and with the next step's maxima.  (A product takes 16 ns of a SIMD; an exponential, its multiplication
// and two additions beside it one more.)
// The exponentials' reference is 2 times the largest weight, moved where a score is above it: weights as factors of V are below 1, the largest in [1/2, 1],
// where bf16 is finest, and their error against float64 is that of rounding exact weights (tests/test_gpu_masked_error.py).  In us, 16384 rows under a window
// of 4096 / 32 trees of 32 rows, and the error by that of exact weights: the maximum itself 1015 / 77.1, 0.98; twice it 995 / 76.6, 1.00; three times 992 / 76.7,
// 1.02; a reference that follows once a score is 2^4 above it 957 / 74.4, 1.06.
// 16384 rows of the 8B heads under a window of 4096: 955 to 1060 us from card to card, 0.91 to 1.01 PFLOP/s, the matrix unit busy 48 % of the cycles; the loop with its products
// alone takes 607.  32 trees of 32 rows behind 512 to 4096 tokens: 76 us, as long as the longest one's steps take.
constexpr int TAB_BLOCKS = 2048;
template <int HD, int KH, bool TREE>
__global__ __launch_bounds__(256 * KH, 2) void masked_wide_kernel(MaskedAttnArgs a) {
    constexpr int BL = 4, NT = 2, STEP = BL * KH;   // blocks of a team in a step, its tiles of 32 keys; blocks of a step
    constexpr int KS = HD / 16, DT = HD / 32, BLK = 16 * HD, BUF = STEP * BLK, T = 256 * KH;
    extern __shared__ __attribute__((aligned(1024))) bf16_t smem_masked[];   // [2] K, [2] V of BUF, [4 KH waves][32][2] floats, [TAB_BLOCKS] ids, flag, [2] counts
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int cg = wave & 3, kh = wave >> 2;
    const int c32 = lane & 31, h = lane >> 5;
    const int G = a.Hq / a.Hkv;
    // kv heads go to the XCDs in turn, so that a head's keys are in one L2 where there are eight of them
    const int hk = blockIdx.x % a.Hkv;
    Piece pc = piece_of(a, blockIdx.x / a.Hkv, hk, MASKED_COLS);
    const Span s = unit_span<TREE>(a, pc.unit);
    if (s.rows <= 0) return;
    const int cols = s.rows * G;
    if (KH == 2 && TREE && a.cut > 1 && !s.dead) {   // (one team: more units than compute units, none is cut)
        pc.cut = tree_cut(a, (s.blocks + 3) >> 2);
        if (pc.piece == 0 && threadIdx.x == 0) a.tickets[MASKED_PIECES + pc.ticket] = pc.cut;   // for those who join them
    }
    if (pc.piece >= pc.cut) return;
    if (s.dead) {
        if (pc.piece == 0)
            for (int i = threadIdx.x; i < cols * HD; i += T) out_at(a, s, i / HD, hk, G)[i % HD] = (bf16_t)0.f;
        return;
    }
    const int n_steps = (s.blocks + STEP - 1) / STEP;
    const int t0 = (int)((int64_t)n_steps * pc.piece / pc.cut), t1 = (int)((int64_t)n_steps * (pc.piece + 1) / pc.cut);
    const int32_t *tab = a.tables + (size_t)s.req * a.max_blk;
    const float sc = a.scale_log2;

    const int col = cg * 32 + c32, row = min(col, cols - 1) / G;
    const Sight see = row_sight<TREE>(a, s, row);
    bf16x8 qf[KS];
    {
        const bf16_t *qp = a.q + (size_t)(s.row0 + row) * a.q_stride + (size_t)(hk * G + min(col, cols - 1) % G) * HD + 8 * h;
#pragma unroll
        for (int i = 0; i < KS; ++i) qf[i] = ld_bf16x8(qp + 16 * i);
    }
    // of the wave's rows: positions of the first and of the last; steps behind what the last one sees are not the wave's
    const int w_first = s.first + min(cg * 32, cols - 1) / G, w_last = s.first + min(cg * 32 + 31, cols - 1) / G;
    const int w_end = cg * 32 >= cols ? t0 : TREE ? t1 : min(t1, ((w_last >> 4) - s.skip) / STEP + 1);

    // Block ids of TAB_BLOCKS counted blocks from step tb on, in LDS: -1: none, or not one of the pool, of which there are some where *s_bad.  (Fetched
    // step by step into registers they would be waited for by a count of the loads behind them, which the compiler takes to be none where some are
    // under a branch: so all loads in flight would be waited for in every step.)
    int32_t *s_tab = (int32_t *)(smem_masked + 4 * BUF) + 4 * KH * 64, *s_bad = s_tab + TAB_BLOCKS;
    auto fill_tab = [&](int tb) {
        for (int i = threadIdx.x; i < min(TAB_BLOCKS, STEP * (t1 - tb)); i += T) {
            const int j = STEP * tb + i;
            int id = -1;
            if (j < s.blocks) {
                id = tab[j < s.sink_blocks ? j : j + s.skip];
                if ((unsigned)id >= (unsigned)a.n_blocks) {
                    atomicOr(a.err_flag, 2);
                    *s_bad = 1;
                    id = -1;
                }
            }
            s_tab[i] = id;
        }
    };
    int tb = t0;   // the first step of s_tab
    // Wave w brings block w of a step, 16 bytes a lane (lane l's at the window's base + 16 l).  K keeps the
    // pool's order; V's chunk (dim, half of 8 tokens) goes to [half][dim].  A block that is missing is read as block 0, masked, and its values are
    // cleared.
    typedef __attribute__((address_space(3))) void lds_void;
    auto id_of = [&](int t) { return s_tab[min(STEP * (t - tb) + wave, TAB_BLOCKS - 1)]; };   // (behind the last step: not used)
    auto head_of = [&](int id) { return ((size_t)max(__builtin_amdgcn_readfirstlane(id), 0) * a.Hkv + hk) * BLK; };
    size_t head_k = 0, head_v = 0;   // of the block that the wave brings next, for K; V follows a step behind
    int id_next = -1;                // asked for a step ahead
    auto k_at = [&](int t) { return smem_masked + ((t - t0) & 1) * BUF; };
    auto v_at = [&](int t) { return smem_masked + (2 + ((t - t0) & 1)) * BUF; };
    auto load_k = [&](int t) {
        head_v = head_k;
        head_k = head_of(id_next);
        const auto buf = __builtin_amdgcn_make_buffer_rsrc((void *)(a.k_pool + head_k), 0, 2 * BLK, 0x00020000);
        bf16_t *d = k_at(t) + wave * BLK;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void *)(d + i * 512), 16, lane * 16, i * 1024, 0, 0);
    };
    auto load_v = [&](int t, size_t head) {
        const auto buf = __builtin_amdgcn_make_buffer_rsrc((void *)(a.v_pool + head), 0, 2 * BLK, 0x00020000);
        bf16_t *d = v_at(t) + wave * BLK;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i)   // 64 dims of a half of the tokens
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (lds_void *)(d + i * 512), 16, lane * 32, (i % (HD / 64)) * 2048 + (i / (HD / 64)) * 16, 0, 0);
    };
    auto klds = [](int r, int cc) { return (r >> 4) * BLK + kpool_chunk_offset(r & 15, cc * 8); };
    auto vlds = [](int blk, int half, int d) { return blk * BLK + half * (8 * HD) + d * 8; };

    // reference (raw score), the same in powers of 2, sum of weights
    float ref = NEG_INF, ms = 0.f, l_run = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

    const float ahead = 1.f / sc;   // one power of 2

    bf16x8 pf[BL];   // weights of the wave's blocks
    constexpr int N_W = BL * 8;
    auto weight = [&](const f32x16 (&st)[NT], int n) {   // the n-th of the lane's weights of a step
        const int j = n / 8, i = n % 8;
        const float p = __builtin_amdgcn_exp2f(fmaf(st[j >> 1][8 * (j & 1) + i], sc, -ms));
        l_run += p;
        pf[j][i] = (bf16_t)p;
        if (i == 7) pf[j] = by_tokens(pf[j]);
    };
    // Fragments of K and V are read R ahead of their products, through one ring: while the last of K are used the first of V are read.  (With the block
    // ids a step ahead 16384 rows under a window of 4096 take 929 us instead of 940, 64 trees of 16 rows 126.5 instead of 129.4; reading the
    // next step's first K beside the last of V as well gives nothing more.)
    constexpr int N_K = NT * KS, N_V = BL * DT, R = 4;
    static_assert(N_K % R == 0 && N_V % R == 0);
    bf16x8 ring[R];
    auto kread = [&](int t, int i) {   // (score tile i % NT, head_dim step i / NT)
        return *(const bf16x8 *)&(k_at(t) + kh * (BL * BLK))[klds(32 * (i % NT) + c32, 2 * (i / NT) + h)];
    };
    auto vread = [&](int t, int i) { return *(const bf16x8 *)&(v_at(t) + kh * (BL * BLK))[vlds(i / DT, h, 32 * (i % DT) + c32)]; };
    auto ring_k = [&](int t) {
#pragma unroll
        for (int i = 0; i < R; ++i) ring[i] = kread(t, i);
    };
    auto ring_v = [&](int t) {
#pragma unroll
        for (int i = 0; i < R; ++i) ring[i] = vread(t, i);
    };
    auto scores = [&](int t, f32x16 (&st)[NT], auto then_v, auto between) {   // then_v: V of step t - 1 next; between(i): what goes beside the i-th product
        f32x16 zero;
#pragma unroll
        for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
        for (int i = 0; i < N_K; ++i) {
            if (i == 0) __builtin_amdgcn_s_setprio(1);   // in front of the other workgroup's waves (16384 rows, window 4096: 975 us without, 963 with)
            if (i == N_K - 1) __builtin_amdgcn_s_setprio(0);
            st[i % NT] = mfma32(ring[i % R], qf[i / NT], i < NT ? zero : st[i % NT]);
            __builtin_amdgcn_sched_barrier(0);
            if (i + R < N_K) ring[i % R] = kread(t, i + R);
            else if (then_v) ring[i % R] = vread(t - 1, i + R - N_K);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    bool bad = false;   // some blocks are none of the pool
    // hides what the wave's rows do not see of step t
    auto mask = [&](int t, f32x16 (&st)[NT]) {
        int pos[BL];
        bool here[BL], full = true;
#pragma unroll
        for (int j = 0; j < BL; ++j) {
            const int e = STEP * t + BL * kh + j, p = 16 * (e < s.sink_blocks ? e : e + s.skip);
            here[j] = e < s.blocks && !(bad && __builtin_amdgcn_readfirstlane(s_tab[STEP * (t - tb) + BL * kh + j]) < 0);
            pos[j] = p;
            full = full && here[j] && (TREE ? p + 15 < s.first : p + 15 <= w_first && (p > w_last - a.window || p + 15 < a.sinks));
        }
        if (full) return;
#pragma unroll
        for (int j = 0; j < BL; ++j) {
            const uint32_t seen = here[j] ? see.template sees16<TREE>(pos[j]) >> (4 * h) : 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = st[j >> 1][8 * (j & 1) + i];
                st[j >> 1][8 * (j & 1) + i] = seen & (1u << ((i >> 2) * 8 + (i & 3))) ? v : NEG_INF;
            }
        }
    };
    auto maximum = [&](const f32x16 (&st)[NT]) {
        float m = NEG_INF;
#pragma unroll
        for (int t2 = 0; t2 < NT; ++t2)
#pragma unroll
            for (int i = 0; i < 16; ++i) m = fmaxf(m, st[t2][i]);
        return m;
    };
    // moves the reference ahead of a score of the step that is above it
    auto follow = [&](float m) {
        const uint32_t mb = __builtin_bit_cast(uint32_t, m);
        const auto sw = __builtin_amdgcn_permlane32_swap(mb, mb, false, false);
        m = fmaxf(__builtin_bit_cast(float, (uint32_t)sw[0]), __builtin_bit_cast(float, (uint32_t)sw[1]));
        if (!__any(m > ref)) return;
        const bool moves = m > ref;
        m += ahead;
        const float alpha = moves ? __builtin_amdgcn_exp2f((ref - m) * sc) : 1.f;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha;
        ref = moves ? m : ref;
        ms = moves ? m * sc : ms;
    };
    // products with V of step t; weights from N0 on are formed beside them (of a block in front of it), then the next step's maximum
    constexpr int N0 = 24;
    auto values = [&](int t, const f32x16 (&cur)[NT], const f32x16 (&nxt)[NT]) {
        // the weights left are due before the last block's products: so many beside each product before those
        constexpr int SLOTS = DT * (BL - 1), EACH = (N_W - N0 + SLOTS - 1) / SLOTS;
        float m = NEG_INF;
#pragma unroll
        for (int i = 0; i < N_V; ++i) {
            o[i % DT] = mfma32(ring[i % R], pf[i / DT], o[i % DT]);
            __builtin_amdgcn_sched_barrier(0);
            if (i + R < N_V) ring[i % R] = vread(t, i + R);
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (i < SLOTS && N0 + i * EACH + e < N_W) weight(cur, N0 + i * EACH + e);
            if (i == SLOTS) m = maximum(nxt);
            __builtin_amdgcn_sched_barrier(0);
        }
        return m;
    };

    if (threadIdx.x < 3) s_bad[threadIdx.x] = 0;
    __syncthreads();
    fill_tab(t0);
#pragma unroll
    for (int i = 0; i < KS; ++i) asm volatile("" : "+v"(qf[i]));   // the queries are here: not to be waited for among the steps' loads
    __syncthreads();
    bad = __builtin_amdgcn_readfirstlane(*s_bad) != 0;
    // All loads and reads of the team's waves so far are done.  Teams use what their own waves bring, so one need not wait for the other, and while
    // one's waves pass from products to exponentials the other's have the matrix unit: a count in LDS in place of the workgroup's barrier (32 trees of 32
    // rows behind 512 to 4096 tokens 81 us with the barrier, 74 so).  All four waves of a team come here equally often, and all are resident: the
    // wait ends.
    int32_t *met = s_bad + 1 + kh;
    int times = 0;
    auto meet = [&]() {
        if (KH == 1) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            return;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (lane == 0) __hip_atomic_fetch_add(met, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        times += 4;
        while (__builtin_amdgcn_readfirstlane(__hip_atomic_load(met, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)) < times) {}
        asm volatile("" ::: "memory");
    };
    // In front of step t's work: K of the step after it and V of its own have landed, nobody reads those of the step before any more; their buffers
    // take K of the step after the next and V of the next.
    const int t_edge = max(s.sink_blocks - 1, 0) / STEP;
    auto turn = [&](int t) {
        // What no row sees of the wave's own block of V is cleared: places behind the end (in the last step), those behind the sinks or before the windows
        // (blocks sink_blocks - 1 and sink_blocks), a missing block whole.
        if (t + 1 >= t1 || bad || (!TREE && (unsigned)(t - t_edge) <= 1)) {
            const int e = STEP * t + wave;
            const bool here = e < s.blocks && !(bad && __builtin_amdgcn_readfirstlane(s_tab[STEP * (t - tb) + wave]) < 0);
            const uint32_t some = here ? unit_sight<TREE>(a, s).template sees16<TREE>(16 * (e < s.sink_blocks ? e : e + s.skip)) : 0u;
            if (some != 0xffffu) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < HD / 32; ++i) {   // 64 dims of a half of the tokens
                    u32x4_m *p = (u32x4_m *)(v_at(t) + wave * BLK + (64 * i + lane) * 8), w = *p;
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] &= keep_pair(some >> (i / (HD / 64) * 8), j);
                    *p = w;
                }
            }
        }
        meet();
        if (STEP * (t + 4 - tb) > TAB_BLOCKS && t + 1 < t1) {   // contexts of more than 32K tokens
            if (KH == 2) __syncthreads();
            tb = t;
            fill_tab(tb);
            __syncthreads();
            bad = __builtin_amdgcn_readfirstlane(*s_bad) != 0;
        }
        if (t + 2 < t1) {
            load_k(t + 2);
            load_v(t + 1, head_v);
            id_next = id_of(t + 3);
        } else if (t + 1 < t1) load_v(t + 1, head_k);
    };
    auto step = [&](int t, f32x16 (&cur)[NT], f32x16 (&nxt)[NT]) {
        turn(t);
        if (t >= w_end) return;
        if (t + 1 < w_end) {
            constexpr int EACH = (N0 + N_K - 1) / N_K;
            ring_k(t + 1);
            scores(t + 1, nxt, std::true_type(), [&](int i) {
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    if (i * EACH + e < N0) weight(cur, i * EACH + e);
            });
            mask(t + 1, nxt);
        } else {
#pragma unroll
            for (int n = 0; n < N0; ++n) weight(cur, n);
            ring_v(t);
        }
        const float m = values(t, cur, nxt);
        if (t + 1 < w_end) follow(m);
    };
    f32x16 sa[NT], sb[NT];
    if (t0 < t1) {
        id_next = id_of(t0);
        load_k(t0);
        id_next = id_of(t0 + 1);
        meet();
        if (t0 + 1 < t1) {
            load_k(t0 + 1);
            load_v(t0, head_v);
            id_next = id_of(t0 + 2);
        } else load_v(t0, head_k);
        if (t0 < w_end) {
            ring_k(t0);
            scores(t0, sa, std::false_type(), [](int) {});
            mask(t0, sa);
            follow(maximum(sa));
        }
    }
    for (int t = t0; t < t1; t += 2) {
        step(t, sa, sb);
        if (t + 1 < t1) step(t + 1, sb, sa);
    }
    l_run += __shfl_xor(l_run, 32, 64);

    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = odd || !(fabsf(o[dt][i]) < __builtin_huge_valf());
    if (__syncthreads_or(odd && col < cols)) {
        careful_unit<HD, TREE>(a, s, hk, STEP * t0, min(STEP * t1, s.blocks), pc, T);
        return;
    }

    if (KH == 2) {
        // both waves of a column rescale to the common reference; the first finishes the first half of head_dim, the second the other, each with the
        // other's part through the buffers (nobody reads those any more)
        f32x4 *x_o = (f32x4 *)smem_masked;   // [8 waves][2 DT][64]
        float *x_ml = (float *)(smem_masked + 4 * BUF), *mine = x_ml + wave * 64, *theirs = x_ml + (wave ^ 4) * 64;
        if (h == 0) {
            mine[2 * c32] = ref;
            mine[2 * c32 + 1] = l_run;
        }
#pragma unroll
        for (int dt = 0; dt < DT / 2; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f32x4 v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = kh == 0 ? o[DT / 2 + dt][4 * j + i] : o[dt][4 * j + i];
                x_o[(wave * (2 * DT) + dt * 4 + j) * 64 + lane] = v;
            }
        __syncthreads();
        const float m_o = theirs[2 * c32], l_o = theirs[2 * c32 + 1];
        const float top = fmaxf(ref, m_o), base = top == NEG_INF ? 0.f : top;
        const float e = __builtin_amdgcn_exp2f((ref - base) * sc), e_o = __builtin_amdgcn_exp2f((m_o - base) * sc);
        l_run = l_run * e + l_o * e_o;
        ref = top;
#pragma unroll
        for (int dt = 0; dt < DT / 2; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 v = x_o[((wave ^ 4) * (2 * DT) + dt * 4 + j) * 64 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[dt][4 * j + i] = (kh == 0 ? o[dt][4 * j + i] : o[DT / 2 + dt][4 * j + i]) * e + v[i] * e_o;
            }
    }
    const int d0 = kh * (HD / KH) + 4 * h;   // this lane's dims: d0 + 32 dt + 8 j + i
    if (KH == 2 && pc.cut > 1) {
        // a column's consecutive sums are written together, through LDS
        constexpr int ROW = HD + 4;
        __syncthreads();   // the other team's part has been read
        float *strip = (float *)smem_masked + cg * (32 * ROW);
#pragma unroll
        for (int dt = 0; dt < DT / KH; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) *(f32x4 *)(strip + c32 * ROW + d0 + 32 * dt + 8 * j) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
        if (h == 0 && kh == 0 && col < cols) *(float2 *)(a.part_ml + 2 * pc.at(pc.piece, col)) = float2{ref, l_run};
        __syncthreads();
        for (int i = kh; i < 32 * (HD / 4) / 64; i += KH) {
            const int item = 64 * i + lane, c = item / (HD / 4), d = item % (HD / 4) * 4;
            if (cg * 32 + c < cols) *(f32x4 *)(a.part_o + pc.at(pc.piece, cg * 32 + c) * HD + d) = *(const f32x4 *)(strip + c * ROW + d);
        }
        return;
    }
    // rows of out are written whole: the wave's columns (of its team's dims) through LDS
    constexpr int ROW = HD + 8;
    if (KH == 2) __syncthreads();   // the other team's part has been read
    bf16_t *strip = smem_masked + cg * (32 * ROW);
    const float inv = l_run > 0.f ? 1.0f / l_run : 0.f;
#pragma unroll
    for (int dt = 0; dt < DT / KH; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (bf16_t)(o[dt][4 * j + i] * inv);
            *(bf16x4 *)(strip + c32 * ROW + d0 + 32 * dt + 8 * j) = v;
        }
    __syncthreads();
    constexpr int CH = HD / 8;
#pragma unroll
    for (int i = 0; i < 32 * CH / (64 * KH); ++i) {
        const int item = 64 * (KH * i + kh) + lane, c = item / CH, d = item % CH * 8;
        if (cg * 32 + c < cols) st_bf16x8(out_at(a, s, cg * 32 + c, hk, G) + d, *(const bf16x8 *)(strip + c * ROW + d));
    }
}

// Brings the pieces of units of many columns together: a thread for four dims of a column.
template <int HD, bool TREE>
__global__ __launch_bounds__(256) void masked_join_kernel(MaskedAttnArgs a) {
    const int G = a.Hq / a.Hkv, hk = blockIdx.x % a.Hkv;
    Piece pc = piece_of(a, blockIdx.x / a.Hkv, hk, MASKED_COLS);
    const Span s = unit_span<TREE>(a, pc.unit);
    if (s.rows <= 0 || s.dead) return;
    if (TREE) pc.cut = a.tickets[MASKED_PIECES + pc.ticket];
    const int item = blockIdx.y * 256 + threadIdx.x, col = item / (HD / 4), d = item % (HD / 4) * 4;
    if (pc.cut == 1 || col >= s.rows * G) return;
    bf16x4 v[1];
    join_columns<1>(a, pc.cut, [&](int, int i, float2 &ml, f32x4 &x) {
        const size_t at = pc.at(i, col);
        ml = *(const float2 *)(a.part_ml + 2 * at);
        x = *(const f32x4 *)(a.part_o + at * HD + d);
    }, v);
    *(bf16x4 *)(out_at(a, s, col, hk, G) + d) = v[0];
}

// Units of up to 32 columns (decode rows, small trees): bound by reading the cache, so nothing is shared and nothing staged.  The waves take
// tiles of 32 keys (two blocks) in turn, straight from the pools into the operands of 32x32x16 products (every load of a wave is a contiguous
// kilobyte, or four pieces of 256 bytes); a tile's keys are asked for as soon as the products with the ones before have been issued, and so are
// its values.  The waves' sums meet in LDS at the end.  8B heads: 64 rows of 512 to 16383 tokens under a window of 4096 take 152 us, 6.3 TB/s (with
// eight waves 154); one row under a window of 1024 8.7 to 8.9 us, in eight pieces.
template <int HD, int NW, bool TREE>
__global__ __launch_bounds__(64 * NW, 2) void masked_few_kernel(MaskedAttnArgs a) {
    constexpr int KS = HD / 16, DT = HD / 32, BLK = 16 * HD, PAD = HD + 4;
    constexpr bool CUTS = NW == 8;   // four waves: more units than compute units, none is cut
    extern __shared__ __attribute__((aligned(16))) float smem_few[];   // [NW][32][PAD], [NW][32][2]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c32 = lane & 31, h = lane >> 5;
    const int G = a.Hq / a.Hkv;
    const int hk = blockIdx.x % a.Hkv;
    const Piece pc = piece_of(a, blockIdx.x / a.Hkv, hk, 32);
    const Span s = unit_span<TREE>(a, pc.unit);
    if (s.rows <= 0) return;
    const int cols = s.rows * G;
    if (s.dead) {
        if (pc.piece == 0)
            for (int i = threadIdx.x; i < cols * HD; i += 64 * NW) out_at(a, s, i / HD, hk, G)[i % HD] = (bf16_t)0.f;
        return;
    }
    const int n_tiles = (s.blocks + 1) >> 1;
    const int t0 = (int)((int64_t)n_tiles * pc.piece / pc.cut), t1 = (int)((int64_t)n_tiles * (pc.piece + 1) / pc.cut);
    const int32_t *tab = a.tables + (size_t)s.req * a.max_blk;
    const float sc = a.scale_log2;
    const int col = c32, row = min(col, cols - 1) / G;
    const int w_last = s.first + s.rows - 1;   // position of the unit's last row (windows)

    // lane l: the id of block l & 1 of a tile; -1: none, or not one of the pool
    auto fetch_ids = [&](int t) {
        const int j = 2 * t + (lane & 1);
        return t < t1 && j < s.blocks ? tab[j < s.sink_blocks ? j : j + s.skip] : -1;
    };
    auto checked = [&](int t, int id) {
        if ((unsigned)id < (unsigned)a.n_blocks) return id;
        if (lane < 2 && t < t1 && 2 * t + lane < s.blocks) atomicOr(a.err_flag, 2);
        return -1;
    };
    bf16x8 kf[KS], vf[2][DT];
    auto head_of = [&](int id) { return ((size_t)max(id, 0) * a.Hkv + hk) * BLK; };   // (a block that is missing: block 0, masked, its values cleared)
    auto load_k = [&](int ids) {
        const size_t h0 = head_of(__builtin_amdgcn_readlane(ids, 0)), h1 = head_of(__builtin_amdgcn_readlane(ids, 1));
        const bf16_t *p = a.k_pool + (c32 < 16 ? h0 : h1) + kpool_chunk_offset(c32 & 15, 8 * h);
#pragma unroll
        for (int i = 0; i < KS; ++i) kf[i] = ld_bf16x8_stream(p + (i >> 1) * 512 + (i & 1) * 256);
    };
    auto load_v = [&](int ids) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const bf16_t *p = a.v_pool + head_of(__builtin_amdgcn_readlane(ids, b)) + c32 * 16 + 8 * h;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[b][dt] = ld_bf16x8_stream(p + dt * 512);
        }
    };
    int t = t0 + wave;
    int ids = checked(t, fetch_ids(t));
    const bool any = t < t1;
    if (any) load_k(ids), load_v(ids);
    int next = fetch_ids(t + NW);
    const Sight see = row_sight<TREE>(a, s, row), all = unit_sight<TREE>(a, s);
    bf16x8 qf[KS];
    {
        const bf16_t *qp = a.q + (size_t)(s.row0 + row) * a.q_stride + (size_t)(hk * G + min(col, cols - 1) % G) * HD + 8 * h;
#pragma unroll
        for (int i = 0; i < KS; ++i) qf[i] = ld_bf16x8(qp + 16 * i);
    }
    float m_run = NEG_INF, l_run = 0.f;   // running maximum of raw scores, running sum
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

    for (; t < t1; t += NW) {
        f32x16 st;
#pragma unroll
        for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
        for (int i = 0; i < KS; ++i) st = mfma32(kf[i], qf[i], st);
        // the next tile, or behind the last one this one again (from the caches)
        const bool more = t + NW < t1;
        const int nids = more ? checked(t + NW, next) : ids;
        next = fetch_ids(t + 2 * NW);
        load_k(nids);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int e = 2 * t + b, p = 16 * (e < s.sink_blocks ? e : e + s.skip);
            const bool there = __builtin_amdgcn_readlane(ids, b) >= 0;
            const bool full = there && (TREE ? p + 15 < s.first : p + 15 <= s.first && (p > w_last - a.window || p + 15 < a.sinks));
            if (!full) {   // uniform
                const uint32_t seen = there ? see.sees16<TREE>(p) >> (4 * h) : 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = st[8 * b + i];
                    st[8 * b + i] = seen & (1u << ((i >> 2) * 8 + (i & 3))) ? x : NEG_INF;
                }
                const uint32_t some = there ? all.sees16<TREE>(p) : 0u;
                if (some != 0xffffu) {   // uniform; the lane's values are those of tokens 8h ..
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t keep = keep_pair(some >> (8 * h), j);
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            u32x4_m w = __builtin_bit_cast(u32x4_m, vf[b][dt]);
                            w[j] &= keep;
                            vf[b][dt] = __builtin_bit_cast(bf16x8, w);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        float m_tile = NEG_INF;
#pragma unroll
        for (int i = 0; i < 16; ++i) m_tile = fmaxf(m_tile, st[i]);
        m_tile = fmaxf(m_tile, __shfl_xor(m_tile, 32, 64));
        const float m_new = fmaxf(m_run, m_tile);
        const float m_safe = m_new == NEG_INF ? 0.f : m_new;
        if (__any(m_new != m_run)) {
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_safe) * sc);
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha;
            m_run = m_new;
        }
        const float ms = m_safe * sc;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            bf16x8 pf;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(st[8 * b + i], sc, -ms));
                l_run += p;
                pf[i] = (bf16_t)p;
            }
            pf = by_tokens(pf);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32(vf[b][dt], pf, o[dt]);
        }
        load_v(nids);
        __builtin_amdgcn_sched_barrier(0);
        ids = nids;
    }
    l_run += __shfl_xor(l_run, 32, 64);

    bool odd = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = odd || !(fabsf(o[dt][i]) < __builtin_huge_valf());
    float *s_o = smem_few, *s_ml = smem_few + NW * 32 * PAD;
    if (col < cols) {
        float *p = s_o + (wave * 32 + col) * PAD + 4 * h;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) *(f32x4 *)(p + 32 * dt + 8 * j) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
        if (h == 0) {
            s_ml[(wave * 32 + col) * 2] = m_run;
            s_ml[(wave * 32 + col) * 2 + 1] = l_run;
        }
    }
    if (__syncthreads_or(odd && col < cols)) {
        careful_unit<HD, TREE>(a, s, hk, 2 * t0, min(2 * t1, s.blocks), pc, 64 * NW);
        if (CUTS && pc.cut > 1) join_pieces<HD, 64 * NW>(a, s, hk, pc);
        return;
    }
    for (int item = threadIdx.x; item < cols * (HD / 4); item += 64 * NW) {
        const int c = item / (HD / 4), d = item % (HD / 4) * 4;
        float top = NEG_INF, l = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, s_ml[(w * 32 + c) * 2]);
        const float base = top == NEG_INF ? 0.f : top;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float e = __builtin_amdgcn_exp2f((s_ml[(w * 32 + c) * 2] - base) * sc);
            l += s_ml[(w * 32 + c) * 2 + 1] * e;
            acc += *(const f32x4 *)(s_o + (w * 32 + c) * PAD + d) * e;
        }
        if (CUTS && pc.cut > 1) {
            const size_t at = pc.at(pc.piece, c);
            const Far far(a);
            far.put_o(at * HD + d, acc);
            if (d == 0) far.put_ml(at, float2{top, l});
            continue;
        }
        const float inv = l > 0.f ? 1.0f / l : 0.f;
        bf16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (bf16_t)(acc[i] * inv);
        *(bf16x4 *)(out_at(a, s, c, hk, G) + d) = v;
    }
    if (CUTS && pc.cut > 1) join_pieces<HD, 64 * NW>(a, s, hk, pc);
}

constexpr int wide_lds(int hd, int kh) { return 4 * kh * 4 * 16 * hd * 2 + 4 * kh * 64 * 4 + (TAB_BLOCKS + 3) * 4; }

constexpr int few_lds(int hd, int nw) { return nw * 32 * (hd + 4 + 2) * 4; }

template <int HD, bool TREE>
void launch(hipStream_t st, const MaskedAttnArgs &a, const MaskedForm &f) {
    const dim3 grid(a.n_units * a.cut * a.Hkv);
    switch (f.kind) {
        case MASKED_FEW4: hipLaunchKernelGGL((masked_few_kernel<HD, 4, TREE>), grid, dim3(256), few_lds(HD, 4), st, a); break;
        case MASKED_FEW8: hipLaunchKernelGGL((masked_few_kernel<HD, 8, TREE>), grid, dim3(512), few_lds(HD, 8), st, a); break;
        case MASKED_WIDE: hipLaunchKernelGGL((masked_wide_kernel<HD, 1, TREE>), grid, dim3(256), wide_lds(HD, 1), st, a); break;
        case MASKED_TEAMS: hipLaunchKernelGGL((masked_wide_kernel<HD, 2, TREE>), grid, dim3(512), wide_lds(HD, 2), st, a); break;
    }
    if (a.cut == 1) return;
    const int cols = a.unit_rows * (a.Hq / a.Hkv);
    const dim3 joins(a.n_units * a.Hkv, (cols * (HD / 4) + 255) / 256);
    if (f.kind == MASKED_TEAMS) hipLaunchKernelGGL((masked_join_kernel<HD, TREE>), joins, dim3(256), 0, st, a);
}

}  // namespace

MaskedForm masked_form(MaskedAttnArgs &a) {
    const int G = a.Hq / a.Hkv;
    const bool tree = a.cu_rows != nullptr;
    int most = 1;   // rows of a request
    if (tree) most = a.max_draft;
    else if (!a.ctx_lens)
        for (int r = 0; r < a.seq.n_req; ++r) most = std::max(most, a.seq.cu[r + 1] - a.seq.cu[r]);
    MaskedForm f{};
    const auto units = [&](int rows) {   // of so many rows
        if (tree) return a.B * ((a.max_draft + rows - 1) / rows);
        if (a.ctx_lens) return a.B;
        int n = 0;
        for (int r = 0; r < a.seq.n_req; ++r) n += (a.seq.cu[r + 1] - a.seq.cu[r] + rows - 1) / rows;
        return n;
    };
    int keys = tree || a.ctx_lens ? a.max_ctx : 0;   // most keys of a row
    for (int r = 0; !tree && !a.ctx_lens && r < a.seq.n_req; ++r) keys = std::max(keys, a.seq.start[r] + a.seq.cu[r + 1] - a.seq.cu[r]);
    if (!tree) keys = (int)std::min<int64_t>(keys, (int64_t)a.window + a.sinks + 32);
    // Units of 32 columns where a request has no more, or where reading the keys again for each of them is little: us with units of 32 / of 128,
    // 8B heads: a tree of 16 behind 900 tokens 12.0 / 16.3, eight of them 17.7 / 19.8, one of 60 behind 3500 19.1 / 22.0, three of 32
    // behind 3000 25.4 / 26.3, four behind 4000 32.1 / 29.2, sixteen behind 500 to 4096 67.9 / 55.9; 100 rows under a window of 2048 19.4 / 21.5,
    // 512 39.0 / 41.1; prompts of 200 rows 9.0 / 12.9, 400 12.1 / 21.1, 600 18.7 / 20.0.
    const bool few = most * G <= 32 || (int64_t)units(32 / G) * a.Hkv * keys <= 256 * 1024;
    a.unit_rows = (few ? 32 : MASKED_COLS) / G;
    a.units_per_req = (a.max_draft + a.unit_rows - 1) / a.unit_rows;
    a.n_units = units(a.unit_rows);
    const int64_t wgs = (int64_t)a.n_units * a.Hkv;
    if (wgs <= 0) return f;
    // Prompts whose rows see most are begun first, so that a launch ends with short units: us without / so, 1500, 100, 2000, 700 and 64 rows behind 0, 3000, 500,
    // 2000 and 9 158 / 129; 700 rows behind 1024, 33 behind 4000 and 1391 of 64/8 heads under a window of 512 63.5 / 58.9.
    if (!tree && !a.ctx_lens) {
        const auto sees = [&](int r) {   // the first row and the last
            const int64_t most_seen = (int64_t)a.window + a.sinks;
            return std::min<int64_t>(a.seq.start[r], most_seen) + std::min<int64_t>(a.seq.start[r] + a.seq.cu[r + 1] - a.seq.cu[r], most_seen);
        };
        for (int r = 0; r < a.seq.n_req; ++r) a.runs[r] = {r, (a.seq.cu[r + 1] - a.seq.cu[r] + a.unit_rows - 1) / a.unit_rows, a.seq.start[r]};
        std::sort(a.runs, a.runs + a.seq.n_req, [&](const MaskedRun &x, const MaskedRun &y) {
            return std::make_pair(sees(x.req), x.req) < std::make_pair(sees(y.req), y.req);
        });
    }
    const int tiles = (int)(((int64_t)keys + 63) / 64);
    const auto cut = [&](int least, int most) {   // pieces of about `least` tiles or more, none but the first for each compute unit
        return (int)std::max<int64_t>(1, std::min<int64_t>({MASKED_PIECES / wgs, most, (tiles + least - 1) / least}));
    };
    // Every workgroup has a compute unit to itself on the whole chip.  A partition may have fewer; the forms are the same there, so that the bits are, though one team
    // is then often faster: us with two teams / one on 256, 192, 128 and 64 units, 32 trees of 32 77 / 93, 98 / 105, 125 / 106, 211 / 183; 2048 rows 58 / 64, 74 / 61,
    // 99 / 79, 195 / 148.
    const bool alone = wgs <= MASKED_PIECES;
    if (few) {
        f.kind = alone ? MASKED_FEW8 : MASKED_FEW4;
        // Eight pieces are asked for together by the one that joins them; more pay for long contexts.  us in 8 / 16 / 32 pieces, 8B heads: a row under a
        // window of 1024 8.8 / 9.7 / 13.0, 4096 13.7 / 13.2 / 14.9, 8192 18.7 / 16.0 / 18.7, 30000 45.5 / 31.1 / 31.2 (24: 29.1); a tree of 8 behind
        // 900 tokens 11.5 / 13.4 / 18.4 (6: 12.0), 4000 17.1 / 17.7 / 21.2, 8000 22.3 / 20.5 / 25.1; 19 rows under a window of 2048 in 8 / 10 pieces
        // 15.4 / 16.7.
        a.cut = cut(2, tiles <= 64 ? 8 : 16);
    } else {
        // Two teams halve the longest unit's time, which two rounds of units end with where most are much shorter: us with two teams / one, 8B heads:
        // a prompt of 1200 rows 32.4 / 37.9, 2048 57.7 / 63.4 (under a window of 1750 57.6 / 58.7, 1536 58.4 / 55.6, 512 42.3 / 31.9), 2048 behind 500
        // 74.9 / 78.8, behind 4000 195 / 187, 1600 beside 100 46.2 / 49.8; 2500 rows (three rounds) 86.3 / 77.9; 64 query heads, 1024 rows 39.8 / 38.0.
        int64_t seen = 0;   // by all rows
        for (int r = 0; !tree && !a.ctx_lens && r < a.seq.n_req; ++r) {
            const int64_t n = a.seq.cu[r + 1] - a.seq.cu[r];
            seen += n * std::min<int64_t>(a.seq.start[r] + n / 2, (int64_t)a.window + a.sinks);
        }
        const bool uneven = !tree && keys >= 1152 && 5 * seen <= 3 * (int64_t)a.seq.cu[a.seq.n_req] * keys;
        f.kind = alone || (uneven && wgs <= 2 * MASKED_PIECES) ? MASKED_TEAMS : MASKED_WIDE;
        a.cut = cut(4, MASKED_MAX_CUT);
    }
    return f;
}

void launch_masked_attention(hipStream_t st, const MaskedAttnArgs &args) {
    MaskedAttnArgs a = args;
    const MaskedForm f = masked_form(a);
    if (a.n_units <= 0) return;
    const bool tree = a.cu_rows != nullptr;
    if (a.hd == 128) {
        if (tree) launch<128, true>(st, a, f);
        else launch<128, false>(st, a, f);
    } else {
        if (tree) launch<64, true>(st, a, f);
        else launch<64, false>(st, a, f);
    }
}

void masked_attention_init() {
    auto set = [](const void *f, int lds) { (void)hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, lds); };
    set((const void *)masked_wide_kernel<128, 1, false>, wide_lds(128, 1));
    set((const void *)masked_wide_kernel<128, 1, true>, wide_lds(128, 1));
    set((const void *)masked_wide_kernel<128, 2, false>, wide_lds(128, 2));
    set((const void *)masked_wide_kernel<128, 2, true>, wide_lds(128, 2));
    set((const void *)masked_wide_kernel<64, 1, false>, wide_lds(64, 1));
    set((const void *)masked_wide_kernel<64, 1, true>, wide_lds(64, 1));
    set((const void *)masked_wide_kernel<64, 2, false>, wide_lds(64, 2));
    set((const void *)masked_wide_kernel<64, 2, true>, wide_lds(64, 2));
    set((const void *)masked_few_kernel<128, 4, false>, few_lds(128, 4));
    set((const void *)masked_few_kernel<128, 4, true>, few_lds(128, 4));
    set((const void *)masked_few_kernel<128, 8, false>, few_lds(128, 8));
    set((const void *)masked_few_kernel<128, 8, true>, few_lds(128, 8));
    set((const void *)masked_few_kernel<64, 8, false>, few_lds(64, 8));
    set((const void *)masked_few_kernel<64, 8, true>, few_lds(64, 8));
}
