// The KV cache held in 4 bits: quantising rows into it, reading them back, and attention over it.
//
// Format.  Groups of 32 consecutive dims of one token's key or value share a scale s = 2^(b - 127), one byte b (255: the group
// holds a NaN or an infinity and reads back as NaN); an element is s times one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, four
// bits.  s is the smallest power of two with max|x| < 7 s: then the nearest level, 6 at most, is never further off than half a
// step between levels (a value in (6, 7) is rounded to 6 as it would be between 6 and 8).  Ties go to the even code.
//
// Layout.  Of a (block of 16 tokens, kv head) 17 * hd bytes in a row:
//   K codes  [hd/32 groups][16 tokens][16]     byte j: dims 2j (low half) and 2j+1 of the group
//   V codes  [4 quads][16][hd/32][4 tokens]    byte (q, j, g, i): dims 32g+2j and 32g+2j+1 of token 4q+i
//   K scales [hd/32][16],  V scales [4 quads][hd/32][4]
// A lane's operand of the matrix instruction that multiplies K (16 rows or 32, 32 dims of a token) is one 16-byte chunk; a
// lane's share of V (4 tokens of a dim pair in every group) is another.  Both halves of a byte belong to one token, so tokens
// can be appended one by one by anybody without reading what is there.
#include <algorithm>

#include "kernels.h"

#define NEG_INF (-__builtin_huge_valf())

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ __forceinline__ uint32_t as_bits(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// ---- the format ---------------------------------------------------------------------------------------------------------

// The scale byte of a group whose largest magnitude has these bf16 bits.  Adding 0x20 carries into the exponent from 1.75 on.
// Clamped so that every value of the group is a normal bf16 (2: 0.5 * 2^-125; 252: 6 * 2^125).
__device__ __forceinline__ uint32_t kv4_scale_byte(uint32_t amax_bits) {
    const int b = (int)((amax_bits + 0x20u) >> 7) - 2;
    return amax_bits >= 0x7f80u ? 255u : (uint32_t)min(max(b, 2), 252);
}
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return as_float(byte << 23); }   // (255: the conversions give NaN)
template <int I>
__device__ __forceinline__ float kv4_scale_of(uint32_t four) { return as_float(((four >> (8 * I)) & 255u) << 23); }

__device__ __forceinline__ uint32_t absmax2(uint32_t m, uint32_t two) {   // of bf16 magnitudes, as bits
    return max(m, max(two & 0x7fffu, (two >> 16) & 0x7fffu));
}
// Eight dims (four bf16 pairs) -> four bytes of codes.
__device__ __forceinline__ uint32_t kv4_codes8(u32x4_t x, float s) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, (uint32_t)x[0]), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, (uint32_t)x[1]), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, (uint32_t)x[2]), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, (uint32_t)x[3]), s, 3);
    return r;
}
// The inverse.
__device__ __forceinline__ u32x4_t kv4_values8(uint32_t codes, float s) {
    return u32x4_t{as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)), as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                   as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)), as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
}

// byte offsets within a (block, kv head)
template <int HD> struct Kv4 {
    static constexpr int G = HD / 32;
    static constexpr int V = 8 * HD, KS = 16 * HD, VS = 16 * HD + HD / 2, BYTES = 17 * HD;
    static __device__ __forceinline__ int k_chunk(int g, int t) { return (g * 16 + t) * 16; }
    static __device__ __forceinline__ int v_byte(int t, int j, int g) { return V + (((t >> 2) * 16 + j) * G + g) * 4 + (t & 3); }
    static __device__ __forceinline__ int k_scale(int g, int t) { return KS + g * 16 + t; }
    static __device__ __forceinline__ int v_scale(int g, int t) { return VS + ((t >> 2) * G + g) * 4 + (t & 3); }
};

// ---- runs of tokens: write and read back ----------------------------------------------------------------------------------
// A workgroup of 2 hd threads takes one (block, kv head) of one request: a thread 16 dims of one token's key (first half of the
// threads) or value.  Bound by memory: 4 hd bytes of bf16 and 17/16 hd of cache a (token, head).
struct RunBlock { int req, bi; };
// The u-th block of the run of blocks that the requests' tokens touch.
__device__ __forceinline__ RunBlock run_block(const SeqInfo &seq, int u) {
    for (int r = 0; r < seq.n_req; ++r) {
        const int len = seq.cu[r + 1] - seq.cu[r];
        if (len <= 0) continue;
        const int b0 = seq.start[r] >> 4, nb = ((seq.start[r] + len - 1) >> 4) - b0 + 1;
        if (u < nb) return {r, b0 + u};
        u -= nb;
    }
    return {-1, 0};
}
static int run_blocks(const SeqInfo &seq) {
    int n = 0;
    for (int r = 0; r < seq.n_req; ++r) {
        const int len = seq.cu[r + 1] - seq.cu[r];
        if (len > 0) n += ((seq.start[r] + len - 1) >> 4) - (seq.start[r] >> 4) + 1;
    }
    return n;
}

template <int HD>
__global__ __launch_bounds__(2 * HD) void kv4_write_kernel(Kv4RowsArgs a) {
    using F = Kv4<HD>;
    __shared__ __attribute__((aligned(16))) uint8_t s_v[8 * HD];
    const int hk = blockIdx.x % a.Hkv, tid = threadIdx.x;
    const RunBlock u = run_block(a.seq, blockIdx.x / a.Hkv);
    if (u.req < 0) return;
    const int blk = a.tables[(size_t)u.req * a.max_blk + u.bi];
    if ((unsigned)blk >= (unsigned)a.n_blocks) {
        if (tid == 0 && hk == 0) atomicOr(a.err_flag, 2);
        return;
    }
    const bool is_v = tid >= HD;
    const int i = is_v ? tid - HD : tid;
    const int t = i / (HD / 16), part = i % (HD / 16), g = part >> 1, half = part & 1;
    const int row = u.bi * 16 + t - a.seq.start[u.req], len = a.seq.cu[u.req + 1] - a.seq.cu[u.req];
    const bool mine = row >= 0 && row < len;
    u32x4_t x0 = {0, 0, 0, 0}, x1 = {0, 0, 0, 0};
    if (mine) {
        const bf16_t *src = (is_v ? a.v : a.k) + (size_t)(a.seq.cu[u.req] + row) * a.row_stride + hk * HD + part * 16;
        x0 = *(const u32x4_t *)src;
        x1 = *(const u32x4_t *)(src + 8);
    }
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) m = absmax2(absmax2(m, x0[j]), x1[j]);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1, 64));   // the group's other half is the neighbouring lane's
    const uint32_t b = kv4_scale_byte(m);
    // (a group that is not finite: its codes do not matter, its scale says so)
    const float s = kv4_scale(min(b, 252u));
    const uint32_t c0 = kv4_codes8(x0, s), c1 = kv4_codes8(x1, s);
    uint8_t *dst = a.pool + ((size_t)blk * a.Hkv + hk) * F::BYTES;
    // whole block: V's bytes change places in LDS and leave 16 at a time; else each by itself, and other tokens' are not touched
    const bool whole = u.bi * 16 >= a.seq.start[u.req] && u.bi * 16 + 16 <= a.seq.start[u.req] + len;
    if (mine) {
        if (!is_v) {
            *(u32x2_t *)(dst + F::k_chunk(g, t) + 8 * half) = u32x2_t{c0, c1};
            if (!half) dst[F::k_scale(g, t)] = (uint8_t)b;
        } else {
            if (!half) dst[F::v_scale(g, t)] = (uint8_t)b;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint8_t c = (uint8_t)((j < 4 ? c0 : c1) >> (8 * (j & 3)));
                const int at = F::v_byte(t, 8 * half + j, g);
                if (whole) s_v[at - F::V] = c;
                else dst[at] = c;
            }
        }
    }
    __syncthreads();
    if (whole && tid < HD / 2) *(u32x4_t *)(dst + F::V + 16 * tid) = *(const u32x4_t *)(s_v + 16 * tid);
}

template <int HD>
__global__ __launch_bounds__(2 * HD) void kv4_read_kernel(Kv4RowsArgs a) {
    using F = Kv4<HD>;
    __shared__ __attribute__((aligned(16))) uint8_t s_v[8 * HD];
    const int hk = blockIdx.x % a.Hkv, tid = threadIdx.x;
    const RunBlock u = run_block(a.seq, blockIdx.x / a.Hkv);
    if (u.req < 0) return;
    const int blk = a.tables[(size_t)u.req * a.max_blk + u.bi];
    const bool ok = (unsigned)blk < (unsigned)a.n_blocks;
    if (!ok && tid == 0 && hk == 0) atomicOr(a.err_flag, 2);
    const uint8_t *src = a.pool + ((size_t)(ok ? blk : 0) * a.Hkv + hk) * F::BYTES;
    const bool is_v = tid >= HD;
    const int i = is_v ? tid - HD : tid;
    const int t = i / (HD / 16), part = i % (HD / 16), g = part >> 1, half = part & 1;
    uint32_t b = src[is_v ? F::v_scale(g, t) : F::k_scale(g, t)];
    u32x2_t c = {0, 0};
    if (!is_v) c = *(const u32x2_t *)(src + F::k_chunk(g, t) + 8 * half);
    if (tid < HD / 2) *(u32x4_t *)(s_v + 16 * tid) = *(const u32x4_t *)(src + F::V + 16 * tid);
    __syncthreads();
    if (is_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c[0] |= (uint32_t)s_v[F::v_byte(t, 8 * half + j, g) - F::V] << (8 * j);
            c[1] |= (uint32_t)s_v[F::v_byte(t, 8 * half + 4 + j, g) - F::V] << (8 * j);
        }
    }
    if (!ok) c = u32x2_t{0, 0}, b = 2;
    const int row = u.bi * 16 + t - a.seq.start[u.req], len = a.seq.cu[u.req + 1] - a.seq.cu[u.req];
    if (row < 0 || row >= len) return;
    const float s = kv4_scale(b);
    bf16_t *dst = (is_v ? a.v_out : a.k_out) + (size_t)(a.seq.cu[u.req] + row) * a.row_stride + hk * HD + part * 16;
    *(u32x4_t *)dst = kv4_values8(c[0], s);
    *(u32x4_t *)(dst + 8) = kv4_values8(c[1], s);
}

void launch_kv4_write(hipStream_t st, const Kv4RowsArgs &a) {
    const int n = run_blocks(a.seq);
    if (n <= 0) return;
    if (a.hd == 128) hipLaunchKernelGGL(kv4_write_kernel<128>, dim3(a.Hkv * n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv4_write_kernel<64>, dim3(a.Hkv * n), dim3(128), 0, st, a);
}

void launch_kv4_read(hipStream_t st, const Kv4RowsArgs &a) {
    const int n = run_blocks(a.seq);
    if (n <= 0) return;
    if (a.hd == 128) hipLaunchKernelGGL(kv4_read_kernel<128>, dim3(a.Hkv * n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv4_read_kernel<64>, dim3(a.Hkv * n), dim3(128), 0, st, a);
}

// ---- one token per request ------------------------------------------------------------------------------------------------
// Half a wave a (row, head)'s key and half its value where head_dim is 64, a wave each where it is 128: a lane is a byte of
// codes, 16 lanes a group.
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xf, 0xf, false));   // rotations within 16 lanes
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xf, 0xf, false));
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x122, 0xf, 0xf, false));
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x121, 0xf, 0xf, false));
}

template <int HD>
__global__ __launch_bounds__(HD) void kv4_append_kernel(Kv4RowsArgs a) {
    using F = Kv4<HD>;
    const int hk = blockIdx.x, row = blockIdx.y;
    const bool is_v = threadIdx.x >= HD / 2;
    const int j = threadIdx.x & (HD / 2 - 1), g = j >> 4;
    const uint32_t x = *(const uint32_t *)((is_v ? a.v : a.k) + (size_t)row * a.row_stride + hk * HD + 2 * j);
    const int pos = a.ctx_lens[row];
    if (pos == -1) return;   // a row without a request
    int blk = -1;
    if (pos >= 0 && (pos >> 4) < a.max_blk) blk = a.tables[(size_t)row * a.max_blk + (pos >> 4)];
    if ((unsigned)blk >= (unsigned)a.n_blocks) {
        if (threadIdx.x == 0 && hk == 0) atomicOr(a.err_flag, 2);
        return;
    }
    const int t = pos & 15;
    const uint32_t b = kv4_scale_byte(max_of_16(absmax2(0, x)));
    const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, x), kv4_scale(min(b, 252u)), 0);
    uint8_t *dst = a.pool + ((size_t)blk * a.Hkv + hk) * F::BYTES;
    dst[is_v ? F::v_byte(t, j & 15, g) : F::k_chunk(g, t) + (j & 15)] = (uint8_t)c;
    if ((j & 15) == 0) dst[is_v ? F::v_scale(g, t) : F::k_scale(g, t)] = (uint8_t)b;
}

void launch_kv4_append(hipStream_t st, const Kv4RowsArgs &a) {
    if (a.B <= 0) return;
    if (a.hd == 128) hipLaunchKernelGGL(kv4_append_kernel<128>, dim3(a.Hkv, a.B), dim3(128), 0, st, a);
    else hipLaunchKernelGGL(kv4_append_kernel<64>, dim3(a.Hkv, a.B), dim3(64), 0, st, a);
}

// ---- attention: what both kinds share ---------------------------------------------------------------------------------------
// Scores.  K stays as it is in the cache: the matrix instruction with block scales takes 4-bit rows, 32 dims and their scale a
// lane.  The query goes in as two e4m3 terms, q = hi + lo / 16: of a bf16's eight significant bits hi takes four and lo the
// rest, exactly, down to 2^-20 of the largest of its 32 dims (smaller ones lose bits there).  Two such products cost what one
// of bf16 operands does, and K needs no conversion.  Their sums are good to 2e-5 of sum|q k| (measured), far less than what
// rounding the softmax weights to bf16 does.
// A scale of 255 makes every score of its token NaN, as a NaN in a bf16 cache would.

// 16 dims of the query (as floats) -> 16 bytes each of hi and lo; mul: the power of two that takes the group's largest into
// [128, 256)
__device__ __forceinline__ void q_split(const float *x, float mul, int *hi, int *lo) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float a = x[4 * w] * mul, b = x[4 * w + 1] * mul, c = x[4 * w + 2] * mul, d = x[4 * w + 3] * mul;
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
        const auto ab = __builtin_amdgcn_cvt_pk_f32_fp8(p, false), cd = __builtin_amdgcn_cvt_pk_f32_fp8(p, true);
        int r = __builtin_amdgcn_cvt_pk_fp8_f32((a - ab[0]) * 16.f, (b - ab[1]) * 16.f, 0, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32((c - cd[0]) * 16.f, (d - cd[1]) * 16.f, r, true);
        hi[w] = p;
        lo[w] = r;
    }
}
__device__ __forceinline__ float absmax16(const float *x) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
    return m;
}
__device__ __forceinline__ bool all_finite16(const float *x) {
    bool f = true;
#pragma unroll
    for (int i = 0; i < 16; ++i) f = f && fabsf(x[i]) < __builtin_huge_valf();   // false for a NaN too
    return f;
}
// Exponent field of the largest magnitude; 255 where it is not finite.
__device__ __forceinline__ uint32_t q_exponent(float amax) { return min(max(as_bits(amax) >> 23, 12u), 255u); }
__device__ __forceinline__ float q_mul(uint32_t e) { return as_float((261u - min(e, 254u)) << 23); }
__device__ __forceinline__ int q_hi_scale(uint32_t e) { return e == 255u ? 255 : (int)e - 7; }
__device__ __forceinline__ int q_lo_scale(uint32_t e) { return e == 255u ? 255 : (int)e - 11; }

__device__ __forceinline__ void load16(const bf16_t *p, float *x) {
    const bf16x8 a = ld_bf16x8(p), b = ld_bf16x8(p + 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = (float)a[i];
        x[8 + i] = (float)b[i];
    }
}

// Four tokens of a dim pair (a dword of codes, a dword of scale bytes) -> the even dim's four values and the odd dim's.
struct V4 { u32x2_t even, odd; };
__device__ __forceinline__ V4 v_values(uint32_t codes, uint32_t scales) {
    const uint32_t x0 = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, kv4_scale_of<0>(scales), 0));
    const uint32_t x1 = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, kv4_scale_of<1>(scales), 1));
    const uint32_t x2 = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, kv4_scale_of<2>(scales), 2));
    const uint32_t x3 = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, kv4_scale_of<3>(scales), 3));
    return {u32x2_t{__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u)},
            u32x2_t{__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u)}};
}
__device__ __forceinline__ bf16x8 join8(u32x2_t a, u32x2_t b) { return __builtin_bit_cast(bf16x8, u32x4_t{a[0], a[1], b[0], b[1]}); }

// Eight columns (a multiple of 8) of an output row.
__device__ __forceinline__ bf16_t *kv4_out(const Kv4AttnArgs &a, int row, int col) {
    return a.out_Mt ? a.out + packed_offset(a.out_row0 + row, col, a.out_Mt) + (col & 7) : a.out + (size_t)row * a.out_stride + col;
}

// ---- attention: one row per request -----------------------------------------------------------------------------------------
// Workgroup = (kv head, request, chunk of the context); its four waves take a quarter of the chunk's tokens each, 32 (two
// blocks) at a time; the G query heads of the kv head are the columns of 16 x 16 tiles.  S^T = K Q^T, then O^T = V^T P^T: a
// lane's eight scores (tokens 4h..4h+3 of both blocks) are the contraction slice that it supplies to the second product.
template <int HD>
__global__ __launch_bounds__(256, 2) void kv4_decode_kernel(Kv4AttnArgs a) {
    using F = Kv4<HD>;
    constexpr int G = F::G;
    extern __shared__ float smem_kv4[];
    const int hk = blockIdx.x, b = blockIdx.z, chunk = blockIdx.y;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c16 = lane & 15, h = lane >> 4;
    const int Gq = a.Hq / a.Hkv;
    float *s_o = smem_kv4;               // [4][HD][Gq]
    float *s_m = smem_kv4 + 4 * HD * Gq; // [4][Gq] maxima, [4][Gq] sums
    float *s_l = s_m + 4 * Gq;

    int n_keys = a.ctx_lens[b] + 1;
    if (n_keys < 0 || n_keys > a.max_ctx) {
        if (tid == 0 && chunk == 0 && hk == 0) atomicOr(a.err_flag, 8);
        n_keys = min(max(n_keys, 0), a.max_ctx);
    }
    if (n_keys == 0) {   // a row without a request
        if (a.n_chunks == 1)
            for (int c = tid * 8; c < Gq * HD; c += 2048) *(u32x4_t *)kv4_out(a, b, hk * Gq * HD + c) = u32x4_t{0, 0, 0, 0};
        return;
    }
    if (chunk * a.chunk >= n_keys) return;
    const int per_wave = a.chunk / 4;
    const int t0 = chunk * a.chunk + wave * per_wave, t1 = min(t0 + per_wave, n_keys);

    // the query's terms: bytes 0-15 of a lane's operand are dims 16h.., bytes 16-31 dims 64 + 16h..
    i32x8 qh, ql;
    int qh_scale, ql_scale;
    {
        float x[2][16];
        const bool col = c16 < Gq;
        const bf16_t *qp = a.q + (size_t)b * a.q_stride + (size_t)(hk * Gq + (col ? c16 : 0)) * HD + 16 * h;
        load16(qp, x[0]);
        if (HD == 128) load16(qp + 64, x[1]);
        uint32_t e[2];
        int hi[8], lo[8];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            if (HD == 64 && p == 1) {
                e[1] = 127;
#pragma unroll
                for (int w = 0; w < 4; ++w) hi[4 + w] = lo[4 + w] = 0;
                break;
            }
            if (!col)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[p][i] = 0.f;
            uint32_t mine = all_finite16(x[p]) ? as_bits(absmax16(x[p])) : 0x7f800000u;
            mine = max(mine, (uint32_t)__shfl_xor((int)mine, 16, 64));
            e[p] = q_exponent(as_float(mine));
            q_split(x[p], q_mul(e[p]), hi + 4 * p, lo + 4 * p);
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            qh[w] = hi[w];
            ql[w] = lo[w];
        }
        // lane quarter h gives the scale of dims 32h..: those of the first 64 are in e[0] of the quarters 2h, of the second in e[1]
        const uint32_t e0 = (uint32_t)__shfl((int)e[0], (2 * (h & 1)) * 16 + c16, 64), e1 = (uint32_t)__shfl((int)e[1], (2 * (h & 1)) * 16 + c16, 64);
        const uint32_t mine = h < 2 ? e0 : e1;
        qh_scale = q_hi_scale(mine);
        ql_scale = q_lo_scale(mine);
    }

    float m_run = NEG_INF, l_run = 0.f;
    f32x4 o[2 * G];   // (group, parity of the dim)
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float sc = a.scale_log2;
    const int32_t *tab = a.tables + (size_t)b * a.max_blk;
    const uint8_t *head = a.pool + (size_t)hk * F::BYTES;
    const size_t blk_stride = (size_t)a.Hkv * F::BYTES;

    for (int base = t0; base < t1; base += 32) {
        u32x4_t kc[2];
        typedef uint32_t gvec __attribute__((ext_vector_type(G)));
        uint32_t ks[2];
        gvec vc[2], vs[2];
        bool ok[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int tok = base + 16 * u;
            int blk = tok < n_keys ? tab[tok >> 4] : -1;
            ok[u] = (unsigned)blk < (unsigned)a.n_blocks;
            if (tok < n_keys && !ok[u] && lane == 0) atomicOr(a.err_flag, 2);
            const uint8_t *p = head + (size_t)(ok[u] ? blk : 0) * blk_stride;
            kc[u] = *(const u32x4_t *)(p + F::k_chunk(h & (G - 1), c16));
            ks[u] = p[F::k_scale(h & (G - 1), c16)];
            vc[u] = *(const gvec *)(p + F::V + (h * 16 + c16) * (4 * G));
            vs[u] = *(const gvec *)(p + F::VS + h * (4 * G));
        }
        f32x4 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const i32x8 k = {(int)kc[u][0], (int)kc[u][1], (int)kc[u][2], (int)kc[u][3], 0, 0, 0, 0};
            s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            s[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, ql, s[u], 4, 0, 0, (int)ks[u], 0, ql_scale);
            s[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, qh, s[u], 4, 0, 0, (int)ks[u], 0, qh_scale);
            const int nv = ok[u] ? min(max(n_keys - (base + 16 * u + 4 * h), 0), 4) : 0;   // valid tokens of this lane's four
            if (nv < 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i >= nv) s[u][i] = NEG_INF;
                const uint32_t keep = nv == 0 ? 0u : 0xffffffffu >> (32 - 8 * nv);
#pragma unroll
                for (int g = 0; g < G; ++g) vs[u][g] &= keep;   // what is behind the context may read as NaN
            }
        }
        float m_tile = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        m_tile = fmaxf(m_tile, __shfl_xor(m_tile, 16, 64));
        m_tile = fmaxf(m_tile, __shfl_xor(m_tile, 32, 64));
        const float m_new = fmaxf(m_run, m_tile), m_safe = m_new == NEG_INF ? 0.f : m_new;
        const float ms = m_safe * sc;
        bf16x8 pf;   // the weights are rounded to bf16 for the second product (at most 2^-9 each); their sum is of the unrounded ones
        float psum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], sc, -ms));
            psum += p;
            pf[i] = (bf16_t)p;
        }
        if (__any(m_new != m_run)) {
            const float alpha = __builtin_amdgcn_exp2f((m_run - m_safe) * sc);
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) o[i] = o[i] * alpha;
            m_run = m_new;
        }
        l_run += psum;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const V4 va = v_values(vc[0][g], vs[0][g]), vb = v_values(vc[1][g], vs[1][g]);
            o[2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join8(va.even, vb.even), pf, o[2 * g], 0, 0, 0);
            o[2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join8(va.odd, vb.odd), pf, o[2 * g + 1], 0, 0, 0);
        }
    }
    l_run += __shfl_xor(l_run, 16, 64);
    l_run += __shfl_xor(l_run, 32, 64);

    // the four waves, in order
    if (c16 < Gq) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s_o[(wave * HD + 32 * g + 2 * (4 * h + i)) * Gq + c16] = o[2 * g][i];
                s_o[(wave * HD + 32 * g + 2 * (4 * h + i) + 1) * Gq + c16] = o[2 * g + 1][i];
            }
        if (h == 0) {
            s_m[wave * Gq + c16] = m_run;
            s_l[wave * Gq + c16] = l_run;
        }
    }
    __syncthreads();
    for (int idx = tid; idx < Gq * HD; idx += 256) {
        const int gg = idx / HD, d = idx % HD;
        const float mx = fmaxf(fmaxf(s_m[gg], s_m[Gq + gg]), fmaxf(s_m[2 * Gq + gg], s_m[3 * Gq + gg])), ms = mx == NEG_INF ? 0.f : mx;
        float acc = 0.f, l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float e = __builtin_amdgcn_exp2f((s_m[w * Gq + gg] - ms) * sc);
            acc += s_o[(w * HD + d) * Gq + gg] * e;
            l += s_l[w * Gq + gg] * e;
        }
        if (a.n_chunks == 1) {
            *kv4_out(a, b, (hk * Gq + gg) * HD + d) = (bf16_t)(l == 0.f ? 0.f : acc / l);   // (0: every block of the row was refused)
        } else {
            const size_t pi = ((size_t)b * a.Hq + hk * Gq + gg) * a.n_chunks + chunk;
            a.part_o[pi * HD + d] = acc;
            if (d == 0) {
                a.part_ml[pi * 2] = mx;
                a.part_ml[pi * 2 + 1] = l;
            }
        }
    }
}

// The pieces of a row (chunks of its context, or key ranges of a prompt's row), in order.  n: pieces of this row.
template <int HD>
__global__ __launch_bounds__(HD) void kv4_merge_kernel(Kv4AttnArgs a) {
    const int hq = blockIdx.x, row = blockIdx.y, d = threadIdx.x;
    int n = a.n_chunks;
    if (a.ctx_lens) {
        const int keys = min(max(a.ctx_lens[row] + 1, 0), a.max_ctx);
        n = (keys + a.chunk - 1) / a.chunk;
    }
    const size_t p0 = ((size_t)row * a.Hq + hq) * a.n_chunks;
    float mx = NEG_INF;
    for (int c = 0; c < n; ++c) mx = fmaxf(mx, a.part_ml[2 * (p0 + c)]);
    const float ms = mx == NEG_INF ? 0.f : mx;
    float acc = 0.f, l = 0.f;
    for (int c = 0; c < n; ++c) {
        const float e = __builtin_amdgcn_exp2f((a.part_ml[2 * (p0 + c)] - ms) * a.scale_log2);
        acc += a.part_o[(p0 + c) * HD + d] * e;
        l += a.part_ml[2 * (p0 + c) + 1] * e;
    }
    *kv4_out(a, row, hq * HD + d) = (bf16_t)(l == 0.f ? 0.f : acc / l);
}

static void launch_kv4_merge(hipStream_t st, const Kv4AttnArgs &a, int rows) {
    if (a.hd == 128) hipLaunchKernelGGL(kv4_merge_kernel<128>, dim3(a.Hq, rows), dim3(128), 0, st, a);
    else hipLaunchKernelGGL(kv4_merge_kernel<64>, dim3(a.Hq, rows), dim3(64), 0, st, a);
}

// Tokens of a chunk: 512, fewer where the launch would not give every compute unit two workgroups.  From the sizes alone.
int kv4_chunk(int B, int Hkv, int max_ctx) {
    int c = 512;
    while (c > 128 && (int64_t)B * Hkv * ((max_ctx + c - 1) / c) < 512) c /= 2;
    return c;
}

void launch_kv4_decode(hipStream_t st, const Kv4AttnArgs &args) {
    Kv4AttnArgs a = args;
    if (a.B <= 0) return;
    a.chunk = kv4_chunk(a.B, a.Hkv, a.max_ctx);
    a.n_chunks = (a.max_ctx + a.chunk - 1) / a.chunk;
    const int Gq = a.Hq / a.Hkv;
    const size_t lds = (size_t)(4 * a.hd * Gq + 8 * Gq) * sizeof(float);
    const dim3 grid(a.Hkv, a.n_chunks, a.B);
    if (a.hd == 128) hipLaunchKernelGGL(kv4_decode_kernel<128>, grid, dim3(256), lds, st, a);
    else hipLaunchKernelGGL(kv4_decode_kernel<64>, grid, dim3(256), lds, st, a);
    if (a.n_chunks > 1) launch_kv4_merge(st, a, a.B);
}

// ---- attention: prompts and chunks of them ----------------------------------------------------------------------------------
// Workgroup = (kv head, 128 columns, key range): a column is a (row, query head) pair, the G heads of the kv head beside each
// other, so that 128 columns are 128 / G neighbouring rows and a chunk of few rows still fills the tiles.  Wave w owns 32
// columns.  Keys come 64 (four blocks) at a time through two LDS buffers: K as its codes, V converted once for the four waves.
// V in LDS: per block two halves [hd][8 tokens], half i the quads i and 2 + i, the dims of a group even ones first: the order
// in which a lane holds its scores, so the weights need no exchange between lanes.
#define KV4_COLS 128
template <int HD> struct Kv4Lds {
    static constexpr int K = 4 * 8 * HD, KS = 4 * (HD / 2), V = 4 * 2 * HD * 16, TILE = K + KS + V;
};

__device__ __forceinline__ int kv4_units(int rows, int G) { return (rows * G + KV4_COLS - 1) / KV4_COLS; }

template <int HD>
__global__ __launch_bounds__(256, 2) void kv4_prefill_kernel(Kv4AttnArgs a) {
    using F = Kv4<HD>;
    using L = Kv4Lds<HD>;
    constexpr int G = F::G, KSTEP = HD / 64, DT = HD / 32;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem_kv4p[];
    const int hk = blockIdx.x % a.Hkv, split = blockIdx.y, Gq = a.Hq / a.Hkv;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c32 = lane & 31, h = lane >> 5;

    int unit = blockIdx.x / a.Hkv, req = 0, units = 0;
    for (; req < a.seq.n_req; ++req) {
        units = kv4_units(a.seq.cu[req + 1] - a.seq.cu[req], Gq);
        if (unit < units) break;
        unit -= units;
    }
    if (req >= a.seq.n_req) return;
    const int row0 = a.seq.cu[req], len = a.seq.cu[req + 1] - row0, prior = a.seq.start[req];
    const int col0 = (units - 1 - unit) * KV4_COLS, n_cols = len * Gq;   // the longest first
    const int col = col0 + 32 * wave + c32;
    const bool valid = col < n_cols;
    const int colc = min(col, n_cols - 1), row = colc / Gq, hq = hk * Gq + colc % Gq;
    const int q_pos = prior + row;
    const int w_min = prior + min(col0 + 32 * wave, n_cols - 1) / Gq, w_max = prior + min(col0 + 32 * wave + 31, n_cols - 1) / Gq;
    const int kv_end = prior + min(col0 + KV4_COLS - 1, n_cols - 1) / Gq + 1;
    const int n_tiles = (kv_end + 63) >> 6;
    // this workgroup's share of the key tiles
    const int kt0 = (int)((int64_t)n_tiles * split / a.n_chunks), kt1 = (int)((int64_t)n_tiles * (split + 1) / a.n_chunks);

    // the query's terms: of each 64 dims bytes 0-15 are dims 16h.., bytes 16-31 dims 32 + 16h..
    i32x8 qh[KSTEP], ql[KSTEP];
    int qhs[KSTEP], qls[KSTEP];
    {
        const bf16_t *qp = a.q + (size_t)(row0 + row) * a.q_stride + (size_t)hq * HD + 16 * h;
#pragma unroll
        for (int s = 0; s < KSTEP; ++s) {
            float x[2][16];
            uint32_t e[2];
            int hi[8], lo[8];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                load16(qp + 64 * s + 32 * p, x[p]);
                uint32_t mine = all_finite16(x[p]) ? as_bits(absmax16(x[p])) : 0x7f800000u;
                mine = max(mine, (uint32_t)__shfl_xor((int)mine, 32, 64));
                e[p] = q_exponent(as_float(mine));
                q_split(x[p], q_mul(e[p]), hi + 4 * p, lo + 4 * p);
            }
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                qh[s][w] = hi[w];
                ql[s][w] = lo[w];
            }
            const uint32_t mine = h ? e[1] : e[0];
            qhs[s] = q_hi_scale(mine);
            qls[s] = q_lo_scale(mine);
        }
    }

    float m_run = NEG_INF, l_run = 0.f;
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    const float sc = a.scale_log2;
    const int32_t *tab = a.tables + (size_t)req * a.max_blk;

    // A wave brings one block of a key tile: a lane HD/8 bytes of K's codes, the codes and scales of two V units (quads v_half
    // and 2 + v_half, dim pair vj, UG groups from vg on), and the lanes of the first HD/8 bytes of K's scales.
    constexpr int UG = G / 2;   // groups of a lane's V unit
    const int vj = lane & 15, vg = ((lane >> 4) & 1) * UG, v_half = lane >> 5;
    // A value that is not finite must not reach the rows before it, whose weight of it is zero: where a scale of V says so, the
    // token's scores are made NaN instead, which only the rows that see it take.
    typedef uint32_t kvec __attribute__((ext_vector_type(HD / 32)));
    typedef uint32_t vvec __attribute__((ext_vector_type(UG)));
    kvec rk;
    uint32_t rks = 0;
    vvec rv[2], rs[2];
    auto fetch = [&](int kt) {
        const int tok0 = kt * 64 + 16 * wave;
        const int blk = tok0 < kv_end ? tab[tok0 >> 4] : -1;
        const bool ok = (unsigned)blk < (unsigned)a.n_blocks;
        if (tok0 < kv_end && !ok && lane == 0) atomicOr(a.err_flag, 2);
        const uint8_t *p = a.pool + ((size_t)(ok ? blk : 0) * a.Hkv + hk) * F::BYTES;
        rk = ((const kvec *)p)[lane];
        if (lane < HD / 8) rks = ok ? ((const uint32_t *)(p + F::KS))[lane] : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int q = v_half + 2 * u;
            rv[u] = *(const vvec *)(p + F::V + ((q * 16 + vj) * G + vg) * 4);
            rs[u] = *(const vvec *)(p + F::VS + (q * G + vg) * 4);
            const int nv = ok ? min(max(kv_end - (tok0 + 4 * q), 0), 4) : 0;   // (what is behind the context may read as NaN)
            const uint32_t keep = nv == 0 ? 0u : 0xffffffffu >> (32 - 8 * nv);
#pragma unroll
            for (int g = 0; g < UG; ++g) rs[u][g] &= keep;
        }
    };
    auto put = [&](int buf) {
        uint8_t *t = smem_kv4p + buf * L::TILE;
        ((kvec *)(t + wave * (8 * HD)))[lane] = rk;
        uint8_t *scales = t + L::K + wave * (HD / 2);
        if (lane < HD / 8) ((uint32_t *)scales)[lane] = rks;
        uint32_t bad[2] = {0, 0};   // bytes of 255
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int g = 0; g < UG; ++g) bad[u] |= ((rs[u][g] & 0x7f7f7f7fu) + 0x01010101u) & rs[u][g] & 0x80808080u;
        if (__any((bad[0] | bad[1]) != 0)) {
            for (int u = 0; u < 2; ++u) {
                const uint32_t ff = (bad[u] >> 7) * 255u;
#pragma unroll
                for (int g = 0; g < UG; ++g) rs[u][g] &= ~ff;
                for (int i = 0; i < 4; ++i)
                    if ((ff >> (8 * i)) & 1) scales[4 * (v_half + 2 * u) + i] = 255;   // of group 0, after the wave's own store above
            }
        }
        bf16x8 *v = (bf16x8 *)(t + L::K + L::KS) + (wave * 2 + v_half) * HD;
#pragma unroll
        for (int g = 0; g < UG; ++g) {
            const V4 x = v_values(rv[0][g], rs[0][g]), y = v_values(rv[1][g], rs[1][g]);
            v[32 * (vg + g) + vj] = join8(x.even, y.even);
            v[32 * (vg + g) + 16 + vj] = join8(x.odd, y.odd);
        }
    };

    if (kt0 < kt1) {
        fetch(kt0);
        put(0);
    }
    __syncthreads();
    for (int kt = kt0; kt < kt1; ++kt) {
        if (kt + 1 < kt1) fetch(kt + 1);
        const int kv0 = kt * 64;
        const uint8_t *t = smem_kv4p + ((kt - kt0) & 1) * L::TILE;
        if (kv0 <= w_max) {
            f32x16 st[2];
#pragma unroll
            for (int t2 = 0; t2 < 2; ++t2) {
#pragma unroll
                for (int i = 0; i < 16; ++i) st[t2][i] = 0.f;
                const int blk = 2 * t2 + (c32 >> 4), tok = c32 & 15;
#pragma unroll
                for (int s = 0; s < KSTEP; ++s) {
                    const u32x4_t kc = *(const u32x4_t *)(t + blk * (8 * HD) + F::k_chunk(2 * s + h, tok));
                    const int ks = t[L::K + blk * (HD / 2) + (2 * s + h) * 16 + tok];
                    const i32x8 k = {(int)kc[0], (int)kc[1], (int)kc[2], (int)kc[3], 0, 0, 0, 0};
                    st[t2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, ql[s], st[t2], 4, 0, 0, ks, 0, qls[s]);
                    st[t2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k, qh[s], st[t2], 4, 0, 0, ks, 0, qhs[s]);
                }
            }
            if (kv0 + 63 > w_min) {   // only tiles that touch the diagonal need the mask
#pragma unroll
                for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (kv0 + 32 * t2 + (i >> 2) * 8 + 4 * h + (i & 3) > q_pos) st[t2][i] = NEG_INF;
            }
            float m_tile = NEG_INF;
#pragma unroll
            for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
                for (int i = 0; i < 16; ++i) m_tile = fmaxf(m_tile, st[t2][i]);
            {
                const auto sw = __builtin_amdgcn_permlane32_swap(as_bits(m_tile), as_bits(m_tile), false, false);
                m_tile = fmaxf(as_float((uint32_t)sw[0]), as_float((uint32_t)sw[1]));
            }
            const float m_new = fmaxf(m_run, m_tile), m_safe = m_new == NEG_INF ? 0.f : m_new;
            if (__any(m_new != m_run)) {
                const float alpha = __builtin_amdgcn_exp2f((m_run - m_safe) * sc);
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha;
                m_run = m_new;
            }
            const float ms = m_safe * sc;
            const bf16x8 *v = (const bf16x8 *)(t + L::K + L::KS);
#pragma unroll
            for (int b4 = 0; b4 < 4; ++b4) {
                bf16x8 pf;   // rounded to bf16 for the product; the sum is of the unrounded weights
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(st[b4 >> 1][8 * (b4 & 1) + i], sc, -ms));
                    l_run += p;
                    pf[i] = (bf16_t)p;
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[(b4 * 2 + h) * HD + 32 * dt + c32], pf, o[dt], 0, 0, 0);
            }
        }
        if (kt + 1 < kt1) put((kt + 1 - kt0) & 1);
        __syncthreads();
    }
    l_run += __shfl_xor(l_run, 32, 64);
    if (!valid) return;
    // rows of o: register i of tile dt is dim 32 dt + 2 (8 (i / 4 & 1) + 4 h + i % 4) + i / 8
    const int out_row = row0 + row;
    if (a.n_chunks == 1) {
        const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                bf16x8 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[2 * i] = (bf16_t)(o[dt][4 * j + i] * inv);
                    w[2 * i + 1] = (bf16_t)(o[dt][8 + 4 * j + i] * inv);
                }
                *(bf16x8 *)kv4_out(a, out_row, hq * HD + 32 * dt + 16 * j + 8 * h) = w;
            }
        return;
    }
    const size_t pi = ((size_t)out_row * a.Hq + hq) * a.n_chunks + split;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x4 *dst = (f32x4 *)(a.part_o + pi * HD + 32 * dt + 16 * j + 8 * h);
            dst[0] = f32x4{o[dt][4 * j], o[dt][8 + 4 * j], o[dt][4 * j + 1], o[dt][8 + 4 * j + 1]};
            dst[1] = f32x4{o[dt][4 * j + 2], o[dt][8 + 4 * j + 2], o[dt][4 * j + 3], o[dt][8 + 4 * j + 3]};
        }
    if (h == 0) {
        a.part_ml[2 * pi] = m_run;
        a.part_ml[2 * pi + 1] = l_run;
    }
}

// Key ranges that a launch's rows are cut into, from the sizes alone: as many as give two workgroups to every compute unit, of 256 keys at least.
int kv4_prefill_splits(const SeqInfo &seq, int Hq, int Hkv, int *units_out) {
    int units = 0, longest = 0;
    for (int r = 0; r < seq.n_req; ++r) {
        const int len = seq.cu[r + 1] - seq.cu[r];
        if (len <= 0) continue;
        units += (len * (Hq / Hkv) + KV4_COLS - 1) / KV4_COLS;
        longest = std::max(longest, seq.start[r] + len);
    }
    *units_out = units;
    if (units == 0) return 1;
    return std::max(1, std::min(KV4_SPLIT_WGS / (units * Hkv), longest / 256));
}

void launch_kv4_prefill(hipStream_t st, const Kv4AttnArgs &args) {
    Kv4AttnArgs a = args;
    int units = 0;
    a.n_chunks = kv4_prefill_splits(a.seq, a.Hq, a.Hkv, &units);
    if (units == 0) return;
    a.ctx_lens = nullptr;
    const dim3 grid(a.Hkv * units, a.n_chunks);
    if (a.hd == 128) hipLaunchKernelGGL(kv4_prefill_kernel<128>, grid, dim3(256), 2 * Kv4Lds<128>::TILE, st, a);
    else hipLaunchKernelGGL(kv4_prefill_kernel<64>, grid, dim3(256), 2 * Kv4Lds<64>::TILE, st, a);
    if (a.n_chunks > 1) launch_kv4_merge(st, a, a.seq.cu[a.seq.n_req]);
}
