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
#include <climits>
#include <type_traits>

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
// Byte I of four as a scale: one instruction (the compiler takes a shift and a mask).
template <int I>
__device__ __forceinline__ float kv4_scale_of(uint32_t four) {
    uint32_t r;
    const uint32_t sh = 23;
    if (I == 0) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(sh), "v"(four));
    if (I == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(sh), "v"(four));
    if (I == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(sh), "v"(four));
    if (I == 3) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(sh), "v"(four));
    return as_float(r);
}

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
// The last of n (1 to 64) ascending numbers, the first of them 0, that is at most u: every lane looks at one.  (The last: an empty
// run begins where the next one does.)
__device__ __forceinline__ int last_at_most(const int32_t *first, int n, int u) {
    const int lane = threadIdx.x & 63;
    return 63 - __builtin_clzll(__ballot(lane < n && first[lane] <= u));
}
// The u-th block of the run of blocks that the requests' tokens touch (u less than their number).
__device__ __forceinline__ RunBlock run_block(const Kv4RowsArgs &a, int u) {
    const int r = last_at_most(a.first, a.seq.n_req, u);
    return {r, (a.seq.start[r] >> 4) + u - a.first[r]};
}
static int run_blocks(Kv4RowsArgs &a) {
    int n = 0;
    for (int r = 0; r < a.seq.n_req; ++r) {
        const int len = a.seq.cu[r + 1] - a.seq.cu[r];
        a.first[r] = n;
        if (len > 0) n += ((a.seq.start[r] + len - 1) >> 4) - (a.seq.start[r] >> 4) + 1;
    }
    return n;
}

template <int HD>
__global__ __launch_bounds__(2 * HD) void kv4_write_kernel(Kv4RowsArgs a) {
    using F = Kv4<HD>;
    __shared__ __attribute__((aligned(16))) uint8_t s_v[8 * HD];
    const int hk = blockIdx.x % a.Hkv, tid = threadIdx.x;
    const RunBlock u = run_block(a, blockIdx.x / a.Hkv);
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
    const RunBlock u = run_block(a, blockIdx.x / a.Hkv);
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

void launch_kv4_write(hipStream_t st, const Kv4RowsArgs &args) {
    Kv4RowsArgs a = args;
    const int n = run_blocks(a);
    if (n <= 0) return;
    if (a.hd == 128) hipLaunchKernelGGL(kv4_write_kernel<128>, dim3(a.Hkv * n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv4_write_kernel<64>, dim3(a.Hkv * n), dim3(128), 0, st, a);
}

void launch_kv4_read(hipStream_t st, const Kv4RowsArgs &args) {
    Kv4RowsArgs a = args;
    const int n = run_blocks(a);
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
    if (pos == -1 || pos >= a.max_pos) return;   // a row without a request, or one without a rotary position (reported by the rotation)
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
// lane.  The query, times log2(e) / sqrt(hd), goes in as three terms of 6 bits (e2m3: multiples of 1/8 below 2, 1/4 below 4, 1/2
// up to 7.5), each a sixteenth of the one before: x = t0 + t1 / 16 + t2 / 256 in units of a power of two that takes the largest
// of the 32 dims into [3.875, 7.75).  What is left of x is at most 2^-12 units, 2^-13.9 of that largest: a dim 2^j below the largest keeps
// 13 - j bits, where a bf16 has 8.  The keys that it meets are themselves off by up to a fifth of the largest of their 32 dims; with
// channels as loud as keys have, the result moves by 1.4e-4 of itself (2-norm), a twelfth of its own rounding to bf16.  With 6-bit operands
// the instruction runs at four times the rate of bf16, so that three products take 3/4 of the time of bf16's, no element of K is
// converted, and the scores come out as the exponents that the softmax wants.  (Two e4m3 terms hold a bf16 exactly, at half the
// rate: 16384 prompt rows 1810 us, 1800 with these.)
// A scale of 255 makes every score of its token NaN, as a NaN in a bf16 cache would; so do not finite queries.
typedef uint32_t u32x6_t __attribute__((ext_vector_type(6)));
struct QTerms {
    u32x6_t t[3];
    int scale;   // bytes 0, 1, 2: of the terms
};
__device__ __forceinline__ i32x8 operand(u32x6_t v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], (int)v[4], (int)v[5], 0, 0}; }
__device__ __forceinline__ i32x8 operand(u32x4_t v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }
// Of 32 dims (p; times c): even and odd ones apart, as the conversion takes them.
__device__ __forceinline__ QTerms q_terms(const bf16_t *p, float c) {
    f32x16 x, y;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x8 v = ld_bf16x8(p + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[4 * i + j] = (float)v[2 * j] * c;
            y[4 * i + j] = (float)v[2 * j + 1] * c;
            m = max(max(m, as_bits(x[4 * i + j]) & 0x7fffffffu), as_bits(y[4 * i + j]) & 0x7fffffffu);
        }
    }
    const bool finite = m < 0x7f800000u;
    const int e = max((int)((m + 0x00080000u) >> 23), 16) - 2;   // 1.9375 * 2^n and more count as 2^(n+1)
    QTerms q;
    q.scale = finite ? e | (e - 4) << 8 | (e - 8) << 16 : 0xffffff;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const float s = as_float((uint32_t)(e - 4 * k) << 23);
        q.t[k] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(x, y, s);
        if (k < 2) {
            typedef float f32x32 __attribute__((ext_vector_type(32)));
            const f32x32 r = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q.t[k], s);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] -= r[2 * i];
                y[i] -= r[2 * i + 1];
            }
        }
    }
    return q;
}

// Four tokens of a dim pair (a dword of codes, a dword of scale bytes) -> the even dim's four values and the odd dim's.
struct V4 { u32x2_t even, odd; };
struct V4Steps {   // in three steps, for code that puts other instructions between them
    float s[4];
    uint32_t x[4];
    __device__ __forceinline__ void scales(uint32_t four) { s[0] = kv4_scale_of<0>(four), s[1] = kv4_scale_of<1>(four), s[2] = kv4_scale_of<2>(four), s[3] = kv4_scale_of<3>(four); }
    // the largest of them and `m`, as bits: 0x7f800000 where one is 255
    __device__ __forceinline__ uint32_t top(uint32_t m) const { return max(max(max(max(m, as_bits(s[0])), as_bits(s[1])), as_bits(s[2])), as_bits(s[3])); }
    __device__ __forceinline__ void convert(uint32_t codes) {
        x[0] = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s[0], 0)), x[1] = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s[1], 1));
        x[2] = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s[2], 2)), x[3] = as_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s[3], 3));
    }
    __device__ __forceinline__ V4 values() const {
        return {u32x2_t{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u)},
                u32x2_t{__builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)}};
    }
};
__device__ __forceinline__ V4 v_values(uint32_t codes, uint32_t scales) {
    V4Steps v;
    v.scales(scales);
    v.convert(codes);
    return v.values();
}
__device__ __forceinline__ bf16x8 join8(u32x2_t a, u32x2_t b) { return __builtin_bit_cast(bf16x8, u32x4_t{a[0], a[1], b[0], b[1]}); }

// Eight columns (a multiple of 8) of an output row.
__device__ __forceinline__ bf16_t *kv4_out(const Kv4AttnArgs &a, int row, int col) {
    return a.out_Mt ? a.out + packed_offset(a.out_row0 + row, col, a.out_Mt) + (col & 7) : a.out + (size_t)row * a.out_stride + col;
}

// Weights are relative to a reference that is moved to the running maximum once a score is this far above it, so they are at most
// 2^4: a bf16 is as fine there as below 1, and the accumulators are rescaled in a few tiles of a long context instead of in two of
// five (16384 prompt rows 1800 -> 1694 us; the error against float64 0.0019 -> 0.0020 of the result).
#define KV4_REF_BEHIND 4.f

// ---- pieces of rows ---------------------------------------------------------------------------------------------------------
// A row of one head that several workgroups compute leaves a piece each: the weighted sum of values, relative to the piece's own
// maximum, that maximum and the sum of weights.  A workgroup joins the pieces of the heads of one kv head of one
// row, in order; a thread takes four dims.  Bound by round trips to memory: up to 8 pieces are asked for at once, more in eights
// behind a pass over the maxima (8B heads, 64 rows of up to 4096 tokens 4.6 us, a row in 32 pieces 4.8; a launch that does nothing
// is 2).
// Of row `row`: n pieces, the j-th of head g of the kv head's is piece at(g, j).
template <int HD, class At>
__device__ __forceinline__ void kv4_join(const Kv4AttnArgs &a, int hk, int row, int n, At at) {
    __shared__ float s[2 * 16];
    const int G = a.Hq / a.Hkv, hq0 = hk * G;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const float2 *ml = (const float2 *)a.part_ml;
    const f32x4 *po = (const f32x4 *)a.part_o;
    auto store = [&](int g, int d4, f32x4 acc, float l) {
        bf16x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (bf16_t)(l == 0.f ? 0.f : acc[j] / l);   // (0: an empty row, or every block of it refused)
        *(bf16x4 *)kv4_out(a, row, (hq0 + g) * HD + 4 * d4) = w;
    };
    if (n <= 8) {
        for (int i = tid; i < G * (HD / 4); i += 256) {
            const int g = i / (HD / 4), d4 = i % (HD / 4);
            f32x4 v[8];
            float2 m[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const size_t c = at(g, max(min(j, n - 1), 0));
                v[j] = po[c * (HD / 4) + d4];
                m[j] = ml[c];
            }
            float mx = NEG_INF, l = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) mx = fmaxf(mx, j < n ? m[j].x : NEG_INF);
            const float ms = mx == NEG_INF ? 0.f : mx;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) {
                    const float e = __builtin_amdgcn_exp2f(m[j].x - ms);
                    acc += v[j] * e;
                    l += m[j].y * e;
                }
            store(g, d4, acc, l);
        }
        return;
    }
    for (int g = wave; g < G; g += 4) {
        float mx = NEG_INF, l = 0.f;
        for (int c = lane; c < n; c += 64) mx = fmaxf(mx, ml[at(g, c)].x);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        const float ms = mx == NEG_INF ? 0.f : mx;
        for (int c = lane; c < n; c += 64) {
            const float2 v = ml[at(g, c)];
            l += v.y * __builtin_amdgcn_exp2f(v.x - ms);
        }
        l = wave_sum(l);
        if (lane == 0) {
            s[2 * g] = ms;
            s[2 * g + 1] = l;
        }
    }
    __syncthreads();
    for (int i = tid; i < G * (HD / 4); i += 256) {
        const int g = i / (HD / 4), d4 = i % (HD / 4);
        const float ms = s[2 * g];
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < n; c0 += 8) {
            f32x4 v[8];
            float m[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = min(c0 + j, n - 1);
                const size_t pc = at(g, c);
                v[j] = po[pc * (HD / 4) + d4];
                m[j] = ml[pc].x;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c0 + j < n) acc += v[j] * __builtin_amdgcn_exp2f(m[j] - ms);
        }
        store(g, d4, acc, s[2 * g + 1]);
    }
}

// ---- attention: one row per request -----------------------------------------------------------------------------------------
// The G query heads of a kv head are the columns of 16 x 16 tiles, the keys come 32 (two blocks) at a time, which a workgroup's
// waves take in turn.  S^T = K Q^T, then O^T = V^T P^T: a lane's eight scores (tokens 4h..4h+3 of both blocks) are the contraction
// slice that it supplies to the second product.  The 4.25 KB of the wave's next 32 tokens are asked for before the present ones are
// computed, from block ids that the wave holds (more of them in flight were slower: 64 rows of up to 8000 tokens 55, two further
// tiles 62 us).
// Workgroup = (kv head, row) or, CUT, (kv head, an equal share of the tokens of all rows): in units of UT tokens, counted by every
// wave for itself, row after row from wherever the share begins.  What of a row is not all of it leaves a piece.
__device__ __forceinline__ float max_of_quarters(float v) {   // over the four lanes of a column
    const auto x = __builtin_amdgcn_permlane16_swap(as_bits(v), as_bits(v), false, false);
    v = fmaxf(as_float((uint32_t)x[0]), as_float((uint32_t)x[1]));
    const auto y = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
    return fmaxf(as_float((uint32_t)y[0]), as_float((uint32_t)y[1]));
}

// units of UT tokens of a row of n
template <int UT> __device__ __forceinline__ int units_of(const Kv4AttnArgs &a, int n) { return (min(max(n, 0), a.max_ctx) + UT - 1) / UT; }

// The piece of a row that begins (or else ends, or is all) in workgroup wg.
__device__ __forceinline__ size_t kv4_piece(const Kv4AttnArgs &a, int hk, int wg, bool begins, int g) {
    return (((size_t)hk * a.wgs + wg) * 2 + begins) * (a.Hq / a.Hkv) + g;
}

template <int HD, int NW, bool CUT>
__global__ __launch_bounds__(64 * NW, NW == 4 && !CUT ? 4 : 2) void kv4_decode_kernel(Kv4AttnArgs a) {
    using F = Kv4<HD>;
    constexpr int G = F::G, NT = 64 * NW, UT = 32 * NW;
    typedef uint32_t gvec __attribute__((ext_vector_type(G)));
    extern __shared__ float smem_kv4[];
    const int hk = blockIdx.x, wg = blockIdx.y;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c16 = lane & 15, h = lane >> 4;
    const int Gq = a.Hq / a.Hkv;

    int row = wg, u0 = 0, left = INT_MAX;   // the first row, its first unit, and how many units the workgroup takes
    if constexpr (CUT) {
        // every wave by itself: a lane counts the units of `per` neighbouring rows, those of the lanes up to it are added up
        const int per = (a.B + 63) / 64, r0 = min(lane * per, a.B), r1 = min(r0 + per, a.B);
        int mine = 0;
        for (int r = r0; r < r1; ++r) {
            const int n = a.ctx_lens[r] + 1;
            if ((n < 0 || n > a.max_ctx) && hk == 0 && wg == 0 && wave == 0) atomicOr(a.err_flag, 8);
            mine += units_of<UT>(a, n);
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o *= 2) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
        const int total = __builtin_amdgcn_readlane(upto, 63), n_wg = min(a.wgs, max(total / a.least, 1)), share = total / n_wg, more = total % n_wg;
        left = share + (wg < more);
        if (wg >= n_wg || left == 0) return;
        const int first = wg * share + min(wg, more), owner = __builtin_ctzll(__ballot(upto > first));
        int at = upto - mine;
        if (lane == owner) {
            row = r0;
            for (int u; first >= at + (u = units_of<UT>(a, a.ctx_lens[row] + 1)); ++row) at += u;
            u0 = first - at;
        }
        row = __builtin_amdgcn_readlane(row, owner);
        u0 = __builtin_amdgcn_readlane(u0, owner);
    }
    const uint8_t *head = a.pool + (size_t)hk * F::BYTES;
    const size_t blk_stride = (size_t)a.Hkv * F::BYTES;
    const uint32_t off_k = F::k_chunk(h & (G - 1), c16), off_ks = F::k_scale(h & (G - 1), c16), off_v = F::V + (h * 16 + c16) * (4 * G), off_vs = F::VS + h * (4 * G);

    for (; row < a.B; ++row, u0 = 0) {
        // the block ids of the wave's first 32 tiles (a lane's id: tile lane / 2 of the wave's, the lower or upper half of it), asked for
        // beside the length, not after it
        const int32_t *tab = a.tables + (size_t)row * a.max_blk;
        const int my_place = 2 * ((lane >> 1) * NW + wave) + (lane & 1);
        int place = u0 * (UT / 16) + my_place;
        int my_blk = tab[min(place, a.max_blk - 1)];
        const int n_given = __builtin_amdgcn_readfirstlane(a.ctx_lens[row]) + 1, n_keys = min(max(n_given, 0), a.max_ctx);

        // the query's terms, a column and 32 dims a lane (columns without a head, and the lanes behind head_dim: zeros)
        QTerms q = q_terms(a.q + (size_t)row * a.q_stride + (size_t)(hk * Gq + min(c16, Gq - 1)) * HD + 32 * (h & (G - 1)), a.scale_log2);
        if (c16 >= Gq || h >= G) q = QTerms{{{}, {}, {}}, 127 | 127 << 8 | 127 << 16};

        if (!CUT && n_given != n_keys && tid == 0 && hk == 0) atomicOr(a.err_flag, 8);
        if (n_keys == 0) {   // a row without a request (of those in a cut launch, the kernel that joins the pieces writes the zeros)
            if (CUT) continue;
            for (int c = tid * 8; c < Gq * HD; c += 8 * NT) *(u32x4_t *)kv4_out(a, row, hk * Gq * HD + c) = u32x4_t{0, 0, 0, 0};
            return;
        }
        const int units = (n_keys + UT - 1) / UT, take = CUT ? min(left, units - u0) : units;
        const int tok0 = u0 * UT, t1 = min((u0 + take) * UT, n_keys), n_tiles = (t1 - tok0 + 31) >> 5;   // of all waves, who take them in turn

        float m_run = NEG_INF, l_run = 0.f;
        f32x4 o[2 * G];   // (group, parity of the dim)
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        struct Buf {
            u32x4_t kc[2];
            uint32_t ks[2];
            gvec vc[2], vs[2];
        };
        int pass = 0;   // first tile of the present ones
        // (always loads, the last tokens again at the end: after a load under a branch, or a way out of the loop between its two halves,
        // the compiler waits for all loads in flight, not for the older ones)
        auto issue = [&](int it, Buf &f) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int blk = __builtin_amdgcn_readlane(my_blk, 2 * it + u);
                const uint8_t *p = head + (size_t)max(blk, 0) * blk_stride;   // a missing block: memory of the pool, masked out
                f.kc[u] = __builtin_nontemporal_load((const u32x4_t *)(p + off_k));
                f.vc[u] = __builtin_nontemporal_load((const gvec *)(p + off_v));
                f.ks[u] = p[off_ks];
                f.vs[u] = *(const gvec *)(p + off_vs);
            }
        };
        auto compute = [&](int it, Buf &f) {
            const int base = tok0 + 32 * (pass + it * NW + wave);
            const int b0 = __builtin_amdgcn_readlane(my_blk, 2 * it), b1 = __builtin_amdgcn_readlane(my_blk, 2 * it + 1);
            f32x4 s[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                s[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(f.kc[u]), operand(q.t[2]), s[u], 4, 2, 0, (int)f.ks[u], 2, q.scale);
                s[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(f.kc[u]), operand(q.t[1]), s[u], 4, 2, 0, (int)f.ks[u], 1, q.scale);
                s[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(f.kc[u]), operand(q.t[0]), s[u], 4, 2, 0, (int)f.ks[u], 0, q.scale);
            }
            if (!(base + 32 <= t1 && b0 >= 0 && b1 >= 0)) {   // uniform
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int nv = (u ? b1 : b0) >= 0 ? min(max(t1 - (base + 16 * u + 4 * h), 0), 4) : 0;   // valid tokens of this lane's four
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i >= nv) s[u][i] = NEG_INF;
                    const uint32_t keep = nv == 0 ? 0u : 0xffffffffu >> (32 - 8 * nv);
#pragma unroll
                    for (int g = 0; g < G; ++g) f.vs[u][g] &= keep;   // what is behind the context may read as NaN
                }
            }
            float m_tile = NEG_INF;   // (one by one: three at a time, and no instructions that only quiet a NaN)
#pragma unroll
            for (int i = 0; i < 8; ++i) m_tile = fmaxf(m_tile, s[i >> 2][i & 3]);
            m_tile = max_of_quarters(m_tile);
            const float m_new = m_tile > m_run + KV4_REF_BEHIND ? m_tile : m_run, ms = m_new == NEG_INF ? 0.f : m_new;
            // The weights are rounded to bf16 for the second product (at most 2^-8 each, as in attention over a bf16 cache: two terms would
            // double the products and their operands); their sum is of the unrounded ones.  With the result's own rounding the
            // deviation from float64 is 0.0020 to 0.0023 (2-norm) instead of 0.0016.
            bf16x8 pf;
            float psum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = __builtin_amdgcn_exp2f(s[i >> 2][i & 3] - ms);
                psum += p;
                pf[i] = (bf16_t)p;
            }
            if (__any(m_new != m_run)) {
                const float alpha = __builtin_amdgcn_exp2f(m_run - ms);
                l_run *= alpha;
#pragma unroll
                for (int i = 0; i < 2 * G; ++i) o[i] = o[i] * alpha;
                m_run = m_new;
            }
            l_run += psum;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const V4 va = v_values(f.vc[0][g], f.vs[0][g]), vb = v_values(f.vc[1][g], f.vs[1][g]);
                o[2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join8(va.even, vb.even), pf, o[2 * g], 0, 0, 0);
                o[2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join8(va.odd, vb.odd), pf, o[2 * g + 1], 0, 0, 0);
            }
        };
        for (;;) {
            if (16 * place >= t1) my_blk = -1;
            else if ((unsigned)my_blk >= (unsigned)a.n_blocks) {
                atomicOr(a.err_flag, 2);
                my_blk = -1;
            }
            const int nit = min((n_tiles - pass - wave + NW - 1) / NW, 32);   // the wave's (0 or less: none)
            if (nit > 0) {
                Buf x, y;
                issue(0, x);
                for (int it = 0; it < nit; it += 2) {
                    issue(min(it + 1, nit - 1), y);
                    __builtin_amdgcn_sched_barrier(0);
                    compute(it, x);
                    __builtin_amdgcn_sched_barrier(0);
                    issue(min(it + 2, nit - 1), x);
                    __builtin_amdgcn_sched_barrier(0);
                    if (it + 1 < nit) compute(it + 1, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            pass += 32 * NW;
            if (pass >= n_tiles) break;
            place += 64 * NW;
            my_blk = tab[min(place, a.max_blk - 1)];
        }
        l_run += __shfl_xor(l_run, 16, 64);
        l_run += __shfl_xor(l_run, 32, 64);

        // the waves, in order
        int Gr = Gq;
        if (CUT) asm volatile("" : "+s"(Gr));   // (or the addresses below, the same for every row, are held in registers all along)
        float *s_o = smem_kv4, *s_m = smem_kv4 + NW * HD * Gr, *s_l = s_m + NW * Gr;   // [NW][HD][Gq], [NW][Gq] maxima, [NW][Gq] sums
        if (c16 < Gr) {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s_o[(wave * HD + 32 * g + 2 * (4 * h + i)) * Gr + c16] = o[2 * g][i];
                    s_o[(wave * HD + 32 * g + 2 * (4 * h + i) + 1) * Gr + c16] = o[2 * g + 1][i];
                }
            if (h == 0) {
                s_m[wave * Gr + c16] = m_run;
                s_l[wave * Gr + c16] = l_run;
            }
        }
        __syncthreads();
        for (int idx = tid; idx < Gr * HD; idx += NT) {
            const int gg = idx / HD, d = idx % HD;
            float mx = NEG_INF;
#pragma unroll
            for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_m[w * Gr + gg]);
            const float ms = mx == NEG_INF ? 0.f : mx;
            float acc = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float e = __builtin_amdgcn_exp2f(s_m[w * Gr + gg] - ms);
                acc += s_o[(w * HD + d) * Gr + gg] * e;
                l += s_l[w * Gr + gg] * e;
            }
            if (!CUT || take == units) {
                *kv4_out(a, row, (hk * Gr + gg) * HD + d) = (bf16_t)(l == 0.f ? 0.f : acc / l);   // (0: every block of the row was refused)
            } else {
                const size_t pi = kv4_piece(a, hk, wg, u0 == 0, gg);
                a.part_o[pi * HD + d] = acc;
                if (d == 0) {
                    a.part_ml[pi * 2] = mx;
                    a.part_ml[pi * 2 + 1] = l;
                }
            }
        }
        if (!CUT) return;
        if (hk == 0 && tid == 0) {
            if (u0 == 0) a.part_row[2 * row] = wg;
            if (u0 + take == units) a.part_row[2 * row + 1] = wg;
        }
        left -= take;
        if (left == 0) return;
        __syncthreads();   // before the next row's waves write theirs
    }
}

template <int HD>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4AttnArgs a) {
    const int row = blockIdx.x / a.Hkv, hk = blockIdx.x % a.Hkv;
    const int first = a.part_row[2 * row], last = a.part_row[2 * row + 1];
    const int n = min(max(a.ctx_lens[row] + 1, 0), a.max_ctx) == 0 ? 0 : last - first + 1;   // (empty rows: nobody wrote first and last)
    if (n == 1) return;
    kv4_join<HD>(a, hk, row, n, [&](int g, int j) { return n == 0 ? 0 : kv4_piece(a, hk, first + j, j == 0, g); });
}

// Which form a decode launch takes, from the sizes alone (pairs: rows times kv heads).  Equal shares cost a launch that joins pieces, and
// where contexts are of unequal lengths a share lies over the border of two of them; a workgroup with a whole row takes 3 us and 3.6 ns
// (eight waves) or 4.9 (four) a token, and the longest row may run alone at the end.  So whole rows where contexts are short, longer
// ones the more pairs there are to hide one; of eight waves where there is at most a workgroup for each compute unit.  One context, its
// calls one behind another; 8B heads, us, whole rows of 8 waves / of 4 / equal shares:
//   1 row of 900 tokens 8.3 / 8.7 / 9.4;  of 1279 9.4 / 10.1 / 9.5;  of 1536 10.5 / 11.8 / 10.2;  of 1664 11.1 / 12.2 / 9.6;  of 2047 11.7 / 13.3 / 9.8
//   1 row of 4000 18.4 / 22.0 / 10.7;  of 32000 110 / 147 / 17;  heads of 64: 1536 9.0 / 10.2 / 9.6;  1664 9.5 / 10.5 / 9.0
//   2 rows of 0 to 1700 11.1 / 12.2 / 12.7;  both of 1700 11.1 / 12.3 / 9.6;  0 to 2600 13.7 / 16.2 / 13.3;  both of 2600 13.7 / 16.2 / 10.5
//   8 rows of 0 to 1700 11.0 / 12.2 / 13.0;  of 200 to 2000 11.8 / 13.4 / 10.8;  of 1000 to 2047 11.8 / 13.4 / 14.5;  of 0 to 2600 13.8 / 16.2 / 13.6
//   16 of 500 to 2000 12.0 / 13.6 / 16.2;  16 of 0 to 3500 17.1 / 20.2 / 18.5;  of 0 to 6000 25.0 / 31.9 / 20.5
//   32 rows (256 pairs) of 0 to 4608 21.8 / 27.0 / 25.4;  all of 4608 29.4 / 30.5 / 34.8;  of 0 to 6144 27.5 / 34.0 / 27.6;  all of 6144 37.2 / 38.2 / 43.2
//   33 rows (264) of 0 to 4096 23.9 / 26.7 / 24.9;  of 0 to 4608 25.8 / 29.7 / 25.0;  all of 4608 46.4 / 39.3 / 35.7;  of 0 to 6144 31.8 / 37.9 / 29.3
//   48 rows of 0 to 4608 31.5 / 34.1 / 32.4;  all of 4608 47.9 / 44.9 / 47.0;  64 of 0 to 4096 35.9 / 33.3 / 36.3;  all of 4096 50.6 / 48.4 / 51.0
//   64 rows of 0 to 6144 49.1 / 48.6 / 46.1;  all of 6144 72.2 / 68.8 / 71.7;  65 rows of heads of 64 of 0 to 4608 18.5 / 23.1 / 22.5
// (Up to 256 pairs every workgroup has a compute unit to itself: rows of up to 6144 are whole there, behind it of up to 4608.  One row
// ends with its last share, so it is cut from 1536 on, several from 2048.)
// Equal shares: of 512 workgroups (64 rows of 4095: 48.6; of 768 55.6, of 1024 51.4), of 2 units at least and as many as make 8 pieces
// of the longest row, or of 8 and more that make 32 (shares of 2 / 4 / 8 units: 8 rows of 200 to 2000 11.0 / 13.3 / 15.4, 4 of 1000 to 4000
// 12.2 / 10.9 / 12.8).
static int kv4_wgs(int Hkv) { return std::max(1, 512 / Hkv); }
int64_t kv4_decode_pieces(int Hkv) { return 2ll * Hkv * kv4_wgs(Hkv); }

Kv4DecodeForm kv4_decode_form(int B, int Hkv, int max_ctx) {
    const int64_t pairs = (int64_t)B * Hkv;
    if (pairs > 256) return max_ctx <= 4608 ? KV4_WHOLE4 : KV4_SHARES;
    return max_ctx <= std::max<int64_t>(B == 1 ? 1536 : 2048, 24 * pairs) ? KV4_WHOLE8 : KV4_SHARES;
}
int kv4_least_share(int max_ctx) {
    const int units = (max_ctx + 127) / 128;
    return std::max({2, std::min(8, (units + 7) / 8), (units + 31) / 32});
}

template <int HD, int NW, bool CUT>
static void launch_kv4_decode_form(hipStream_t st, const Kv4AttnArgs &a) {
    const int Gq = a.Hq / a.Hkv;
    hipLaunchKernelGGL((kv4_decode_kernel<HD, NW, CUT>), dim3(a.Hkv, CUT ? a.wgs : a.B), dim3(64 * NW), (size_t)(NW * HD * Gq + 2 * NW * Gq) * sizeof(float), st, a);
}

void launch_kv4_decode(hipStream_t st, const Kv4AttnArgs &args) {
    Kv4AttnArgs a = args;
    if (a.B <= 0) return;
    const Kv4DecodeForm form = kv4_decode_form(a.B, a.Hkv, a.max_ctx);
    a.wgs = form == KV4_SHARES ? kv4_wgs(a.Hkv) : 0;
    a.least = kv4_least_share(a.max_ctx);
    if (a.wgs) {
        if (a.hd == 128) launch_kv4_decode_form<128, 4, true>(st, a);
        else launch_kv4_decode_form<64, 4, true>(st, a);
    } else if (form == KV4_WHOLE8) {
        if (a.hd == 128) launch_kv4_decode_form<128, 8, false>(st, a);
        else launch_kv4_decode_form<64, 8, false>(st, a);
    } else {
        if (a.hd == 128) launch_kv4_decode_form<128, 4, false>(st, a);
        else launch_kv4_decode_form<64, 4, false>(st, a);
    }
    if (a.wgs) {
        if (a.hd == 128) hipLaunchKernelGGL(kv4_merge_kernel<128>, dim3(a.Hkv * a.B), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(kv4_merge_kernel<64>, dim3(a.Hkv * a.B), dim3(256), 0, st, a);
    }
}

void kv4_kernels_init() {
    (void)hipFuncSetAttribute((const void *)kv4_decode_kernel<128, 8, false>, hipFuncAttributeMaxDynamicSharedMemorySize, 8 * (128 + 2) * 16 * 4);
}

// ---- attention: prompts and chunks of them ----------------------------------------------------------------------------------
// Workgroup = (kv head, 128 or 256 columns, key range): a column is a (row, query head) pair, the G heads of the kv head beside
// each other, so that 128 columns are 128 / G neighbouring rows and a chunk of few rows still fills the tiles.  Wave w owns 32
// columns.  Keys come 64 (four blocks) at a time through two LDS buffers: K as its codes, V converted once for all the waves.
// V in LDS: per block two halves [hd][8 tokens], half i the quads i and 2 + i, the dims of a group even ones first: the order
// in which a lane holds its scores, so the weights need no exchange between lanes.
#define KV4_MIN_TILES 4   // key tiles of a piece at least
template <int HD> struct Kv4Lds {
    static constexpr int K = 4 * 8 * HD, KS = 4 * (HD / 2), V = 4 * 2 * HD * 16, TILE = K + KS + V;
};

template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv4_prefill_kernel(Kv4PromptArgs a) {
    using F = Kv4<HD>;
    using L = Kv4Lds<HD>;
    constexpr int COLS = 32 * NW, WPB = NW / 4;   // waves that bring a block
    static_assert(WPB == 1 || HD == 128, "a lane's share of a block");
    constexpr int G = F::G, KSTEP = HD / 64, DT = HD / 32;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem_kv4p[];
    const int hk = blockIdx.x % a.Hkv, Gq = a.Hq / a.Hkv;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c32 = lane & 31, h = lane >> 5;

    const int at = (a.fold > 0 && (int)blockIdx.x >= a.fold ? (int)(gridDim.x - 1 - (blockIdx.x - a.fold)) : (int)blockIdx.x) / a.Hkv;
    const int req = last_at_most(a.first, a.seq.n_req, at);
    const int cut = a.cut[req], unit = (at - a.first[req]) / cut, split = (at - a.first[req]) % cut;
    const int row0 = a.seq.cu[req], len = a.seq.cu[req + 1] - row0, prior = a.seq.start[req];
    const int n_cols = len * Gq, col0 = ((n_cols + COLS - 1) / COLS - 1 - unit) * COLS;   // the longest first
    const int col = col0 + 32 * wave + c32;
    const bool valid = col < n_cols;
    const int colc = min(col, n_cols - 1), row = colc / Gq, hq = hk * Gq + colc % Gq;
    const int q_pos = prior + row;
    const int w_min = prior + min(col0 + 32 * wave, n_cols - 1) / Gq;
    const int kv_end = prior + min(col0 + COLS - 1, n_cols - 1) / Gq + 1;
    const int n_tiles = (kv_end + 63) >> 6;
    // this workgroup's share of the key tiles
    const int kt0 = (int)((int64_t)n_tiles * split / cut), kt1 = (int)((int64_t)n_tiles * (split + 1) / cut);

    QTerms q[KSTEP];   // of dims 64 s + 32 h ..
#pragma unroll
    for (int s = 0; s < KSTEP; ++s) q[s] = q_terms(a.q + (size_t)(row0 + row) * a.q_stride + (size_t)hq * HD + 64 * s + 32 * h, a.scale_log2);

    // Scores are computed relative to a reference, from whose negative the products start: the row's first maximum, moved to the
    // running one once a score is KV4_REF_BEHIND above it (limit; -inf while the row has seen no key).
    f32x16 minus_ref = {};
    float limit = NEG_INF, l_run = 0.f, l_odd = 0.f;   // the sum of weights in two parts
    f32x16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    const int32_t *tab = a.tables + (size_t)req * a.max_blk;

    // A wave (of eight: two) brings one block of a key tile: a lane its part of K's codes, the codes and scales of two V units (quads v_half
    // and 2 + v_half, dim pair vj, UG groups from vg on) and a dword of K's scales.
    constexpr int UG = G / (2 * WPB);   // groups of a lane's V unit
    const int wb = wave / WPB, wp = wave % WPB;   // the wave's block, and which share of it
    const int vj = lane & 15, vg = (2 * wp + ((lane >> 4) & 1)) * UG, v_half = lane >> 5;
    const int k_scales = WPB == 1 ? lane & (HD / 8 - 1) : 4 * (wp + 2 * ((lane >> 2) & 1)) + (lane & 3);
    typedef uint32_t kvec __attribute__((ext_vector_type(HD / 32 / WPB)));
    typedef uint32_t vvec __attribute__((ext_vector_type(UG)));
    kvec rk;
    uint32_t rks;
    vvec rv[2], rs[2];
    // A lane's block of the tile to fetch next (the lane & 3-th), asked for a tile ahead (behind the context: its last one, which nobody
    // looks at).  So every wave knows which of all four are none of the pool: their tokens are masked.
    int next_blk = 0;
    uint32_t r_none = 0, none = 0;   // those, a bit each, of what was fetched and of the tile that comes next
    auto block_at = [&](int kt) { return tab[min(kt * 4 + (lane & 3), (kv_end - 1) >> 4)]; };
    auto fetch = [&](int kt) {   // and asks for the block ids of the tile after it
        r_none = (uint32_t)__ballot((unsigned)next_blk >= (unsigned)a.n_blocks) & 15;
        const int blk = __builtin_amdgcn_readlane(next_blk, wb);
        const uint8_t *p = a.pool + ((size_t)((r_none >> wb) & 1 ? 0 : blk) * a.Hkv + hk) * F::BYTES;
        rk = *(const kvec *)(p + (uint32_t)((64 * wp + lane) * (HD / 8 / WPB)));
        rks = *(const uint32_t *)(p + (uint32_t)(F::KS + 4 * k_scales));
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            rv[u] = *(const vvec *)(p + (uint32_t)(F::V + (((v_half + 2 * u) * 16 + vj) * G + vg) * 4));
            rs[u] = *(const vvec *)(p + (uint32_t)(F::VS + ((v_half + 2 * u) * G + vg) * 4));
        }
        next_blk = block_at(min(kt + 1, kt1 - 1));
    };
    auto refuse = [&]() {   // a block that is none: nothing that reads as NaN
        if (!((r_none >> wb) & 1)) return;
        if (lane == 0) atomicOr(a.err_flag, 2);
        rks = 0;
        rs[0] = rs[1] = 0;
    };
    // What was fetched goes to LDS in parts, which the first product's instructions lie between: K; then of each group the values
    // of two quads and their stores.  (No branch among them: what the products give is used behind it, and the compiler would move
    // them there.)
    constexpr int PARTS = 6 * UG, SLOTS = 6 * KSTEP;
    V4Steps step;
    V4 px;
    uint32_t top = 0;
    auto put = [&](int part, uint8_t *t) {
        uint8_t *scales = t + L::K + wb * (HD / 2);
        bf16x8 *v = (bf16x8 *)(t + L::K + L::KS) + (wb * 2 + v_half) * HD + 32 * vg + vj;
        const int g = part / 6, u = part / 3 % 2;
        if (part == 0) {
            *(kvec *)(t + wb * (8 * HD) + (64 * wp + lane) * (HD / 8 / WPB)) = rk;
            ((uint32_t *)scales)[k_scales] = rks;
            top = 0;
        }
        if (part % 3 == 0) {
            step.scales(rs[u][g]);
        } else if (part % 3 == 1) {
            top = step.top(top);
            step.convert(rv[u][g]);
        } else if (u == 0) {
            px = step.values();
        } else {
            const V4 py = step.values();
            v[32 * g] = join8(px.even, py.even);
            v[32 * g + 16] = join8(px.odd, py.odd);
        }
    };
    // A value that is not finite must not reach the rows before it, whose weight of it is zero: the token's scores are made NaN
    // instead, which only the rows that see it take.
    auto put_nan = [&](uint8_t *t) {
        if (!__any(top >= 0x7f800000u)) return;
        uint8_t *scales = t + L::K + wb * (HD / 2);
        bf16x8 *v = (bf16x8 *)(t + L::K + L::KS) + (wb * 2 + v_half) * HD + 32 * vg + vj;
        for (int u = 0; u < 2; ++u) {
            uint32_t ff = 0;   // bytes of 255
#pragma unroll
            for (int g = 0; g < UG; ++g) ff |= ((rs[u][g] & 0x7f7f7f7fu) + 0x01010101u) & rs[u][g] & 0x80808080u;
            ff = (ff >> 7) * 255u;
            rs[u] &= ~ff;
            for (int i = 0; i < 4; ++i)
                if ((ff >> (8 * i)) & 1) scales[16 * wp + 4 * (v_half + 2 * u) + i] = 255;   // of a group whose scales the wave itself stored above
        }
#pragma unroll
        for (int g = 0; g < UG; ++g) {
            const V4 x = v_values(rv[0][g], rs[0][g]), y = v_values(rv[1][g], rs[1][g]);
            v[32 * g] = join8(x.even, y.even);
            v[32 * g + 16] = join8(x.odd, y.odd);
        }
    };

    // A key tile: the tile in buffer B is used while the next one, which is in registers, goes to the other buffer and the one
    // after that is fetched.  The order of instructions is written out: with two waves a SIMD the matrix unit idles whenever both
    // wait for vector work at a time.
    const int k_base = (c32 >> 4) * (8 * HD) + F::k_chunk(h, c32 & 15), s_base = (c32 >> 4) * (HD / 2) + h * 16 + (c32 & 15), v_base = (h * HD + c32) * 16;
    auto tile = [&](int kt, auto btag) {
        constexpr int B = decltype(btag)::value;
        uint8_t *t = smem_kv4p + B * L::TILE, *other = smem_kv4p + (1 - B) * L::TILE;
        const int kv0 = kt * 64;
        const uint32_t hidden = none;
        refuse();
        none = r_none;
        u32x4_t kc[2][KSTEP];
        int ks[2][KSTEP];
#pragma unroll
        for (int s = 0; s < KSTEP; ++s)
#pragma unroll
            for (int t2 = 0; t2 < 2; ++t2) {
                kc[t2][s] = *(const u32x4_t *)(t + k_base + t2 * (16 * HD) + s * 512);
                ks[t2][s] = t[s_base + L::K + t2 * HD + s * 32];
            }
        f32x16 st[2];
        __builtin_amdgcn_s_setprio(1);   // a wave with products goes before one with softmax (16384 rows 1845 -> 1810 us)
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {   // step s of head_dim, the query's smallest term first, the two score tiles in turn
            const int t2 = i & 1, s = i / 6, k = 2 - (i >> 1) % 3;
            const f32x16 from = i < 2 ? minus_ref : st[t2];
            if (k == 2) st[t2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(kc[t2][s]), operand(q[s].t[2]), from, 4, 2, 0, ks[t2][s], 2, q[s].scale);
            if (k == 1) st[t2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(kc[t2][s]), operand(q[s].t[1]), from, 4, 2, 0, ks[t2][s], 1, q[s].scale);
            if (k == 0) st[t2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(kc[t2][s]), operand(q[s].t[0]), from, 4, 2, 0, ks[t2][s], 0, q[s].scale);
            __builtin_amdgcn_sched_barrier(0);
            if (i % (SLOTS / PARTS) == 0) put(i / (SLOTS / PARTS), other);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        asm volatile("" : "+v"(st[0]), "+v"(st[1]));   // the products stay in front of the branch
        put_nan(other);
        fetch(min(kt + 2, kt1 - 1));
        // Only tiles that touch the diagonal, or lack a block, need the mask (one for both: with a branch of its own for a missing block
        // 16384 rows took 1659 us, so 1645, without it 1633).
        if (kv0 + 63 > w_min || hidden) {
#pragma unroll
            for (int b4 = 0; b4 < 4; ++b4) {
                const int last = (hidden >> b4) & 1 ? -1 : q_pos;
#pragma unroll
                for (int i = 8 * (b4 & 1); i < 8 * (b4 & 1) + 8; ++i)
                    if (kv0 + 32 * (b4 >> 1) + (i >> 2) * 8 + 4 * h + (i & 3) > last) st[b4 >> 1][i] = NEG_INF;
            }
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
        if (__any(m_tile > limit)) {
            const bool moves = m_tile > limit;
            const float by = moves ? m_tile : 0.f, alpha = limit == NEG_INF ? 1.f : __builtin_amdgcn_exp2f(-by);
            l_run *= alpha;
            l_odd *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = o[dt] * alpha;
            minus_ref -= by;
            st[0] -= by;
            st[1] -= by;
            if (moves) limit = KV4_REF_BEHIND;
        }
        // weights of a block, a pair at a time, rounded to bf16 for the product (at most 2^-8 each, as in decode); their sum is of the
        // unrounded ones (plain additions: the dot instruction, half as many, does not run beside the matrix unit)
        u32x4_t pw[2];
        auto weights = [&](int b4, int w0, int n) {
#pragma unroll
            for (int w = w0; w < w0 + n; ++w) {
                const float p0 = __builtin_amdgcn_exp2f(st[b4 >> 1][8 * (b4 & 1) + 2 * w]), p1 = __builtin_amdgcn_exp2f(st[b4 >> 1][8 * (b4 & 1) + 2 * w + 1]);
                l_run += p0;
                l_odd += p1;
                bf16x2 p;
                p[0] = (bf16_t)p0;
                p[1] = (bf16_t)p1;
                pw[b4 & 1][w] = as_bits(p);
            }
        };
        constexpr int NV = 4 * DT, R = 4;   // V's fragments are read R - 1 ahead of their products
        bf16x8 vf[R];
        auto values = [&](int f) { return *(const bf16x8 *)(t + v_base + L::K + L::KS + (f / DT) * (32 * HD) + (f % DT) * 512); };
#pragma unroll
        for (int f = 0; f < R - 1; ++f) vf[f] = values(f);
        weights(0, 0, 4);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            const int b4 = f / DT, dt = f % DT;
            if (f + R - 1 < NV) vf[(f + R - 1) % R] = values(f + R - 1);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[f % R], __builtin_bit_cast(bf16x8, pw[b4 & 1]), o[dt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (b4 < 3) weights(b4 + 1, dt * (4 / DT), 4 / DT);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    if (kt0 < kt1) {
        next_blk = block_at(kt0);
        fetch(kt0);
        refuse();
        none = r_none;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) put(i, smem_kv4p);
        put_nan(smem_kv4p);
        fetch(min(kt0 + 1, kt1 - 1));
    }
    __syncthreads();
    for (int kt = kt0; kt < kt1; kt += 2) {
        tile(kt, std::integral_constant<int, 0>{});
        __syncthreads();
        if (kt + 1 < kt1) {
            tile(kt + 1, std::integral_constant<int, 1>{});
            __syncthreads();
        }
    }
    l_run += l_odd;
    l_run += __shfl_xor(l_run, 32, 64);
    if (!valid) return;
    // rows of o: register i of tile dt is dim 32 dt + 2 (8 (i / 4 & 1) + 4 h + i % 4) + i / 8
    const int out_row = row0 + row;
    if (cut == 1) {
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
    const size_t pi = a.base[req] + ((size_t)row * a.Hq + hq) * cut + split;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            f32x4 *dst = (f32x4 *)(a.part_o + pi * HD + 32 * dt + 16 * j + 8 * h);
            dst[0] = f32x4{o[dt][4 * j], o[dt][8 + 4 * j], o[dt][4 * j + 1], o[dt][8 + 4 * j + 1]};
            dst[1] = f32x4{o[dt][4 * j + 2], o[dt][8 + 4 * j + 2], o[dt][4 * j + 3], o[dt][8 + 4 * j + 3]};
        }
    if (h == 0) {
        a.part_ml[2 * pi] = limit == NEG_INF ? NEG_INF : -minus_ref[0];
        a.part_ml[2 * pi + 1] = l_run;
    }
}

// The rows that were cut.
template <int HD>
__global__ __launch_bounds__(256) void kv4_prompt_merge_kernel(Kv4PromptArgs a) {
    const int hk = blockIdx.x % a.Hkv, at = blockIdx.x / a.Hkv, req = last_at_most(a.row, a.seq.n_req, at), row = at - a.row[req], cut = a.cut[req];
    const size_t p0 = a.base[req] + ((size_t)row * a.Hq + hk * (a.Hq / a.Hkv)) * cut;
    kv4_join<HD>(a, hk, a.seq.cu[req] + row, cut, [&](int g, int j) { return p0 + g * cut + j; });
}

// How many pieces the keys of each request's units are cut into, from the sizes alone: the number of key tiles of a piece that
// makes the launch shortest by this account, in us.  A compute unit is taken to need 0.85 a tile (head_dim 128) with two workgroups of
// four waves, 0.95 with one, 1.65 with one of eight; the longest piece is the tail.  Pieces are joined by a launch of their own, 5 us, and pass
// through memory as float32, 0.2 us a MB written and read.  These are numbers that put the forms in the measured order, not the times of a
// tile (a wave that has a SIMD to itself takes 1.3 us): 2048 rows are 35 by the account and 46 as measured.  8B heads, us, uncut / the
// longest unit in 2, 4 pieces / in more (chosen):
//   19 rows behind 6005 tokens 97 / 57, 35 / 9: 24, 24: 19 (24);  512 behind 8000 135 / 84, 78 (4);  2000 rows beside 100 behind 8000 146 / 95, 72 (4)
//   512 behind 1024 31 (1) / 32;  512 rows 16 (1) / 24;  1024 rows 25 (1) / 36, 44;  2048 rows 46 (1) / 74
//   70B heads, 700 rows behind 1024, 33 behind 4000 and 1391: 93 / 81 (2);  heads of 64, 19 behind 6005 76 / 46, 29 / 9: 21, 24: 18 (24)
// Returns the workgroups for each kv head, *rows_cut the rows to join.
static int kv4_prompt_cuts(Kv4PromptArgs &a, int cols, int *rows_cut) {
    const int G = a.Hq / a.Hkv;
    const double tile_us = a.hd != 128 ? 0.5 : cols == 128 ? 0.85 : 1.65;
    int units = 0, most = 0;
    double tiles = 0;
    auto n_units = [&](int r) { return ((a.seq.cu[r + 1] - a.seq.cu[r]) * G + cols - 1) / cols; };
    auto longest = [&](int r) { return (a.seq.start[r] + a.seq.cu[r + 1] - a.seq.cu[r] + 63) / 64; };   // key tiles of its last unit
    for (int r = 0; r < a.seq.n_req; ++r)
        if (const int u = n_units(r)) {
            units += u;
            tiles += 0.5 * u * ((a.seq.start[r] + 63) / 64 + longest(r) + 1);
            most = std::max(most, longest(r));
        }
    if (units == 0) return 0;
    const double even = tiles * a.Hkv / 256 * tile_us;
    const bool folds = units * a.Hkv > 256 && units * a.Hkv <= 512;
    int best = most;   // key tiles of a piece at most
    double best_us = 0;
    for (int c = 1; c <= 64; c += std::max(1, c / 2)) {   // pieces of the longest unit
        const int share = (most + c - 1) / c;
        if (c > 1 && share < KV4_MIN_TILES) break;
        int n = 0, pieces = 0;
        double mb = 0;
        for (int r = 0; r < a.seq.n_req; ++r) {
            const int u = n_units(r), cut = u ? (longest(r) + share - 1) / share : 1;
            n += u * cut;
            if (cut > 1) {
                pieces += u * a.Hkv * cut;
                mb += 1e-6 * (a.seq.cu[r + 1] - a.seq.cu[r]) * a.Hq * cut * a.hd * 4;
            }
        }
        if (pieces * cols > KV4_PIECES * 128) break;
        const double tail = share * tile_us * (cols == 256 ? 1.0 : n * a.Hkv <= 256 ? 1.12 : folds && c == 1 ? 1.3 : 1.95);
        const double us = std::max(even, tail) + (pieces ? 5 + 0.4 * mb : 0);
        if (c == 1 || us < best_us) best = share, best_us = us;
    }
    int n = 0, rows = 0, pieces = 0;
    for (int r = 0; r < a.seq.n_req; ++r) {
        const int u = n_units(r), cut = u ? (longest(r) + best - 1) / best : 1;
        a.first[r] = n;
        a.base[r] = pieces * cols;
        a.row[r] = rows;
        a.cut[r] = cut;
        n += u * cut;
        if (cut > 1) {
            pieces += u * a.Hkv * cut;
            rows += a.seq.cu[r + 1] - a.seq.cu[r];
        }
    }
    // workgroups that all run at once, two a compute unit: the shorter half in rising order, beside the longer (2048 rows 52.7 -> 48.0 us)
    a.fold = folds && n == units ? 256 : 0;
    *rows_cut = rows;
    return n;
}

Kv4PromptPlan kv4_prompt_plan(Kv4PromptArgs &a) {
    // Eight waves of 32 columns convert a value once for 256 columns instead of 128, but have their compute unit to themselves: where
    // there are enough of them for the last round not to matter.  8B heads, us, four / eight waves (workgroups of eight):
    //   2048 rows (256) 47 / 57;  4096 (512) 133 / 146;  6000 (752) 263 / 264;  8192 (1024) 471 / 450;  12000 (1504) 978 / 936;  16384 1785 / 1707
    int units = 0;
    for (int r = 0; r < a.seq.n_req; ++r) units += ((a.seq.cu[r + 1] - a.seq.cu[r]) * (a.Hq / a.Hkv) + 255) / 256;
    const int cols = a.hd == 128 && units * a.Hkv >= 1024 ? 256 : 128;
    int rows = 0;
    const int n = kv4_prompt_cuts(a, cols, &rows);
    return {cols, n, rows};
}

void launch_kv4_prefill(hipStream_t st, const Kv4PromptArgs &args) {
    Kv4PromptArgs a = args;
    const auto [cols, n, rows] = kv4_prompt_plan(a);
    if (n == 0) return;
    if (cols == 256) hipLaunchKernelGGL((kv4_prefill_kernel<128, 8>), dim3(a.Hkv * n), dim3(512), 2 * Kv4Lds<128>::TILE, st, a);
    else if (a.hd == 128) hipLaunchKernelGGL((kv4_prefill_kernel<128, 4>), dim3(a.Hkv * n), dim3(256), 2 * Kv4Lds<128>::TILE, st, a);
    else hipLaunchKernelGGL((kv4_prefill_kernel<64, 4>), dim3(a.Hkv * n), dim3(256), 2 * Kv4Lds<64>::TILE, st, a);
    if (rows == 0) return;
    if (a.hd == 128) hipLaunchKernelGGL(kv4_prompt_merge_kernel<128>, dim3(a.Hkv * rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(kv4_prompt_merge_kernel<64>, dim3(a.Hkv * rows), dim3(256), 0, st, a);
}
