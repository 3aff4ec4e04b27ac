// Device pieces shared by the kernels that contract queries with 8-bit prefix tiles.
//
// A tile is 32 tokens of one head's keys or values: 32 * HD codes, contiguous in the record, one scale.  Query rows are
// the N of the tensor-core products (mma.sync m16n8k16, f16 in, fp32 out), so that 1 .. 8 rows cost one column tile and
// no more:
//     S^T [tokens x rows] = K [tokens x hd] Q^T          A = keys,     B = queries
//     O^T [hd x rows]     = V^T [hd x tokens] P^T        A = values^T, B = weights
// Every e4m3 value is an f16 value (3 mantissa bits, exponents -9 .. 8): codes are widened exactly, two per instruction, straight
// from the words a lane reads from shared memory (the conversion runs at 63 pairs a clock and SM, the product at 957 MAC;
// mma.sync on e4m3 operands is no way around it: it is that same conversion and product inside, 2.5 times the instructions).
// The order of the contracted index is free as long as both operands agree.
//   Keys: lane (g = lane / 4, t = lane % 4) takes the HD / 4 consecutive columns t * HD / 4 .. of two tokens, so its queries
//   are HD / 4 consecutive elements, too.  Rows g and g + 8 of the A operand are tokens row_token(g) and row_token(g) + 2 ...
//   Values: ... because ldmatrix (16 x 16 bytes, transposed) gives lane (g, t) the codes of tokens 4t .. 4t + 3 of columns g and
//   g + 8: widened pairwise they are the A operand as they stand, if contraction slots 2t, 2t + 1, 2t + 8, 2t + 9 are these tokens.
#pragma once
#include "prefix8_internal.h"
#include "ptx_helpers.cuh"

#include <cuda_fp16.h>
#include <math.h>

namespace ebrl {
namespace p8 {

constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t widen(uint32_t two)   // the e4m3 pair in the low half -> f16x2
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return r;
}
// Two 16 x 16 byte matrices, transposed: lanes 0 - 15 give the row addresses of the first, 16 - 31 of the second.  Lane (g, t) gets
// rows 4t .. 4t + 3 of columns g and g + 8 of each.
__device__ __forceinline__ void load_columns(uint32_t a, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v)   // an 8 x 8 matrix of 16-bit values held two per lane
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// The second f16 term of a pair: what rounding to the first left over.
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t first)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&first));
    return pack_f16(lo - f.x, hi - f.y);
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, uint32_t nbytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(nbytes) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void prefetch_l1(const void *p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}

// A block's scale as the readers use it: the sign marks a block that holds a NaN, which poisons what reads it as a whole, whatever
// becomes of the codes' own NaN on the way (a maximum drops it).
__device__ __forceinline__ float read_scale(float s) { return __float_as_uint(s) >> 31 ? __uint_as_float(0x7fffffffu) : s; }

// The token (of 16) that is row g of the keys' operand; row g + 8 is the one two further on.
__device__ __forceinline__ int row_token(int g) { return 4 * (g >> 1) + (g & 1); }

// Where byte `off` of token `tok` of a tile stands in shared memory: 128-byte lines whose eight 16-byte pieces are permuted
// so that the key reads (two tokens per phase, four at head_dim 32) and the value reads (the same columns of eight tokens)
// touch every bank once.  The pattern repeats every 8 tokens.
template <int HD> __device__ __forceinline__ uint32_t tile_addr(int tok, int off)
{
    const int lin = tok * HD + off, line = lin >> 7, piece = (lin >> 4) & 7;
    const int sw = HD == 128 ? (line & 7) : (HD == 64 ? (line & 3) : (line & 1) * 5);
    return (uint32_t)(line * 128 + ((piece ^ sw) << 4) + (lin & 15));
}

// Requests a tile (its first `valid` tokens; the others become zeros) into the slot at dst.
template <int HD> __device__ __forceinline__ void request_tile(uint32_t dst, const char *src, int valid, int lane)
{
    constexpr int N = 2 * HD / 32;                 // 16-byte pieces per lane
    if (valid >= BLOCK) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int lin = (i * 32 + lane) * 16;
            cp16(dst + tile_addr<HD>(lin / HD, lin % HD), src + lin);
        }
    } else {
        const int bytes = valid * HD;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int lin = (i * 32 + lane) * 16;
            cp16(dst + tile_addr<HD>(lin / HD, lin % HD), lin < bytes ? src + lin : src, lin < bytes ? 16u : 0u);
        }
    }
}

// One lane's share of a column tile of queries as B operands: row g, columns t * HD / 4 .., scaled by a power of two so that the
// row's largest element lies in [2^14, 2^15).  bf16 queries then are f16 values exactly unless they are 2^28 smaller than the row's
// largest (then 2^-40 of that is lost); fp32 queries are split into two f16 terms (22 bits).
// q[s]: the operands of step s (16 columns): {b0, b1 of the first term, of the second}.
// `negate` puts the sign of the softmax scale into the queries, so that what scores are multiplied by is never negative.
// Returns the factor that undoes the scaling.
template <bool F32> constexpr int QW = F32 ? 4 : 2;   // words per step
template <int HD, bool F32> __device__ __forceinline__ float load_q(const void *q, bool there, bool negate, int t, uint32_t (*out)[QW<F32>])
{
    constexpr int N = HD / 4;
    float x[N];
    if (there) {
        if constexpr (F32) {
            const float4 *p = reinterpret_cast<const float4 *>((const float *)q + t * N);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float4 v = p[i];
                x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
            }
        } else {
            const uint4 *p = reinterpret_cast<const uint4 *>((const __nv_bfloat16 *)q + t * N);
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const uint4 v = p[i];
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
                    x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = 0.f;
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(x[i]));
    m = fmaxf(m, __shfl_xor_sync(FULL, m, 1));
    m = fmaxf(m, __shfl_xor_sync(FULL, m, 2));
    const int e = (int)(__float_as_uint(m) >> 23);            // biased exponent of the largest
    const int up = (m == 0.f || e == 255) ? 0 : min(14 + 127 - e, 127);
    const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= negate ? -mul : mul;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float a = x[4 * s + 2 * j], b = x[4 * s + 2 * j + 1];
            out[s][j] = pack_f16(a, b);
            if constexpr (F32) out[s][2 + j] = pack_rest(a, b, out[s][j]);
        }
    return 1.f / mul;   // a power of two: exact
}

// One lane's words of two keys of a 16-token half tile: its rows g and g + 8 of the A operand.
template <int HD> struct KeyWords {
    uint32_t a[HD / 16], b[HD / 16];
    static constexpr int OFFS = HD == 128 ? 4 : 2;
    __device__ __forceinline__ void load(uint32_t slot, const uint32_t *off, int half)
    {
        const uint32_t base = slot + (uint32_t)(half * 16 * HD);
        if constexpr (HD == 128) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 x = lds128(base + off[j]), y = lds128(base + off[2 + j]);
                a[4 * j] = x.x; a[4 * j + 1] = x.y; a[4 * j + 2] = x.z; a[4 * j + 3] = x.w;
                b[4 * j] = y.x; b[4 * j + 1] = y.y; b[4 * j + 2] = y.z; b[4 * j + 3] = y.w;
            }
        } else if constexpr (HD == 64) {
            const uint4 x = lds128(base + off[0]), y = lds128(base + off[1]);
            a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w;
            b[0] = y.x; b[1] = y.y; b[2] = y.z; b[3] = y.w;
        } else {
            const uint2 x = lds64(base + off[0]), y = lds64(base + off[1]);
            a[0] = x.x; a[1] = x.y;
            b[0] = y.x; b[1] = y.y;
        }
    }
    static __device__ __forceinline__ void offsets(uint32_t *off, int g, int t)
    {
#pragma unroll
        for (int i = 0; i < OFFS; ++i) {
            const int tok = row_token(g) + 2 * (i / (OFFS / 2)), piece = OFFS == 4 ? i % 2 : 0;
            off[i] = tile_addr<HD>(tok, t * (HD / 4) + 16 * piece);
        }
    }
};

// Raw scores of a tile's two halves (16 tokens each) and NT column tiles: s = keys x queries.  q(step, nt, w) hands out the queries'
// operands.  Halves side by side: 2 NT independent chains of products hide one another's latency.
// The tensor core truncates its sums.  APART: the second terms add up by themselves, so that only the first terms' sum loses bits at its
// size, and meet it in fp32 (weights of 16 x 20 - 32 tokens x 4 heads of 64 x 8 fp32
// rows 6.3e-7 -> 2.4e-7 off; time: see weigh).
template <int HD, int NT, bool F32, bool APART = false, typename Q> __device__ __forceinline__ void score(float (*s)[NT][4], const KeyWords<HD> *k, Q &&q)
{
    constexpr bool TWO = F32 && APART;
    float rest[TWO ? 2 : 1][TWO ? NT : 1][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[h][nt][c] = 0.f;
                if constexpr (TWO) rest[h][nt][c] = 0.f;
            }
#pragma unroll
    for (int st = 0; st < HD / 16; ++st) {
        uint32_t a[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            a[h][0] = widen(k[h].a[st]); a[h][1] = widen(k[h].b[st]); a[h][2] = widen(k[h].a[st] >> 16); a[h][3] = widen(k[h].b[st] >> 16);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            uint32_t w[QW<F32>];
            q(st, nt, w);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (F32) mma(TWO ? rest[TWO ? h : 0][TWO ? nt : 0] : s[h][nt], a[h][0], a[h][1], a[h][2], a[h][3], w[2], w[3]);
                mma(s[h][nt], a[h][0], a[h][1], a[h][2], a[h][3], w[0], w[1]);
            }
        }
    }
    if constexpr (TWO) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[h][nt][c] += rest[h][nt][c];
    }
}

}  // namespace p8
}  // namespace ebrl
