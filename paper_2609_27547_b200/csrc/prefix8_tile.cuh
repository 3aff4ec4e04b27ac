// Device pieces shared by the kernels that contract queries with 8-bit prefix tiles.
//
// A tile is 32 tokens of one head's keys or values: 32 * HD codes, contiguous in the record, one scale.  Query rows are
// the N of the tensor-core products (mma.sync m16n8k16, f16 in, fp32 out), so that 1 .. 8 rows cost one column tile and
// no more:
//     S^T [tokens x rows] = K [tokens x hd] Q^T          A = keys,     B = queries
//     O^T [hd x rows]     = V^T [hd x tokens] P^T        A = values^T, B = weights
// Every e4m3 value is an f16 value (3 mantissa bits, exponents -9 .. 8), so codes are widened exactly, straight from the words a
// lane reads from shared memory, in two ways that run side by side:
//   widen   the conversion instruction, one pair each; it runs on the quarter-rate unit at 8 pairs a clock and SM (measured: with it
//           alone that unit is 82 % busy and the stream stops at half of the copy bandwidth, which needs 11.5 pairs)
//   spread  integer instructions: sign and magnitude put at their places in the f16 give the value times 2^-8 (subnormals
//           included), 3 to 4 instructions a pair on the full-rate units
// A quarter of the pairs take the first way.  The 2^8 between them is taken up by the queries' and the output's factors.  The order of the contracted index is free as long
// as both operands agree: lane (g = lane / 4, t = lane % 4) takes the HD / 4 consecutive columns t * HD / 4 .. of tokens g
// and g + 8 as its key operand (so its queries are HD / 4 consecutive elements, too), and the HD / 8 consecutive columns
// g * HD / 8 .. of tokens 2t, 2t + 1, 2t + 8, 2t + 9 as its value operand (so its outputs are consecutive).
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
// Bytes 0 and 2 (even) or 1 and 3 (odd) of four codes as f16x2, times 2^-8: exponent and mantissa of e4m3 are the low seven bits,
// those of f16 bits 13 .. 7 once the exponent's top bit is 0, and the biases differ by 8.
__device__ __forceinline__ uint32_t spread_even(uint32_t w) { return ((w << 7) & 0x3f803f80u) | ((w << 8) & 0x80008000u); }
__device__ __forceinline__ uint32_t spread_odd(uint32_t w) { return ((w >> 1) & 0x3f803f80u) | (w & 0x80008000u); }
// Which steps of the contraction over head_dim (keys) and which 16-column tiles of the output (values) take the conversion unit.
__host__ __device__ constexpr bool by_unit(int i) { return (i & 3) == 3; }

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
    return r;
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
__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}

// A block's scale as the readers use it: the sign marks a block that holds a NaN, which poisons what reads it as a whole (the
// integer way of widening would take a NaN code for 480).
__device__ __forceinline__ float read_scale(float s) { return __float_as_uint(s) >> 31 ? __uint_as_float(0x7fffffffu) : s; }

// Where byte `off` of token `tok` of a tile stands in shared memory: 128-byte lines whose eight 16-byte pieces are permuted
// so that the key reads (one or two tokens per phase) and the value reads (tokens 0, 2, 4, 6 per phase) touch every bank
// once.  The pattern repeats every 8 tokens: address(tok + 8 k, off) = address(tok, off) + 8 k HD.
template <int HD> __device__ __forceinline__ uint32_t tile_addr(int tok, int off)
{
    const int lin = tok * HD + off, line = lin >> 7, piece = (lin >> 4) & 7;
    const int sw = HD == 128 ? (line & 7) : (HD == 64 ? (line & 3) << 1 : (line & 1) << 1);
    return (uint32_t)(line * 128 + ((piece ^ sw) << 4) + (lin & 15));
}

// Requests a tile (its first `valid` tokens; the others become zeros) into the slot at dst.
template <int HD> __device__ __forceinline__ void request_tile(uint32_t dst, const char *src, int valid, int lane)
{
    constexpr int N = 2 * HD / 32;                 // 16-byte pieces per lane
    const int bytes = valid * HD;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int lin = (i * 32 + lane) * 16;
        const uint32_t at = dst + tile_addr<HD>(lin / HD, lin % HD);
        cp16(at, lin < bytes ? src + lin : src, lin < bytes ? 16u : 0u);
    }
}

// One lane's share of the queries of a row tile as B operands: row g of each column tile, columns t * HD / 4 .., scaled by a
// power of two so that the row's largest element lies in [2^6, 2^7) where keys are widened by the conversion unit and in [2^14, 2^15)
// where they come 2^8 smaller.  bf16 queries then are f16 values exactly unless they are 2^20 smaller than the row's largest
// (then 2^-31 of it is lost); fp32 queries are split into two f16 terms (22 bits).  Returns the factor that undoes it.
template <int HD, bool F32> __device__ __forceinline__ float load_q(const void *q, bool there, int t, uint32_t (*hi)[2], uint32_t (*lo)[2])
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
    const int up = (m == 0.f || e == 255) ? 0 : min(6 + 127 - e, 119);
    const float mul = __uint_as_float((uint32_t)(up + 127) << 23);
#pragma unroll
    for (int s = 0; s < HD / 16; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // the two columns that share a register of the keys: neighbours, or (spread) every other one
            const float k = by_unit(s) ? mul : mul * 256.f;
            const float a = x[4 * s + (by_unit(s) ? 2 * j : j)] * k, b = x[4 * s + (by_unit(s) ? 2 * j + 1 : j + 2)] * k;
            hi[s][j] = pack_f16(a, b);
            if constexpr (F32) lo[s][j] = pack_rest(a, b, hi[s][j]);
        }
    return 1.f / mul;   // a power of two: exact
}

// A pair of keys' words -> the A operand of one step.
__device__ __forceinline__ void key_operand(int step, uint32_t a, uint32_t b, uint32_t *f)
{
    if (by_unit(step)) { f[0] = widen(a); f[1] = widen(b); f[2] = widen(a >> 16); f[3] = widen(b >> 16); }
    else { f[0] = spread_even(a); f[1] = spread_even(b); f[2] = spread_odd(a); f[3] = spread_odd(b); }
}

// One lane's words of the keys g and g + 8 of a 16-token half tile; kaddr = the tile's slot + tile_addr(g, t * HD / 4).
template <int HD> struct KeyWords {
    uint32_t a[HD / 16], b[HD / 16];
    __device__ __forceinline__ void load(uint32_t slot, const uint32_t *off, int half)
    {
        const uint32_t base = slot + (uint32_t)(half * 16 * HD);
        if constexpr (HD == 128) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 x = lds128(base + off[j]), y = lds128(base + off[j] + 8 * HD);
                a[4 * j] = x.x; a[4 * j + 1] = x.y; a[4 * j + 2] = x.z; a[4 * j + 3] = x.w;
                b[4 * j] = y.x; b[4 * j + 1] = y.y; b[4 * j + 2] = y.z; b[4 * j + 3] = y.w;
            }
        } else if constexpr (HD == 64) {
            const uint4 x = lds128(base + off[0]), y = lds128(base + off[0] + 8 * HD);
            a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w;
            b[0] = y.x; b[1] = y.y; b[2] = y.z; b[3] = y.w;
        } else {
            const uint2 x = lds64(base + off[0]), y = lds64(base + off[0] + 8 * HD);
            a[0] = x.x; a[1] = x.y;
            b[0] = y.x; b[1] = y.y;
        }
    }
    static __device__ __forceinline__ void offsets(uint32_t *off, int g, int t)
    {
        off[0] = tile_addr<HD>(g, t * (HD / 4));
        off[1] = HD == 128 ? tile_addr<HD>(g, t * (HD / 4) + 16) : 0u;
    }
};

}  // namespace p8
}  // namespace ebrl
