// Softmax attention of few query rows over paged keys and values (include/ebrl_pages.h): out = softmax(scale q k^T) v.
//
//   Item = (sequence, piece of it, key/value head, 16 or 32 query rows), worked on by ONE WARP: its own running softmax and its
//   own ring of stages (32 tokens of keys and values each, 16 at fp32 heads of 64 and 128) filled by cp.async, no barrier.  Calls that would leave
//   SMs empty share an item among a TEAM of warps (the CTA), each an even share of the tokens, joined in shared memory; long
//   sequences are cut into pieces besides, joined by a second kernel.
//   Query rows are (token, member) pairs of the heads that share a key/value head, so each key and value is read once for all of them.
//   A token that no row may see (hidden, behind the length, on a page that is not there) is filled with zeros by the copy itself, so
//   whatever stands there meets no product.
//
//   bf16, 16 rows: HBM.  192 x 512 - 2048 tokens x 4 heads of 128, one token each: 78 us for 473 MB, 6.1 TB/s, 0.93 of a copy (four warps per SM with three stages
//   each 96, six with two 78; a team of two, an item each 105: a warp's chain of copies, products and exponentials takes 1.7 us a tile, so that the longest item is
//   what is waited for).  1 x 256 tokens x 16 heads of 64: 6 us with teams of eight, 11.6 without.
//   fp32: three tf32 products for each, a k-step's added up by themselves and then in registers (chained through, the tensor core's truncation made the result
//   2.4e-6 wrong instead of 2.8e-7).  96 x 64 - 512 tokens x 4 heads of 64, 16 - 64 rows: 62 us, of which the products would take 17: eight warps of 255
//   registers per SM issue an instruction every four cycles each, and no more of them fit.
#include "pages_internal.h"
#include "ptx_helpers.cuh"

#include <cuda_bf16.h>
#include <math.h>

namespace ebrl {
namespace pg {

constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <int HD, int MT, bool F32> struct Cfg {
    static constexpr int ES = F32 ? 4 : 2, RB = HD * ES;                 // bytes of a row
    static constexpr int TK = F32 && HD >= 64 ? 16 : 32;                 // tokens of a tile
    static constexpr int TILE = TK * RB, Q_BYTES = 16 * MT * RB;
    static constexpr int WARPS = HD == 128 ? (F32 ? 4 : (MT == 1 ? 6 : 5)) : (RB >= 128 ? 8 : 12);   // per SM
    static constexpr int ROOM = (224 * 1024 / WARPS - Q_BYTES) / (2 * TILE);
    static constexpr int STAGES = ROOM < 4 ? ROOM : 4;
    static constexpr int WARP_BYTES = STAGES * 2 * TILE + Q_BYTES;
    static_assert(STAGES >= 2 && STAGES * 2 * TILE >= 16 * MT * (HD * 4 + 8), "ring");   // (a team's results are joined in the rings)
};

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
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t *r)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ float lds32(uint32_t a)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void mma_bf16(float *c, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float *c, const uint32_t *a, const uint32_t *b)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_tf32_first(float *c, const uint32_t *a, const uint32_t *b)   // c = a b
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "f"(0.f));
}
// x as two tf32 terms: the first rounded to 11 bits (2^-11 of x is left), the second cut to 11 bits by the tensor core, which ignores the
// low 13 (2^-21 of x is lost).  Plain integer instructions: the conversion instruction runs at a sixteenth of their rate.
__device__ __forceinline__ void two_terms(float x, uint32_t &hi, uint32_t &lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Where 16-byte piece `p` of row `r` of a tile stands: pieces are permuted so that eight rows' same piece (what ldmatrix reads) and
// four rows' pairs of pieces (what the fp32 values' reads take) touch every bank once.
template <int RB> __device__ __forceinline__ uint32_t tile_at(int r, int p)
{
    if constexpr (RB >= 128) return (uint32_t)(r * RB + ((p ^ (r & 7)) << 4));
    else return (uint32_t)(r * RB + ((p ^ ((r >> 1) & 3)) << 4));
}

template <int HD, int MT, bool F32, bool TEAM>
__global__ void __launch_bounds__(Cfg<HD, MT, F32>::WARPS * 32, 1)
attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendSeqs sq)
{
    using C = Cfg<HD, MT, F32>;
    constexpr int RB = C::RB, TK = C::TK, PIECES = RB / 16, ROWS = 16 * MT, NT = TK / 8, NV = HD / 8;
    extern __shared__ __align__(1024) char smem[];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring = ptx::smem_u32(smem + (size_t)warp * C::WARP_BYTES), q_at = ring + C::STAGES * 2 * C::TILE;
    __shared__ unsigned stage_word[C::WARPS][C::STAGES];
    const int kvh = a.g.kvh, G = a.G;
    const float sc = a.scale * LOG2E;
    // Where a lane reads: piece p of its row stands at the address of piece 0 (or 1) with the bits of 16 p flipped.
    const uint32_t q_off = tile_at<RB>(lane & 15, lane >> 4), k_off = tile_at<RB>((lane & 7) + ((lane >> 4) << 3), (lane >> 3) & 1);
    const uint32_t v_off[2] = {F32 ? tile_at<RB>(2 * t, g >> 2) + (g & 3) * 4 : q_off, F32 ? tile_at<RB>(2 * t + 1, g >> 2) + (g & 3) * 4 : 0};
    pdl_launch_dependents();

    for (int x = TEAM ? blockIdx.x : warp * gridDim.x + blockIdx.x; x < sq.items; x += gridDim.x * (TEAM ? 1 : warps)) {
        // which item this is
        const AttendSeq seq = sq.s[find_seq(sq.n, x, [&](int i) { return sq.s[i].item; })];
        const int m = seq.m, len = seq.len, R = m * G, RT = (R + ROWS - 1) / ROWS;
        int rest = x - seq.item;
        const int rt = rest % RT; rest /= RT;
        const int kh = rest % kvh, piece = rest / kvh;
        const int r0 = rt * ROWS, r1 = min(R, r0 + ROWS);                 // its rows; row = token * G + member
        const int first = len - m;                                        // position of query 0
        // the tokens that some row of the item sees: lo .. hi
        const Span span = seen_by(len, m, G, r0, r1, a.causal, a.window, a.split, piece);
        int lo = span.lo, hi = span.hi;
        const int seen = lo;                                              // no row sees a token below
        lo = lo / TK * TK;
        if constexpr (TEAM) {   // this warp's even share
            const int part = (hi - lo + warps * TK - 1) / (warps * TK) * TK;
            lo += warp * part;
            hi = min(hi, lo + part);
        }
        const int tiles = hi > lo ? (hi - lo + TK - 1) / TK : 0;

        // queries into shared memory
        for (int c = lane; c < ROWS * PIECES; c += 32) {
            const int r = c / PIECES, p = c % PIECES, row = min(r0 + r, R - 1), tok = row / G;
            const char *src = a.q + (((long long)seq.row + tok) * a.q_stride + (long long)(kh * G + row - tok * G) * HD) * C::ES + p * 16;
            cp16(q_at + tile_at<RB>(r, p), src, r0 + r < R ? 16 : 0);
        }

        // A batch of 32 mask words' pages and bits, one per lane; the next one is on its way while this one is used.
        const int *tab = a.p.table + seq.tab * a.p.stride;
        const int word0 = lo / WORD, words = (hi + WORD - 1) / WORD;
        auto look_up = [&](int base, int &page, unsigned &bits) {
            const int w = base + lane;
            page = -1;
            bits = 0;
            if (w < words) {
                const int pg = tab[(w * WORD) >> a.g.t_shift];
                if ((unsigned)pg < (unsigned)a.p.n_pages) {
                    page = pg;
                    bits = *reinterpret_cast<const unsigned *>(a.p.pool + (size_t)pg * a.g.bytes + a.g.mask + ((w * WORD & (a.g.T - 1)) >> 3));
                    if (w * WORD < seen) bits = w * WORD + WORD > seen ? bits & (FULL << (seen - w * WORD)) : 0;
                    if (w * WORD < lo) bits &= FULL << (lo - w * WORD);
                    if (w * WORD + WORD > hi) bits &= FULL >> (w * WORD + WORD - hi);
                }
            }
        };
        int page, page2, batch = word0;
        unsigned bits, bits2;
        if (tiles) { look_up(batch, page, bits); look_up(batch + 32, page2, bits2); }
        int issued = 0;
        const size_t head_k = a.g.at(a.layer, 0, kh), head_v = a.g.at(a.layer, 1, kh);
        auto issue = [&]() {   // one commit group, empty when nothing is left
            if (issued < tiles) {
                const int tok = lo + issued * TK, w = tok / WORD;
                if (w - batch >= 32) {
                    batch += 32;
                    page = page2; bits = bits2;
                    look_up(batch + 32, page2, bits2);
                }
                const int pg = __shfl_sync(FULL, page, w - batch);
                unsigned see = __shfl_sync(FULL, bits, w - batch);
                if (TK == 16) see = (tok & 16 ? see >> 16 : see) & 0xffffu;
                const char *base = a.p.pool + (pg >= 0 ? (size_t)pg * a.g.bytes + (size_t)(tok & (a.g.T - 1)) * RB : 0);
                const uint32_t dst = ring + (uint32_t)(issued % C::STAGES * 2 * C::TILE);
                if (lane == 0) stage_word[warp][issued % C::STAGES] = see;
                if (see) {
#pragma unroll 4
                    for (int c = lane; c < TK * PIECES; c += 32) {
                        const int r = c / PIECES, p = c % PIECES;
                        const uint32_t n = (see >> r) & 1 ? 16 : 0, at = tile_at<RB>(r, p);
                        cp16(dst + at, base + head_k + r * RB + p * 16, n);
                        cp16(dst + C::TILE + at, base + head_v + r * RB + p * 16, n);
                    }
                }
                ++issued;
            }
            cp_commit();
        };
#pragma unroll
        for (int j = 0; j < C::STAGES - 1; ++j) issue();

        float O[MT][NV][4], M[MT][2], L[MT][2];
        int last[MT][2];                     // the last token (exclusive) that a row sees, and the first one
        int from[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int n = 0; n < NV; ++n) { O[i][n][0] = O[i][n][1] = O[i][n][2] = O[i][n][3] = 0.f; }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                M[i][e] = -INFINITY; L[i][e] = 0.f;
                const int tok = min(r0 + i * 16 + e * 8 + g, R - 1) / G;
                last[i][e] = a.causal ? first + tok + 1 : 0x7fffffff;
                from[i][e] = first_seen(first + tok, a.window);
            }
        }
        const int all_last = a.causal ? first + r0 / G + 1 : 0x7fffffff;                  // tokens below are seen by every row ...
        const int all_from = first_seen(first + (r1 - 1) / G, a.window);                  // ... and from here on

        for (int j = 0; j < tiles; ++j) {
            cp_wait<C::STAGES - 2>();
            __syncwarp();      // tile j is there for every lane, and every lane has read tile j - 1, whose stage is filled next
            issue();
            const uint32_t kt = ring + (uint32_t)(j % C::STAGES * 2 * C::TILE), vt = kt + C::TILE;
            const unsigned see = stage_word[warp][j % C::STAGES];
            if (see) {
                float S[MT][NT][4];
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n) { S[i][n][0] = S[i][n][1] = S[i][n][2] = S[i][n][3] = 0.f; }
                if constexpr (!F32) {
#pragma unroll
                    for (int k = 0; k < HD / 16; ++k) {
                        uint32_t qa[MT][4];
#pragma unroll
                        for (int i = 0; i < MT; ++i) ldsm4((q_at + i * 16 * RB + q_off) ^ (k * 32), qa[i]);
#pragma unroll
                        for (int n = 0; n < NT; n += 2) {
                            uint32_t kb[4];
                            ldsm4((kt + n * 8 * RB + k_off) ^ (k * 32), kb);
#pragma unroll
                            for (int i = 0; i < MT; ++i) { mma_bf16(S[i][n], qa[i], kb[0], kb[1]); mma_bf16(S[i][n + 1], qa[i], kb[2], kb[3]); }
                        }
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < HD / 8; ++k) {
                        uint32_t qa[4], qh[MT][4], ql[MT][4];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            ldsm4((q_at + i * 16 * RB + q_off) ^ (k * 32), qa);
#pragma unroll
                            for (int e = 0; e < 4; ++e) two_terms(__uint_as_float(qa[e]), qh[i][e], ql[i][e]);
                        }
                        // the products of one k-step by themselves, then added: the tensor core's own sums are truncated
                        float c[MT][NT][4];
                        uint32_t kh_[NT][2], kl[NT][2];
#pragma unroll
                        for (int n = 0; n < NT; n += 2) {
                            uint32_t kb[4];
                            ldsm4((kt + n * 8 * RB + k_off) ^ (k * 32), kb);
#pragma unroll
                            for (int e = 0; e < 4; ++e) two_terms(__uint_as_float(kb[e]), kh_[n + e / 2][e & 1], kl[n + e / 2][e & 1]);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < MT; ++i) mma_tf32_first(c[i][n], ql[i], kh_[n]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < MT; ++i) mma_tf32(c[i][n], qh[i], kl[n]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < MT; ++i) mma_tf32(c[i][n], qh[i], kh_[n]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < MT; ++i)
#pragma unroll
                                for (int e = 0; e < 4; ++e) S[i][n][e] += c[i][n][e];
                    }
                }
                // scores in units of log 2, what a row does not see at -inf
                const int tok = lo + j * TK;
                const bool whole = see == (TK == 32 ? FULL : 0xffffu) && tok + TK <= all_last && tok >= all_from;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = n * 8 + 2 * t + (e & 1);
                            S[i][n][e] = __fmul_rn(S[i][n][e], sc);       // (rounded, as the maxima are: scores beyond 2^23 would else be off from them)
                            if (!whole && !(((see >> c) & 1) && tok + c < last[i][e >> 1] && tok + c >= from[i][e >> 1])) S[i][n][e] = -INFINITY;
                        }
                bool moved = false;
                float f[MT][2];
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = S[i][0][2 * e];
#pragma unroll
                        for (int n = 0; n < NT; ++n) top = fmaxf(top, fmaxf(S[i][n][2 * e], S[i][n][2 * e + 1]));
                        top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
                        f[i][e] = 1.f;
                        if (top > M[i][e]) {
                            f[i][e] = ex2(M[i][e] - top);     // (0 the first time)
                            M[i][e] = top;
                            moved = true;
                        }
                    }
                if (__any_sync(FULL, moved)) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        L[i][0] *= f[i][0]; L[i][1] *= f[i][1];
#pragma unroll
                        for (int n = 0; n < NV; ++n) { O[i][n][0] *= f[i][0]; O[i][n][1] *= f[i][0]; O[i][n][2] *= f[i][1]; O[i][n][3] *= f[i][1]; }
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float ref = M[i][e] == -INFINITY ? 0.f : M[i][e];
                        float sum = 0.f;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            S[i][n][2 * e] = ex2(S[i][n][2 * e] - ref);
                            S[i][n][2 * e + 1] = ex2(S[i][n][2 * e + 1] - ref);
                            sum += S[i][n][2 * e] + S[i][n][2 * e + 1];
                        }
                        L[i][e] += sum;
                    }
                if constexpr (!F32) {
                    // Weights become bf16, because the values that they meet are (half a step is 2^-8 of a weight; the sum that divides them is not rounded): results are
                    // 1.8e-3 to 2.0e-3 off, of which their own rounding is 1.7e-3.  Two terms would be half as many products again.
#pragma unroll
                    for (int k = 0; k < TK / 16; ++k) {
                        uint32_t pa[MT][4];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            pa[i][0] = pack_bf16(S[i][2 * k][0], S[i][2 * k][1]);
                            pa[i][1] = pack_bf16(S[i][2 * k][2], S[i][2 * k][3]);
                            pa[i][2] = pack_bf16(S[i][2 * k + 1][0], S[i][2 * k + 1][1]);
                            pa[i][3] = pack_bf16(S[i][2 * k + 1][2], S[i][2 * k + 1][3]);
                        }
#pragma unroll
                        for (int n = 0; n < NV; n += 2) {
                            uint32_t vb[4];
                            ldsm4t((vt + k * 16 * RB + v_off[0]) ^ (n * 16), vb);
#pragma unroll
                            for (int i = 0; i < MT; ++i) { mma_bf16(O[i][n], pa[i], vb[0], vb[1]); mma_bf16(O[i][n + 1], pa[i], vb[2], vb[3]); }
                        }
                    }
                } else {
                    // the contraction's slots t and t + 4 are tokens 2t and 2t + 1: weights stay where the scores were
#pragma unroll
                    for (int k = 0; k < TK / 8; ++k) {
                        uint32_t ph[MT][4], pl[MT][4];
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            two_terms(S[i][k][0], ph[i][0], pl[i][0]); two_terms(S[i][k][2], ph[i][1], pl[i][1]);
                            two_terms(S[i][k][1], ph[i][2], pl[i][2]); two_terms(S[i][k][3], ph[i][3], pl[i][3]);
                        }
#pragma unroll
                        for (int n0 = 0; n0 < NV; n0 += 4) {
                            float c[MT][4][4];
                            uint32_t vh[4][2], vl[4][2];
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    two_terms(lds32((vt + k * 8 * RB + v_off[e]) ^ ((n0 + n) * 32)), vh[n][e], vl[n][e]);
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int i = 0; i < MT; ++i) mma_tf32_first(c[i][n], pl[i], vh[n]);
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int i = 0; i < MT; ++i) mma_tf32(c[i][n], ph[i], vl[n]);
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int i = 0; i < MT; ++i) mma_tf32(c[i][n], ph[i], vh[n]);
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int i = 0; i < MT; ++i)
#pragma unroll
                                    for (int e = 0; e < 4; ++e) O[i][n0 + n][e] += c[i][n][e];
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                L[i][e] += __shfl_xor_sync(FULL, L[i][e], 1);
                L[i][e] += __shfl_xor_sync(FULL, L[i][e], 2);
            }
        cp_wait<0>();
        __syncwarp();

        // Where a row's result goes: the output, or the piece's partial result.
        const bool cut = a.split && seq.part >= 0;
        auto finish = [&](int row, int col, const float *v, int nv, float top, float sum) {   // nv consecutive columns of a row
            const int tok = row / G, head = kh * G + row - tok * G;
            if (cut) {
                const size_t at = ((size_t)seq.part + (size_t)piece * m + tok) * a.heads + head;
                for (int c = 0; c < nv; ++c) a.part_o[at * HD + col + c] = v[c];
                if (col == 0) { a.part_ml[2 * at] = top; a.part_ml[2 * at + 1] = sum; }
                return;
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const size_t r = (size_t)seq.row + tok;
            char *o = a.out + (r * a.o_stride + (size_t)head * HD + col) * C::ES;
            if constexpr (F32) { for (int c = 0; c < nv; ++c) ((float *)o)[c] = v[c] * inv; }
            else { for (int c = 0; c < nv; c += 2) ((uint32_t *)o)[c / 2] = pack_bf16(v[c] * inv, v[c + 1] * inv); }
            if (a.lse && col == 0) a.lse[r * a.heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
        };
        if constexpr (!TEAM) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = r0 + i * 16 + e * 8 + g;
                    if (row < r1)
#pragma unroll
                        for (int n = 0; n < NV; ++n) finish(row, n * 8 + 2 * t, &O[i][n][2 * e], 2, M[i][e], L[i][e]);
                }
        } else {
            // every warp's sums into its own ring, which is idle now; rows are then dealt out to the warps, sums taken in warp order
            float *mine = reinterpret_cast<float *>(smem + (size_t)warp * C::WARP_BYTES);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = i * 16 + e * 8 + g;
#pragma unroll
                    for (int n = 0; n < NV; ++n) *reinterpret_cast<float2 *>(mine + r * HD + n * 8 + 2 * t) = make_float2(O[i][n][2 * e], O[i][n][2 * e + 1]);
                    if (t == 0) { mine[ROWS * HD + 2 * r] = M[i][e]; mine[ROWS * HD + 2 * r + 1] = L[i][e]; }
                }
            __syncthreads();
            constexpr int PER = HD / 32;      // columns of a lane
            for (int r = warp; r < r1 - r0; r += warps) {
                float top = -INFINITY, sum = 0.f, v[PER < 2 ? 2 : PER] = {};
                for (int w = 0; w < warps; ++w) top = fmaxf(top, reinterpret_cast<const float *>(smem + (size_t)w * C::WARP_BYTES)[ROWS * HD + 2 * r]);
                const float ref = top == -INFINITY ? 0.f : top;
                constexpr int W = PER < 2 ? 2 : PER;            // (two columns at least are written at once)
                if (lane * W < HD) {
                    for (int w = 0; w < warps; ++w) {
                        const float *o = reinterpret_cast<const float *>(smem + (size_t)w * C::WARP_BYTES);
                        const float f = ex2(o[ROWS * HD + 2 * r] - ref);
                        sum = fmaf(f, o[ROWS * HD + 2 * r + 1], sum);
#pragma unroll
                        for (int c = 0; c < W; ++c) v[c] = fmaf(f, o[r * HD + lane * W + c], v[c]);
                    }
                    finish(r0 + r, lane * W, v, W, top, sum);
                }
            }
            __syncthreads();
        }
    }
    pdl_wait();      // (the end of this kernel is to be that of the ones beside it, too)
}

// Joins the pieces of cut sequences: one warp per (query, head), sums in a fixed order.
template <int HD, bool F32>
__global__ void __launch_bounds__(256) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ AttendSeqs sq)
{
    constexpr int W = HD / 32;
    const int lane = threadIdx.x & 31;
    pdl_wait();      // (set up while the last pieces are being worked on)
    const long long rows = (long long)sq.items * a.heads;      // (items: the queries of the cut sequences, counted in sq.item)
    for (long long x = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); x < rows; x += (long long)gridDim.x * 8) {
        const int r = (int)(x / a.heads), head = (int)(x - (long long)r * a.heads);
        const AttendSeq seq = sq.s[find_seq(sq.n, r, [&](int i) { return sq.s[i].item; })];
        const int tok = r - seq.item, m = seq.m, np = pieces_of(seq.len, m, a.window, a.split);
        const size_t at0 = ((size_t)seq.part + tok) * a.heads + head, step = (size_t)m * a.heads;
        float top = -INFINITY, sum = 0.f;
        bool there = true;                         // (a piece whose kernel gave up a wait has NaN for a reference)
        for (int p = lane; p < np; p += 32) {      // relative to the piece whose weights add up to most, so that its sums are no larger than its values
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (at0 + p * step));
            top = fmaxf(top, ml.x + log2f(ml.y));
            there = there && ml.x == ml.x;
        }
        if (!__all_sync(FULL, there)) continue;
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
        const float ref = top == -INFINITY ? 0.f : top;
        float v[W] = {};
        for (int base = 0; base < np; base += 32) {      // each lane weighs a piece
            const int mine = base + lane, n = min(32, np - base);
            const float2 ml = mine < np ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * (at0 + mine * step)) : make_float2(-INFINITY, 0.f);
            const float f_mine = ex2(ml.x - ref);
            sum = fmaf(f_mine, ml.y, sum);
            const float *o = a.part_o + (at0 + base * step) * HD + lane * W;
            for (int p0 = 0; p0 < n; p0 += 16) {         // (16 pieces at once: two 65 k-token histories 64 us, four at once 69)
                float x[16][W];
#pragma unroll
                for (int p = 0; p < 16; ++p)
#pragma unroll
                    for (int c = 0; c < W; ++c) x[p][c] = p0 + p < n ? o[(p0 + p) * step * HD + c] : 0.f;
#pragma unroll
                for (int p = 0; p < 16; ++p) {
                    const float f = __shfl_sync(FULL, f_mine, p0 + p);
#pragma unroll
                    for (int c = 0; c < W; ++c) v[c] = fmaf(f, x[p][c], v[c]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const size_t row = (size_t)seq.row + tok, at = row * a.o_stride + (size_t)head * HD + lane * W;
#pragma unroll
        for (int c = 0; c < W; ++c) {
            if constexpr (F32) ((float *)a.out)[at + c] = v[c] * inv;
            else ((__nv_bfloat16 *)a.out)[at + c] = __float2bfloat16_rn(v[c] * inv);
        }
        if (a.lse && lane == 0) a.lse[row * a.heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
}

int attend_rows(int rows) { return rows <= 16 ? 16 : 32; }
int attend_warps(int hd, bool f32, int rows) { return hd == 128 ? (f32 ? 4 : (rows == 16 ? 6 : 5)) : (hd * (f32 ? 4 : 2) >= 128 ? 8 : 12); }

namespace {

template <int HD, int MT, bool F32, bool TEAM> cudaError_t go(const AttendArgs &a, const AttendSeqs &s, int quota, bool beside, cudaStream_t st)
{
    using C = Cfg<HD, MT, F32>;
    static std::atomic<bool> set[64];   // (calls may come from several threads; setting it twice is harmless)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        cudaError_t err = cudaFuncSetAttribute(attend_kernel<HD, MT, F32, TEAM>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::WARPS * C::WARP_BYTES);
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    // Under a quota: persistent CTAs with all of an SM's warps.  Else one CTA per item: the hardware hands out the next as one ends.
    const int warps = TEAM ? a.team : (quota ? C::WARPS : 1), grid = quota && !TEAM && s.items > quota ? quota : s.items;
    const Beside with(beside);
    return launch_kernel(attend_kernel<HD, MT, F32, TEAM>, grid, warps * 32, (size_t)(warps * C::WARP_BYTES), st, 1, a, s);
}

template <int HD, bool F32> cudaError_t pick(const AttendArgs &a, const AttendSeqs &s, int rows, int quota, bool beside, cudaStream_t st)
{
    if (a.team > 1) return rows == 16 ? go<HD, 1, F32, true>(a, s, quota, beside, st) : go<HD, 2, F32, true>(a, s, quota, beside, st);
    return rows == 16 ? go<HD, 1, F32, false>(a, s, quota, beside, st) : go<HD, 2, F32, false>(a, s, quota, beside, st);
}

}  // namespace

cudaError_t launch_attend(const AttendArgs &a, const AttendSeqs &s, bool f32, int rows, int quota, bool beside, cudaStream_t st)
{
    if (s.items == 0) return cudaSuccess;
    switch (a.g.hd) {
    case 128: return f32 ? pick<128, true>(a, s, rows, quota, beside, st) : pick<128, false>(a, s, rows, quota, beside, st);
    case 64: return f32 ? pick<64, true>(a, s, rows, quota, beside, st) : pick<64, false>(a, s, rows, quota, beside, st);
    default: return f32 ? pick<32, true>(a, s, rows, quota, beside, st) : pick<32, false>(a, s, rows, quota, beside, st);
    }
}

template <bool F32> static cudaError_t join(const AttendArgs &a, const AttendSeqs &s, int grid, cudaStream_t st)
{
    switch (a.g.hd) {
    case 128: return launch_kernel(attend_join_kernel<128, F32>, grid, 256, 0, st, 1, a, s);
    case 64: return launch_kernel(attend_join_kernel<64, F32>, grid, 256, 0, st, 1, a, s);
    default: return launch_kernel(attend_join_kernel<32, F32>, grid, 256, 0, st, 1, a, s);
    }
}

cudaError_t launch_attend_join(const AttendArgs &a, const AttendSeqs &s, bool f32, int quota, int sms, cudaStream_t st)
{
    if (s.items == 0) return cudaSuccess;
    const long long need = ((long long)s.items * a.heads + 7) / 8, cap = quota ? quota : (long long)sms * 8;
    const int grid = (int)(need < cap ? need : cap);
    const Beside early(quota == 0);      // (under a quota its CTAs would wait on SMs beside the pieces')
    return f32 ? join<true>(a, s, grid, st) : join<false>(a, s, grid, st);
}

}  // namespace pg
}  // namespace ebrl
