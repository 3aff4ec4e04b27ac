// Softmax attention over 8-bit prefix records (include/ebrl_prefix8.h): out = softmax(scale q k^T) v, k = code * scale.
//
// Bound: HBM.  Each code is read once and used by the 1 .. 32 query rows of a row tile, far left of the ridge even on mma.sync, so
// what counts is that bytes are always in flight and that a code costs few instructions.
//
//   Item = (environment, piece of its prefix, key/value head, row tile), worked on by ONE WARP: its own running softmax, its
//   own ring of tile slots (keys and values alternate) filled by cp.async, no barrier, no partial results to join unless a prefix is
//   cut.  A record's head is contiguous, so a tile is one straight 4 KB run at head_dim 128.
//   SMs hold 16 warps at 8 rows, 12 at 16, 8 at 32 (what registers allow); 130 - 190 KB of tiles are in flight per SM, three
//   times what HBM latency asks for.  With all SMs to itself the launch is one CTA per item, which lets the hardware even out
//   ragged prefixes; under an SM quota it is a persistent grid of `quota` CTAs that hold all of an SM's warps.
//   (Four warps per item, joined in shared memory, were 1.6 times slower on 512 x 768 tokens x 16 heads: an item was
//   over before its set-up and join were paid for.)
//
//   Running maximum, lazily: a row's reference is raised only when a score exceeds it by 2^14 / 2^6; until then the weights
//   2^(s - ref) stay below 2^14, which f16 holds with the same 11 bits.  The common tile needs one vote and no
//   shuffles.  Weights aim at 2^6 rather than 1, so that those 2^-20 of the largest are still normal f16 numbers.
//   A block's value scale is applied in fp32 to the block's own product (tmp), not to the weights: any finite scales work.
//
//   bf16 queries are exact (prefix8_tile.cuh), weights are rounded to f16: 11 bits, an eighth of the output's own rounding.  fp32 queries: queries and weights in two f16 terms each (22 bits).  Sums are fp32.
#include "prefix8_tile.cuh"
#include "rowops.cuh"

#include <float.h>

namespace ebrl {
namespace p8 {

template <int HD, int NT, bool F32> struct AttendCfg {
    static constexpr int WARPS = HD == 128 ? (NT == 1 ? 12 : (F32 && NT == 4 ? 7 : 8)) : (NT == 1 ? (F32 ? 12 : 16) : (NT == 2 ? (F32 ? 8 : 10) : (F32 ? 7 : 8)));    // per SM
    static constexpr int TILE = BLOCK * HD;
    // queries in shared memory where registers hold the outputs of 32 rows, or of 16 beside two f16 terms: per warp
    static constexpr bool QS = NT == 4 || (F32 && NT == 2);
    static constexpr int QBYTES = QS ? HD / 16 * NT * 32 * 4 * QW<F32> : 0;
    static constexpr int ROOM = (224 * 1024 / WARPS - QBYTES - 128) / TILE;
    static constexpr int SLOTS = ROOM < 8 ? ROOM : 8;                 // 3 .. 8 tiles per warp
    static constexpr int WARP_BYTES = SLOTS * TILE + QBYTES + 128;    // ring, queries, and per slot the tile's scale and mask
    static_assert(SLOTS >= 3, "ring");
};

template <int HD, int NT, bool F32>
__global__ void __launch_bounds__(AttendCfg<HD, NT, F32>::WARPS * 32, 1)
attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    using C = AttendCfg<HD, NT, F32>;
    constexpr int MT = HD / 16, W = HD / 32, ST = HD / 16;
    extern __shared__ __align__(128) char smem[];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const uint32_t ring_u = ptx::smem_u32(smem + (size_t)warp * C::WARP_BYTES);
    const uint32_t q_u = ring_u + C::SLOTS * C::TILE, tail_u = q_u + C::QBYTES;
    const int G = a.r.G, R = a.r.H * G, RT = (R + NT * 8 - 1) / (NT * 8), kvh = a.r.rec.kvh;
    const int n_envs = a.r.meta ? a.r.n_envs : ev.n;
    const long long items = (long long)n_envs * kvh * a.n_split * RT;
    uint32_t koff[2], voff[2];
    KeyWords<HD>::offsets(koff, g, t);
    voff[0] = tile_addr<HD>(2 * t, g * (HD / 8));
    voff[1] = tile_addr<HD>(2 * t + 1, g * (HD / 8));
    pdl_launch_dependents();
    pdl_wait();

    // items go round the CTAs first, so that the last round spreads over all SMs
    for (long long item = (long long)warp * gridDim.x + blockIdx.x; item < items; item += (long long)gridDim.x * warps) {
        unsigned x = (unsigned)item;
        const int rt = (int)(x % (unsigned)RT); x /= (unsigned)RT;
        const int kh = (int)(x % (unsigned)kvh); x /= (unsigned)kvh;
        const int sp = (int)(x % (unsigned)a.n_split), env = (int)(x / (unsigned)a.n_split);
        const char *rec;
        int len;
        if (a.r.meta) { rec = (const char *)a.r.meta[env].kv; len = a.r.meta[env].P; }
        else { rec = a.r.pool + (size_t)ev.slot[env] * a.r.rec.bytes; len = ev.len[env]; }
        const int t0 = sp * a.split, t1 = a.n_split == 1 ? len : min(len, t0 + a.split);
        if (sp > 0 && t0 >= len) continue;
        const int ntile = (t1 - t0 + BLOCK - 1) / BLOCK;
        const char *kp = rec + a.r.rec.head(a.r.layer, 0, kh) + (size_t)t0 * HD, *vp = rec + a.r.rec.head(a.r.layer, 1, kh) + (size_t)t0 * HD;
        const char *ksp = rec + a.r.rec.head_scales(a.r.layer, 0, kh) + t0 / BLOCK * 4, *vsp = rec + a.r.rec.head_scales(a.r.layer, 1, kh) + t0 / BLOCK * 4;
        const char *mkp = rec + a.r.rec.mask + t0 / BLOCK * 4;

        // position j of the item's stream: keys (even) or values (odd) of tile j / 2 with their scale and, beside the keys, the
        // mask word; one commit group each, empty past the end
        int jt = 0;
        auto issue = [&](int plane, int slot) {
            if (jt < ntile) {
                const uint32_t dst = ring_u + (uint32_t)(slot * C::TILE), tail = tail_u + (uint32_t)(slot * 8);
                request_tile<HD>(dst, (plane ? vp : kp) + (size_t)jt * C::TILE, t1 - t0 - jt * BLOCK, lane);
                if (lane == 0) cp4(tail, (plane ? vsp : ksp) + (size_t)jt * 4);
                if (lane == 1 && plane == 0) cp4(tail + 4, mkp + (size_t)jt * 4);
                jt += plane;
            }
            cp_commit();
        };
#pragma unroll
        for (int j = 0; j < C::SLOTS - 1; ++j) issue(j & 1, j);

        // queries
        uint32_t q[C::QS ? 1 : NT][ST][QW<F32>];
        float fr[NT][2];   // what takes a raw product of row 2t (+ 1) of column tile nt to a score in units of log 2 (times the key scale)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = rt * NT * 8 + nt * 8 + g, tok = r / G;
            const size_t off = (size_t)env * a.r.q_env + (size_t)tok * a.r.q_tok + (size_t)(kh * G + r - tok * G) * HD;
            const void *p = F32 ? (const void *)((const float *)a.r.q + off) : (const void *)((const __nv_bfloat16 *)a.r.q + off);
            uint32_t b[ST][QW<F32>];
            const float f = load_q<HD, F32>(p, r < R, a.r.scale < 0.f, t, b) * (fabsf(a.r.scale) * LOG2E);
            fr[nt][0] = __shfl_sync(FULL, f, 8 * t);
            fr[nt][1] = __shfl_sync(FULL, f, 8 * t + 4);
#pragma unroll
            for (int st = 0; st < ST; ++st) {
                if constexpr (C::QS) {
                    const uint32_t at = q_u + (uint32_t)(((st * NT + nt) * 32 + lane) * 4 * QW<F32>);
                    if constexpr (F32) sts128(at, b[st][0], b[st][1], b[st][2], b[st][3]);
                    else sts64(at, b[st][0], b[st][1]);
                } else {
#pragma unroll
                    for (int c = 0; c < QW<F32>; ++c) q[nt][st][c] = b[st][c];
                }
            }
        }
        // (a lane reads back from shared memory what it wrote itself)
        auto query = [&](int st, int nt, uint32_t *w) {
            if constexpr (C::QS) {
                const uint32_t at = q_u + (uint32_t)(((st * NT + nt) * 32 + lane) * 4 * QW<F32>);
                if constexpr (F32) { const uint4 u = lds128(at); w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; }
                else { const uint2 u = lds64(at); w[0] = u.x; w[1] = u.y; }
            } else {
#pragma unroll
                for (int c = 0; c < QW<F32>; ++c) w[c] = q[nt][st][c];
            }
        };

        float o[MT][NT][4], mr[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mr[nt][0] = mr[nt][1] = -FLT_MAX;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[m][nt][c] = 0.f;
        }
        int slot = 0;
        for (int i = 0; i < ntile; ++i) {
            cp_wait<C::SLOTS - 2>();
            __syncwarp();            // the tile is there for every lane, and every lane is done with the slot requested next
            issue((C::SLOTS - 1) & 1, slot == 0 ? C::SLOTS - 1 : slot - 1);
            const uint32_t kslot = ring_u + (uint32_t)(slot * C::TILE);
            const uint2 tail = lds64(tail_u + (uint32_t)(slot * 8));
            slot = slot + 1 == C::SLOTS ? 0 : slot + 1;
            const float ks = read_scale(__uint_as_float(tail.x));
            uint32_t mk = tail.y;
            if (i == ntile - 1 && ((t1 - t0) & (BLOCK - 1))) mk &= (1u << ((t1 - t0) & (BLOCK - 1))) - 1u;

            uint32_t pb[2][NT][2], pl[F32 ? 2 : 1][NT][2];
            if (mk) {
                float s[2][NT][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    KeyWords<HD> kw;
                    kw.load(kslot, koff, h);
                    score<HD, NT, F32>(s[h], kw, query);
                }
                const bool hides = mk != FULL;
                if (hides) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool s0 = (mk >> (16 * h + g)) & 1, s1 = (mk >> (16 * h + 8 + g)) & 1;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (!s0) s[h][nt][0] = s[h][nt][1] = -FLT_MAX;
                            if (!s1) s[h][nt][2] = s[h][nt][3] = -FLT_MAX;
                        }
                    }
                }
                float c[NT][2], top[NT][2];
                bool above = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        c[nt][j] = ks * fr[nt][j];
                        top[nt][j] = c[nt][j] * fmaxf(fmaxf(s[0][nt][j], s[0][nt][j + 2]), fmaxf(s[1][nt][j], s[1][nt][j + 2]));
                        above |= top[nt][j] > mr[nt][j] + 14.f;
                    }
                if (__any_sync(FULL, above)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float corr[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float m = top[nt][j];
                            m = fmaxf(m, __shfl_xor_sync(FULL, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(FULL, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(FULL, m, 16));
                            const float nm = m > mr[nt][j] + 14.f ? m - 6.f : mr[nt][j];
                            corr[j] = ex2(mr[nt][j] - nm);
                            mr[nt][j] = nm;
                            l[nt][j] *= corr[j];
                        }
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            o[m][nt][0] *= corr[0]; o[m][nt][1] *= corr[1]; o[m][nt][2] *= corr[0]; o[m][nt][3] *= corr[1];
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float p0 = ex2(fmaf(s[h][nt][0], c[nt][0], -mr[nt][0])), p1 = ex2(fmaf(s[h][nt][1], c[nt][1], -mr[nt][1]));
                        float p2 = ex2(fmaf(s[h][nt][2], c[nt][0], -mr[nt][0])), p3 = ex2(fmaf(s[h][nt][3], c[nt][1], -mr[nt][1]));
                        if (hides) {   // (their scores are no more than very low: a factor of 0 makes them 0)
                            if (!((mk >> (16 * h + g)) & 1)) p0 = p1 = 0.f;
                            if (!((mk >> (16 * h + 8 + g)) & 1)) p2 = p3 = 0.f;
                        }
                        l[nt][0] += p0 + p2;
                        l[nt][1] += p1 + p3;
                        const uint32_t w0 = pack_f16(p0, p1), w1 = pack_f16(p2, p3);
                        if constexpr (F32) {
                            pl[h][nt][0] = transpose8(pack_rest(p0, p1, w0));
                            pl[h][nt][1] = transpose8(pack_rest(p2, p3, w1));
                        }
                        pb[h][nt][0] = transpose8(w0);
                        pb[h][nt][1] = transpose8(w1);
                    }
            }

            cp_wait<C::SLOTS - 2>();
            __syncwarp();
            issue(C::SLOTS & 1, slot == 0 ? C::SLOTS - 1 : slot - 1);
            const uint32_t vslot = ring_u + (uint32_t)(slot * C::TILE);
            const float vs = read_scale(__uint_as_float(lds32(tail_u + (uint32_t)(slot * 8))));
            slot = slot + 1 == C::SLOTS ? 0 : slot + 1;
            if (mk) {
                uint32_t v[2][4][W];   // tokens 2t, 2t + 1, 2t + 8, 2t + 9 of each half
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t at = vslot + voff[k & 1] + (uint32_t)((16 * h + 8 * (k >> 1)) * HD);
                        if constexpr (W == 4) { const uint4 u = lds128(at); v[h][k][0] = u.x; v[h][k][1] = u.y; v[h][k][2] = u.z; v[h][k][3] = u.w; }
                        else if constexpr (W == 2) { const uint2 u = lds64(at); v[h][k][0] = u.x; v[h][k][1] = u.y; }
                        else v[h][k][0] = lds32(at);
                    }
#pragma unroll
                for (int wd = 0; wd < W; ++wd)
#pragma unroll
                    for (int sub = 0; sub < 2; ++sub) {
                        const int m = 2 * wd + sub;
                        uint32_t f[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // two columns, the codes of two tokens side by side
                            const uint32_t p = prmt(v[h][0][wd], v[h][1][wd], sub ? 0x7362u : 0x5140u), r = prmt(v[h][2][wd], v[h][3][wd], sub ? 0x7362u : 0x5140u);
                            f[h][0] = widen(p); f[h][1] = widen(p >> 16); f[h][2] = widen(r); f[h][3] = widen(r >> 16);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            float tmp[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                if constexpr (F32) mma(tmp, f[h][0], f[h][1], f[h][2], f[h][3], pl[h][nt][0], pl[h][nt][1]);
                                mma(tmp, f[h][0], f[h][1], f[h][2], f[h][3], pb[h][nt][0], pb[h][nt][1]);
                            }
#pragma unroll
                            for (int k = 0; k < 4; ++k) o[m][nt][k] = fmaf(vs, tmp[k], o[m][nt][k]);
                        }
                    }
            }
        }
        cp_wait<0>();      // only empty groups are left; the ring is free
        __syncwarp();

        // rows 2t and 2t + 1 of each column tile, columns g * HD / 8 ..
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float L = l[nt][j];
                L += __shfl_xor_sync(FULL, L, 4);
                L += __shfl_xor_sync(FULL, L, 8);
                L += __shfl_xor_sync(FULL, L, 16);
                const int r = rt * NT * 8 + nt * 8 + 2 * t + j, tok = r / G, head = kh * G + r - tok * G;
                if (r >= R) continue;
                if (a.n_split > 1) {
                    const size_t at = ((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + (size_t)tok * a.r.heads + head;
                    float *dst = a.part_o + at * HD + g * (HD / 8);
#pragma unroll
                    for (int k = 0; k < HD / 32; ++k)
                        *reinterpret_cast<float4 *>(dst + 4 * k) = make_float4(o[2 * k][nt][j], o[2 * k][nt][j + 2], o[2 * k + 1][nt][j], o[2 * k + 1][nt][j + 2]);
                    if (g == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(mr[nt][j], L);
                    continue;
                }
                const float inv = L == 0.f ? 0.f : 1.f / L;
                const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + g * (HD / 8);
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < HD / 32; ++k) {
                        const float4 u = make_float4(o[2 * k][nt][j] * inv, o[2 * k][nt][j + 2] * inv, o[2 * k + 1][nt][j] * inv, o[2 * k + 1][nt][j + 2] * inv);
                        if (a.split_out) store_split4(a.out, a.out_t1, a.out_t2, off + 4 * k, u.x, u.y, u.z, u.w);
                        else *reinterpret_cast<float4 *>((float *)a.out + off + 4 * k) = u;
                    }
                } else {
                    uint32_t w[HD / 16];
#pragma unroll
                    for (int k = 0; k < HD / 16; ++k) {
                        const __nv_bfloat162 u = __floats2bfloat162_rn(o[k][nt][j] * inv, o[k][nt][j + 2] * inv);
                        w[k] = *reinterpret_cast<const uint32_t *>(&u);
                    }
                    __nv_bfloat16 *dst = (__nv_bfloat16 *)a.out + off;
                    if constexpr (HD == 128) {
                        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4 *>(dst + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    } else if constexpr (HD == 64) *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                    else *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
                }
                if (a.lse && g == 0) a.lse[((size_t)env * a.r.H + tok) * a.r.heads + head] = L == 0.f ? -INFINITY : (mr[nt][j] + log2f(L)) * LN2;
            }
    }
}

// Joins the pieces of long prefixes: one CTA per query row, the pieces divided over its eight warps, sums in warp order.
// Traffic is the pieces' results only (1 / 64 of the cache at 896-token pieces and 4 rows).
template <int HD, bool F32>
__global__ void __launch_bounds__(256) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    constexpr int V = HD / 32;
    __shared__ float so[8][HD], sl[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, RH = a.r.H * a.r.heads;
    const long long rows = (long long)ev.n * RH;
    pdl_launch_dependents();
    pdl_wait();
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const int env = (int)(row / RH), rr = (int)(row - (long long)env * RH), tok = rr / a.r.heads, head = rr - tok * a.r.heads;
        const int np = max(1, (ev.len[env] + a.split - 1) / a.split);
        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (size_t)env * a.n_split * RH + rr;
        const float *po = a.part_o + ((size_t)env * a.n_split * RH + rr) * HD + lane * V;
        float M = -FLT_MAX;
        for (int p = lane; p < np; p += 32) M = fmaxf(M, ml[(size_t)p * RH].x);
        M = warp_max(M);
        float acc[V], L = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll 4
        for (int p = warp; p < np; p += 8) {
            const float2 u = ml[(size_t)p * RH];
            const float f = ex2(u.x - M);
            L = fmaf(f, u.y, L);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(f, po[(size_t)p * RH * HD + i], acc[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) so[warp][lane * V + i] = acc[i];
        if (lane == 0) sl[warp] = L;
        __syncthreads();
        if (threadIdx.x < HD) {
            float s = 0.f, z = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) { s += so[w][threadIdx.x]; z += sl[w]; }
            const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + threadIdx.x;
            const float v = z == 0.f ? 0.f : s / z;
            if constexpr (F32) ((float *)a.out)[off] = v;
            else ((__nv_bfloat16 *)a.out)[off] = __float2bfloat16_rn(v);
            if (a.lse && threadIdx.x == 0) a.lse[(size_t)env * RH + rr] = z == 0.f ? -INFINITY : (M + log2f(z)) * LN2;
        }
        __syncthreads();
    }
}

namespace {

template <int HD, int NT, bool F32> cudaError_t go(const AttendArgs &a, const Envs &e, int grid, cudaStream_t st)
{
    using C = AttendCfg<HD, NT, F32>;
    static bool set[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        cudaError_t err = cudaFuncSetAttribute(attend_kernel<HD, NT, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::WARPS * C::WARP_BYTES);
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    const long long n = a.r.meta ? a.r.n_envs : e.n;
    const long long items = n * a.r.rec.kvh * a.n_split * ((a.r.H * a.r.G + NT * 8 - 1) / (NT * 8));
    if (items == 0) return cudaSuccess;
    const int warps = grid ? C::WARPS : 1;
    const long long cap = grid ? grid : 1 << 20;   // items go round the CTAs first: a grid of `quota` CTAs uses as many SMs as it has items
    return launch_kernel(attend_kernel<HD, NT, F32>, (int)(items < cap ? items : cap), warps * 32, (size_t)(warps * C::WARP_BYTES), st, 1, a, e);
}

template <int HD> cudaError_t pick(const AttendArgs &a, const Envs &e, bool f32, int grid, cudaStream_t st)
{
    const int nt = row_tile(a.r.H * a.r.G) / 8;
    if (f32) return nt == 1 ? go<HD, 1, true>(a, e, grid, st) : (nt == 2 ? go<HD, 2, true>(a, e, grid, st) : go<HD, 4, true>(a, e, grid, st));
    return nt == 1 ? go<HD, 1, false>(a, e, grid, st) : (nt == 2 ? go<HD, 2, false>(a, e, grid, st) : go<HD, 4, false>(a, e, grid, st));
}

}  // namespace

int attend_warps(int rows, bool f32)
{
    const int nt = row_tile(rows) / 8;
    return f32 ? (nt == 1 ? AttendCfg<128, 1, true>::WARPS : (nt == 2 ? AttendCfg<128, 2, true>::WARPS : AttendCfg<128, 4, true>::WARPS))
               : (nt == 1 ? AttendCfg<128, 1, false>::WARPS : (nt == 2 ? AttendCfg<128, 2, false>::WARPS : AttendCfg<128, 4, false>::WARPS));
}

cudaError_t launch_attend(const AttendArgs &a, const Envs &e, bool f32, int grid, cudaStream_t st)
{
    return a.r.rec.hd == 128 ? pick<128>(a, e, f32, grid, st) : (a.r.rec.hd == 64 ? pick<64>(a, e, f32, grid, st) : pick<32>(a, e, f32, grid, st));
}

cudaError_t launch_attend_join(const AttendArgs &a, const Envs &e, bool f32, int grid, int n_sms, cudaStream_t st)
{
    const long long rows = (long long)e.n * a.r.H * a.r.heads;
    const long long cap = grid ? grid : (long long)n_sms * 8;
    const int g = (int)(rows < cap ? rows : cap);
    if (g == 0) return cudaSuccess;
    switch (a.r.rec.hd) {
    case 128: return f32 ? launch_kernel(attend_join_kernel<128, true>, g, 256, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<128, false>, g, 256, 0, st, 1, a, e);
    case 64: return f32 ? launch_kernel(attend_join_kernel<64, true>, g, 256, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<64, false>, g, 256, 0, st, 1, a, e);
    default: return f32 ? launch_kernel(attend_join_kernel<32, true>, g, 256, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<32, false>, g, 256, 0, st, 1, a, e);
    }
}

}  // namespace p8
}  // namespace ebrl
