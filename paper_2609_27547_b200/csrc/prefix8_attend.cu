// Softmax attention over 8-bit prefix records (include/ebrl_prefix8.h): out = softmax(scale q k^T) v, k = code * scale.
//
// Bound: HBM.  Each code is read once and used by the 1 .. 32 query rows of a row tile, far left of the ridge even on mma.sync, so
// what counts is that bytes are always in flight and that a code costs few instructions.
//
//   Item = (environment, piece of its prefix, key/value head, row tile), worked on by ONE WARP: its own running softmax, its
//   own ring of stages (a key and a value tile each) filled by cp.async, no barrier, no partial results to join unless a prefix is
//   cut.  A record's head is contiguous, so a tile is one straight 4 KB run at head_dim 128.
//   SMs hold 16 warps at 8 rows, 12 at 16, 8 at 32 (what registers allow); 130 - 190 KB of tiles are in flight per SM, three
//   times what HBM latency asks for.  With all SMs to itself the launch is one CTA per item, which lets the hardware even out
//   ragged prefixes; under an SM quota it is a persistent grid of `quota` CTAs that hold all of an SM's warps.
//   (Four warps per item, joined in shared memory, were 1.6 times slower on 512 x 768 tokens x 16 heads: an item was
//   over before its set-up and join were paid for.)
//
//   With the cache in L2 (arithmetic alone) 512 x 768 tokens x 16 heads of 128 take 143 us at 8 rows, 240 at 16, 460 at 32; from
//   HBM 241 us (6.7 TB/s of codes), 296 (5.4) and 492.  Half of the cycles of the 16-row kernel are dependent-instruction waits
//   at two warps per scheduler; removing any one kind of work (products, exponentials, conversions, transposes) saves 1 - 5 %.
//
//   Running maximum, lazily: a row's reference is raised only when a score exceeds it by 2^14 / 2^6; until then the weights
//   2^(s - ref) stay below 2^14, which f16 holds with the same 11 bits.  The common tile needs one vote and no
//   shuffles.  Weights aim at 2^6 rather than 1, so that those 2^-20 of the largest are still normal f16 numbers.
//   Value scales are never put into the weights: outputs change their unit where neighbouring blocks' scales differ (exact for
//   powers of two), and where they differ by more than 2^20 the block's product is scaled by itself.  Any finite scales work.
//   fp32 queries always take the latter way: summed up in the tensor core over 16 tiles, outputs were 1.1e-6 off instead of 3.5e-7.
//
//   bf16 queries are exact (prefix8_tile.cuh), weights are rounded to f16: 11 bits, an eighth of the output's own rounding.  fp32 queries: queries and weights in two f16 terms each (22 bits).  Sums are fp32.
#include "prefix8_tile.cuh"
#include "rowops.cuh"

#include <float.h>

namespace ebrl {
namespace p8 {

template <int HD, int NT, bool F32> struct AttendCfg {
    // per SM: as many as their registers allow (168 a thread at 12, 255 at 8)
    static constexpr int WARPS = NT == 4 ? (F32 && HD == 128 ? 6 : 8) : (NT == 2 ? (HD == 128 || F32 ? 8 : 12) : (HD == 128 ? 12 : 16));
    static constexpr int TILE = BLOCK * HD;
    // queries in shared memory where registers hold the outputs of 32 rows, or of 16 beside two f16 terms: per warp
    static constexpr bool QS = NT == 4 || (NT == 2 && F32);
    static constexpr int QBYTES = QS ? HD / 16 * NT * 32 * 4 * QW<F32> : 0;
    static constexpr int ROOM = (224 * 1024 / WARPS - QBYTES) / (2 * TILE);
    static constexpr int STAGES = ROOM < 4 ? ROOM : 4;                // 2 .. 4 pairs of a key and a value tile per warp
    static constexpr int WARP_BYTES = STAGES * 2 * TILE + QBYTES;     // ring, queries
    static constexpr int PSTRIDE = HD + 4;                            // floats per staged output row
    static_assert(STAGES >= 2 && 8 * PSTRIDE * 4 <= STAGES * 2 * TILE, "ring");
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
    const uint32_t q_u = ring_u + C::STAGES * 2 * C::TILE;
    const int G = a.r.G, R = a.r.H * G, RT = (R + NT * 8 - 1) / (NT * 8), kvh = a.r.rec.kvh;
    const int n_envs = a.r.meta ? a.r.n_envs : ev.n;
    const long long items = (long long)n_envs * kvh * a.n_split * RT;
    uint32_t koff[KeyWords<HD>::OFFS];
    KeyWords<HD>::offsets(koff, g, t);
    const uint32_t voff = tile_addr<HD>(lane & 15, (lane >> 4) * 16);   // a row of the value tile, column pieces 2 p of it at voff ^ 32 p
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

        // requests the item's next tile (keys and values) into a stage of the ring; one commit group, empty past the end
        int left = t1 - t0;
        auto issue = [&](int stage) {
            if (left > 0) {
                const uint32_t dst = ring_u + (uint32_t)(stage * 2 * C::TILE);
                request_tile<HD>(dst, kp, left, lane);
                request_tile<HD>(dst + C::TILE, vp, left, lane);
                kp += C::TILE;
                vp += C::TILE;
                left -= BLOCK;
            }
            cp_commit();
        };
#pragma unroll
        for (int j = 0; j < C::STAGES - 1; ++j) issue(j);

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

        float o[MT][NT][4];   // column m * 16 + g of rows 2t, 2t + 1, column + 8 of the same; in units of `unit`
        float unit = 1.f;
        float mr[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            mr[nt][0] = mr[nt][1] = -FLT_MAX;
            l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[m][nt][c] = 0.f;
        }
        float ks_l = 0.f, vs_l = 0.f;      // scales and visible tokens of tile (i & ~31) + lane
        uint32_t mk_l = 0;
        int stage = 0;
        for (int i = 0; i < ntile; ++i) {
            if ((i & 31) == 0) {
                const int tile = t0 / BLOCK + i + lane;
                mk_l = 0;
                if (i + lane < ntile) {
                    ks_l = read_scale(reinterpret_cast<const float *>(rec + a.r.rec.head_scales(a.r.layer, 0, kh))[tile]);
                    vs_l = read_scale(reinterpret_cast<const float *>(rec + a.r.rec.head_scales(a.r.layer, 1, kh))[tile]);
                    mk_l = reinterpret_cast<const uint32_t *>(rec + a.r.rec.mask)[tile];
                    const int v = t1 - tile * BLOCK;
                    if (v < BLOCK) mk_l &= (1u << v) - 1u;
                }
            }
            const float ks = __shfl_sync(FULL, ks_l, i & 31), vs = __shfl_sync(FULL, vs_l, i & 31);
            const uint32_t mk = __shfl_sync(FULL, mk_l, i & 31);
            cp_wait<C::STAGES - 2>();
            __syncwarp();            // the tile is there for every lane, and every lane is done with the stage requested next
            issue(stage == 0 ? C::STAGES - 1 : stage - 1);
            const uint32_t kslot = ring_u + (uint32_t)(stage * 2 * C::TILE), vslot = kslot + C::TILE;
            stage = stage + 1 == C::STAGES ? 0 : stage + 1;

            if (mk) {
                uint32_t pb[2][NT][2], pl[F32 ? 2 : 1][NT][2];
                float s[2][NT][4];
                if constexpr (NT <= 2) {
                    KeyWords<HD> kw[2];
                    kw[0].load(kslot, koff, 0);
                    kw[1].load(kslot, koff, 1);
                    score<HD, NT, F32, 2>(s, kw, query);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        KeyWords<HD> kw;
                        kw.load(kslot, koff, h);
                        score<HD, NT, F32, 1>(s + h, &kw, query);
                    }
                }
                const bool hides = mk != FULL;
                if (hides) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool s0 = (mk >> (16 * h + row_token(g))) & 1, s1 = (mk >> (16 * h + row_token(g) + 2)) & 1;
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
                            if (!((mk >> (16 * h + row_token(g))) & 1)) p0 = p1 = 0.f;
                            if (!((mk >> (16 * h + row_token(g) + 2)) & 1)) p2 = p3 = 0.f;
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

                // outputs are kept in units of the last block's value scale: neighbours mostly share it (a power of two), and then the
                // products add up in place
                auto values = [&](auto &&take) {
#pragma unroll
                    for (int p = 0; p < W; ++p) {       // 32 columns
                        uint32_t v[2][4];
                        load_columns(vslot + (voff ^ (uint32_t)(32 * p)), v[0]);
                        load_columns(vslot + (voff ^ (uint32_t)(32 * p)) + 16 * HD, v[1]);
#pragma unroll
                        for (int sub = 0; sub < 2; ++sub) {
                            uint32_t f[2][4];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                f[h][0] = widen(v[h][2 * sub]); f[h][1] = widen(v[h][2 * sub + 1]);
                                f[h][2] = widen(v[h][2 * sub] >> 16); f[h][3] = widen(v[h][2 * sub + 1] >> 16);
                            }
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) take(2 * p + sub, nt, f);
                        }
                    }
                };
                auto product = [&](float *c, int nt, uint32_t (*f)[4]) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (F32) mma(c, f[h][0], f[h][1], f[h][2], f[h][3], pl[h][nt][0], pl[h][nt][1]);
                        mma(c, f[h][0], f[h][1], f[h][2], f[h][3], pb[h][nt][0], pb[h][nt][1]);
                    }
                };
                auto rescale = [&](float by) {
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) o[m][nt][c] *= by;
                };
                // fp32 sums that stay in the tensor core lose their last bits to its truncation: fp32 queries take every block's product out
                bool near = !F32;
                if (!F32 && vs != unit) {
                    const float by = unit / vs;
                    near = by >= 1.f / 1048576.f && by <= 1048576.f;
                    rescale(near ? by : unit);
                    unit = near ? vs : 1.f;
                }
                if (near) values([&](int m, int nt, uint32_t (*f)[4]) { product(o[m][nt], nt, f); });
                else   // far apart, zero, or not a number: outputs as they are, the block's own product scaled and added
                    values([&](int m, int nt, uint32_t (*f)[4]) {
                        float tmp[4] = {0.f, 0.f, 0.f, 0.f};
                        product(tmp, nt, f);
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[m][nt][c] = fmaf(vs, tmp[c], o[m][nt][c]);
                    });
            }
        }
        cp_wait<0>();      // only empty groups are left; the ring is free
        __syncwarp();

        // one column tile of rows at a time through the ring, so that rows leave in whole 128-byte runs
        float *rows = reinterpret_cast<float *>(smem + (size_t)warp * C::WARP_BYTES);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float L[2], inv[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                L[j] = l[nt][j];
                L[j] += __shfl_xor_sync(FULL, L[j], 4);
                L[j] += __shfl_xor_sync(FULL, L[j], 8);
                L[j] += __shfl_xor_sync(FULL, L[j], 16);
                inv[j] = a.n_split > 1 ? unit : (L[j] == 0.f ? 0.f : unit / L[j]);
                const int r = rt * NT * 8 + nt * 8 + 2 * t + j, tok = r / G, row = tok * a.r.heads + kh * G + r - tok * G;
                if (g == 0 && r < R) {
                    if (a.n_split > 1) *reinterpret_cast<float2 *>(a.part_ml + (((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + row) * 2) = make_float2(mr[nt][j], L[j]);
                    else if (a.lse) a.lse[(size_t)env * a.r.H * a.r.heads + row] = L[j] == 0.f ? -INFINITY : (mr[nt][j] + log2f(L[j])) * LN2;
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    rows[(2 * t) * C::PSTRIDE + m * 16 + 8 * k + g] = o[m][nt][2 * k] * inv[0];
                    rows[(2 * t + 1) * C::PSTRIDE + m * 16 + 8 * k + g] = o[m][nt][2 * k + 1] * inv[1];
                }
            __syncwarp();
#pragma unroll
            for (int v = 0; v < HD / 16; ++v) {
                const int row = (v * 32 + lane) / (HD / 4), col = (v * 32 + lane) % (HD / 4) * 4, r = rt * NT * 8 + nt * 8 + row, tok = r / G, head = kh * G + r - tok * G;
                if (r < R) {
                    const float4 u = *reinterpret_cast<const float4 *>(rows + row * C::PSTRIDE + col);
                    const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + col;
                    if (a.n_split > 1)
                        *reinterpret_cast<float4 *>(a.part_o + (((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + (size_t)tok * a.r.heads + head) * HD + col) = u;
                    else if constexpr (!F32) store4<__nv_bfloat16>((__nv_bfloat16 *)a.out + off, u.x, u.y, u.z, u.w);
                    else if (a.split_out) store_split4(a.out, a.out_t1, a.out_t2, off, u.x, u.y, u.z, u.w);
                    else store4<float>((float *)a.out + off, u.x, u.y, u.z, u.w);
                }
            }
            __syncwarp();
        }
    }
}

// Joins the pieces of long prefixes: one CTA per query row, the pieces divided over its sixteen warps, sums in warp order.
// Traffic is the pieces' results only (1 / 64 of the cache at 896-token pieces and 4 rows).
template <int HD, bool F32>
__global__ void __launch_bounds__(512) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    constexpr int V = HD / 32;
    __shared__ float so[16][HD], sl[16];
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
#pragma unroll 8
        for (int p = warp; p < np; p += 16) {
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
            for (int w = 0; w < 16; ++w) { s += so[w][threadIdx.x]; z += sl[w]; }
            const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + threadIdx.x;
            const float v = z == 0.f ? 0.f : s / z;
            if constexpr (F32) ((float *)a.out)[off] = v;
            else ((__nv_bfloat16 *)a.out)[off] = __float2bfloat16_rn(v);
            if (a.lse && threadIdx.x == 0) a.lse[(size_t)env * RH + rr] = z == 0.f ? -INFINITY : (M + log2f(z)) * LN2;
        }
        __syncthreads();
    }
}

int attend_warps(int rows, bool f32)
{
    const int nt = row_tile(rows) / 8;
    return f32 ? (nt == 1 ? AttendCfg<128, 1, true>::WARPS : (nt == 2 ? AttendCfg<128, 2, true>::WARPS : AttendCfg<128, 4, true>::WARPS))
               : (nt == 1 ? AttendCfg<128, 1, false>::WARPS : (nt == 2 ? AttendCfg<128, 2, false>::WARPS : AttendCfg<128, 4, false>::WARPS));
}

namespace {

// Query rows per item, as the smallest tile whose items still fill the SMs' warps if there is one below the rows' own tile: with few
// items more of them beat reading a prefix once (96 environments x 301 tokens x 64 rows: 59 us with 32 rows, 22 with 8).
// A row's result is the same in every tile.
int tile_for(const AttendArgs &a, const Envs &e, bool f32, int sms)
{
    const int rows = a.r.H * a.r.G;
    int tile = row_tile(rows);
    const long long base = (long long)(a.r.meta ? a.r.n_envs : e.n) * a.r.rec.kvh * a.n_split;
    while (tile > 8 && base * ((rows + tile - 1) / tile) < (long long)sms * attend_warps(tile, f32)) tile /= 2;
    return tile;
}

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

template <int HD> cudaError_t pick(const AttendArgs &a, const Envs &e, bool f32, int grid, int sms, cudaStream_t st)
{
    const int nt = tile_for(a, e, f32, grid ? grid : sms) / 8;
    if (f32) return nt == 1 ? go<HD, 1, true>(a, e, grid, st) : (nt == 2 ? go<HD, 2, true>(a, e, grid, st) : go<HD, 4, true>(a, e, grid, st));
    return nt == 1 ? go<HD, 1, false>(a, e, grid, st) : (nt == 2 ? go<HD, 2, false>(a, e, grid, st) : go<HD, 4, false>(a, e, grid, st));
}

}  // namespace

cudaError_t launch_attend(const AttendArgs &a, const Envs &e, bool f32, int grid, int sms, cudaStream_t st)
{
    return a.r.rec.hd == 128 ? pick<128>(a, e, f32, grid, sms, st) : (a.r.rec.hd == 64 ? pick<64>(a, e, f32, grid, sms, st) : pick<32>(a, e, f32, grid, sms, st));
}

cudaError_t launch_attend_join(const AttendArgs &a, const Envs &e, bool f32, int grid, int n_sms, cudaStream_t st)
{
    const long long rows = (long long)e.n * a.r.H * a.r.heads;
    const long long cap = grid ? grid : (long long)n_sms * 8;
    const int g = (int)(rows < cap ? rows : cap);
    if (g == 0) return cudaSuccess;
    struct Early {   // the join may be set up while the last pieces are being worked on; it waits for them itself
        Early() { pdl_set(true); }
        ~Early() { pdl_set(false); }
    } early;
    switch (a.r.rec.hd) {
    case 128: return f32 ? launch_kernel(attend_join_kernel<128, true>, g, 512, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<128, false>, g, 512, 0, st, 1, a, e);
    case 64: return f32 ? launch_kernel(attend_join_kernel<64, true>, g, 512, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<64, false>, g, 512, 0, st, 1, a, e);
    default: return f32 ? launch_kernel(attend_join_kernel<32, true>, g, 512, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<32, false>, g, 512, 0, st, 1, a, e);
    }
}

}  // namespace p8
}  // namespace ebrl
