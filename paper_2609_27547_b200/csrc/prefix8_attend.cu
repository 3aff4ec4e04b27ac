// Softmax attention over 8-bit prefix records (include/ebrl_prefix8.h): out = softmax(scale q k^T) v, k = code * scale.
//
// Bound: HBM.  Each code is read once and used by the 1 .. 32 query rows of a row tile -- 32 flops per byte at 8 rows, far left of
// the ridge even on mma.sync (955 MAC/clk/SM measured; 16 rows at full copy bandwidth need 370) -- so what counts is that
// bytes are always in flight and that a code costs few instructions.
//
//   Item = (environment, piece of its prefix, key/value head, row tile), worked on by a TEAM of four warps; a team shares
//   nothing with another one.  Warp w takes the tiles (32 tokens) w, w + 4, ... with its own running softmax and its own ring of
//   tile slots (keys and values alternate) filled by cp.async: a record's head is contiguous, so a tile is one straight
//   4 KB run at head_dim 128, and no warp ever waits for another one before the end of the item.  There the four partial results
//   are joined in shared memory, in warp order.
//   SMs hold 4 teams at 8 rows, 3 at 16, 2 at 32 (what registers allow); 96 - 190 KB of tiles are in flight per SM, three
//   times what HBM latency asks for.  With all SMs to itself the launch is one CTA per team, which lets the hardware
//   even out ragged prefixes; under an SM quota it is a persistent grid of `quota` CTAs that hold all of an SM's teams.
//
//   Running maximum, lazily: a row's reference is raised only when a score exceeds it by 2^14 / 2^6; until then the weights
//   2^(s - ref) stay below 2^14, which f16 holds with the same 11 bits.  The common tile needs one vote and no
//   shuffles.  Weights aim at 2^6 rather than 1, so that those 2^-20 of the largest are still normal f16 numbers.
//   A block's value scale is applied in fp32 to the block's own product (tmp), not to the weights: any finite scales work.
//
//   fp32 queries: q and the weights are held in two f16 terms each (22 bits; 2^-23 relative), the codes are exact in f16,
//   sums are fp32.  bf16 queries: q exact, weights rounded to 11 bits, an eighth of the output's own rounding.
#include "prefix8_tile.cuh"
#include "rowops.cuh"

#include <float.h>

namespace ebrl {
namespace p8 {

template <int HD, int NT, bool F32> struct AttendCfg {
    static constexpr int TEAMS = F32 ? (NT == 1 ? 3 : 2) : (NT == 1 ? 4 : (NT == 2 ? 3 : 2));
    static constexpr int TILE = BLOCK * HD;
    static constexpr int RING = HD == 32 ? 8192 : 49152 / TEAMS;      // bytes per warp
    static constexpr int SLOTS = RING / TILE;                         // 3, 4, 6 at head_dim 128
    static constexpr bool QS = NT >= 2;                               // queries in shared memory: registers hold the outputs
    static constexpr int QBYTES = QS ? (HD / 16) * NT * 2 * 32 * 4 * (F32 ? 2 : 1) + NT * 8 * 4 : 0;   // per team, + row factors
    static constexpr int PSTRIDE = HD + 4;                            // floats per row of a warp's partial result
    static_assert(SLOTS >= 3, "ring");
    static_assert(NT * 8 * (PSTRIDE + 2) * 4 <= RING, "a warp's partial result fits its ring");
    static constexpr int smem(int teams) { return teams * (4 * RING + QBYTES); }
};

// barriers by literal number: a number in a register would claim all sixteen of the CTA
__device__ __forceinline__ void team_sync(int team)
{
    if (team == 0) asm volatile("bar.sync 1, 128;" ::: "memory");
    else if (team == 1) asm volatile("bar.sync 2, 128;" ::: "memory");
    else if (team == 2) asm volatile("bar.sync 3, 128;" ::: "memory");
    else asm volatile("bar.sync 4, 128;" ::: "memory");
}

template <int HD, int NT, bool F32>
__global__ void __launch_bounds__(AttendCfg<HD, NT, F32>::TEAMS * 128, 1)
attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    using C = AttendCfg<HD, NT, F32>;
    constexpr int KS = HD / 16, MT = HD / 16, W = HD / 32;
    extern __shared__ __align__(128) char smem[];
    const int teams = blockDim.x >> 7, team = threadIdx.x >> 7, tid = threadIdx.x & 127, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    char *ring = smem + (size_t)(team * 4 + warp) * C::RING;
    const uint32_t ring_u = ptx::smem_u32(ring);
    char *qsm = smem + (size_t)teams * 4 * C::RING + team * C::QBYTES;
    const uint32_t qsm_u = ptx::smem_u32(qsm);
    const float *qf = reinterpret_cast<const float *>(qsm + C::QBYTES - NT * 8 * 4);
    const int G = a.r.G, R = a.r.H * G, RT = (R + NT * 8 - 1) / (NT * 8), kvh = a.r.rec.kvh;
    const int n_envs = a.r.meta ? a.r.n_envs : ev.n;
    const long long items = (long long)n_envs * kvh * a.n_split * RT;
    uint32_t koff[2], voff[2];
    KeyWords<HD>::offsets(koff, g, t);
    voff[0] = tile_addr<HD>(2 * t, g * (HD / 8));
    voff[1] = tile_addr<HD>(2 * t + 1, g * (HD / 8));
    pdl_launch_dependents();
    pdl_wait();

    for (long long item = (long long)blockIdx.x * teams + team; item < items; item += (long long)gridDim.x * teams) {
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
        const int ntile = (t1 - t0 + BLOCK - 1) / BLOCK, mine = ntile > warp ? (ntile - warp + 3) / 4 : 0;
        const char *kp = rec + a.r.rec.head(a.r.layer, 0, kh) + (size_t)t0 * HD, *vp = rec + a.r.rec.head(a.r.layer, 1, kh) + (size_t)t0 * HD;

        // slot j of the warp's stream: keys (even) or values (odd) of its tile j / 2; one commit group each, empty past the end
        auto issue = [&](int j, int slot) {
            if (j < 2 * mine) {
                const int tile = warp + 4 * (j >> 1);
                request_tile<HD>(ring_u + (uint32_t)(slot * C::TILE), ((j & 1) ? vp : kp) + (size_t)tile * C::TILE, min(BLOCK, t1 - t0 - tile * BLOCK), lane);
            }
            cp_commit();
        };
#pragma unroll
        for (int j = 0; j < C::SLOTS - 1; ++j) issue(j, j);

        // queries
        uint32_t qh[C::QS ? 1 : NT][KS][2], ql[C::QS || !F32 ? 1 : NT][KS][2];
        float fr[NT][2];   // what takes a raw product of row 2t (+ 1) of column tile nt to a score in units of log 2 (times the key scale)
        auto q_row = [&](int nt, uint32_t (*hi)[2], uint32_t (*lo)[2]) {
            const int r = rt * NT * 8 + nt * 8 + g, tok = r / G;
            const size_t off = (size_t)env * a.r.q_env + (size_t)tok * a.r.q_tok + (size_t)(kh * G + r - tok * G) * HD;
            const void *p = F32 ? (const void *)((const float *)a.r.q + off) : (const void *)((const __nv_bfloat16 *)a.r.q + off);
            return load_q<HD, F32>(p, r < R, t, hi, lo) * (a.r.scale * LOG2E);
        };
        if constexpr (!C::QS) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float f = q_row(nt, qh[nt], ql[F32 ? nt : 0]);
                fr[nt][0] = __shfl_sync(FULL, f, 8 * t);
                fr[nt][1] = __shfl_sync(FULL, f, 8 * t + 4);
            }
        } else {
            // warp w brings column tile w; words of two column tiles side by side: [term][step][pair][lane][4]
            if (warp < NT) {
                uint32_t hi[KS][2], lo[KS][2];
                const float f = q_row(warp, hi, lo);
                uint32_t *dst = reinterpret_cast<uint32_t *>(qsm);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    uint32_t *d = dst + ((s * (NT / 2) + (warp >> 1)) * 32 + lane) * 4 + (warp & 1) * 2;
                    *reinterpret_cast<uint2 *>(d) = make_uint2(hi[s][0], hi[s][1]);
                    if constexpr (F32) *reinterpret_cast<uint2 *>(d + KS * (NT / 2) * 32 * 4) = make_uint2(lo[s][0], lo[s][1]);
                }
                if (t == 0) const_cast<float *>(qf)[warp * 8 + g] = f;
            }
            team_sync(team);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) { fr[nt][0] = qf[nt * 8 + 2 * t]; fr[nt][1] = qf[nt * 8 + 2 * t + 1]; }
        }

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
        float ks_l = 0.f, vs_l = 0.f;      // scales and visible tokens of this warp's tiles i0 + lane
        uint32_t mk_l = 0;
        const float *ksp = reinterpret_cast<const float *>(rec + a.r.rec.head_scales(a.r.layer, 0, kh)) + t0 / BLOCK;
        const float *vsp = reinterpret_cast<const float *>(rec + a.r.rec.head_scales(a.r.layer, 1, kh)) + t0 / BLOCK;
        const uint32_t *mkp = reinterpret_cast<const uint32_t *>(rec + a.r.rec.mask) + t0 / BLOCK;
        int slot = 0;
        for (int i = 0; i < mine; ++i) {
            if ((i & 31) == 0) {
                const int tile = warp + 4 * (i + lane);
                mk_l = 0;
                if (tile < ntile) {
                    ks_l = read_scale(ksp[tile]); vs_l = read_scale(vsp[tile]); mk_l = mkp[tile];
                    const int v = t1 - t0 - tile * BLOCK;
                    if (v < BLOCK) mk_l &= (1u << v) - 1u;
                }
            }
            const float ks = __shfl_sync(FULL, ks_l, i & 31), vs = __shfl_sync(FULL, vs_l, i & 31);
            const uint32_t mk = __shfl_sync(FULL, mk_l, i & 31);

            cp_wait<C::SLOTS - 2>();
            __syncwarp();            // the tile is there for every lane, and every lane is done with the slot requested next
            issue(2 * i + C::SLOTS - 1, slot == 0 ? C::SLOTS - 1 : slot - 1);
            const uint32_t kslot = ring_u + (uint32_t)(slot * C::TILE);
            slot = slot + 1 == C::SLOTS ? 0 : slot + 1;

            uint32_t pb[2][NT][2], pl[F32 ? 2 : 1][NT][2];
            if (mk) {
                float s[2][NT][4];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[h][nt][c] = 0.f;
                if constexpr (C::QS) {
                    KeyWords<HD> kw[2];
                    kw[0].load(kslot, koff, 0);
                    kw[1].load(kslot, koff, 1);
#pragma unroll
                    for (int st = 0; st < KS; ++st) {
                        uint32_t f[2][4];
                        key_operand(st, kw[0].a[st], kw[0].b[st], f[0]);
                        key_operand(st, kw[1].a[st], kw[1].b[st], f[1]);
#pragma unroll
                        for (int term = 0; term < (F32 ? 2 : 1); ++term)
#pragma unroll
                            for (int pr = 0; pr < NT / 2; ++pr) {
                                const uint4 b = lds128(qsm_u + (uint32_t)((((term * KS + st) * (NT / 2) + pr) * 32 + lane) * 16));
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    mma(s[h][2 * pr], f[h][0], f[h][1], f[h][2], f[h][3], b.x, b.y);
                                    mma(s[h][2 * pr + 1], f[h][0], f[h][1], f[h][2], f[h][3], b.z, b.w);
                                }
                            }
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        KeyWords<HD> kw;
                        kw.load(kslot, koff, h);
#pragma unroll
                        for (int st = 0; st < KS; ++st) {
                            uint32_t f[4];
                            key_operand(st, kw.a[st], kw.b[st], f);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma(s[h][nt], f[0], f[1], f[2], f[3], qh[nt][st][0], qh[nt][st][1]);
                                if constexpr (F32) mma(s[h][nt], f[0], f[1], f[2], f[3], ql[nt][st][0], ql[nt][st][1]);
                            }
                        }
                    }
                }
                bool above = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float c0 = ks * fr[nt][0], c1 = ks * fr[nt][1];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        s[h][nt][0] *= c0; s[h][nt][1] *= c1; s[h][nt][2] *= c0; s[h][nt][3] *= c1;
                    }
                }
                if (mk != FULL) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const bool s0 = (mk >> (16 * h + g)) & 1, s1 = (mk >> (16 * h + 8 + g)) & 1;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (!s0) s[h][nt][0] = s[h][nt][1] = -INFINITY;
                            if (!s1) s[h][nt][2] = s[h][nt][3] = -INFINITY;
                        }
                    }
                }
                float top[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        top[nt][j] = fmaxf(fmaxf(s[0][nt][j], s[0][nt][j + 2]), fmaxf(s[1][nt][j], s[1][nt][j + 2]));
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
                        const float p0 = ex2(s[h][nt][0] - mr[nt][0]), p1 = ex2(s[h][nt][1] - mr[nt][1]);
                        const float p2 = ex2(s[h][nt][2] - mr[nt][0]), p3 = ex2(s[h][nt][3] - mr[nt][1]);
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
            issue(2 * i + C::SLOTS, slot == 0 ? C::SLOTS - 1 : slot - 1);
            const uint32_t vslot = ring_u + (uint32_t)(slot * C::TILE);
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
                        // two columns of two tokens each, the tokens side by side for the conversion unit, a byte apart for spreading
                        const uint32_t sel = by_unit(m) ? (sub ? 0x7362u : 0x5140u) : (sub ? 0x7632u : 0x5410u);
                        const float vf = by_unit(m) ? vs : vs * 256.f;
                        uint32_t f[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t p = prmt(v[h][0][wd], v[h][1][wd], sel), r = prmt(v[h][2][wd], v[h][3][wd], sel);
                            if (by_unit(m)) { f[h][0] = widen(p); f[h][1] = widen(p >> 16); f[h][2] = widen(r); f[h][3] = widen(r >> 16); }
                            else { f[h][0] = spread_even(p); f[h][1] = spread_odd(p); f[h][2] = spread_even(r); f[h][3] = spread_odd(r); }
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
                            for (int c = 0; c < 4; ++c) o[m][nt][c] = fmaf(vf, tmp[c], o[m][nt][c]);
                        }
                    }
            }
        }
        cp_wait<0>();      // only empty groups are left; the ring is free
        __syncwarp();

        // the warp's partial result into its ring, then the team's join
        float *part = reinterpret_cast<float *>(ring), *ml = part + NT * 8 * C::PSTRIDE;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float s = l[nt][j];
                s += __shfl_xor_sync(FULL, s, 4);
                s += __shfl_xor_sync(FULL, s, 8);
                s += __shfl_xor_sync(FULL, s, 16);
                const int row = nt * 8 + 2 * t + j;
                if (g == 0) { ml[2 * row] = mr[nt][j]; ml[2 * row + 1] = s; }
                float *dst = part + row * C::PSTRIDE + g * (HD / 8);
#pragma unroll
                for (int q = 0; q < HD / 32; ++q)
                    *reinterpret_cast<float4 *>(dst + 4 * q) = make_float4(o[2 * q][nt][j], o[2 * q][nt][j + 2], o[2 * q + 1][nt][j], o[2 * q + 1][nt][j + 2]);
            }
        team_sync(team);
        const int rows = min(NT * 8, R - rt * NT * 8);
        const float *p0 = reinterpret_cast<const float *>(smem + (size_t)team * 4 * C::RING);
        for (int v = tid; v < rows * (HD / 4); v += 128) {
            const int row = v / (HD / 4), col = (v % (HD / 4)) * 4, r = rt * NT * 8 + row, tok = r / G, head = kh * G + r - tok * G;
            float m[4], M = -FLT_MAX, L = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                m[w] = p0[(size_t)w * (C::RING / 4) + NT * 8 * C::PSTRIDE + 2 * row];
                M = m[w] > M ? m[w] : M;
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float *pw = p0 + (size_t)w * (C::RING / 4);
                const float f = ex2(m[w] - M);
                const float4 u = *reinterpret_cast<const float4 *>(pw + row * C::PSTRIDE + col);
                L = fmaf(f, pw[NT * 8 * C::PSTRIDE + 2 * row + 1], L);
                acc.x = fmaf(f, u.x, acc.x); acc.y = fmaf(f, u.y, acc.y); acc.z = fmaf(f, u.z, acc.z); acc.w = fmaf(f, u.w, acc.w);
            }
            if (a.n_split > 1) {
                const size_t at = ((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + (size_t)tok * a.r.heads + head;
                *reinterpret_cast<float4 *>(a.part_o + at * HD + col) = acc;
                if (col == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(M, L);
                continue;
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            acc.x *= inv; acc.y *= inv; acc.z *= inv; acc.w *= inv;
            const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + col;
            if constexpr (F32) {
                if (a.split_out) store_split4(a.out, a.out_t1, a.out_t2, off, acc.x, acc.y, acc.z, acc.w);
                else store4<float>((float *)a.out + off, acc.x, acc.y, acc.z, acc.w);
            } else {
                store4<__nv_bfloat16>((__nv_bfloat16 *)a.out + off, acc.x, acc.y, acc.z, acc.w);
            }
            if (a.lse && col == 0) a.lse[((size_t)env * a.r.H + tok) * a.r.heads + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
        }
        team_sync(team);   // the rings (and the staged queries) are free for the next item
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
        cudaError_t err = cudaFuncSetAttribute(attend_kernel<HD, NT, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::smem(C::TEAMS));
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    const long long n = a.r.meta ? a.r.n_envs : e.n;
    const long long items = n * a.r.rec.kvh * a.n_split * ((a.r.H * a.r.G + NT * 8 - 1) / (NT * 8));
    if (items == 0) return cudaSuccess;
    const int teams = grid ? C::TEAMS : 1;
    const long long need = (items + teams - 1) / teams, cap = grid ? grid : 1 << 20;
    return launch_kernel(attend_kernel<HD, NT, F32>, (int)(need < cap ? need : cap), teams * 128, (size_t)C::smem(teams), st, 1, a, e);
}

template <int HD> cudaError_t pick(const AttendArgs &a, const Envs &e, bool f32, int grid, cudaStream_t st)
{
    const int nt = row_tile(a.r.H * a.r.G) / 8;
    if (f32) return nt == 1 ? go<HD, 1, true>(a, e, grid, st) : (nt == 2 ? go<HD, 2, true>(a, e, grid, st) : go<HD, 4, true>(a, e, grid, st));
    return nt == 1 ? go<HD, 1, false>(a, e, grid, st) : (nt == 2 ? go<HD, 2, false>(a, e, grid, st) : go<HD, 4, false>(a, e, grid, st));
}

}  // namespace

int attend_teams(int hd, int rows, bool f32)
{
    (void)hd;
    const int nt = row_tile(rows) / 8;
    return f32 ? (nt == 1 ? AttendCfg<128, 1, true>::TEAMS : AttendCfg<128, 2, true>::TEAMS)
               : (nt == 1 ? AttendCfg<128, 1, false>::TEAMS : (nt == 2 ? AttendCfg<128, 2, false>::TEAMS : AttendCfg<128, 4, false>::TEAMS));
}

cudaError_t launch_attend(const AttendArgs &a, const Envs &e, bool f32, int max_len, int grid, cudaStream_t st)
{
    (void)max_len;
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
