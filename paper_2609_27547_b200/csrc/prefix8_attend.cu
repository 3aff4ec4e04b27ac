// Softmax attention over 8-bit prefix records (include/ebrl_prefix8.h): out = softmax(scale q k^T) v, k = code * scale.
//
// Bound: HBM.  Each code is read once and used by the 1 .. 16 query rows of a row tile, far left of the ridge even on mma.sync, so
// what counts is that bytes are always in flight and that a code costs few instructions.
//
//   Item = (environment, piece of its prefix, key/value head, row tile), worked on by ONE WARP: its own running softmax, its
//   own ring of stages (a key and a value tile each) filled by cp.async, no barrier, no partial results to join unless a prefix is
//   cut.  A record's head is contiguous, so a tile is one straight 4 KB run at head_dim 128.
//   At head_dim 128 SMs hold 12 warps at 8 rows and 8 at 16, at 64 they hold 16 and 12 (what registers allow); 96 - 130 KB of
//   tiles are in flight per SM, twice what HBM latency asks for, and a warp's requests run on from one item into the next
//   (512 x 768 tokens x 16 heads x 16 rows: 314 -> 294 us).  Where prefixes are alike, or under an SM quota, warps are persistent;
//   where they differ the launch is one CTA per item, which lets the hardware even them out.
//   Calls that would leave most of the SMs empty share an item among a TEAM of 2, 4 or 8 warps (the CTA): each an even share of
//   the tokens, joined in warp order through the rings, which are idle by then (1 x 256 tokens x 16 heads of 64: 8.4 -> 6.0 us).  With the
//   SMs full a team of four is 1.5 times slower: an item is over before its set-up and join are paid for.
//
//   With the cache in L2 (arithmetic alone) 512 x 768 tokens x 16 heads of 128 take 150 us at 8 rows and 228 at 16; from HBM
//   240 us (6.7 TB/s of codes) and 286 (5.6; 294 at the power cap).  At 16 rows the legacy tensor path is what it waits for: a product
//   occupies a quarter-SM for 9 cycles (64 a tile), fp32 instructions do not run beside it (conversions and exponentials do),
//   and the sum of both is 740 of the 1250 cycles a tile takes.
//
//   Running maximum, lazily: a row's reference is raised only when a score exceeds it by 2^14 / 2^6; until then the weights
//   2^(s - ref) stay below 2^14, which f16 holds with the same 11 bits.  The common tile needs one vote and no
//   shuffles.  Weights aim at 2^6 rather than 1, so that those 2^-20 of the largest are still normal f16 numbers.
//   Value scales are never put into the weights: outputs change their unit where neighbouring blocks' scales differ (exact for
//   powers of two), and a block whose scale is 2^20 below the largest so far has its product scaled by itself.  Any finite scales work, zero and
//   subnormal ones too (such a block is scaled by itself).
//   fp32 queries always take the latter way: summed up in the tensor core over 16 tiles, outputs were 1.1e-6 off instead of 3.5e-7.
//
//   bf16 queries are exact (prefix8_tile.cuh), weights are rounded to f16: 11 bits, an eighth of the output's own rounding.
//   fp32 queries: queries and weights in two f16 terms each (22 bits).  Sums are fp32.
#include "prefix8_tile.cuh"
#include "rowops.cuh"

#include <float.h>

namespace ebrl {
namespace p8 {

template <int HD, int NT> struct AttendCfg {
    // per SM: as many as their registers allow (128 a thread at 16, 168 at 12, 255 at 8)
    static constexpr int WARPS = HD == 128 ? (NT == 1 ? 12 : 8) : (NT == 1 ? 16 : 12);
    static constexpr int TILE = BLOCK * HD;
    static constexpr int ROOM = 224 * 1024 / WARPS / (2 * TILE);
    static constexpr int STAGES = ROOM < 4 ? ROOM : 4;                // 2 .. 4 pairs of a key and a value tile per warp
    static constexpr int WARP_BYTES = STAGES * 2 * TILE;              // its ring
    static_assert(STAGES >= 2, "ring");
};

template <int HD, int NT, bool F32, bool TEAM>
__global__ void __launch_bounds__(AttendCfg<HD, NT>::WARPS * 32, 1)
attend_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    using C = AttendCfg<HD, NT>;
    constexpr int MT = HD / 16, W = HD / 32, ST = HD / 16;
    extern __shared__ __align__(128) char smem[];
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const uint32_t ring_u = ptx::smem_u32(smem + (size_t)warp * C::WARP_BYTES);
    const int G = a.r.G, R = a.r.H * G, RT = (R + NT * 8 - 1) / (NT * 8), kvh = a.r.rec.kvh;
    const int n_envs = a.r.meta ? a.r.n_envs : ev.n;
    const long long items = (long long)n_envs * kvh * a.n_split * RT;
    uint32_t koff[KeyWords<HD>::OFFS];
    KeyWords<HD>::offsets(koff, g, t);
    const uint32_t voff = tile_addr<HD>(lane & 15, (lane >> 4) * 16);   // a row of the value tile, column pieces 2 p of it at voff ^ 32 p
    pdl_launch_dependents();
    pdl_wait();

    // what item `i` is: its row tile, head, piece, environment, record and tokens t0 .. t1 (none past the prefix's end)
    struct Item { int rt, kh, sp, env, len, t0, t1; const char *rec; };
    auto item_of = [&](unsigned x) {
        Item it;
        it.rt = (int)(x % (unsigned)RT); x /= (unsigned)RT;
        it.kh = (int)(x % (unsigned)kvh); x /= (unsigned)kvh;
        it.sp = (int)(x % (unsigned)a.n_split); it.env = (int)(x / (unsigned)a.n_split);
        if (a.r.meta) { it.rec = (const char *)a.r.meta[it.env].kv; it.len = a.r.meta[it.env].P; }
        else { it.rec = a.r.pool + (size_t)ev.slot[it.env] * a.r.rec.bytes; it.len = ev.len[it.env]; }
        it.t0 = it.sp * a.split;
        it.t1 = a.n_split == 1 ? it.len : min(it.len, it.t0 + a.split);
        if constexpr (TEAM) {   // this warp's even share
            const int part = (it.t1 - it.t0 + warps * BLOCK - 1) / (warps * BLOCK) * BLOCK;
            it.t0 += warp * part;
            it.t1 = min(it.t1, it.t0 + part);
        }
        return it;
    };
    auto q_at = [&](const Item &it, int row) {   // offset of query row `row` of the item's kv head, in elements
        const int tok = row / G;
        return (size_t)it.env * a.r.q_env + (size_t)tok * a.r.q_tok + (size_t)(it.kh * G + row - tok * G) * HD;
    };
    // items go round the CTAs first, so that the last round spreads over all SMs
    const unsigned first = TEAM ? blockIdx.x : (unsigned)warp * gridDim.x + blockIdx.x, stride = gridDim.x * (TEAM ? 1u : (unsigned)warps);

    // The requests run STAGES - 1 tiles ahead of the arithmetic, from one item into the next: while an item's last tiles are worked on the next
    // one's first tiles (and its queries, scales and mask, into L1) are on their way.
    unsigned asked = first;     // the item being requested; its next tile, and the tokens that are left from there on
    const char *kp = nullptr, *vp = nullptr;
    int left = 0;
    auto seek = [&]() {
        while (asked < (unsigned)items) {
            const Item it = item_of(asked);
            left = it.t1 - it.t0;
            if (left > 0) {
                kp = it.rec + a.r.rec.head(a.r.layer, 0, it.kh) + (size_t)it.t0 * HD;
                vp = it.rec + a.r.rec.head(a.r.layer, 1, it.kh) + (size_t)it.t0 * HD;
                constexpr int LINES = HD * (F32 ? 4 : 2) > 128 ? HD * (F32 ? 4 : 2) / 128 : 1;   // 128-byte lines of a query row
#pragma unroll
                for (int i = 0; i < (NT * 8 * LINES + 31) / 32; ++i) {
                    const int row = it.rt * NT * 8 + (i * 32 + lane) / LINES;
                    if (i * 32 + lane < NT * 8 * LINES && row < R) prefetch_l1((const char *)a.r.q + q_at(it, row) * (F32 ? 4 : 2) + (lane % LINES) * 128);
                }
                if (lane < 3) prefetch_l1((lane < 2 ? it.rec + a.r.rec.head_scales(a.r.layer, lane, it.kh) : it.rec + a.r.rec.mask) + it.t0 / BLOCK * 4);
                return;
            }
            asked += stride;
        }
        left = 0;
    };
    seek();
    auto issue = [&](int stage) {   // one commit group, empty when nothing is left
        if (left > 0) {
            const uint32_t dst = ring_u + (uint32_t)(stage * 2 * C::TILE);
            request_tile<HD>(dst, kp, left, lane);
            request_tile<HD>(dst + C::TILE, vp, left, lane);
            kp += C::TILE;
            vp += C::TILE;
            left -= BLOCK;
            if (left <= 0) { asked += stride; seek(); }
        }
        cp_commit();
    };
#pragma unroll
    for (int j = 0; j < C::STAGES - 1; ++j) issue(j);
    int stage = 0;

    for (unsigned item = first; item < (unsigned)items; item += stride) {
        const Item it = item_of(item);
        const int rt = it.rt, kh = it.kh, sp = it.sp, env = it.env, t0 = it.t0, t1 = it.t1;
        const char *rec = it.rec;
        if (sp > 0 && sp * a.split >= it.len) continue;
        const int ntile = (t1 - t0 + BLOCK - 1) / BLOCK;   // (0 or less for a team's warp that got none)

        // queries
        uint32_t q[NT][ST][QW<F32>];
        float fr[NT][2];   // what takes a raw product of row 2t (+ 1) of column tile nt to a score in units of log 2 (times the key scale)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = rt * NT * 8 + nt * 8 + g;
            const size_t off = q_at(it, r < R ? r : 0);
            const void *p = F32 ? (const void *)((const float *)a.r.q + off) : (const void *)((const __nv_bfloat16 *)a.r.q + off);
            const float f = load_q<HD, F32>(p, r < R, a.r.scale < 0.f, t, q[nt]) * (fabsf(a.r.scale) * LOG2E);
            fr[nt][0] = __shfl_sync(FULL, f, 8 * t);
            fr[nt][1] = __shfl_sync(FULL, f, 8 * t + 4);
        }
        auto query = [&](int st, int nt, uint32_t *w) {
#pragma unroll
            for (int c = 0; c < QW<F32>; ++c) w[c] = q[nt][st][c];
        };

        float o[MT][NT][4];   // column m * 16 + g of rows 2t, 2t + 1, column + 8 of the same; in units of `unit`
        float unit = FLT_MIN, inv_unit = 1.f / FLT_MIN, most = FLT_MIN;   // (a smaller scale never is the unit); the largest scale so far
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
        auto rescale = [&](float by) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[m][nt][c] *= by;
        };
        float ks_l = 0.f, vs_l = 0.f;      // scales and visible tokens of tile (i & ~31) + lane
        uint32_t mk_l = 0;
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
                KeyWords<HD> kw[2];
                kw[0].load(kslot, koff, 0);
                kw[1].load(kslot, koff, 1);
                score<HD, NT, F32>(s, kw, query);
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
                // fp32 sums that stay in the tensor core lose their last bits to its truncation: fp32 queries take every block's product out
                bool near = !F32;
                if (F32 ? vs > unit : vs != unit) {
                    most = fmaxf(most, vs);
                    if (F32 || (near = vs >= fmaxf(most * 0x1p-20f, FLT_MIN))) {   // (bounded, so that outputs of large blocks stay in range, and 1 / vs)
                        inv_unit = 1.f / vs;
                        rescale(unit * inv_unit);
                        unit = vs;
                    }
                }
                if (near) values([&](int m, int nt, uint32_t (*f)[4]) { product(o[m][nt], nt, f); });
                else {   // far below the others, or not a number: the block's own product scaled and added
                    const float by = vs * inv_unit;
                    values([&](int m, int nt, uint32_t (*f)[4]) {
                        float tmp[4] = {0.f, 0.f, 0.f, 0.f};
                        product(tmp, nt, f);
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[m][nt][c] = fmaf(by, tmp[c], o[m][nt][c]);
                    });
                }
            }
        }
        // Outputs: lane (g, t) has columns g of rows 2t, 2t + 1 of 8 x 8 matrices; transposed it has columns 2t, 2t + 1 of row g.
        auto store_ml = [&](int nt, int j, float m, float L) {
            const int r = rt * NT * 8 + nt * 8 + 2 * t + j, tok = r / G, row = tok * a.r.heads + kh * G + r - tok * G;
            if (g == 0 && r < R) {
                if (a.n_split > 1) *reinterpret_cast<float2 *>(a.part_ml + (((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + row) * 2) = make_float2(m, L);
                else if (a.lse) a.lse[(size_t)env * a.r.H * a.r.heads + row] = L == 0.f ? -INFINITY : (m + log2f(L)) * LN2;
            }
        };
        struct At { bool there; size_t off; float *part; };
        auto row_at = [&](int nt) {
            const int r = rt * NT * 8 + nt * 8 + g, tok = r / G, head = kh * G + r - tok * G;
            return At{r < R, (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + 2 * t,
                      a.part_o + (((size_t)env * a.n_split + sp) * ((size_t)a.r.H * a.r.heads) + (size_t)tok * a.r.heads + head) * HD + 2 * t};
        };
        auto store_o = [&](const At &at, int col, float x, float y) {   // rows' softmax-weighted means
            if (F32 || a.n_split > 1) {   // upper and lower halves apart
                const uint32_t xu = __float_as_uint(x), yu = __float_as_uint(y);
                const uint32_t hi = transpose8(__byte_perm(xu, yu, 0x7632)), lo = transpose8(__byte_perm(xu, yu, 0x5410));
                const float2 v = make_float2(__uint_as_float(__byte_perm(lo, hi, 0x5410)), __uint_as_float(__byte_perm(lo, hi, 0x7632)));
                if (at.there) {
                    if (a.n_split > 1) *reinterpret_cast<float2 *>(at.part + col) = v;
                    else if (a.split_out) store_split2(a.out, a.out_t1, a.out_t2, at.off + col, v.x, v.y);
                    else *reinterpret_cast<float2 *>((float *)a.out + at.off + col) = v;
                }
            } else {
                const __nv_bfloat162 u = __floats2bfloat162_rn(x, y);
                const uint32_t w = transpose8(*reinterpret_cast<const uint32_t *>(&u));
                if (at.there) *reinterpret_cast<uint32_t *>((__nv_bfloat16 *)a.out + at.off + col) = w;
            }
        };
        auto sum = [&](float L) {
            L += __shfl_xor_sync(FULL, L, 4);
            L += __shfl_xor_sync(FULL, L, 8);
            return L + __shfl_xor_sync(FULL, L, 16);
        };
        if constexpr (!TEAM) {
            if (unit < 0x1p-64f) {   // (unit / L has to keep its 24 bits)
                rescale(0x1p-64f);
                unit *= 0x1p64f;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float inv[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float L = sum(l[nt][j]);
                    inv[j] = L == 0.f ? 0.f : unit / L;
                    store_ml(nt, j, mr[nt][j], L);
                }
                const At at = row_at(nt);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int k = 0; k < 2; ++k) store_o(at, m * 16 + 8 * k, o[m][nt][2 * k] * inv[0], o[m][nt][2 * k + 1] * inv[1]);
            }
        } else {   // (one item per CTA: nothing is requested any more) join the team's pieces through its rings, in warp order
            constexpr int ML = NT * 8 * HD * 4;   // a warp's outputs, then its rows' (reference, sum) and its unit
            static_assert(ML + NT * 8 * 8 + 4 <= C::WARP_BYTES, "join");
            auto of = [&](int w) { return smem + (size_t)w * C::WARP_BYTES; };
            auto ml = [&](int w, int nt, int j) { return *reinterpret_cast<const float2 *>(of(w) + ML + (nt * 8 + 2 * t + j) * 8); };
            cp_wait<0>();
            __syncwarp();
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<float4 *>(of(warp) + ((m * NT + nt) * 32 + lane) * 16) = make_float4(o[m][nt][0], o[m][nt][1], o[m][nt][2], o[m][nt][3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float L = sum(l[nt][j]);
                    if (g == 0) *reinterpret_cast<float2 *>(of(warp) + ML + (nt * 8 + 2 * t + j) * 8) = make_float2(mr[nt][j], L);
                }
            if (lane == 0) *reinterpret_cast<float *>(of(warp) + ML + NT * 8 * 8) = unit;
            __syncthreads();
            float largest = 0.f;   // of the units; where all are small, sums are formed 2^64 as large, so that neither they nor their factors lose bits
            for (int w = 0; w < warps; ++w) largest = fmaxf(largest, *reinterpret_cast<const float *>(of(w) + ML + NT * 8 * 8));
            const float up = largest < 0x1p-64f ? 0x1p64f : 1.f, down = 1.f / up;
            float M[NT][2], inv[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float mx = -FLT_MAX, z = 0.f;
                    for (int w = 0; w < warps; ++w) mx = fmaxf(mx, ml(w, nt, j).x);
                    for (int w = 0; w < warps; ++w) { const float2 v = ml(w, nt, j); z = fmaf(ex2(v.x - mx), v.y, z); }
                    M[nt][j] = mx;
                    inv[nt][j] = z == 0.f ? 0.f : 1.f / z;
                    if (warp == 0) store_ml(nt, j, mx, z);
                }
            for (int m = warp; m < MT; m += warps) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float x[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int w = 0; w < warps; ++w) {
                        const float4 v = *reinterpret_cast<const float4 *>(of(w) + ((m * NT + nt) * 32 + lane) * 16);
                        const float u = *reinterpret_cast<const float *>(of(w) + ML + NT * 8 * 8) * up;
                        const float f0 = ex2(ml(w, nt, 0).x - M[nt][0]) * inv[nt][0] * u, f1 = ex2(ml(w, nt, 1).x - M[nt][1]) * inv[nt][1] * u;
                        x[0] = fmaf(f0, v.x, x[0]); x[1] = fmaf(f1, v.y, x[1]); x[2] = fmaf(f0, v.z, x[2]); x[3] = fmaf(f1, v.w, x[3]);
                    }
                    const At at = row_at(nt);
                    store_o(at, m * 16, x[0] * down, x[1] * down);
                    store_o(at, m * 16 + 8, x[2] * down, x[3] * down);
                }
            }
        }
    }
    cp_wait<0>();      // only empty groups are left
}

// Joins the pieces of long prefixes: WPR warps per query row (16 where there are many pieces: latency; 1 where there are few: rows),
// the pieces divided over them, sums in warp order.  Traffic is the pieces' results only (1 / 32 of the cache at 384-token pieces and
// 4 rows).
template <int HD, bool F32, int WPR>
__global__ void __launch_bounds__(512) attend_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ Envs ev)
{
    constexpr int V = HD / 32, RPC = 16 / WPR;
    __shared__ float so[16][HD];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, RH = a.r.H * a.r.heads, sub = warp % WPR;
    const long long rows = (long long)ev.n * RH;
    pdl_launch_dependents();
    pdl_wait();
    for (long long row0 = (long long)blockIdx.x * RPC; row0 < rows; row0 += (long long)gridDim.x * RPC) {
        const long long row = row0 + warp / WPR;
        const bool there = row < rows;
        const int env = there ? (int)(row / RH) : 0, rr = there ? (int)(row - (long long)env * RH) : 0, tok = rr / a.r.heads, head = rr - tok * a.r.heads;
        const int np = there ? max(1, (ev.len[env] + a.split - 1) / a.split) : 0;
        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (size_t)env * a.n_split * RH + rr;
        const float *po = a.part_o + ((size_t)env * a.n_split * RH + rr) * HD + lane * V;
        float M = -FLT_MAX, L = 0.f;
        for (int p = lane; p < np; p += 32) M = fmaxf(M, ml[(size_t)p * RH].x);
        M = warp_max(M);
        for (int p = lane; p < np; p += 32) { const float2 u = ml[(size_t)p * RH]; L = fmaf(ex2(u.x - M), u.y, L); }
        L = warp_sum(L);
        const float inv = L == 0.f ? 0.f : 1.f / L;
        float acc[V];
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
#pragma unroll 8
        for (int p = sub; p < np; p += WPR) {
            const float2 u = ml[(size_t)p * RH];
            const float f = ex2(u.x - M) * u.y * inv;
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = fmaf(f, po[(size_t)p * RH * HD + i], acc[i]);
        }
        auto store = [&](int col, float v) {
            const size_t off = (size_t)env * a.o_env + (size_t)tok * a.o_tok + (size_t)head * HD + col;
            if constexpr (F32) ((float *)a.out)[off] = v;
            else ((__nv_bfloat16 *)a.out)[off] = __float2bfloat16_rn(v);
            if (a.lse && col == 0) a.lse[(size_t)env * RH + rr] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
        };
        if constexpr (WPR == 1) {
            if (there) {
#pragma unroll
                for (int i = 0; i < V; ++i) store(lane * V + i, acc[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) so[warp][lane * V + i] = acc[i];
            __syncthreads();
            if (threadIdx.x < HD) {   // (one row per CTA: every thread knows it)
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < 16; ++w) s += so[w][threadIdx.x];
                store(threadIdx.x, s);
            }
            __syncthreads();
        }
    }
}

int attend_warps(int hd, int tile) { return hd == 128 ? (tile == 8 ? AttendCfg<128, 1>::WARPS : AttendCfg<128, 2>::WARPS) : (tile == 8 ? AttendCfg<64, 1>::WARPS : AttendCfg<64, 2>::WARPS); }

// Query rows per item: 8, or 16 where that fills its rows and long prefixes make up for fewer warps per SM.  Rows beyond a tile are
// further items next to this one: they read the same keys and values from L2.  A row's result is the same in every tile.
// Measured, us with 8 / 16 (/ 32, which is gone) rows per item, 16 heads:
//   head_dim 128, 128 x 768 tokens:  16 rows 91 / 83 / 124,  32 rows 146 / 132 / 134,  64 rows 280 / 241 / 251
//                 256 x 256 tokens:  16 rows 71 / 77 / 116,  32 rows 124 / 124 / 134;  512 x 64: 16 rows 70 / 87 / 120
//   head_dim 64,  128 x 768 tokens:  16 rows 50 / 61 / 77,   32 rows  89 /  82 /  82,  64 rows 169 / 141 / 155;  512 x 768: 16 rows 180 / 161
//                 256 x 256 tokens:  16 rows 44 / 48 / 76,   32 rows  79 /  75 /  87;  512 x 64: 32 rows 83 / 91 / 101
//   fp32, 64:     128 x 768 tokens:  16 rows 62 / 68 / 109,  32 rows 114 / 114 / 116: always 8
int attend_tile(int hd, int rows, bool f32, int max_len)
{
    const bool fills = (rows - 1) % 16 >= 8;
    const bool pays = max_len >= 512 || (hd < 128 && rows >= 32 && max_len >= 256);
    return !f32 && fills && pays ? 16 : 8;
}

namespace {

// ... and where items of 16 rows would not keep every warp busy one and a half times, items of 8 (the 50 / 61 above).
int tile_for(const AttendArgs &a, const Envs &e, bool f32, int sms)
{
    const int rows = a.r.H * a.r.G, tile = attend_tile(a.r.rec.hd, rows, f32, a.max_len);
    const long long items = (long long)(a.r.meta ? a.r.n_envs : e.n) * a.r.rec.kvh * a.n_split * ((rows + tile - 1) / tile);
    return 2 * items < 3LL * sms * attend_warps(a.r.rec.hd, tile) ? 8 : tile;
}

template <int HD, int NT, bool F32, bool TEAM = false> cudaError_t go(const AttendArgs &a, const Envs &e, int grid, int sms, cudaStream_t st)
{
    using C = AttendCfg<HD, NT>;
    static std::atomic<bool> set[64];   // (calls may come from several threads; setting it twice is harmless)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        cudaError_t err = cudaFuncSetAttribute(attend_kernel<HD, NT, F32, TEAM>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::WARPS * C::WARP_BYTES);
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    const long long n = a.r.meta ? a.r.n_envs : e.n;
    const long long items = n * a.r.rec.kvh * a.n_split * ((a.r.H * a.r.G + NT * 8 - 1) / (NT * 8));
    if (items == 0) return cudaSuccess;
    // Under a quota: persistent CTAs with all of an SM's warps.  Else one-warp CTAs: as many as the SMs hold where prefixes are alike (the
    // ring then runs on from item to item), one per item where they are not (the hardware hands out the next as one ends).
    const int warps = TEAM ? a.team : (grid ? C::WARPS : 1);
    const long long cap = TEAM ? items : (grid ? grid : (a.alike ? (long long)sms * C::WARPS : 1 << 20));   // (a team takes one item: the join uses its rings)
    return launch_kernel(attend_kernel<HD, NT, F32, TEAM>, (int)(items < cap ? items : cap), warps * 32, (size_t)(warps * C::WARP_BYTES), st, 1, a, e);
}

template <int HD> cudaError_t pick(const AttendArgs &a, const Envs &e, bool f32, int grid, int sms, cudaStream_t st)
{
    if (a.team > 1) return f32 ? go<HD, 1, true, true>(a, e, grid, sms, st) : go<HD, 1, false, true>(a, e, grid, sms, st);
    if (f32) return go<HD, 1, true>(a, e, grid, sms, st);
    return tile_for(a, e, f32, grid ? grid : sms) == 8 ? go<HD, 1, false>(a, e, grid, sms, st) : go<HD, 2, false>(a, e, grid, sms, st);
}

}  // namespace

cudaError_t launch_attend(const AttendArgs &a, const Envs &e, bool f32, int grid, int sms, cudaStream_t st)
{
    return a.r.rec.hd == 128 ? pick<128>(a, e, f32, grid, sms, st) : (a.r.rec.hd == 64 ? pick<64>(a, e, f32, grid, sms, st) : pick<32>(a, e, f32, grid, sms, st));
}

template <int HD, int WPR> static cudaError_t join(const AttendArgs &a, const Envs &e, bool f32, int g, cudaStream_t st)
{
    return f32 ? launch_kernel(attend_join_kernel<HD, true, WPR>, g, 512, 0, st, 1, a, e) : launch_kernel(attend_join_kernel<HD, false, WPR>, g, 512, 0, st, 1, a, e);
}

cudaError_t launch_attend_join(const AttendArgs &a, const Envs &e, bool f32, int grid, int n_sms, cudaStream_t st)
{
    const bool many = a.n_split > 16;
    const long long rows = (long long)e.n * a.r.H * a.r.heads, need = many ? rows : (rows + 15) / 16;
    const long long cap = grid ? grid : (long long)n_sms * 4;
    const int g = (int)(need < cap ? need : cap);
    if (g == 0) return cudaSuccess;
    struct Early {   // the join may be set up while the last pieces are being worked on; it waits for them itself
        const bool before = pdl_enabled();
        Early(bool on) { pdl_set(on); }
        ~Early() { pdl_set(before); }
    } early(grid == 0);   // (under a quota its CTAs would wait on SMs beside the attention's)
    switch (a.r.rec.hd) {
    case 128: return many ? join<128, 16>(a, e, f32, g, st) : join<128, 1>(a, e, f32, g, st);
    case 64: return many ? join<64, 16>(a, e, f32, g, st) : join<64, 1>(a, e, f32, g, st);
    default: return many ? join<32, 16>(a, e, f32, g, st) : join<32, 1>(a, e, f32, g, st);
    }
}

}  // namespace p8
}  // namespace ebrl
