// The weight each prefix token got (include/ebrl_prefix8.h): w[t] = sum over heads and query rows of exp(scale q k_t - lse).
//
// Bound: HBM -- the key codes are read once, a token's weight is written once.  A second pass over the keys is half of the
// attention's own traffic; gathering the weights inside attention would need either the scores of all heads in memory
// (16 rows x 4 B per token and head against 128 B of codes) or atomics across heads, whose order changes the last bits.
//
// A CTA owns some tiles x TW of one environment and walks every (key/value head, row tile): its eight warps are HW parallel
// heads x TW token groups (HW = 8 with eight heads or more).  A warp keeps its head's queries in registers for up to twelve
// tiles, adds a token's weights up over the quad's rows by three exchanges, and over its heads in shared memory, in
// words of its own.  At the end the parallel heads are added in warp order: a fixed order whatever the tiles per warp, no atomics.
// The key tiles of a warp's heads are one stream through a ring of cp.async slots, so the ring stays full across heads.
#include "prefix8_tile.cuh"

namespace ebrl {
namespace p8 {

constexpr int MAX_TILES = 12;   // per warp

template <int HD, int NT, bool F32> struct WeighCfg {
    static constexpr int CTAS = F32 && (NT > 1 || HD == 128) ? 1 : 2;   // per SM
    static constexpr int TILE = BLOCK * HD, RING = HD == 32 ? 8192 : (CTAS == 2 ? 12288 : 24576), SLOTS = RING / TILE < 8 ? RING / TILE : 8;
    static constexpr int SMEM = 8 * RING;
};

template <int HD, int NT, bool F32>
__global__ void __launch_bounds__(256, WeighCfg<HD, NT, F32>::CTAS)
weigh_kernel(const __grid_constant__ WeighArgs a, const __grid_constant__ Envs ev, int hw_log2, int n_chunk, int tiles)
{
    using C = WeighCfg<HD, NT, F32>;
    extern __shared__ __align__(128) char smem[];
    __shared__ float red[8][MAX_TILES * BLOCK];   // per warp: the sums of its tokens over its heads
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring_u = ptx::smem_u32(smem + (size_t)warp * C::RING);
    const int G = a.r.G, R = a.r.H * G, RT = (R + NT * 8 - 1) / (NT * 8), kvh = a.r.rec.kvh, units = kvh * RT;
    const int tok_w = tiles * BLOCK;   // tokens per warp
    const int HW = 1 << hw_log2, TW = 8 >> hw_log2, hw = warp & (HW - 1), tw = warp >> hw_log2;
    const int n_envs = a.r.meta ? a.r.n_envs : ev.n;
    const long long items = (long long)n_envs * n_chunk;
    uint32_t koff[KeyWords<HD>::OFFS];
    KeyWords<HD>::offsets(koff, g, t);
    pdl_launch_dependents();
    pdl_wait();

    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int env = (int)(item / n_chunk), chunk = (int)(item - (long long)env * n_chunk);
        const char *rec;
        float *wp;
        int len;
        if (a.r.meta) { rec = (const char *)a.r.meta[env].kv; len = a.r.meta[env].P; wp = a.r.meta[env].weight; }
        else {
            rec = a.r.pool + (size_t)ev.slot[env] * a.r.rec.bytes;
            len = ev.len[env];
            wp = a.weight + (size_t)ev.slot[env] * a.stride;
        }
        const int c0 = chunk * TW * tok_w;                     // first token of the CTA
        if (c0 >= len || !wp) continue;                      // (the same for the whole CTA)
        const int b0 = c0 + tw * tok_w;                        // ... and of the warp
        const int live = b0 >= len ? 0 : min(tiles, (len - b0 + BLOCK - 1) / BLOCK);
        const int mine = hw < units ? (units - hw + HW - 1) >> hw_log2 : 0;   // this warp's (head, row tile) units: hw, hw + HW, ...
        const int loads = mine * live;
        // load j of the warp's stream: tile j % live of its unit j / live
        int iu = hw, it = 0;
        auto issue = [&](int j, int slot) {
            if (j < loads) {
                const char *src = rec + a.r.rec.head(a.r.layer, 0, iu / RT) + (size_t)(b0 + it * BLOCK) * HD;
                request_tile<HD>(ring_u + (uint32_t)(slot * C::TILE), src, min(BLOCK, len - b0 - it * BLOCK), lane);
                if (++it == live) { it = 0; iu += HW; }
            }
            cp_commit();
        };
#pragma unroll
        for (int j = 0; j < C::SLOTS - 1; ++j) issue(j, j);

        uint32_t seen = 0;   // lane l: visible tokens of tile l
        if (lane < live) {
            seen = reinterpret_cast<const uint32_t *>(rec + a.r.rec.mask)[b0 / BLOCK + lane];
            const int v = len - b0 - lane * BLOCK;
            if (v < BLOCK) seen &= (1u << v) - 1u;
        }
        for (int k = lane; k < tok_w; k += 32) red[warp][k] = 0.f;
        __syncwarp();

        int slot = 0, j = 0;
        for (int u = 0; u < mine; ++u) {
            if (live == 0) break;
            const int unit = hw + u * HW, kh = unit / RT, rt = unit - kh * RT;
            uint32_t q[NT][HD / 16][QW<F32>];
            float fr[NT][2], ls[NT][2];
            if (u + 1 < mine) {   // the next unit's queries on their way into L1
                constexpr int LINES = HD * (F32 ? 4 : 2) / 128 > 0 ? HD * (F32 ? 4 : 2) / 128 : 1;   // 128-byte lines of a row
                const int un = unit + HW, kn = un / RT, rn = un - kn * RT;
#pragma unroll
                for (int i = lane; i < NT * 8 * LINES; i += 32) {
                    const int r = rn * NT * 8 + i / LINES, tok = r / G;
                    const size_t off = (size_t)env * a.r.q_env + (size_t)tok * a.r.q_tok + (size_t)(kn * G + r - tok * G) * HD;
                    if (r < R) prefetch_l1((const char *)a.r.q + off * (F32 ? 4 : 2) + (i % LINES) * 128);
                }
            }
            const float ks_l = lane < live ? read_scale(reinterpret_cast<const float *>(rec + a.r.rec.head_scales(a.r.layer, 0, kh))[b0 / BLOCK + lane]) : 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = rt * NT * 8 + nt * 8 + g, tok = r / G, head = kh * G + r - tok * G;
                const size_t off = (size_t)env * a.r.q_env + (size_t)tok * a.r.q_tok + (size_t)head * HD;
                const void *p = F32 ? (const void *)((const float *)a.r.q + off) : (const void *)((const __nv_bfloat16 *)a.r.q + off);
                const float f = load_q<HD, F32>(p, r < R, a.r.scale < 0.f, t, q[nt]) * fabsf(a.r.scale);
                // rows that saw nothing (lse = -inf) and rows past the last one add 2^-inf
                float l = r < R ? a.lse[(size_t)env * a.l_env + (size_t)tok * a.l_tok + (size_t)head * a.l_head] : -INFINITY;
                l = l == -INFINITY ? INFINITY : l;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    fr[nt][c] = __shfl_sync(FULL, f, 8 * t + 4 * c);
                    ls[nt][c] = __shfl_sync(FULL, l, 8 * t + 4 * c);
                }
            }
            for (int i = 0; i < live; ++i) {
                const float ks = __shfl_sync(FULL, ks_l, i);
                cp_wait<C::SLOTS - 2>();
                __syncwarp();
                issue(j + C::SLOTS - 1, slot == 0 ? C::SLOTS - 1 : slot - 1);
                const uint32_t at = ring_u + (uint32_t)(slot * C::TILE);
                slot = slot + 1 == C::SLOTS ? 0 : slot + 1;
                ++j;
                KeyWords<HD> kw[2];
                kw[0].load(at, koff, 0);
                kw[1].load(at, koff, 1);
                float s[2][NT][4];
                score<HD, NT, F32, true>(s, kw, [&](int st, int nt, uint32_t *w) {
#pragma unroll
                    for (int c = 0; c < QW<F32>; ++c) w[c] = q[nt][st][c];
                });
                float v[4] = {0.f, 0.f, 0.f, 0.f};   // token 16 h + row_token(g) + 2 c at v[2 h + c], over this lane's rows
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        // (the difference in natural units: ks * fr is exact for a power of two, lse as it was given)
                        const float c0 = ks * fr[nt][0], c1 = ks * fr[nt][1];
                        v[2 * h] += ex2(LOG2E * fmaf(s[h][nt][0], c0, -ls[nt][0])) + ex2(LOG2E * fmaf(s[h][nt][1], c1, -ls[nt][1]));
                        v[2 * h + 1] += ex2(LOG2E * fmaf(s[h][nt][2], c0, -ls[nt][0])) + ex2(LOG2E * fmaf(s[h][nt][3], c1, -ls[nt][1]));
                    }
                // over the quad by halving exchanges: lane t ends with the total of v[t]
                const float a0 = (t & 2 ? v[2] : v[0]) + __shfl_xor_sync(FULL, t & 2 ? v[0] : v[2], 2);
                const float a1 = (t & 2 ? v[3] : v[1]) + __shfl_xor_sync(FULL, t & 2 ? v[1] : v[3], 2);
                const float sum = (t & 1 ? a1 : a0) + __shfl_xor_sync(FULL, t & 1 ? a0 : a1, 1);
                red[warp][i * 32 + 16 * (t >> 1) + row_token(g) + 2 * (t & 1)] += sum;   // (a word of its own for every lane)
            }
        }
        cp_wait<0>();
        __syncwarp();
        for (int k = lane; k < live * 32; k += 32) {   // hidden tokens got nothing
            const uint32_t m = __shfl_sync(FULL, seen, k >> 5);
            if (!((m >> lane) & 1)) red[warp][k] = 0.f;
        }
        __syncthreads();
        for (int k = threadIdx.x; k < TW * tok_w; k += 256) {
            const int tok = c0 + k, group = k / tok_w, first = group << hw_log2;
            if (tok < len) {
                float v = 0.f;
                for (int h = 0; h < HW; ++h) v += red[first + h][k - group * tok_w];
                wp[tok] = a.accumulate ? wp[tok] + v : v;
            }
        }
        __syncthreads();   // red and the rings are free
    }
}

namespace {

template <int HD, int NT, bool F32> cudaError_t go(const WeighArgs &a, const Envs &e, int max_len, int grid, int sms, cudaStream_t st)
{
    using C = WeighCfg<HD, NT, F32>;
    static std::atomic<bool> set[64];   // (calls may come from several threads; setting it twice is harmless)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        cudaError_t err = cudaFuncSetAttribute(weigh_kernel<HD, NT, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    const int units = a.r.rec.kvh * ((a.r.H * a.r.G + NT * 8 - 1) / (NT * 8));
    const int hw = units >= 8 ? 3 : (units >= 4 ? 2 : (units >= 2 ? 1 : 0));
    // Tiles per warp: up to 12, evenly (a head's queries are brought in once for all of them: 4, 8, 12 tiles took 107, 90, 84 us on
    // 256 x 734 tokens x 16 heads x 16 rows), but fewer where that gives the SMs less than two CTAs each.
    const int n = a.r.meta ? a.r.n_envs : e.n, TW = 8 >> hw, all = (max_len + BLOCK - 1) / BLOCK, most = (all + TW - 1) / TW;
    if (n == 0 || all == 0) return cudaSuccess;
    int n_chunk = (most + MAX_TILES - 1) / MAX_TILES;
    const int wanted = (2 * (grid ? grid : sms) + n - 1) / n;
    if (n_chunk < wanted) n_chunk = wanted < most ? wanted : most;
    const int tiles = (most + n_chunk - 1) / n_chunk;
    n_chunk = (most + tiles - 1) / tiles;
    const long long items = (long long)n * n_chunk, cap = grid ? grid : 1 << 20;
    return launch_kernel(weigh_kernel<HD, NT, F32>, (int)(items < cap ? items : cap), 256, (size_t)C::SMEM, st, 1, a, e, hw, n_chunk, tiles);
}

// Query rows per product, from the call's rows, head and type alone, so that a batch's other lengths change no bits.  Measured,
// us with 8 / 16 / 32 on 128 x 768 tokens x 16 heads (two CTAs per SM but for 32 rows and the fp32 forms that hold no more than
// one): bf16 of 128, 8 rows 48 / 52 / 81, 16 rows 62 / 56 / 87, 32 rows 112 / 89 / 96; bf16 of 64, 8 rows 30 / 36 / 61, 32 rows
// 90 / 66 / 77.  fp32 of 128, 8 rows 60 / 73 / 118, 32 rows 183 / 135 / 138 (since second
// terms add up apart 60 at 8 rows, 85 at 16 and 146 at 32 in the tiles chosen here).  fp32 of 64 (and of 32 alike), 8 rows 34 / 54 / 76, 32
// rows 101 / 104 / 91 (512 x 64 tokens: 54 / 73 / 70), 64 rows 189 / 194 / 164 (97 / 129 / 122): one size for them all.
template <int HD> cudaError_t pick(const WeighArgs &a, const Envs &e, bool f32, int max_len, int grid, int sms, cudaStream_t st)
{
    const int rows = a.r.H * a.r.G;
    if (f32 && (HD < 128 || rows <= 8)) return go<HD, 1, true>(a, e, max_len, grid, sms, st);
    if (f32) return go<HD, HD < 128 ? 1 : 2, true>(a, e, max_len, grid, sms, st);
    return rows <= 8 ? go<HD, 1, false>(a, e, max_len, grid, sms, st) : go<HD, 2, false>(a, e, max_len, grid, sms, st);
}

}  // namespace

cudaError_t launch_weigh(const WeighArgs &a, const Envs &e, bool f32, int max_len, int grid, int sms, cudaStream_t st)
{
    return a.r.rec.hd == 128 ? pick<128>(a, e, f32, max_len, grid, sms, st) : (a.r.rec.hd == 64 ? pick<64>(a, e, f32, max_len, grid, sms, st) : pick<32>(a, e, f32, max_len, grid, sms, st));
}

}  // namespace p8
}  // namespace ebrl
