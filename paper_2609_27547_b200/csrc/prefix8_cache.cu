// Writing and shortening 8-bit prefix records (include/ebrl_prefix8.h): quantize and evict.
#include "prefix8_internal.h"
#include "rowops.cuh"

#include <cuda_fp16.h>
#include <math.h>

namespace ebrl {
namespace p8 {

namespace {

// The block scale: the power of two s with amax / s in (224, 448] (448 = 1.75 * 2^8 is the largest e4m3 value), so that
// dividing by it is exact and a later change of scale moves exponents only.  1 for 0; the smallest normal number bounds it below.
__device__ __forceinline__ float block_scale(float amax)
{
    if (amax == 0.f) return 1.f;
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - ((b & 0x7fffffu) <= 0x600000u ? 8 : 7);   // amax = m 2^(e' - 127), m <= 1.75 or above
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// Two fp32 values -> two e4m3 codes (a in the low byte), to nearest even, saturated; NaN stays NaN.
__device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
    return r;
}
// Two e4m3 codes as f16, one code's value, two codes' values.
__device__ __forceinline__ uint32_t code_half2(uint32_t two)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return r;
}
__device__ __forceinline__ float2 code_pair(uint32_t two)
{
    const uint32_t r = code_half2(two);
    return __half22float2(*reinterpret_cast<const __half2 *>(&r));
}
__device__ __forceinline__ float code_value(uint32_t c) { return code_pair(c).x; }
// Two codes times a power of two, as codes; NaN stays NaN.
__device__ __forceinline__ uint32_t times2(uint32_t two, __half2 f)
{
    const uint32_t r = code_half2(two);
    const __half2 p = __hmul2(*reinterpret_cast<const __half2 *>(&r), f);
    uint16_t o;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(o) : "r"(*reinterpret_cast<const uint32_t *>(&p)));
    return o;
}
__device__ __forceinline__ float finite_abs(float x)
{
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;   // (false for NaN)
}

}  // namespace

// One warp per (environment, layer, plane, block of 32 tokens, head), heads next to one another in a CTA so that it reads whole
// rows.  The block lives in registers between the maximum and the rounding: planes are read once.
// Bound: HBM, esz + 1 bytes per element.  A lane's loads are 16 bytes; 8 (bf16, head_dim 64) to 32 (fp32, 128) of them
// are in flight per lane.
template <int HD, bool F32>
__global__ void __launch_bounds__(256) quantize_kernel(const __grid_constant__ QuantEnvs ev, Record rec, char *pool, long long row_stride, int max_blocks)
{
    constexpr int V = F32 ? 4 : 8, LPR = HD / V, RPI = 32 / LPR, N = 32 / RPI;   // elements per load, lanes per row, rows per load, loads
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lp = rec.kv_layers * 2;
    const long long items = (long long)ev.n * max_blocks * lp * rec.kvh;
    for (long long item = (long long)blockIdx.x * 8 + warp; item < items; item += (long long)gridDim.x * 8) {
        long long x = item;
        const int h = (int)(x % rec.kvh); x /= rec.kvh;
        const int p = (int)(x % lp); x /= lp;
        const int blk = (int)(x % max_blocks), env = (int)(x / max_blocks);
        const int len = ev.len[env], t0 = blk * BLOCK;
        if (t0 >= len) continue;
        char *r = pool + (size_t)ev.slot[env] * rec.bytes;
        // tokens of this block that queries see
        uint32_t seen = len - t0 >= BLOCK ? 0xffffffffu : (1u << (len - t0)) - 1u;
        if (ev.mask[env]) seen &= __ballot_sync(0xffffffffu, t0 + lane < len && ev.mask[env][t0 + lane] != 0);
        if (p == 0 && h == 0 && lane == 0) reinterpret_cast<uint32_t *>(r + rec.mask)[blk] = seen;
        const size_t first = ((size_t)p * ev.plane_rows[env] + t0) * row_stride + (size_t)h * HD + (lane % LPR) * V;
        uint4 raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int tok = i * RPI + lane / LPR;
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if ((seen >> tok) & 1) {
                const size_t at = first + (size_t)tok * row_stride;
                raw[i] = __ldcs(reinterpret_cast<const uint4 *>(F32 ? (const void *)((const float *)ev.planes[env] + at) : (const void *)((const __nv_bfloat16 *)ev.planes[env] + at)));
            }
        }
        // magnitudes are ordered like their bits; two bf16 ones are compared in one instruction
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (F32) top = max(max(top, max(raw[i].x & 0x7fffffffu, raw[i].y & 0x7fffffffu)), max(raw[i].z & 0x7fffffffu, raw[i].w & 0x7fffffffu));
            else top = __vmaxu2(__vmaxu2(top, __vmaxu2(raw[i].x & 0x7fff7fffu, raw[i].y & 0x7fff7fffu)), __vmaxu2(raw[i].z & 0x7fff7fffu, raw[i].w & 0x7fff7fffu));
        }
        if constexpr (!F32) top = max(top << 16, top & 0xffff0000u);
        top = __reduce_max_sync(0xffffffffu, top);
        bool nan = false;
        if (top >= 0x7f800000u) {   // not all finite: the largest finite one instead
            uint32_t fin = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const uint32_t m = (F32 ? w[j % 4] : (j & 1 ? w[j / 2] & 0xffff0000u : w[(j / 2) % 4] << 16)) & 0x7fffffffu;
                    nan |= m > 0x7f800000u;
                    if (m < 0x7f800000u) fin = max(fin, m);
                }
            }
            top = __reduce_max_sync(0xffffffffu, fin);
            nan = __any_sync(0xffffffffu, nan);
        }
        const float amax = __uint_as_float(top);
        const float s = block_scale(amax), inv = 1.f / s;   // both powers of two: products with inv are exact
        if (lane == 0) reinterpret_cast<float *>(r + rec.scales)[((size_t)p * rec.kvh + h) * rec.nb + blk] = nan ? -s : s;
        char *dst = r + ((size_t)p * rec.kvh + h) * rec.plane + (size_t)t0 * HD + (lane % LPR) * V;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int tok = i * RPI + lane / LPR;
            if (t0 + tok < len) {
                char *to = dst + (size_t)tok * HD;
                if constexpr (F32) {
                    *reinterpret_cast<uint32_t *>(to) = narrow2(__uint_as_float(raw[i].x) * inv, __uint_as_float(raw[i].y) * inv) |
                                                        narrow2(__uint_as_float(raw[i].z) * inv, __uint_as_float(raw[i].w) * inv) << 16;
                } else {
                    auto two = [&](uint32_t w) { return narrow2(__uint_as_float(w << 16) * inv, __uint_as_float(w & 0xffff0000u) * inv); };
                    *reinterpret_cast<uint2 *>(to) = make_uint2(two(raw[i].x) | two(raw[i].y) << 16, two(raw[i].z) | two(raw[i].w) << 16);
                }
            }
        }
    }
}

cudaError_t launch_quantize(const Record &rec, char *pool, long long row_stride, bool f32, const QuantEnvs &e, int max_len, int grid, cudaStream_t st)
{
    const int max_blocks = (max_len + BLOCK - 1) / BLOCK;
    const long long items = (long long)e.n * max_blocks * rec.kv_layers * 2 * rec.kvh, need = (items + 7) / 8, cap = grid ? grid : 1 << 20;
    if (items == 0) return cudaSuccess;
    const int g = (int)(need < cap ? need : cap);
#define EBRL_Q(HD) (f32 ? launch_kernel(quantize_kernel<HD, true>, g, 256, 0, st, 1, e, rec, pool, row_stride, max_blocks) \
                        : launch_kernel(quantize_kernel<HD, false>, g, 256, 0, st, 1, e, rec, pool, row_stride, max_blocks))
    return rec.hd == 128 ? EBRL_Q(128) : (rec.hd == 64 ? EBRL_Q(64) : EBRL_Q(32));
#undef EBRL_Q
}

// ---- evict ------------------------------------------------------------------------------------------------------------

// An order-preserving integer of a token's weight: protected like +inf; hidden tokens and NaN like -inf; -0 like +0.
__device__ __forceinline__ uint32_t weight_key(const EvictArgs &a, const float *w, const uint32_t *mask, int t, int len)
{
    float x = w[t] + 0.f;
    if (!((mask[t >> 5] >> (t & 31)) & 1) || !(x == x)) x = -INFINITY;
    if (t < a.protect_first || t >= len - a.protect_last) x = INFINITY;
    const uint32_t u = __float_as_uint(x);
    return (u >> 31) ? ~u : u | 0x80000000u;
}

// Which tokens stay: one CTA per environment.  The key of the last kept token is found byte by byte (four passes of a
// 256-bin histogram over the keys, which stay in shared memory up to SELECT_KEYS tokens and are made anew from the weights beyond),
// then one pass in token order lists what is above it and the first of what ties with it.  The mask and the weights follow in chunks that are read as a whole before they are
// written: a kept token never moves to a higher index, so working in place is safe.
// Bound: latency -- 4 B per token against 256 B of codes in the second kernel.
constexpr int SELECT_KEYS = 49152;

__global__ void __launch_bounds__(1024) select_kernel(const __grid_constant__ EvictArgs a, const __grid_constant__ EvictEnvs ev, int room)
{
    extern __shared__ uint32_t keys[];   // [room]
    __shared__ int hist[256];
    __shared__ uint32_t wsum[32];
    __shared__ uint32_t s_prefix;
    __shared__ int s_need;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int env = blockIdx.x; env < ev.n; env += gridDim.x) {
        const int len = ev.len[env], keep = ev.keep[env];
        if (keep == 0) continue;
        const char *src = a.src + (size_t)ev.slot[env] * a.rec.bytes;
        const float *w = a.weight + (size_t)ev.slot[env] * a.weight_stride;
        const uint32_t *mask = reinterpret_cast<const uint32_t *>(src + a.rec.mask);
        int *kept = a.kept + (size_t)env * a.kept_stride;
        uint32_t prefix = 0;      // the bytes of the last kept key found so far
        int need = keep;          // how many tokens are kept among those that start with them
        const bool cached = len <= room;
        if (keep < len && cached) {
#pragma unroll 4
            for (int t = threadIdx.x; t < len; t += 1024) keys[t] = weight_key(a, w, mask, t, len);
            __syncthreads();
        }
        auto key_of = [&](int t) { return cached ? keys[t] : weight_key(a, w, mask, t, len); };
        if (keep < len) {
            for (int shift = 24; shift >= 0; shift -= 8) {
                if (threadIdx.x < 256) hist[threadIdx.x] = 0;
                __syncthreads();
#pragma unroll 4
                for (int t = threadIdx.x; t < len; t += 1024) {
                    const uint32_t k = key_of(t);
                    if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);   // counts: the order does not matter
                }
                __syncthreads();
                if (warp == 0) {
                    // bins from the top, eight per lane: the bin in which the count reaches `need`
                    int c[8], sum = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) { c[i] = hist[255 - (lane * 8 + i)]; sum += c[i]; }
                    int before = sum;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += v; }
                    before -= sum;
                    if (before < need && before + sum >= need) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (before < need && before + c[i] >= need) { s_prefix = prefix | (uint32_t)(255 - (lane * 8 + i)) << shift; s_need = need - before; }
                            before += c[i];
                        }
                    }
                }
                __syncthreads();
                prefix = s_prefix;
                need = min(max(s_need, 0), keep);   // (it is, unless the weights change meanwhile: see below)
            }
        }
        // tokens in order, four to a thread: above the last kept key, or the first `need` that equal it.  Positions come from a scan of
        // both counts at once (16 bits each: a round has 4096 tokens).
        int done_above = 0, done_equal = 0;
        for (int base = 0; base < len; base += 4096) {
            const int t0 = base + 4 * threadIdx.x;
            uint32_t flags = 0, mine = 0;     // bit i: above, bit 4 + i: equal
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (t0 + i >= len) continue;
                const uint32_t k = keep == len ? 1u : key_of(t0 + i);
                const bool above = keep == len || k > prefix, equal = keep != len && k == prefix;
                flags |= (uint32_t)above << i | (uint32_t)equal << (4 + i);
                mine += (uint32_t)above + ((uint32_t)equal << 16);
            }
            uint32_t upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
            __syncthreads();
            if (lane == 31) wsum[warp] = upto;
            __syncthreads();
            uint32_t all = wsum[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, all, o); if (lane >= o) all += v; }
            const uint32_t before = (warp ? __shfl_sync(0xffffffffu, all, warp - 1) : 0u) + upto - mine, total = __shfl_sync(0xffffffffu, all, 31);
            int na = done_above + (int)(before & 0xffffu), ne = done_equal + (int)(before >> 16);
            done_above += (int)(total & 0xffffu);
            done_equal += (int)(total >> 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool above = (flags >> i) & 1, equal = (flags >> (4 + i)) & 1;
                const int at = na + min(ne, need);
                if ((above || (equal && ne < need)) && at < keep) kept[at] = t0 + i;
                na += above;
                ne += equal;
            }
        }
        // Weights that someone changes while the passes read them (a caller's race) may have given too few or too many: the list is cut above and
        // filled here, so that whatever it holds lies in the prefix and no access leaves the arrays.
        for (int j = done_above + min(done_equal, need) + threadIdx.x; j < keep; j += 1024) kept[j] = len - 1;
        __syncthreads();   // the list is there for the whole CTA
        uint32_t *to_mask = reinterpret_cast<uint32_t *>(a.dst + (size_t)ev.slot[env] * a.rec.bytes + a.rec.mask);
        float *to_w = a.weight_out ? a.weight_out + (size_t)ev.slot[env] * a.weight_out_stride : nullptr;
        for (int base = 0; base < keep; base += 1024) {
            const int j = base + threadIdx.x;
            int idx = 0;
            float x = 0.f;
            bool vis = false;
            if (j < keep) { idx = kept[j]; x = w[idx]; vis = (mask[idx >> 5] >> (idx & 31)) & 1; }
            const uint32_t word = __ballot_sync(0xffffffffu, vis);
            __syncthreads();
            if (j < keep && to_w) to_w[j] = x;
            if (lane == 0 && j < keep) to_mask[j >> 5] = word;
            __syncthreads();
        }
    }
}

// The kept rows of one (environment, layer, plane, head), a warp per new block: gather, largest value, new scale, round, write.
// A lane holds 16-byte pieces of rows, so a row is one coalesced read.  A CTA reads the eight blocks of a chunk before
// it writes any of them, and takes chunks in order when the record is shortened in place (n_part = 1): sources never lie before
// the rows being written.  Otherwise the chunks are spread over n_part CTAs.
// Bound: HBM, 2 bytes per kept code.
template <int HD>
__global__ void __launch_bounds__(256, 4) gather_kernel(const __grid_constant__ EvictArgs a, const __grid_constant__ EvictEnvs ev, int n_part)
{
    constexpr int LPR = HD / 16, RPI = 32 / LPR, N = 32 / RPI;   // lanes per row, rows per load, loads per lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = a.rec.kv_layers * 2 * a.rec.kvh;
    const long long items = (long long)ev.n * heads * n_part;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        long long x = item;
        const int part = (int)(x % n_part); x /= n_part;
        const int h = (int)(x % heads), env = (int)(x / heads);
        const int keep = ev.keep[env];
        const int *kept = a.kept + (size_t)env * a.kept_stride;
        const size_t rec_off = (size_t)ev.slot[env] * a.rec.bytes, head_off = rec_off + (size_t)h * a.rec.plane, sc_off = rec_off + a.rec.scales + (size_t)h * a.rec.nb * 4;
        const char *src = a.src + head_off;
        const float *ssc = reinterpret_cast<const float *>(a.src + sc_off);
        for (int base = part * 8 * BLOCK; base < keep; base += n_part * 8 * BLOCK) {   // (the same for the whole CTA)
            const int b0 = base + warp * BLOCK;
            uint4 v[N];
            float sc[N];
            const int mine = b0 + lane < keep ? kept[b0 + lane] : -1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int idx = __shfl_sync(0xffffffffu, mine, i * RPI + lane / LPR);
                v[i] = make_uint4(0u, 0u, 0u, 0u);
                sc[i] = 0.f;
                if (idx >= 0) {
                    v[i] = *reinterpret_cast<const uint4 *>(src + (size_t)idx * HD + (lane % LPR) * 16);
                    sc[i] = fabsf(ssc[idx >> 5]);
                }
            }
            float amax = 0.f;
            bool nan = false;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // codes without their sign are ordered like their values, 0x7f (NaN) above all; two codes are compared in one instruction
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                uint32_t even = 0, odd = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) { even = __vmaxu2(even, w[j] & 0x007f007fu); odd = __vmaxu2(odd, w[j] & 0x7f007f00u); }
                const uint32_t m = __vmaxu2(even, odd >> 8), top = max(m & 0xffffu, m >> 16);
                nan |= top == 0x7fu;
                amax = fmaxf(amax, code_value(top) * sc[i]);   // (a NaN is dropped)
            }
            const bool any_nan = __any_sync(0xffffffffu, nan);
            // Products may pass fp32's largest number (quantize keeps 3.4e38 as 256 x 2^120): then all are taken 2^-9 as large, and so is the scale.
            const bool vast = __any_sync(0xffffffffu, amax == INFINITY);
            const float pre = vast ? 0x1p-9f : 1.f;
            if (any_nan || vast) {   // the largest that is a number
                amax = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    for (int j = 0; j < 16; ++j) {
                        const uint32_t c = (w[j >> 2] >> (8 * (j & 3))) & 0x7fu;
                        if (c != 0x7fu) amax = fmaxf(amax, finite_abs(code_value(c) * pre * sc[i]));
                    }
                }
            }
            amax = warp_max(amax);
            float s = block_scale(amax);
            if (vast) s = fminf(s, 0x1p118f);   // (2^127 is the largest scale)
            const float inv = 1.f / s;
            // whether every row changes its scale by a power of two that f16 holds
            bool fine = true;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float by = pre * sc[i] * inv;
                fine &= sc[i] == 0.f || ((__float_as_uint(by) & 0x007fffffu) == 0 && by >= 1.f / 16384.f && by <= 16384.f);
            }
            fine = __all_sync(0xffffffffu, fine);
            __syncthreads();   // every block of the chunk has been read
            if (b0 < keep) {
                char *dst = a.dst + head_off;
                if (lane == 0) *reinterpret_cast<float *>(a.dst + sc_off + (size_t)(b0 >> 5) * 4) = (any_nan ? -s : s) * (vast ? 0x1p9f : 1.f);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int row = b0 + i * RPI + lane / LPR;
                    if (row < keep) {
                        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                        uint32_t o[4];
                        const float by = pre * sc[i] * inv;
                        if (fine) {
                            // codes are f16 values, a power of two of one is, too (or far below the smallest code)
                            const __half2 f = __float2half2_rn(by);
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[j] = times2(w[j], f) | times2(w[j] >> 16, f) << 16;
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint32_t r = 0;
#pragma unroll
                                for (int q = 0; q < 2; ++q) {
                                    const float2 f = code_pair((w[j] >> (16 * q)) & 0xffffu);
                                    r |= narrow2(f.x * pre * sc[i] * inv, f.y * pre * sc[i] * inv) << (16 * q);
                                }
                                o[j] = r;
                            }
                        }
                        *reinterpret_cast<uint4 *>(dst + (size_t)row * HD + (lane % LPR) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                    }
                }
            }
        }
    }
}

cudaError_t launch_evict(const EvictArgs &a, const EvictEnvs &e, int max_keep, int grid, int n_sms, cudaStream_t st)
{
    if (e.n == 0 || max_keep == 0) return cudaSuccess;
    const int g1 = grid && grid < e.n ? grid : e.n;
    int longest = 0;
    for (int i = 0; i < e.n; ++i) longest = longest > e.len[i] ? longest : e.len[i];
    const int room = longest < SELECT_KEYS ? longest : SELECT_KEYS;
    static std::atomic<bool> set[64];   // (calls may come from several threads; setting it twice is harmless)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        const cudaError_t e2 = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SELECT_KEYS * 4);
        if (e2 != cudaSuccess) return e2;
        set[dev] = true;
    }
    cudaError_t err = launch_kernel(select_kernel, g1, 1024, (size_t)room * 4, st, 1, a, e, room);
    if (err != cudaSuccess) return err;
    const int chunks = (max_keep + 8 * BLOCK - 1) / (8 * BLOCK);
    const long long heads = (long long)e.n * a.rec.kv_layers * 2 * a.rec.kvh;
    // in place the chunks of a head are one CTA's, in order; otherwise each is a CTA's
    const long long part = a.src == a.dst ? 1 : chunks;
    const long long items = heads * part, cap = grid ? grid : 1 << 20;
    const int g2 = (int)(items < cap ? items : cap);
    switch (a.rec.hd) {
    case 128: return launch_kernel(gather_kernel<128>, g2, 256, 0, st, 1, a, e, (int)part);
    case 64: return launch_kernel(gather_kernel<64>, g2, 256, 0, st, 1, a, e, (int)part);
    default: return launch_kernel(gather_kernel<32>, g2, 256, 0, st, 1, a, e, (int)part);
    }
}

}  // namespace p8
}  // namespace ebrl
