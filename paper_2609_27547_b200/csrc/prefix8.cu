// The C boundary of the 8-bit prefix cache operators (include/ebrl_prefix8.h): argument checks, the choice of pieces, and the
// launches.  Nothing here touches the device before every argument has been checked.
#include "prefix8_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <string>
#include <vector>

using namespace ebrl;
using namespace ebrl::p8;

namespace ebrl {
namespace p8 {

Record record_of(const ebrl_prefix8_layout_t &l)
{
    Record r{};
    r.kv_layers = l.kv_layers; r.kvh = l.n_kv_heads; r.hd = l.head_dim;
    r.nb = (l.capacity + BLOCK - 1) / BLOCK;
    r.rows = r.nb * BLOCK;
    r.plane = (size_t)r.rows * r.hd;
    const size_t heads = (size_t)r.kv_layers * 2 * r.kvh;
    r.scales = heads * r.plane;
    r.mask = r.scales + heads * r.nb * 4;
    r.bytes = (r.mask + (size_t)r.nb * 4 + 127) & ~(size_t)127;
    return r;
}

}  // namespace p8
}  // namespace ebrl

namespace {

thread_local char t_error[256];

ebrl_status_t fail(ebrl_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(t_error, sizeof t_error, fmt, ap);
    va_end(ap);
    return st;
}

#define BAD(...) return fail(EBRL_ERR_INVALID_ARG, __VA_ARGS__)

ebrl_status_t check_layout(const ebrl_prefix8_layout_t *l)
{
    if (!l) BAD("layout is NULL");
    if (l->kv_layers < 1 || l->n_kv_heads < 1 || l->capacity < 1) BAD("kv_layers, n_kv_heads and capacity must be positive");
    if (l->head_dim != 32 && l->head_dim != 64 && l->head_dim != 128) return fail(EBRL_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
    if (l->capacity > 1 << 24 || l->kv_layers > 1 << 12 || l->n_kv_heads > 1 << 12)
        return fail(EBRL_ERR_UNSUPPORTED, "capacity is limited to 2^24 tokens, kv_layers and n_kv_heads to 4096");
    return EBRL_OK;
}

// What every operator takes: the pool, the slots and the lengths.  `writes`: slots must differ.
ebrl_status_t check_envs(const ebrl_prefix8_layout_t *l, const void *pool, int32_t n_slots, int32_t n, const int32_t *slots,
                         const int32_t *len, int32_t sm_quota, bool writes)
{
    const ebrl_status_t st = check_layout(l);
    if (st != EBRL_OK) return st;
    if (n < 0 || n_slots < 0) BAD("n and n_slots must not be negative");
    if (sm_quota < 0) return fail(EBRL_ERR_QUOTA, "sm_quota < 0");
    if (n == 0) return EBRL_OK;
    if (!pool || ((uintptr_t)pool & 15)) BAD("the pool is NULL or not 16-byte aligned");
    if (!len) BAD("len is NULL");
    if (!slots && n > n_slots) BAD("%d environments, but %d slots", n, n_slots);
    std::vector<bool> used(writes && slots ? n_slots : 0);
    for (int i = 0; i < n; ++i) {
        if (len[i] < 0 || len[i] > l->capacity) BAD("len[%d] = %d is outside 0..capacity", i, len[i]);
        if (slots) {
            if (slots[i] < 0 || slots[i] >= n_slots) BAD("slots[%d] = %d is outside 0..n_slots - 1", i, slots[i]);
            if (writes) {
                if (used[slots[i]]) BAD("slot %d is named twice", slots[i]);
                used[slots[i]] = true;
            }
        }
    }
    return EBRL_OK;
}

size_t esize(int dtype) { return dtype == EBRL_BF16 ? 2 : 4; }

// Whether n x H rows of `width` elements with these strides lie apart from one another.
bool rows_apart(int64_t n, int64_t H, int64_t env, int64_t tok, int64_t width)
{
    if (n <= 1 && H <= 1) return true;
    if (n <= 1) return tok >= width;
    if (H <= 1) return env >= width;
    return (tok >= width && env >= (H - 1) * tok + width) || (env >= width && tok >= (n - 1) * env + width);
}

// Whether rows with these strides start at multiples of 16 bytes from the first; the stride of a single environment or token does not matter.
bool strides_fit(int64_t n, int64_t H, int64_t env, int64_t tok, int64_t es)
{
    return (n <= 1 || (env >= 0 && env * es % 16 == 0)) && (H <= 1 || (tok >= 0 && tok * es % 16 == 0));
}

ebrl_status_t check_queries(const ebrl_prefix8_layout_t *l, int32_t n, int32_t layer, const void *q, int32_t dtype, int32_t H, int32_t heads,
                            int64_t q_env, int64_t q_tok, float scale, bool none_too = false)
{
    if (layer < 0 || layer >= l->kv_layers) BAD("layer %d is outside 0..kv_layers - 1", layer);
    if (dtype != EBRL_F32 && dtype != EBRL_BF16) BAD("unknown q_dtype");
    const int least = none_too ? 0 : 1;
    if (H < least || heads < least || heads % l->n_kv_heads) BAD("H must be positive and n_heads a positive multiple of n_kv_heads");
    if (H > 1024 || heads > 1 << 16) return fail(EBRL_ERR_UNSUPPORTED, "H is limited to 1024 and n_heads to 65536");
    if (H == 0 || heads == 0) return EBRL_OK;
    if (!q || ((uintptr_t)q & 15)) BAD("q is NULL or not 16-byte aligned");
    if (!strides_fit(n, H, q_env, q_tok, (int64_t)esize(dtype)))
        BAD("query strides must be multiples of 16 bytes and not negative");
    if (!std::isfinite(scale)) BAD("scale must be finite");
    return EBRL_OK;
}

// The SMs of the current device; also checks the quota.
ebrl_status_t device_sms(int32_t quota, int *sms)
{
    static std::atomic<int> known[64];   // (calls may come from several threads)
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); return fail(EBRL_ERR_CUDA, "no usable CUDA device"); }
    if (!known[dev]) {
        int v = 0;
        const cudaError_t e = cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) { cudaGetLastError(); return fail(EBRL_ERR_CUDA, "no usable CUDA device: %s", cudaGetErrorString(e)); }
        known[dev] = v;
    }
    *sms = known[dev];
    if (quota > *sms) return fail(EBRL_ERR_QUOTA, "sm_quota %d on a device of %d SMs", quota, *sms);
    return EBRL_OK;
}

ebrl_status_t launched(cudaError_t e)
{
    if (e == cudaSuccess) return EBRL_OK;
    cudaGetLastError();
    return fail(EBRL_ERR_CUDA, "kernel launch failed: %s", cudaGetErrorString(e));
}

int longest(const int32_t *len, int n)
{
    int m = 0;
    for (int i = 0; i < n; ++i) m = std::max(m, (int)len[i]);
    return m;
}

// How prefixes are cut: tokens per piece, pieces of the longest prefix, warps that share a piece (a team: one CTA, joined in
// shared memory).  Left to itself (asked = 0), a call is cut where its items, weighed by their length, fill half of the warps that
// the SMs hold or less: among a team of as many warps as fill them once, and where eight are too few and prefixes longer than 4096
// tokens, into pieces of a team of four each.  Pieces cost a workspace and a second launch (7 us of the host's time), a team costs neither.
// Measured, us on the device, one warp / this rule: 1 x 256 tokens x 16 heads of 64, 1 row 8.4 / 6.0; 4 x 6303 x 8 heads of 128, 128 rows
// 146 / 81; 278 x 1732 x 2 heads of 64, 8 rows 49 / 30; two 65 k-token prefixes x 4 heads of 128, 4 rows 1394 / 30 (pieces of 384 tokens without
// teams 34).  Where SMs are half full short prefixes are not worth a team (512 x 64 - 512 x 4 heads, 8 rows, fp32: 1, 2, 4 warps
// 26, 29, 38; 96 x 0 - 301 x 2 heads of 32, 64 rows: 9.8, 14.7, 16.5), hence the least number of tiles; teams of eight at head_dim 128 leave 4 of
// 12 warps idle.  110 random calls: geometric mean 21.3 -> 15.6.
struct Cut { int split, n_split, team; };

Cut cut(const ebrl_prefix8_layout_t &l, int n, const int32_t *len, int H, int heads, int asked, int quota, int sms, bool f32)
{
    const int most = longest(len, n), rows = H * (heads / l.n_kv_heads);
    Cut c = {std::max(most, 1), 1, 1};
    if (asked < 0 || most == 0) return c;
    if (asked > 0) {
        if (most > asked) { c.split = asked; c.n_split = (most + asked - 1) / asked; }
        return c;
    }
    // Under a quota: persistent CTAs with a warp for each piece; as many pieces as there are warps for, not below 256 tokens.  Measured, us on the
    // device, never cut / this rule, quota 16 and 74: 1 x 1024 tokens x 16 heads of 64, 8 rows 19.9 / 12.4, 19.9 / 12.1; 16 x 2000 x 4 heads of
    // 128, 8 rows 45 / 36, 46 / 20; two 65 k-token prefixes x 4 heads of 128, 4 rows 1396 / 107, 1396 / 35; 64 x 768 x 16 heads of 128, 16 rows
    // (not cut) 258, 67.  It loses where items fill nearly half the warps: 4 x 6303 x 8 heads of 128, 128 rows at 74 SMs 177 / 190, 32 x 768 x 16
    // heads of 64, 8 fp32 rows 23.7 / 28.1.
    if (quota) {
        sms = std::min(sms, quota);
        long long items = 0;
        for (int i = 0; i < n; ++i) items += len[i] > 0;
        const int tile = attend_tile(l.head_dim, rows, f32, most);
        items *= (long long)l.n_kv_heads * ((rows + tile - 1) / tile);
        const long long warps = (long long)sms * attend_warps(l.head_dim, tile);
        if (items * 2 > warps) return c;
        const long long parts = std::min<long long>(warps / items, most / 256);
        if (parts < 2) return c;
        c.split = (int)((most + parts - 1) / parts + 127) / 128 * 128;
        c.n_split = (most + c.split - 1) / c.split;
        return c;
    }
    double tokens = 0;
    long long items = 0;
    for (int i = 0; i < n; ++i) { tokens += len[i]; items += len[i] > 0; }
    const int warps = attend_warps(l.head_dim, 8);
    const double per = (double)l.n_kv_heads * ((rows + 7) / 8) / ((double)sms * warps);   // items of 8 rows of an environment: their part of the SMs' warps
    const double fill = tokens / most * per, room = 2 / (items * per);   // (no more than two warps for each of theirs, however short most prefixes are)
    if (most > 4096 && fill * 8 <= 1) {
        const int pieces = (int)std::min(std::min(1 / (fill * 4), room / 4), most / 512.);
        if (pieces > 1) {
            c.split = ((most + pieces - 1) / pieces + 127) / 128 * 128;
            c.n_split = (most + c.split - 1) / c.split;
            c.team = 4;
            return c;
        }
    }
    c.team = fill * (warps % 8 ? warps : 8) <= 1 ? 8 : (fill <= .3 ? 4 : (fill <= .5 ? 2 : 1));
    const int least = fill <= .04 ? 1 : (fill <= .125 ? 2 : (fill <= .3 ? 8 : 20));   // tiles for every warp of the longest
    while (c.team > 1 && (c.team > room || most <= least * (c.team - 1) * BLOCK)) c.team /= 2;
    return c;
}

uint64_t part_rows(int n, int n_split, int H, int heads) { return n_split > 1 ? (uint64_t)n * n_split * H * heads : 0; }

// No exception leaves the library.
template <typename F> ebrl_status_t guarded(F &&f)
{
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return fail(EBRL_ERR_NOMEM, "out of host memory");
    } catch (const std::exception &e) {
        return fail(EBRL_ERR_INVALID_ARG, "%s", e.what());
    }
}

bool overlap(const void *a, uint64_t na, const void *b, uint64_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

// Whether two arrays of n rows of `width` fp32 values share memory.  Rows of one stride may lie between one another.
bool rows_overlap(const float *a, int64_t stride_a, const float *b, int64_t stride_b, int64_t n, int64_t width)
{
    auto bytes = [&](int64_t stride) { return (uint64_t)((n - 1) * stride + width) * 4; };
    if (!overlap(a, bytes(stride_a), b, bytes(stride_b))) return false;
    if (stride_a != stride_b) return true;
    const uint64_t stride = (uint64_t)stride_a * 4, w = (uint64_t)width * 4;
    const uint64_t apart = ((uintptr_t)a > (uintptr_t)b ? (uintptr_t)a - (uintptr_t)b : (uintptr_t)b - (uintptr_t)a) % stride;
    return apart < w || stride - apart < w;
}

thread_local Envs t_envs;
thread_local QuantEnvs t_quant;
thread_local EvictEnvs t_evict;

const Envs &some_envs(int first, int n, const int32_t *slots, const int32_t *len)
{
    t_envs.n = n;
    for (int i = 0; i < n; ++i) { t_envs.slot[i] = slots ? slots[first + i] : first + i; t_envs.len[i] = len[first + i]; }
    return t_envs;
}

}  // namespace

extern "C" {

uint64_t ebrl_prefix8_record_bytes(const ebrl_prefix8_layout_t *layout)
{
    return check_layout(layout) == EBRL_OK ? (uint64_t)record_of(*layout).bytes : 0;
}

const char *ebrl_prefix8_last_error(void) { return t_error; }

ebrl_status_t ebrl_prefix8_quantize(const ebrl_prefix8_layout_t *layout, void *pool, int32_t n_slots, int32_t n, const int32_t *slots,
                                    const void *const *planes, const int32_t *len, const int32_t *plane_rows, int64_t row_stride,
                                    int32_t src_dtype, const uint8_t *const *mask, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_envs(layout, pool, n_slots, n, slots, len, sm_quota, true);
        if (st != EBRL_OK || n == 0) return st;
        if (src_dtype != EBRL_F32 && src_dtype != EBRL_BF16) BAD("unknown src_dtype");
        const int64_t d = (int64_t)layout->n_kv_heads * layout->head_dim;
        if (row_stride == 0) row_stride = d;
        if (row_stride < d || row_stride * (int64_t)esize(src_dtype) % 16) BAD("row_stride must be at least %lld elements and a multiple of 16 bytes", (long long)d);
        if (!planes) BAD("planes is NULL");
        for (int i = 0; i < n; ++i) {
            if (len[i] == 0) continue;
            if (!planes[i] || ((uintptr_t)planes[i] & 15)) BAD("planes[%d] is NULL or not 16-byte aligned", i);
            if (plane_rows && plane_rows[i] < len[i]) BAD("plane_rows[%d] < len[%d]", i, i);
        }
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        const Record rec = record_of(*layout);
        for (int first = 0; first < n; first += QUANT_ENVS) {
            QuantEnvs &e = t_quant;
            e.n = std::min(QUANT_ENVS, n - first);
            for (int i = 0; i < e.n; ++i) {
                const int k = first + i;
                e.planes[i] = planes[k]; e.mask[i] = mask ? mask[k] : nullptr;
                e.slot[i] = slots ? slots[k] : k; e.len[i] = len[k]; e.plane_rows[i] = plane_rows ? plane_rows[k] : len[k];
            }
            st = launched(launch_quantize(rec, (char *)pool, row_stride, src_dtype == EBRL_F32, e, longest(e.len, e.n), sm_quota, (cudaStream_t)stream));
            if (st != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

uint64_t ebrl_prefix8_attend_workspace(const ebrl_prefix8_layout_t *layout, int32_t n, const int32_t *len, int32_t H, int32_t n_heads,
                                       int32_t split_tokens, int32_t sm_quota)
{
    if (check_layout(layout) != EBRL_OK || n <= 0 || !len || H < 1 || n_heads < 1 || n_heads % layout->n_kv_heads) return 0;
    int sms = 0;
    if (device_sms(0, &sms) != EBRL_OK) return 0;
    uint64_t most = 0;   // of either query type
    for (int f32 = 0; f32 < 2; ++f32) {
        const Cut c = cut(*layout, n, len, H, n_heads, split_tokens, std::max<int>(sm_quota, 0), sms, f32 != 0);
        most = std::max(most, part_rows(n, c.n_split, H, n_heads) * (layout->head_dim + 2) * 4);
    }
    return most;
}

ebrl_status_t ebrl_prefix8_attend(const ebrl_prefix8_layout_t *layout, const void *pool, int32_t n_slots, int32_t n, const int32_t *slots,
                                  const int32_t *len, int32_t layer, const void *q, int32_t q_dtype, int32_t H, int32_t n_heads,
                                  int64_t q_env_stride, int64_t q_token_stride, void *out, int64_t o_env_stride, int64_t o_token_stride,
                                  float *lse, float scale, int32_t split_tokens, void *workspace, uint64_t workspace_bytes,
                                  int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_envs(layout, pool, n_slots, n, slots, len, sm_quota, false);
        if (st != EBRL_OK || n == 0) return st;
        if ((st = check_queries(layout, n, layer, q, q_dtype, H, n_heads, q_env_stride, q_token_stride, scale)) != EBRL_OK) return st;
        if (!out || ((uintptr_t)out & 15)) BAD("out is NULL or not 16-byte aligned");
        if (lse && ((uintptr_t)lse & 3)) BAD("lse is not 4-byte aligned");
        const int64_t es = (int64_t)esize(q_dtype), width = (int64_t)n_heads * layout->head_dim;
        if (!strides_fit(n, H, o_env_stride, o_token_stride, es)) BAD("output strides must be multiples of 16 bytes and not negative");
        if (!rows_apart(n, H, o_env_stride, o_token_stride, width)) BAD("output rows overlap one another");
        if (out == q && ((n > 1 && o_env_stride != q_env_stride) || (H > 1 && o_token_stride != q_token_stride)))
            BAD("out may be q only with the same strides");
        if (split_tokens < -1 || split_tokens % 128 > 0) BAD("split_tokens is -1, 0 or a positive multiple of 128");
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        const bool f32 = q_dtype == EBRL_F32;
        const Cut c = cut(*layout, n, len, H, n_heads, split_tokens, sm_quota, sms, f32);
        const int n_split = c.n_split;
        const int rows = H * (n_heads / layout->n_kv_heads);
        if ((int64_t)std::min(n, CHUNK_ENVS) * layout->n_kv_heads * n_split * ((rows + 7) / 8) > INT32_MAX)
            return fail(EBRL_ERR_UNSUPPORTED, "too many pieces in one call");
        const uint64_t pr = part_rows(n, n_split, H, n_heads), need = pr * (layout->head_dim + 2) * 4;
        if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need))
            BAD("a 16-byte aligned workspace of %llu bytes is needed", (unsigned long long)need);
        AttendArgs a{};
        a.r.rec = record_of(*layout); a.r.pool = (const char *)pool; a.r.layer = layer;
        a.r.q_env = q_env_stride; a.r.q_tok = q_token_stride; a.r.H = H; a.r.heads = n_heads; a.r.G = n_heads / layout->n_kv_heads; a.r.scale = scale;
        a.o_env = o_env_stride; a.o_tok = o_token_stride;
        a.split = c.split; a.n_split = n_split; a.team = c.team;
        for (int first = 0; first < n; first += CHUNK_ENVS) {
            const Envs &e = some_envs(first, std::min(CHUNK_ENVS, n - first), slots, len);
            a.max_len = longest(e.len, e.n);
            a.alike = std::all_of(e.len, e.len + e.n, [&](int v) { return v == a.max_len; });
            a.r.q = (const char *)q + first * q_env_stride * es;
            a.out = (char *)out + first * o_env_stride * es;
            a.lse = lse ? lse + (size_t)first * H * n_heads : nullptr;
            if (need) {
                const size_t at = (size_t)first * n_split * H * n_heads;
                a.part_o = (float *)workspace + at * layout->head_dim;
                a.part_ml = (float *)workspace + pr * layout->head_dim + at * 2;
            }
            if ((st = launched(launch_attend(a, e, f32, sm_quota, sms, (cudaStream_t)stream))) != EBRL_OK) return st;
            if (n_split > 1 && (st = launched(launch_attend_join(a, e, f32, sm_quota, sms, (cudaStream_t)stream))) != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_prefix8_weigh(const ebrl_prefix8_layout_t *layout, const void *pool, int32_t n_slots, int32_t n, const int32_t *slots,
                                 const int32_t *len, int32_t layer, const void *q, int32_t q_dtype, int32_t H, int32_t n_heads,
                                 int64_t q_env_stride, int64_t q_token_stride, const float *lse, int64_t lse_env_stride,
                                 int64_t lse_token_stride, int64_t lse_head_stride, float scale, float *weight, int64_t weight_stride, int32_t accumulate, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_envs(layout, pool, n_slots, n, slots, len, sm_quota, true);
        if (st != EBRL_OK || n == 0) return st;
        const bool rows = H != 0 && n_heads != 0;   // (without rows there is nothing to read, but a sum to write)
        if ((st = check_queries(layout, n, layer, q, q_dtype, H, n_heads, q_env_stride, q_token_stride, scale, true)) != EBRL_OK) return st;
        if ((rows && !lse) || !weight || (((uintptr_t)lse | (uintptr_t)weight) & 3)) BAD("lse or weight is NULL or not 4-byte aligned");
        if (rows && (lse_env_stride < 0 || lse_token_stride < 0 || lse_head_stride < 0)) BAD("lse strides must not be negative");
        if (weight_stride < layout->capacity) BAD("weight_stride < capacity");
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        if (!rows && accumulate) return EBRL_OK;
        WeighArgs a{};
        a.r.rec = record_of(*layout); a.r.pool = (const char *)pool; a.r.layer = layer;
        a.r.q_env = q_env_stride; a.r.q_tok = q_token_stride; a.r.H = H; a.r.heads = n_heads; a.r.G = n_heads / layout->n_kv_heads; a.r.scale = scale;
        a.l_env = lse_env_stride; a.l_tok = lse_token_stride; a.l_head = lse_head_stride;
        a.weight = weight; a.stride = weight_stride; a.accumulate = accumulate != 0;
        for (int first = 0; first < n; first += CHUNK_ENVS) {
            const Envs &e = some_envs(first, std::min(CHUNK_ENVS, n - first), slots, len);
            a.r.q = (const char *)q + first * q_env_stride * (int64_t)esize(q_dtype);
            a.lse = lse + first * lse_env_stride;
            if ((st = launched(launch_weigh(a, e, q_dtype == EBRL_F32, longest(e.len, e.n), sm_quota, sms, (cudaStream_t)stream))) != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_prefix8_evict(const ebrl_prefix8_layout_t *layout, const void *src, void *dst, int32_t n_slots, int32_t n,
                                 const int32_t *slots, const int32_t *len, const int32_t *keep, int32_t protect_first, int32_t protect_last,
                                 const float *weight, int64_t weight_stride, float *weight_out, int64_t weight_out_stride, int32_t *kept,
                                 int64_t kept_stride, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_envs(layout, src, n_slots, n, slots, len, sm_quota, true);
        if (st != EBRL_OK || n == 0) return st;
        const Record rec = record_of(*layout);
        if (!dst || ((uintptr_t)dst & 15)) BAD("dst is NULL or not 16-byte aligned");
        if (dst != src && overlap(src, rec.bytes * (uint64_t)n_slots, dst, rec.bytes * (uint64_t)n_slots)) BAD("dst overlaps src without being it");
        if (!keep) BAD("keep is NULL");
        if (protect_first < 0 || protect_last < 0) BAD("protect_first and protect_last must not be negative");
        if (!weight || !kept || (((uintptr_t)weight | (uintptr_t)weight_out | (uintptr_t)kept) & 3)) BAD("weight or kept is NULL, or an array is not 4-byte aligned");
        if (weight_stride < layout->capacity || (weight_out && weight_out_stride < layout->capacity)) BAD("weight strides must be at least capacity");
        if (weight_out == weight ? weight_out_stride != weight_stride
                                 : weight_out && rows_overlap(weight, weight_stride, weight_out, weight_out_stride, n_slots, layout->capacity))
            BAD("weight_out overlaps weight without being it");
        for (int i = 0; i < n; ++i) {
            if (keep[i] < 0) BAD("keep[%d] < 0", i);
            if (std::min(keep[i], len[i]) > kept_stride) BAD("kept_stride is less than the new length of environment %d", i);
        }
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        EvictArgs a{};
        a.rec = rec; a.src = (const char *)src; a.dst = (char *)dst;
        a.protect_first = protect_first; a.protect_last = protect_last;
        a.weight = weight; a.weight_stride = weight_stride; a.weight_out = weight_out; a.weight_out_stride = weight_out_stride;
        a.kept_stride = kept_stride;
        for (int first = 0; first < n; first += EVICT_ENVS) {
            EvictEnvs &e = t_evict;
            e.n = std::min(EVICT_ENVS, n - first);
            int most = 0;
            for (int i = 0; i < e.n; ++i) {
                e.slot[i] = slots ? slots[first + i] : first + i;
                e.len[i] = len[first + i];
                e.keep[i] = std::min(keep[first + i], len[first + i]);
                most = std::max(most, e.keep[i]);
            }
            a.kept = kept + first * kept_stride;
            if ((st = launched(launch_evict(a, e, most, sm_quota, sms, (cudaStream_t)stream))) != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

}  // extern "C"
