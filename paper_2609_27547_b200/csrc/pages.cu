// The C boundary of the operators on paged caches (include/ebrl_pages.h): argument checks, the choice of pieces, and the launches.
// Nothing here touches the device before every argument has been checked.
#include "pages_internal.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <vector>

using namespace ebrl;
using namespace ebrl::pg;

namespace ebrl {
namespace pg {

char *error_text()
{
    static thread_local char text[256];
    return text;
}

Geometry geometry_of(const ebrl_pages_layout_t &l)
{
    Geometry g{};
    g.layers = l.kv_layers; g.kvh = l.n_kv_heads; g.hd = l.head_dim; g.T = l.page_tokens; g.es = l.dtype == EBRL_BF16 ? 2 : 4;
    while (1 << g.t_shift < g.T) ++g.t_shift;
    g.head = (size_t)g.T * g.hd * g.es;
    g.mask = (size_t)g.layers * 2 * g.kvh * g.head;
    g.bytes = (g.mask + (size_t)g.T / 8 + 127) & ~(size_t)127;
    return g;
}

}  // namespace pg
}  // namespace ebrl

namespace {

ebrl_status_t fail(ebrl_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(error_text(), 256, fmt, ap);
    va_end(ap);
    return st;
}

#define BAD(...) return fail(EBRL_ERR_INVALID_ARG, __VA_ARGS__)

ebrl_status_t check_layout(const ebrl_pages_layout_t *l)
{
    if (!l) BAD("layout is NULL");
    if (l->kv_layers < 1 || l->n_kv_heads < 1) BAD("kv_layers and n_kv_heads must be positive");
    if (l->dtype != EBRL_F32 && l->dtype != EBRL_BF16) BAD("unknown dtype");
    if (l->head_dim != 32 && l->head_dim != 64 && l->head_dim != 128) return fail(EBRL_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
    if (l->page_tokens != 32 && l->page_tokens != 64 && l->page_tokens != 128 && l->page_tokens != 256)
        return fail(EBRL_ERR_UNSUPPORTED, "page_tokens must be 32, 64, 128 or 256");
    if (l->kv_layers > 1 << 12 || l->n_kv_heads > 1 << 12) return fail(EBRL_ERR_UNSUPPORTED, "kv_layers and n_kv_heads are limited to 4096");
    return EBRL_OK;
}

ebrl_status_t check_pool(const ebrl_pages_layout_t *l, const void *pool, int32_t n_pages, int32_t n, int32_t sm_quota)
{
    const ebrl_status_t st = check_layout(l);
    if (st != EBRL_OK) return st;
    if (n < 0 || n_pages < 0) BAD("n and n_pages must not be negative");
    if (sm_quota < 0) return fail(EBRL_ERR_QUOTA, "sm_quota < 0");
    if (n == 0) return EBRL_OK;
    if (!pool || ((uintptr_t)pool & 15)) BAD("the pool is NULL or not 16-byte aligned");
    if (n_pages < 1) BAD("the pool has no pages");
    return EBRL_OK;
}

// What every operator on sequences takes: the table and the lengths.
ebrl_status_t check_seqs(const ebrl_pages_layout_t *l, int32_t n, const int32_t *table, int64_t table_stride, const int32_t *len)
{
    if (!len) BAD("len is NULL");
    bool any = false;                 // (a table without columns has no address)
    for (int i = 0; i < n; ++i) any = any || len[i] > 0;
    if ((!table && any) || ((uintptr_t)table & 3)) BAD("table is NULL or not 4-byte aligned");
    if (table_stride < 0) BAD("table_stride must not be negative");
    for (int i = 0; i < n; ++i) {
        if (len[i] < 0 || len[i] > 1 << 30) BAD("len[%d] = %d is outside 0..2^30", i, len[i]);
        if ((len[i] + (int64_t)l->page_tokens - 1) / l->page_tokens > table_stride) BAD("len[%d] = %d needs more than %lld pages", i, len[i], (long long)table_stride);
    }
    return EBRL_OK;
}

// The packed rows of a call: their number, or -1 where there are too many.
int64_t total_rows(int32_t n, const int32_t *count)
{
    int64_t t = 0;
    for (int i = 0; i < n; ++i) t += count[i];
    return t <= INT32_MAX ? t : -1;
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

thread_local AppendSeqs t_append;
thread_local GatherSeqs t_gather;
thread_local AttendSeqs t_attend;
thread_local CopyPages t_copy;
thread_local uint64_t t_drop_limit = 0;     // tests of the give-up path

// ---- attend: kernels, pieces ----

// Sequences of one call that one kernel takes: those whose query rows fill items of so many rows.
struct Group {
    int rows = 0;                    // query rows of an item
    std::vector<int> seqs;
    int split = 0, team = 1;
};

// A sequence of more rows is taken by the tensor-memory kernel.  Measured, us, one warp per item / that kernel, 64 x 2000 tokens x 4 heads: heads of 128, 16 rows
// 55 / -, 32 rows 83 / 53, 64 rows 159 / 54; of 64, 32 rows 41 / 42, 64 rows 115 / 42; of 32, 64 rows 65 / 61 (with two tiles per CTA).
int chunk_from(int hd) { return hd == 128 ? 16 : 32; }

// Its rows per item.  Two tiles that share what is loaded pay where the products take the time, and are never much worse there: heads of 128, 4 x 2000 new
// tokens over 8 - 16 k x 16 heads 751 us against 779 in CTAs of one tile, 64 x 100 over 600 88 against 86.  Heads of 64 and 32 wait for the exponentials either way:
// 4 x 2048 over 8 k 432 against 412, 64 x 100 over 600 75 against 70 (59 since such CTAs are persistent).
int chunk_rows(int hd, int64_t rows) { return hd == 128 && rows > SMALL_CHUNK_ROWS ? CHUNK_ROWS : SMALL_CHUNK_ROWS; }

struct Plan {
    Group groups[4];                 // CHUNK_ROWS, SMALL_CHUNK_ROWS, 32 rows, 16 rows: in this order, so that short items fill up what long ones leave
    std::vector<int64_t> row;        // first packed query of each sequence
    uint64_t pairs = 0;              // (query, piece) pairs of the sequences that are cut
};

int tiles_of(int len, int m, int window)   // mask words that a sequence's longest item sees
{
    return (len - first_token(len, m, window) + WORD - 1) / WORD;
}

// How long a group takes, in tiles, where `slots` items are worked on at a time, each sequence is cut into pieces of `piece` tiles and an item is shared by a
// team of warps: the longest piece, or an even share of all there is and, where there is more than one round, half a piece that some wait for.  An item's
// beginning and end cost 3 tiles.
double time_of(const std::vector<int> &tiles, const std::vector<int64_t> &items, double slots, int piece, int team)
{
    double all = 0, count = 0;
    int longest = 0;
    for (size_t k = 0; k < tiles.size(); ++k) {
        const int n = (tiles[k] + piece - 1) / piece;
        longest = std::max(longest, std::min(piece, tiles[k]));
        count += (double)items[k] * n;
        all += (double)items[k] * ((double)tiles[k] / team + 3 * n);
    }
    const double one = (double)longest / team + 3;
    return std::max(one, all / slots + (count > slots ? one / 2 : 0));
}

// How a group's sequences are cut.  Left to itself (asked = 0): an item is shared by the team of warps for which time_of is least (16 or 32 rows, no quota), and
// long sequences are cut into the pieces for which it is, where that saves more than the join costs.
void cut(const ebrl_pages_layout_t &l, Group &g, const int32_t *m, const int32_t *len, int G, int window, int asked, int quota, int sms)
{
    if (asked < 0) return;
    if (asked > 0) { g.split = asked; return; }
    const bool chunk = g.rows >= SMALL_CHUNK_ROWS;
    const int warps = chunk ? (quota ? 1 : CHUNK_ROWS / g.rows) : attend_warps(l.head_dim, l.dtype == EBRL_F32, g.rows);   // items that an SM works on at a time
    const int tile = chunk ? 4 : 1;                                                        // mask words of a tile
    const int at_once = quota ? std::min(sms, quota) : sms;
    auto slots = [&](int team) { return (double)at_once * (warps / team); };
    std::vector<int> tiles;
    std::vector<int64_t> items;
    double all = 0;
    int longest = 1;
    double rows = 0;                                                                       // of all heads
    for (int i : g.seqs) {
        rows += (double)m[i] * G * l.n_kv_heads;
        tiles.push_back((tiles_of(len[i], m[i], window) + tile - 1) / tile);
        items.push_back((int64_t)l.n_kv_heads * (((int64_t)m[i] * G + g.rows - 1) / g.rows));
        all += (double)items.back();
        longest = std::max(longest, tiles.back());
    }
    if (all >= 8 * slots(1)) return;                    // (many rounds: nothing to gain)
    double best = time_of(tiles, items, slots(1), longest, 1);
    if (!chunk && !quota)
        for (int team = 2; team <= std::min(8, warps); team *= 2) {
            const double t = time_of(tiles, items, slots(team), longest, team) + 1;              // (their join)
            if (t < .95 * best) { best = t; g.team = team; }
        }
    if (tiles.size() > 64 || longest * tile < 32) return;
    const int team = chunk || quota ? 1 : 4, step = chunk ? 1 : 4;                         // pieces are multiples of 128 tokens
    for (int pieces = 2; pieces <= 64 && longest / pieces >= 4 * team; ++pieces) {
        const int piece = ((longest + pieces - 1) / pieces + step - 1) / step * step;
        // the join: a launch, and the partial results written and read, 8 MB in the time of a tile (1 - 2 us)
        const double t = time_of(tiles, items, slots(team), piece, team) + 6 + rows * pieces * l.head_dim * 8 / 8e6;
        if (t < .95 * best) { best = t; g.team = team; g.split = piece * tile * WORD; }
    }
}

void plan(Plan &p, const ebrl_pages_layout_t &l, int32_t n, const int32_t *m, const int32_t *len, int n_heads, int window, int asked, int quota, int sms, bool chunks)
{
    const int G = n_heads / l.n_kv_heads;
    int64_t at = 0;
    p.row.resize((size_t)n);
    for (int i = 0; i < n; ++i) {
        p.row[i] = at;
        at += m[i];
        if (m[i] == 0) continue;
        const int64_t all = (int64_t)m[i] * G;
        const int rows = chunks && all > chunk_from(l.head_dim) ? chunk_rows(l.head_dim, all) : attend_rows((int)std::min<int64_t>(all, 1 << 20));
        Group &g = p.groups[rows == 16 ? 3 : (rows == 32 ? 2 : (rows == SMALL_CHUNK_ROWS ? 1 : 0))];
        g.rows = rows;
        g.seqs.push_back(i);
    }
    for (Group &g : p.groups) {
        if (g.seqs.empty()) continue;
        cut(l, g, m, len, G, window, asked, quota, sms);
        // longest first: what is handed out last is short
        std::stable_sort(g.seqs.begin(), g.seqs.end(), [&](int a, int b) { return len[a] > len[b]; });
        for (int i : g.seqs) {
            const int np = pieces_of(len[i], m[i], window, g.split);
            if (np > 1) p.pairs += (uint64_t)np * m[i];
        }
    }
}

ebrl_status_t check_attend_counts(const ebrl_pages_layout_t *l, int32_t n, const int32_t *new_tokens, int32_t n_heads, int32_t causal, int32_t window,
                                  int32_t split_tokens)
{
    if (!new_tokens) BAD("new_tokens is NULL");
    if (n_heads < 1 || n_heads % l->n_kv_heads) BAD("n_heads must be a positive multiple of n_kv_heads");
    if (n_heads > 1 << 16 || n_heads / l->n_kv_heads > 128) return fail(EBRL_ERR_UNSUPPORTED, "n_heads is limited to 65536 and to 128 for each key/value head");
    for (int i = 0; i < n; ++i)
        if (new_tokens[i] < 0) BAD("new_tokens[%d] < 0", i);
    const int64_t rows = total_rows(n, new_tokens);
    if (rows < 0) return fail(EBRL_ERR_UNSUPPORTED, "more than 2^31 - 1 queries in one call");
    for (int i = 0; i < n; ++i)
        if ((int64_t)new_tokens[i] * (n_heads / l->n_kv_heads) > INT32_MAX / 2) return fail(EBRL_ERR_UNSUPPORTED, "new_tokens[%d] is too large", i);
    if (window < 0) BAD("window must not be negative");
    if (window > 0 && !causal) BAD("a window needs causal");
    if (split_tokens < -1 || split_tokens % 128 > 0) BAD("split_tokens is -1, 0 or a positive multiple of 128");
    return EBRL_OK;
}

// A call's window and pieces, small enough for 32-bit arithmetic.
void bound(int32_t n, const int32_t *len, int32_t &window, int32_t &split_tokens)
{
    const int longest = *std::max_element(len, len + n);
    window = bounded_window(window, longest);
    split_tokens = bounded_split(split_tokens, longest);
}

uint64_t part_bytes(const ebrl_pages_layout_t &l, uint64_t pairs, int n_heads) { return pairs * n_heads * (l.head_dim + 2) * 4; }

}  // namespace

extern "C" {

uint64_t ebrl_pages_page_bytes(const ebrl_pages_layout_t *layout)
{
    return check_layout(layout) == EBRL_OK ? (uint64_t)geometry_of(*layout).bytes : 0;
}

const char *ebrl_pages_last_error(void) { return error_text(); }

ebrl_status_t ebrl_pages_check(void)
{
    int sms = 0, status = 0;
    const ebrl_status_t st = device_sms(0, &sms);
    if (st != EBRL_OK) return st;
    const cudaError_t e = take_status(&status);
    if (e != cudaSuccess) { cudaGetLastError(); return fail(EBRL_ERR_CUDA, "%s", cudaGetErrorString(e)); }
    return status ? fail(EBRL_ERR_TIMEOUT, "a kernel's wait for its own copies ran out") : EBRL_OK;
}

void ebrl_pages_test_drop_copies(uint64_t limit_ns) { t_drop_limit = std::min<uint64_t>(limit_ns, 2000000000ull); }

ebrl_status_t ebrl_pages_append(const ebrl_pages_layout_t *layout, void *pool, int32_t n_pages, int32_t n, const int32_t *table, int64_t table_stride,
                                const int32_t *new_tokens, const int32_t *len, int32_t layer, const void *k, int64_t k_stride, const void *v,
                                int64_t v_stride, const uint8_t *mask, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_pool(layout, pool, n_pages, n, sm_quota);
        if (st != EBRL_OK || n == 0) return st;
        if ((st = check_seqs(layout, n, table, table_stride, len)) != EBRL_OK) return st;
        if (layer < 0 || layer >= layout->kv_layers) BAD("layer %d is outside 0..kv_layers - 1", layer);
        if (!new_tokens) BAD("new_tokens is NULL");
        for (int i = 0; i < n; ++i)
            if (new_tokens[i] < 0 || new_tokens[i] > len[i]) BAD("new_tokens[%d] = %d is outside 0..len", i, new_tokens[i]);
        const int64_t rows = total_rows(n, new_tokens);
        if (rows < 0) return fail(EBRL_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens in one call");
        if (rows == 0) return EBRL_OK;
        const Geometry g = geometry_of(*layout);
        if (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) BAD("k or v is NULL or not 16-byte aligned");
        if (rows > 1 && (k_stride < 0 || v_stride < 0 || (k_stride * g.es | v_stride * g.es) % 16)) BAD("strides must be multiples of 16 bytes and not negative");
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        AppendArgs a{};
        a.g = g;
        a.p = {(char *)pool, n_pages, table, table_stride};
        a.layer = layer; a.k = (const char *)k; a.v = (const char *)v;
        a.k_stride = k_stride * g.es; a.v_stride = v_stride * g.es; a.mask = mask;
        AppendSeqs &s = t_append;
        int row = 0;
        s.n = s.items = 0;
        auto flush = [&]() {
            const ebrl_status_t r = launched(launch_append(a, s, sm_quota, (cudaStream_t)stream));
            s.n = s.items = 0;
            return r;
        };
        for (int i = 0; i < n; ++i) {
            if (new_tokens[i] == 0) continue;
            const int start = len[i] - new_tokens[i];
            s.s[s.n] = {s.items, row, new_tokens[i], len[i], i};
            s.items += (len[i] + WORD - 1) / WORD - start / WORD;
            row += new_tokens[i];
            if (++s.n == SEQS && (st = flush()) != EBRL_OK) return st;
        }
        return s.n ? flush() : EBRL_OK;
    });
}

uint64_t ebrl_pages_attend_workspace(const ebrl_pages_layout_t *layout, int32_t n, const int32_t *new_tokens, const int32_t *len, int32_t n_heads,
                                     int32_t causal, int32_t window, int32_t split_tokens, int32_t sm_quota)
{
    uint64_t bytes = 0;
    guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_layout(layout);
        if (st != EBRL_OK) return st;
        if (n <= 0 || !len) BAD("n or len");
        if ((st = check_attend_counts(layout, n, new_tokens, n_heads, causal, window, split_tokens)) != EBRL_OK) return st;
        for (int i = 0; i < n; ++i)
            if (len[i] < 0 || len[i] > 1 << 30) BAD("len[%d] = %d is outside 0..2^30", i, len[i]);
        int sms = 0;
        if ((st = device_sms(0, &sms)) != EBRL_OK) return st;
        bound(n, len, window, split_tokens);
        for (int chunks = 0; chunks < 2; ++chunks) {   // of either kernel: which one it is may depend on the scale
            Plan p;
            plan(p, *layout, n, new_tokens, len, n_heads, window, split_tokens, std::max<int>(sm_quota, 0), sms, chunks && chunk_supported(geometry_of(*layout), 0, 1.f));
            bytes = std::max(bytes, part_bytes(*layout, p.pairs, n_heads));
        }
        return EBRL_OK;
    });
    return bytes;
}

ebrl_status_t ebrl_pages_attend(const ebrl_pages_layout_t *layout, const void *pool, int32_t n_pages, int32_t n, const int32_t *table,
                                int64_t table_stride, const int32_t *new_tokens, const int32_t *len, int32_t layer, const void *q, int64_t q_stride,
                                int32_t n_heads, void *out, int64_t o_stride, float *lse, float scale, int32_t causal, int32_t window,
                                int32_t split_tokens, void *workspace, uint64_t workspace_bytes, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_pool(layout, pool, n_pages, n, sm_quota);
        if (st != EBRL_OK || n == 0) return st;
        if ((st = check_seqs(layout, n, table, table_stride, len)) != EBRL_OK) return st;
        if (layer < 0 || layer >= layout->kv_layers) BAD("layer %d is outside 0..kv_layers - 1", layer);
        if ((st = check_attend_counts(layout, n, new_tokens, n_heads, causal, window, split_tokens)) != EBRL_OK) return st;
        const int64_t rows = total_rows(n, new_tokens);
        if (rows == 0) return EBRL_OK;
        const Geometry g = geometry_of(*layout);
        const int64_t width = (int64_t)n_heads * g.hd;
        if (!q || ((uintptr_t)q & 15)) BAD("q is NULL or not 16-byte aligned");
        if (!out || ((uintptr_t)out & 15)) BAD("out is NULL or not 16-byte aligned");
        if (lse && ((uintptr_t)lse & 3)) BAD("lse is not 4-byte aligned");
        if (rows > 1 && (q_stride < 0 || o_stride < 0 || q_stride * g.es % 16 || o_stride * g.es % 16)) BAD("strides must be multiples of 16 bytes and not negative");
        if (rows > 1 && o_stride < width) BAD("output rows overlap one another");
        if (rows > 1 && out == q && o_stride != q_stride) BAD("out may be q only with the same stride");
        if (!std::isfinite(scale * 1.4426950408889634f)) BAD("scale must be finite, and below 2.3e38");   // (scores are taken in units of log 2)
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        bound(n, len, window, split_tokens);
        Plan p;
        plan(p, *layout, n, new_tokens, len, n_heads, window, split_tokens, sm_quota, sms, chunk_supported(g, n_pages, scale));
        const uint64_t need = part_bytes(*layout, p.pairs, n_heads);
        if (p.pairs > INT32_MAX) return fail(EBRL_ERR_UNSUPPORTED, "too many pieces in one call");
        auto items_of = [&](const Group &gr, int i) {
            return (((int64_t)new_tokens[i] * (n_heads / g.kvh) + gr.rows - 1) / gr.rows) * g.kvh * pieces_of(len[i], new_tokens[i], window, gr.split);
        };
        for (const Group &gr : p.groups)
            for (int i : gr.seqs)
                if (items_of(gr, i) > 1 << 30) return fail(EBRL_ERR_UNSUPPORTED, "too many query rows, heads and pieces in sequence %d", i);
        if (need && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < need))
            BAD("a 16-byte aligned workspace of %llu bytes is needed", (unsigned long long)need);
        AttendArgs a{};
        a.g = g;
        a.p = {(char *)pool, n_pages, table, table_stride};
        a.layer = layer; a.heads = n_heads; a.G = n_heads / g.kvh;
        a.q = (const char *)q; a.out = (char *)out; a.q_stride = q_stride; a.o_stride = o_stride;
        a.lse = lse; a.scale = scale; a.up = std::min(8.f / std::max(scale * 1.4426950408889634f, FLT_MIN * .125f), FLT_MAX); a.causal = causal != 0; a.window = window;
        a.limit_ns = t_drop_limit ? t_drop_limit : 4000000000ull;
        a.test_drop_copies = t_drop_limit != 0;
        a.part_o = (float *)workspace;
        a.part_ml = (float *)workspace + p.pairs * n_heads * g.hd;
        const bool f32 = layout->dtype == EBRL_F32;
        AttendSeqs &s = t_attend;
        int64_t pair = 0;
        bool beside = false;             // whether a kernel of this call is before this one (a quota allows one at a time; a join waits for all)
        for (const Group &gr : p.groups) {
            a.split = gr.split; a.team = gr.team;
            for (size_t at = 0; at < gr.seqs.size();) {
                int64_t items = 0;
                s.n = 0;
                bool any = false;
                for (; at < gr.seqs.size() && s.n < SEQS; ++at) {
                    const int i = gr.seqs[at], np = pieces_of(len[i], new_tokens[i], window, gr.split);
                    const int64_t mine = items_of(gr, i);
                    if (items + mine > 1 << 30) break;
                    s.s[s.n] = {(int)items, (int)p.row[i], new_tokens[i], len[i], i, np > 1 ? (int)pair : -1};
                    if (np > 1) { pair += (int64_t)np * new_tokens[i]; any = true; }
                    items += mine;
                    ++s.n;
                }
                s.items = (int)items;
                st = launched(gr.rows >= SMALL_CHUNK_ROWS ? launch_chunk(a, s, gr.rows, sm_quota, sms, beside, (cudaStream_t)stream)
                                                    : launch_attend(a, s, f32, gr.rows, sm_quota, beside, (cudaStream_t)stream));
                beside = sm_quota == 0 && !any;
                if (st != EBRL_OK) return st;
                if (!any) continue;
                // the join's items are the queries of the cut sequences
                int k = 0, queries = 0;
                for (int j = 0; j < s.n; ++j) {
                    if (s.s[j].part < 0) continue;
                    s.s[k] = s.s[j];
                    s.s[k].item = queries;
                    queries += s.s[k].m;
                    ++k;
                }
                s.n = k;
                s.items = queries;
                if ((st = launched(launch_attend_join(a, s, f32, sm_quota, sms, (cudaStream_t)stream))) != EBRL_OK) return st;
            }
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_copy(const ebrl_pages_layout_t *layout, const void *src, int32_t src_pages, void *dst, int32_t dst_pages, int32_t n,
                              const int32_t *from, const int32_t *to, const int32_t *tokens, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_pool(layout, src, src_pages, n, sm_quota);
        if (st == EBRL_OK) st = check_pool(layout, dst, dst_pages, n, sm_quota);
        if (st != EBRL_OK || n == 0) return st;
        if (!from || !to) BAD("from or to is NULL");
        const Geometry g = geometry_of(*layout);
        if (dst != src && overlap(src, g.bytes * (uint64_t)src_pages, dst, g.bytes * (uint64_t)dst_pages)) BAD("dst overlaps src without being it");
        std::vector<bool> written((size_t)dst_pages);
        for (int i = 0; i < n; ++i) {
            if (from[i] < 0 || from[i] >= src_pages) BAD("from[%d] = %d is outside 0..%d", i, from[i], src_pages - 1);
            if (to[i] < 0 || to[i] >= dst_pages) BAD("to[%d] = %d is outside 0..%d", i, to[i], dst_pages - 1);
            if (tokens && (tokens[i] < 0 || tokens[i] > g.T)) BAD("tokens[%d] = %d is outside 0..page_tokens", i, tokens[i]);
            if (written[to[i]]) BAD("page %d is written twice", to[i]);
            written[to[i]] = true;
        }
        if (dst == src)
            for (int i = 0; i < n; ++i)
                if (from[i] < dst_pages && written[from[i]]) BAD("page %d is both read and written", from[i]);
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        for (int first = 0; first < n; first += COPY_PAGES) {
            CopyPages &c = t_copy;
            c.n = std::min(COPY_PAGES, n - first);
            for (int i = 0; i < c.n; ++i) { c.from[i] = from[first + i]; c.to[i] = to[first + i]; c.tokens[i] = tokens ? tokens[first + i] : g.T; }
            if ((st = launched(launch_copy(g, (const char *)src, (char *)dst, c, sm_quota, (cudaStream_t)stream))) != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_gather(const ebrl_pages_layout_t *layout, const void *pool, int32_t n_pages, int32_t n, const int32_t *table,
                                int64_t table_stride, const int32_t *len, void *const *planes, const int32_t *plane_rows, int64_t row_stride,
                                uint8_t *const *mask, int32_t sm_quota, void *stream)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_pool(layout, pool, n_pages, n, sm_quota);
        if (st != EBRL_OK || n == 0) return st;
        if ((st = check_seqs(layout, n, table, table_stride, len)) != EBRL_OK) return st;
        const Geometry g = geometry_of(*layout);
        const int64_t d = (int64_t)g.kvh * g.hd;
        if (row_stride == 0) row_stride = d;
        if (row_stride < d || row_stride * g.es % 16) BAD("row_stride must be at least %lld elements and a multiple of 16 bytes", (long long)d);
        if (!planes) BAD("planes is NULL");
        for (int i = 0; i < n; ++i) {
            if (len[i] == 0) continue;
            if (!planes[i] || ((uintptr_t)planes[i] & 15)) BAD("planes[%d] is NULL or not 16-byte aligned", i);
            if (plane_rows && plane_rows[i] < len[i]) BAD("plane_rows[%d] < len[%d]", i, i);
        }
        int sms = 0;
        if ((st = device_sms(sm_quota, &sms)) != EBRL_OK) return st;
        const Pages p = {(char *)const_cast<void *>(pool), n_pages, table, table_stride};
        for (int first = 0; first < n; first += GATHER_SEQS) {
            GatherSeqs &s = t_gather;
            s.n = std::min(GATHER_SEQS, n - first);
            s.first = first;
            s.items = 0;
            for (int i = 0; i < s.n; ++i) {
                const int k = first + i;
                s.s[i] = {planes[k], mask ? mask[k] : nullptr, s.items, len[k], plane_rows ? plane_rows[k] : len[k]};
                s.items += (len[k] + WORD - 1) / WORD;
            }
            if ((st = launched(launch_gather(g, p, row_stride * g.es, s, sm_quota, (cudaStream_t)stream))) != EBRL_OK) return st;
        }
        return EBRL_OK;
    });
}

}  // extern "C"
