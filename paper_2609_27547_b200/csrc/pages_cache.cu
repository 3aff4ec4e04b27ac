// Moving tokens in and out of pages (include/ebrl_pages.h): append, copy, gather.
//
// Bound: HBM, one read and one write of each element.  All three move 16-byte pieces; the head-major page meets token-major rows in
// append and gather, where a run of one head (64 - 512 bytes) is contiguous on both sides, so no transpose through shared
// memory is needed.  An item is the part of one mask word's 32 tokens that fits SLICE columns of one plane: the page is looked up once, and
// whoever takes slice 0 of plane 0 owns the word's bits.
#include "pages_internal.h"

namespace ebrl {
namespace pg {

constexpr int THREADS = 256, QUOTA_THREADS = 1024;   // under a quota one CTA has an SM to itself
constexpr int SLICE = 1024;                          // bytes of a token's row that an item moves

__device__ __forceinline__ uint4 read16(const char *p) { return __ldcs(reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ void write16(char *p, uint4 v) { *reinterpret_cast<uint4 *>(p) = v; }

__global__ void append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ AppendSeqs s, int slices)
{
    const int row_bytes = a.g.kvh * a.g.hd * a.g.es, head_bytes = a.g.hd * a.g.es;
    const long long items = (long long)s.items * 2 * slices;
    for (long long x = blockIdx.x; x < items; x += gridDim.x) {
        const int slice = (int)(x % slices), plane = (int)(x / slices) & 1, word = (int)(x / (2 * slices));
        const AppendSeqs::Seq q = s.s[find_seq(s.n, word, [&](int i) { return s.s[i].item; })];
        const int start = q.len - q.new_tokens, base = (start / WORD + word - q.item) * WORD;   // (the word's first token)
        const int t0 = max(start, base), t1 = min(q.len, base + WORD);
        const int page = a.p.table[q.tab * a.p.stride + (base >> a.g.t_shift)];
        if ((unsigned)page >= (unsigned)a.p.n_pages) continue;
        char *at = a.p.pool + (size_t)page * a.g.bytes;
        const long long row0 = (long long)q.row - start;                            // packed row of token t: row0 + t
        const int slot0 = base & (a.g.T - 1);
        if (plane == 0 && slice == 0 && threadIdx.x < 32) {
            const int t = base + threadIdx.x;
            const bool mine = t >= t0 && t < t1, see = mine && (!a.mask || a.mask[row0 + t]);
            const unsigned m = __ballot_sync(0xffffffffu, mine), v = __ballot_sync(0xffffffffu, see);
            if (threadIdx.x == 0) {
                unsigned *w = reinterpret_cast<unsigned *>(at + a.g.mask) + slot0 / WORD;
                *w = m == 0xffffffffu ? v : ((*w & ~m) | v);
            }
        }
        const int c0 = slice * SLICE, c1 = min(row_bytes, c0 + SLICE), per = (c1 - c0) / 16, n = (t1 - t0) * per;
        const char *src = plane ? a.v : a.k;
        const long long stride = plane ? a.v_stride : a.k_stride;
        char *dst = at + a.g.at(a.layer, plane, 0);
#pragma unroll 4
        for (int c = threadIdx.x; c < n; c += blockDim.x) {
            const int r = c / per, col = c0 + (c - r * per) * 16, t = t0 + r;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (!a.mask || a.mask[row0 + t]) v = read16(src + (row0 + t) * stride + col);
            const int h = col / head_bytes;
            write16(dst + (size_t)h * a.g.head + (size_t)(slot0 + t - base) * head_bytes + (col - h * head_bytes), v);
        }
    }
}

// The first `tokens` rows of every head of a page, in chunks of the same number of pieces.
__global__ void copy_kernel(const __grid_constant__ Geometry g, const char *src, char *dst, const __grid_constant__ CopyPages c, int chunks, int chunk)
{
    const int head_bytes = g.hd * g.es;
    const unsigned heads = (unsigned)(g.layers * 2 * g.kvh);
    const long long items = (long long)c.n * chunks;
    for (long long x = blockIdx.x; x < items; x += gridDim.x) {
        const int i = (int)(x / chunks), k = c.tokens[i];
        const unsigned per = (unsigned)(k * head_bytes / 16);                          // pieces of a head
        const unsigned long long all = (unsigned long long)heads * per, first = (unsigned long long)(x % chunks) * chunk;
        const char *a = src + (size_t)c.from[i] * g.bytes;
        char *b = dst + (size_t)c.to[i] * g.bytes;
        if (first == 0 && threadIdx.x < (k + WORD - 1) / WORD) {
            const unsigned w = reinterpret_cast<const unsigned *>(a + g.mask)[threadIdx.x];
            unsigned *to = reinterpret_cast<unsigned *>(b + g.mask) + threadIdx.x;
            const int left = k - (int)threadIdx.x * WORD;
            const unsigned m = left >= WORD ? 0xffffffffu : (1u << left) - 1;
            *to = m == 0xffffffffu ? w : ((*to & ~m) | (w & m));
        }
        if (first >= all) continue;
        const unsigned n = (unsigned)min((unsigned long long)chunk, all - first);
        // (head, piece in it) of the chunk's first piece; the quotients of the others are small numbers'
        const unsigned h0 = (unsigned)(first / per), o0 = (unsigned)(first - (unsigned long long)h0 * per);
#pragma unroll 8
        for (unsigned u = threadIdx.x; u < n; u += blockDim.x) {
            const unsigned h = (o0 + u) / per, o = o0 + u - h * per;
            const size_t off = (size_t)(h0 + h) * g.head + (size_t)o * 16;
            write16(b + off, read16(a + off));
        }
    }
}

__global__ void gather_kernel(const __grid_constant__ Geometry g, const __grid_constant__ Pages p, long long row_stride, const __grid_constant__ GatherSeqs s, int slices)
{
    const int row_bytes = g.kvh * g.hd * g.es, head_bytes = g.hd * g.es, planes = g.layers * 2;
    const long long items = (long long)s.items * planes * slices;
    for (long long x = blockIdx.x; x < items; x += gridDim.x) {
        const int slice = (int)(x % slices), plane = (int)(x / slices % planes), word = (int)(x / ((long long)slices * planes));
        const int i = find_seq(s.n, word, [&](int k) { return s.s[k].item; });
        const GatherSeqs::Seq q = s.s[i];
        const int base = (word - q.item) * WORD, t1 = min(q.len, base + WORD);
        const int page = p.table[(s.first + i) * p.stride + (base >> g.t_shift)], slot0 = base & (g.T - 1);
        const bool there = (unsigned)page < (unsigned)p.n_pages;
        const char *at = p.pool + (there ? (size_t)page * g.bytes : 0);
        const unsigned see = there ? reinterpret_cast<const unsigned *>(at + g.mask)[slot0 / WORD] : 0u;
        if (plane == 0 && slice == 0 && q.mask && threadIdx.x < t1 - base) q.mask[base + threadIdx.x] = (see >> threadIdx.x) & 1;
        const int c0 = slice * SLICE, c1 = min(row_bytes, c0 + SLICE), per = (c1 - c0) / 16, n = (t1 - base) * per;
        const char *src = at + (size_t)plane * g.kvh * g.head;
        char *dst = (char *)q.planes + ((size_t)plane * q.plane_rows + base) * row_stride;
#pragma unroll 4
        for (int c = threadIdx.x; c < n; c += blockDim.x) {
            const int r = c / per, col = c0 + (c - r * per) * 16, h = col / head_bytes;
            uint4 v = make_uint4(0, 0, 0, 0);
            if ((see >> r) & 1) v = read16(src + (size_t)h * g.head + (size_t)(slot0 + r) * head_bytes + (col - h * head_bytes));
            write16(dst + (size_t)r * row_stride + col, v);
        }
    }
}

static int grid_for(long long items, int quota) { return (int)(quota ? (items < quota ? items : quota) : (items < 1 << 30 ? items : 1 << 30)); }

cudaError_t launch_append(const AppendArgs &a, const AppendSeqs &s, int quota, cudaStream_t st)
{
    if (s.items == 0) return cudaSuccess;
    const int slices = (a.g.kvh * a.g.hd * a.g.es + SLICE - 1) / SLICE;
    append_kernel<<<grid_for((long long)s.items * 2 * slices, quota), quota ? QUOTA_THREADS : THREADS, 0, st>>>(a, s, slices);
    return cudaGetLastError();
}

cudaError_t launch_copy(const Geometry &g, const char *src, char *dst, const CopyPages &c, int quota, cudaStream_t st)
{
    int most = 0;
    for (int i = 0; i < c.n; ++i) most = c.tokens[i] > most ? c.tokens[i] : most;
    if (c.n == 0 || most == 0) return cudaSuccess;
    const long long all = (long long)g.layers * 2 * g.kvh * (most * g.hd * g.es / 16);
    const int chunk = 2048;                                       // 32 KB: eight pieces for each of 256 threads
    const int chunks = (int)((all + chunk - 1) / chunk);
    copy_kernel<<<grid_for((long long)c.n * chunks, quota), quota ? QUOTA_THREADS : THREADS, 0, st>>>(g, src, dst, c, chunks, chunk);
    return cudaGetLastError();
}

cudaError_t launch_gather(const Geometry &g, const Pages &p, long long row_stride, const GatherSeqs &s, int quota, cudaStream_t st)
{
    if (s.items == 0) return cudaSuccess;
    const int slices = (g.kvh * g.hd * g.es + SLICE - 1) / SLICE;
    gather_kernel<<<grid_for((long long)s.items * g.layers * 2 * slices, quota), quota ? QUOTA_THREADS : THREADS, 0, st>>>(g, p, row_stride, s, slices);
    return cudaGetLastError();
}

}  // namespace pg
}  // namespace ebrl
