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

// An item's pieces: up to 32 rows of `per` pieces each, as (row, piece) without a division.
struct Split {
    unsigned per, inv;
    __device__ __forceinline__ explicit Split(int n) : per(n), inv((1u << 18) / n + 1) {}
    __device__ __forceinline__ int row(unsigned c) const { return (int)((c * inv) >> 18); }       // (exact for c < 2048, n <= 64)
};
constexpr int BATCH = 4;         // reads that a thread has in flight before it writes

__global__ void append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ AppendSeqs s, int slices)
{
    const int row_bytes = a.g.kvh * a.g.hd * a.g.es, head_shift = 31 - __clz(a.g.hd * a.g.es), lane = threadIdx.x & 31;
    const long long items = (long long)s.items * 2 * slices;
    for (long long x = blockIdx.x; x < items; x += gridDim.x) {
        const int slice = (int)(x % slices), plane = (int)(x / slices) & 1, word = (int)(x / (2 * slices));
        const AppendSeqs::Seq q = s.s[find_seq(s.n, word, [&](int i) { return s.s[i].item; })];
        const int start = q.len - q.new_tokens, base = (start / WORD + word - q.item) * WORD;   // (the word's first token)
        const int t0 = max(start, base), t1 = min(q.len, base + WORD);
        const int page = a.p.table[q.tab * a.p.stride + (base >> a.g.t_shift)];
        const long long row0 = (long long)q.row - start;                               // packed row of token t: row0 + t
        const bool mine = base + lane >= t0 && base + lane < t1;
        const unsigned m = __ballot_sync(0xffffffffu, mine), v = __ballot_sync(0xffffffffu, mine && (!a.mask || a.mask[row0 + base + lane]));
        if ((unsigned)page >= (unsigned)a.p.n_pages) continue;
        char *at = a.p.pool + (size_t)page * a.g.bytes;
        const int slot0 = base & (a.g.T - 1);
        if (plane == 0 && slice == 0 && threadIdx.x == 0) {
            unsigned *w = reinterpret_cast<unsigned *>(at + a.g.mask) + slot0 / WORD;
            *w = m == 0xffffffffu ? v : ((*w & ~m) | v);
        }
        const int c0 = slice * SLICE, c1 = min(row_bytes, c0 + SLICE);
        const Split split((c1 - c0) / 16);
        const unsigned n = (unsigned)(t1 - t0) * split.per;
        const long long stride = plane ? a.v_stride : a.k_stride;
        const char *src = (plane ? a.v : a.k) + (row0 + t0) * stride + c0;
        char *dst = at + a.g.at(a.layer, plane, 0) + ((size_t)(slot0 + t0 - base) << head_shift);
        for (unsigned c = threadIdx.x; c < n; c += BATCH * blockDim.x) {
            uint4 x4[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const unsigned k = c + i * blockDim.x;
                x4[i] = make_uint4(0, 0, 0, 0);
                const int r = split.row(k);
                if (k < n && (v >> (r + t0 - base)) & 1) x4[i] = read16(src + r * stride + (k - r * split.per) * 16);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const unsigned k = c + i * blockDim.x;
                const int r = split.row(k), col = c0 + (int)(k - r * split.per) * 16, h = col >> head_shift;
                if (k < n) write16(dst + (size_t)h * a.g.head + ((size_t)r << head_shift) + (col - (h << head_shift)), x4[i]);
            }
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
    const int row_bytes = g.kvh * g.hd * g.es, head_shift = 31 - __clz(g.hd * g.es), planes = g.layers * 2;
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
        const int c0 = slice * SLICE, c1 = min(row_bytes, c0 + SLICE);
        const Split split((c1 - c0) / 16);
        const unsigned n = (unsigned)(t1 - base) * split.per;
        const char *src = at + (size_t)plane * g.kvh * g.head + ((size_t)slot0 << head_shift);
        char *dst = (char *)q.planes + ((size_t)plane * q.plane_rows + base) * row_stride + c0;
        for (unsigned c = threadIdx.x; c < n; c += BATCH * blockDim.x) {
            uint4 x4[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const unsigned k = c + i * blockDim.x;
                x4[i] = make_uint4(0, 0, 0, 0);
                const int r = split.row(k), col = c0 + (int)(k - r * split.per) * 16, h = col >> head_shift;
                if (k < n && (see >> r) & 1) x4[i] = read16(src + (size_t)h * g.head + ((size_t)r << head_shift) + (col - (h << head_shift)));
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const unsigned k = c + i * blockDim.x;
                const int r = split.row(k);
                if (k < n) write16(dst + (size_t)r * row_stride + (k - r * split.per) * 16, x4[i]);
            }
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
