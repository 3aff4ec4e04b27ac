// Internal declarations of the operators on paged caches (include/ebrl_pages.h).
#pragma once

#include "../../include/ebrl_pages.h"
#include "actgen_internal.h"
#include "pages_span.h"

#include <atomic>

namespace ebrl {
namespace pg {

constexpr int WORD = 32;          // tokens of a mask word; what the kernels look a page up for
constexpr int SEQS = 1024;        // sequences per launch: what is known of them travels as kernel parameters (up to 28 KB)

char *error_text();               // of this thread, 256 bytes

// What the kernels need to find a token.
struct Geometry {
    int layers, kvh, hd, T, es;             // T = tokens of a page, es = bytes of an element
    int t_shift;                            // T = 1 << t_shift
    size_t head, mask, bytes;               // bytes of one head's [T][hd]; offset of the mask words; bytes of a page
    __host__ __device__ size_t at(int layer, int p, int h) const { return (((size_t)layer * 2 + p) * kvh + h) * head; }
};
Geometry geometry_of(const ebrl_pages_layout_t &l);

// Where a sequence's pages are.
struct Pages {
    char *pool;
    int n_pages;
    const int *table;
    long long stride;
};

// ---- append, copy, gather (pages_cache.cu) ----

struct AppendSeqs {
    int n, items;                            // an item: a mask word that new tokens fall into
    struct Seq { int item, row, new_tokens, len, tab; } s[SEQS];   // first item; first packed row; row of the table
};
struct AppendArgs {
    Geometry g;
    Pages p;
    int layer;
    const char *k, *v;
    long long k_stride, v_stride;            // bytes
    const uint8_t *mask;
};
cudaError_t launch_append(const AppendArgs &a, const AppendSeqs &s, int quota, cudaStream_t st);

constexpr int COPY_PAGES = 2048;
struct CopyPages { int n, from[COPY_PAGES], to[COPY_PAGES], tokens[COPY_PAGES]; };
cudaError_t launch_copy(const Geometry &g, const char *src, char *dst, const CopyPages &c, int quota, cudaStream_t st);

constexpr int GATHER_SEQS = 512;  // (32 bytes each)
struct GatherSeqs {
    int n, items;                            // an item: 32 tokens
    struct Seq { void *planes; uint8_t *mask; int item, len, plane_rows; } s[GATHER_SEQS];
    int first;                               // row of the table of sequence 0
};
cudaError_t launch_gather(const Geometry &g, const Pages &p, long long row_stride, const GatherSeqs &s, int quota, cudaStream_t st);

// ---- attend ----

struct AttendSeq {
    int item, row, m, len, tab;                        // first item; first packed query; queries; length; row of the table
    int part;                                          // first (query, piece) pair of the partial results; -1: not cut
};
struct AttendSeqs {
    int n, items;
    AttendSeq s[SEQS];
};
struct AttendArgs {
    Geometry g;
    Pages p;
    int layer, heads, G;                               // G = heads / kv heads
    const char *q;
    char *out;
    long long q_stride, o_stride;                      // elements
    float *lse;
    float scale, up;                                   // up: what moves a score by 8 in units of log 2; the largest number where there is none (a subnormal scale)
    int causal, window;
    int split;                                         // tokens of a piece; 0: not cut
    int team;                                          // warps that share an item
    unsigned long long limit_ns;                       // bound of a wait
    int test_drop_copies;                              // tests of the give-up path: the copying warp issues nothing
    float *part_o, *part_ml;                           // [pair][heads][hd] sums, [pair][heads][2] (reference, NaN where there is no result; sum of weights)
};

// A launch that may begin as soon as the CTAs of the one before it have begun (beside: they share nothing but what both read), and ends after it: the kernels
// of one call take turns at the SMs without a gap.
struct Beside {
    const bool before = pdl_enabled();
    explicit Beside(bool on) { pdl_set(on); }
    ~Beside() { pdl_set(before); }
    Beside(const Beside &) = delete;
    Beside &operator=(const Beside &) = delete;
};

int attend_rows(int rows);                             // query rows of an item
int attend_warps(int hd, bool f32, int rows);          // warps that an SM holds
cudaError_t launch_attend(const AttendArgs &a, const AttendSeqs &s, bool f32, int rows, int quota, bool beside, cudaStream_t st);
cudaError_t launch_attend_join(const AttendArgs &a, const AttendSeqs &s, bool f32, int quota, int sms, cudaStream_t st);

// The same for many query rows, bf16 (pages_chunk.cu): an item is a CTA of 256 of them, or one of 128, of which an SM holds two.
constexpr int CHUNK_ROWS = 256, SMALL_CHUNK_ROWS = 128;
bool chunk_supported(const Geometry &g, int n_pages, float scale);
cudaError_t launch_chunk(const AttendArgs &a, const AttendSeqs &s, int rows, int quota, int sms, bool beside, cudaStream_t st);

// Whether a bounded wait ran out on the current device since the last call (waits for the device).
cudaError_t take_status(int *status);

#ifdef __CUDACC__
// The last of n (at most 1024) whose first item, at(i), is not above x; by all lanes of a warp.  Two looks at 32 of them at once: a search by halves
// meets a miss of the constant cache, where kernel parameters are read, at every step (a microsecond each at a launch's start).
template <typename F> __device__ __forceinline__ int find_seq(int n, int x, F at)
{
    const int lane = threadIdx.x & 31, step = (n + 31) / 32;
    int i = lane * step, base = (__popc(__ballot_sync(0xffffffffu, i < n && at(i) <= x)) - 1) * step;
    if (step > 1) {
        i = base + lane;
        base += __popc(__ballot_sync(0xffffffffu, lane < step && i < n && at(i) <= x)) - 1;
    }
    return base;
}
#endif

}  // namespace pg
}  // namespace ebrl
