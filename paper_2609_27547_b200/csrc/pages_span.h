// Which tokens of a sequence the queries of attend see (include/ebrl_pages.h): host and device arithmetic, in 32 bits.  Plain C++, so that tests build it by itself.
//
// A sequence has len <= 2^30 tokens and m < 2^30 queries; query j stands at position len - m + j, which is negative where there are more queries than tokens.
// With a window below len and pieces below len, as bounded_window and bounded_split leave them, no sum here passes 2^31 either way.
#pragma once

#ifdef __CUDACC__
#define EBRL_HD __host__ __device__ __forceinline__
#else
#define EBRL_HD inline
#endif

namespace ebrl {
namespace pg {

// A window that is not shorter than the longest sequence of the call limits nothing: no query stands behind that sequence's last token.
inline int bounded_window(int window, int longest) { return window < longest ? window : 0; }
// Pieces that are not shorter than it cut nothing.
inline int bounded_split(int split_tokens, int longest) { return split_tokens > 0 && split_tokens >= longest ? -1 : split_tokens; }

// The first token that a query at position `at` sees.
EBRL_HD int first_seen(int at, int window) { return window ? at + 1 - window : -0x7fffffff; }

// The first token that a query of the sequence sees (rounded down to 128): where its first piece begins.
EBRL_HD int first_token(int len, int m, int window)
{
    const int lo = window ? len - m + 1 - window : 0;
    return lo > 0 ? lo / 128 * 128 : 0;
}
EBRL_HD int pieces_of(int len, int m, int window, int split)
{
    const int n = len - first_token(len, m, window);
    return split && n > split ? (int)(((long long)n + split - 1) / split) : 1;
}

// The tokens lo .. hi of one piece that some of the rows r0 .. r1 - 1 sees (row = query * G + member of the head group); none where hi <= lo.
struct Span { int lo, hi; };
EBRL_HD Span seen_by(int len, int m, int G, int r0, int r1, bool causal, int window, int split, int piece)
{
    const int first = len - m;                                        // position of query 0
    Span s = {first_token(len, m, window), len};
    if (split) {
        s.lo += piece * split;
        if (s.lo + split < s.hi) s.hi = s.lo + split;
    }
    if (causal) {
        const int end = first + (r1 - 1) / G + 1;
        if (end < s.hi) s.hi = end;
        if (window) {
            const int from = first_seen(first + r0 / G, window);
            if (from > s.lo) s.lo = from;
        }
    }
    return s;
}

}  // namespace pg
}  // namespace ebrl
