// Driver for the token ranges of attend (pages_span.h) built with UndefinedBehaviorSanitizer, which sees a signed sum that wraps: lengths, numbers of queries, windows
// and pieces over everything that a call may say, against the definition in 64 bits.  tests/test_pages_limits_host.py compiles it.
#include "../paper_2609_27547_b200/csrc/pages_span.h"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

using namespace ebrl::pg;

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "CHECK failed at line %d: %s (len %d m %d G %d window %d split %d longest %d)\n", __LINE__, #cond, len, m, G, window, split, longest); std::exit(2); } } while (0)

int main()
{
    const int top = 0x7fffffff, lens[] = {0, 1, 10, 127, 128, 1000, 65537, (1 << 30) - 1, 1 << 30}, gs[] = {1, 3, 128};
    const int windows[] = {0, 1, 10, 128, 1000000, 1 << 30, top - 1, top}, splits[] = {-1, 0, 128, 1024, 1 << 30, 2147483520};
    long long calls = 0;
    for (int len : lens) for (int G : gs) for (int window : windows) for (int split : splits) for (int more : {0, 5, 1 << 29}) {
        const int longest = std::min(1 << 30, len + more), most = top / 2 / G;
        for (int m : {1, 2, len, len + 1, len + 3, len + 300, most - 1, most}) {
            if (m < 1 || m > most) continue;
            const int w = bounded_window(window, longest), s = std::max(0, bounded_split(split, longest));
            CHECK(w >= 0 && (w == 0 || w == window) && (s == 0 || s == split));
            const int np = pieces_of(len, m, w, s), R = m * G;
            CHECK(np >= 1);
            for (int piece : {0, np / 2, np - 1}) for (int r0 : {0, R / 2 / 128 * 128, (R - 1) / 128 * 128}) {
                const int r1 = std::min(R - r0, 128) + r0;
                for (bool causal : {true, false}) {
                    if (!causal && window) continue;
                    const Span got = seen_by(len, m, G, r0, r1, causal, w, s, piece);
                    // by the definition: a row's tokens, those of all rows, of those the piece's part (pieces begin where the sequence's first query's window does)
                    const long long pos0 = (long long)len - m + r0 / G, pos1 = (long long)len - m + (r1 - 1) / G;
                    long long lo = 0, hi = len;
                    if (causal) hi = std::min<long long>(hi, pos1 + 1);
                    if (window) lo = std::max<long long>(0, pos0 - window + 1);
                    const long long start = window ? std::max<long long>(0, (long long)len - m - window + 1) / 128 * 128 : 0;
                    if (s) {
                        lo = std::max(lo, start + (long long)piece * s);
                        hi = std::min(hi, start + (long long)(piece + 1) * s);
                    }
                    CHECK(first_token(len, m, w) == start);
                    CHECK((lo >= hi && got.lo >= got.hi) || (got.lo == lo && got.hi == hi));
                    // the limits of single rows
                    for (int r : {r0, r1 - 1}) {
                        const int at = len - m + r / G;
                        const long long from = window ? (long long)at + 1 - window : -1;
                        CHECK(std::max<long long>(0, first_seen(at, w)) == std::max<long long>(0, from));
                    }
                    ++calls;
                }
            }
        }
    }
    std::printf("pages span driver: ok, %lld ranges\n", calls);
    return 0;
}
