// Driver for the book of a paged cache (host only) built with AddressSanitizer and UndefinedBehaviorSanitizer: a long run of random calls, valid and
// not; after each, every page's count is what the tables say.  tests/test_pages_sanitizers.py compiles it with the source as plain C++.
#include "../include/ebrl_pages.h"

#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>

namespace ebrl { namespace pg { char *error_text() { static char text[256]; return text; } } }

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "CHECK failed at line %d: %s\n", __LINE__, #cond); std::exit(2); } } while (0)

int main()
{
    unsigned seed = 1;
    auto rnd = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (unsigned)n); };
    for (int round = 0; round < 10; ++round) {
        const int T = 32, n_pages = 1 + rnd(200), n_seqs = 1 + rnd(12);
        ebrl_pages_book_t book = nullptr;
        CHECK(ebrl_pages_book_create(n_pages, T, n_seqs, &book) == EBRL_OK);
        for (int step = 0; step < 150; ++step) {
            const int k = rnd(4);
            std::vector<int32_t> a(k), b(k), from(n_pages + k), to(n_pages + k), tokens(n_pages + k);
            int32_t moves = -1;
            for (int i = 0; i < k; ++i) { a[i] = rnd(n_seqs + 1) - rnd(2); b[i] = rnd(40) == 0 ? -1 : rnd(500); }
            switch (rnd(5)) {
            case 0: case 1:
                for (int i = 0; i < k; ++i) b[i] = ebrl_pages_book_len(book, a[i]) + rnd(100) - (rnd(20) == 0);
                ebrl_pages_book_extend(book, k, a.data(), b.data(), from.data(), to.data(), tokens.data(), &moves);
                break;
            case 2: for (int i = 0; i < k; ++i) b[i] = rnd(n_seqs); ebrl_pages_book_fork(book, k, a.data(), b.data()); break;
            case 3: for (int i = 0; i < k; ++i) b[i] = rnd(2) ? 0 : rnd(300); ebrl_pages_book_shorten(book, k, a.data(), b.data()); break;
            default: ebrl_pages_book_compact(book, rnd(n_pages + 1), from.data(), to.data(), tokens.data(), &moves);
            }
            std::set<int32_t> pages;
            for (int s = 0; s < n_seqs; ++s) {
                std::vector<int32_t> row(n_pages + 1);
                const int32_t seq = s;
                CHECK(ebrl_pages_book_table(book, 1, &seq, row.data(), n_pages + 1) == EBRL_OK);
                const int32_t len = ebrl_pages_book_len(book, s);
                for (int j = 0; j <= n_pages; ++j) {
                    CHECK((row[j] >= 0) == (j * T < len));
                    if (row[j] >= 0) { CHECK(row[j] < n_pages); pages.insert(row[j]); }
                }
            }
            CHECK((int)pages.size() == ebrl_pages_book_used(book));
        }
        ebrl_pages_book_t other = nullptr;
        CHECK(ebrl_pages_book_clone(book, &other) == EBRL_OK);
        ebrl_pages_book_destroy(book);
        ebrl_pages_book_destroy(other);
    }
    std::printf("pages book driver: ok\n");
    return 0;
}
