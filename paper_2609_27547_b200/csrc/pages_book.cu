// Host-only: the book of a paged cache (include/ebrl_pages.h): which pages belong to which sequence, what forks share, and the moves
// that extending a shared page and compaction ask for.  No device code.
//
// A page's count says how many sequences name it.  Free pages are a bitmap: the lowest is found from the lowest word that may hold
// one, so handing out and taking back a page cost O(1) but for the words that are skipped, each skipped once per time it fills up.
#include "../../include/ebrl_pages.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <new>
#include <vector>

struct ebrl_pages_book {
    struct Seq { int32_t len = 0; std::vector<int32_t> pages; };
    int32_t n_pages = 0, page_tokens = 0, used = 0;
    std::vector<Seq> seqs;
    std::vector<int32_t> count;        // sequences that name a page
    std::vector<uint64_t> free_bits;   // bit p % 64 of word p / 64: page p is free
    size_t low = 0;                    // no word below holds a free page

    int32_t pages_for(int32_t len) const { return (int32_t)(((int64_t)len + page_tokens - 1) / page_tokens); }
    int32_t take()
    {
        while (!free_bits[low]) ++low;
        const int32_t p = (int32_t)(low * 64 + __builtin_ctzll(free_bits[low]));
        free_bits[low] &= free_bits[low] - 1;
        count[p] = 1;
        ++used;
        return p;
    }
    void drop(int32_t p)
    {
        if (--count[p]) return;
        free_bits[p / 64] |= 1ull << (p % 64);
        low = std::min(low, (size_t)p / 64);
        --used;
    }
};

namespace ebrl {
namespace pg {
char *error_text();            // of this thread, 256 bytes (shared with the operators)
}
}

namespace {

using Book = ebrl_pages_book;

ebrl_status_t fail(ebrl_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(ebrl::pg::error_text(), 256, fmt, ap);
    va_end(ap);
    return st;
}

#define BAD(...) return fail(EBRL_ERR_INVALID_ARG, __VA_ARGS__)

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

// n sequences of a book, each named once where `once`.
ebrl_status_t check_seqs(const Book *b, int32_t n, const int32_t *seqs, bool once)
{
    if (!b) BAD("the book is NULL");
    if (n < 0) BAD("n must not be negative");
    if (n && !seqs) BAD("the sequences are NULL");
    std::vector<bool> seen(once ? b->seqs.size() : 0);
    for (int i = 0; i < n; ++i) {
        if (seqs[i] < 0 || (size_t)seqs[i] >= b->seqs.size()) BAD("there is no sequence %d", seqs[i]);
        if (once) {
            if (seen[seqs[i]]) BAD("sequence %d is named twice", seqs[i]);
            seen[seqs[i]] = true;
        }
    }
    return EBRL_OK;
}

}  // namespace

extern "C" {

ebrl_status_t ebrl_pages_book_create(int32_t n_pages, int32_t page_tokens, int32_t max_sequences, ebrl_pages_book_t *out)
{
    return guarded([&]() -> ebrl_status_t {
        if (!out) BAD("out is NULL");
        *out = nullptr;
        if (n_pages < 0 || max_sequences < 0) BAD("n_pages and max_sequences must not be negative");
        if (page_tokens < 1) BAD("page_tokens must be positive");
        Book *b = new Book;
        try {
            b->n_pages = n_pages;
            b->page_tokens = page_tokens;
            b->seqs.resize((size_t)max_sequences);
            b->count.assign((size_t)n_pages, 0);
            b->free_bits.assign((size_t)n_pages / 64 + 1, 0);
            for (int32_t p = 0; p < n_pages; ++p) b->free_bits[p / 64] |= 1ull << (p % 64);
        } catch (...) {
            delete b;
            throw;
        }
        *out = b;
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_book_clone(ebrl_pages_book_t book, ebrl_pages_book_t *out)
{
    return guarded([&]() -> ebrl_status_t {
        if (!out) BAD("out is NULL");
        *out = nullptr;
        if (!book) BAD("the book is NULL");
        *out = new Book(*book);
        return EBRL_OK;
    });
}

void ebrl_pages_book_destroy(ebrl_pages_book_t book) { delete book; }

ebrl_status_t ebrl_pages_book_extend(ebrl_pages_book_t b, int32_t n, const int32_t *seqs, const int32_t *len, int32_t *from, int32_t *to, int32_t *tokens,
                                     int32_t *n_moves)
{
    return guarded([&]() -> ebrl_status_t {
        const ebrl_status_t st = check_seqs(b, n, seqs, true);
        if (st != EBRL_OK) return st;
        if (!n_moves || (n && (!len || !from || !to || !tokens))) BAD("len, n_moves or the arrays of moves are NULL");
        // What it takes.  Of k sequences of the call that share a page and write to it, all but the last one that names it need a copy.
        int64_t need = 0;
        std::vector<int32_t> leaving;   // (pages in the order of the call, to be counted)
        for (int i = 0; i < n; ++i) {
            const Book::Seq &s = b->seqs[seqs[i]];
            if (len[i] < s.len) BAD("sequence %d is %d tokens long, which is more than %d", seqs[i], s.len, len[i]);
            need += b->pages_for(len[i]) - (int32_t)s.pages.size();
            if (len[i] > s.len && s.len % b->page_tokens && b->count[s.pages.back()] > 1) leaving.push_back(s.pages.back());
        }
        std::sort(leaving.begin(), leaving.end());
        for (size_t i = 0, j; i < leaving.size(); i = j) {
            for (j = i; j < leaving.size() && leaving[j] == leaving[i];) ++j;
            need += std::min<int64_t>((int64_t)(j - i), b->count[leaving[i]] - 1);
        }
        if (need > b->n_pages - b->used) return fail(EBRL_ERR_NOMEM, "%lld pages are needed, %d are free", (long long)need, b->n_pages - b->used);
        for (int i = 0; i < n; ++i) b->seqs[seqs[i]].pages.reserve((size_t)b->pages_for(len[i]));   // (nothing fails from here on)
        int32_t k = 0;
        for (int i = 0; i < n; ++i) {
            Book::Seq &s = b->seqs[seqs[i]];
            const int32_t part = s.len % b->page_tokens;
            if (len[i] > s.len && part && b->count[s.pages.back()] > 1) {
                const int32_t p = b->take();
                from[k] = s.pages.back(); to[k] = p; tokens[k] = part;
                ++k;
                b->drop(s.pages.back());
                s.pages.back() = p;
            }
            while ((int32_t)s.pages.size() < b->pages_for(len[i])) s.pages.push_back(b->take());
            s.len = len[i];
        }
        *n_moves = k;
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_book_fork(ebrl_pages_book_t b, int32_t n, const int32_t *from, const int32_t *to)
{
    return guarded([&]() -> ebrl_status_t {
        ebrl_status_t st = check_seqs(b, n, from, false);
        if (st == EBRL_OK) st = check_seqs(b, n, to, true);
        if (st != EBRL_OK) return st;
        std::vector<bool> read(b->seqs.size());
        for (int i = 0; i < n; ++i) read[from[i]] = true;
        for (int i = 0; i < n; ++i) {
            if (b->seqs[to[i]].len || !b->seqs[to[i]].pages.empty()) BAD("sequence %d is not empty", to[i]);
            if (read[to[i]]) BAD("sequence %d is both forked from and to", to[i]);
        }
        std::vector<std::vector<int32_t>> pages((size_t)n);
        for (int i = 0; i < n; ++i) pages[i] = b->seqs[from[i]].pages;   // (nothing fails from here on)
        for (int i = 0; i < n; ++i) {
            for (int32_t p : pages[i]) ++b->count[p];
            b->seqs[to[i]].len = b->seqs[from[i]].len;
            b->seqs[to[i]].pages.swap(pages[i]);
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_book_shorten(ebrl_pages_book_t b, int32_t n, const int32_t *seqs, const int32_t *len)
{
    return guarded([&]() -> ebrl_status_t {
        const ebrl_status_t st = check_seqs(b, n, seqs, true);
        if (st != EBRL_OK) return st;
        if (n && !len) BAD("len is NULL");
        for (int i = 0; i < n; ++i)
            if (len[i] < 0 || len[i] > b->seqs[seqs[i]].len) BAD("sequence %d is %d tokens long and cannot be cut to %d", seqs[i], b->seqs[seqs[i]].len, len[i]);
        for (int i = 0; i < n; ++i) {
            Book::Seq &s = b->seqs[seqs[i]];
            while ((int32_t)s.pages.size() > b->pages_for(len[i])) {
                b->drop(s.pages.back());
                s.pages.pop_back();
            }
            s.len = len[i];
        }
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_book_compact(ebrl_pages_book_t b, int32_t room, int32_t *from, int32_t *to, int32_t *tokens, int32_t *n_moves)
{
    return guarded([&]() -> ebrl_status_t {
        if (!b) BAD("the book is NULL");
        if (room < 0) BAD("room must not be negative");
        if (!n_moves || (room && (!from || !to || !tokens))) BAD("n_moves or the arrays of moves are NULL");
        std::vector<int32_t> there((size_t)b->n_pages, -1), fill((size_t)b->n_pages, 0);   // where a page goes; tokens of it in use
        for (const Book::Seq &s : b->seqs)
            for (size_t j = 0; j < s.pages.size(); ++j)
                fill[s.pages[j]] = std::max(fill[s.pages[j]], (int32_t)std::min<int64_t>(b->page_tokens, s.len - (int64_t)j * b->page_tokens));
        int32_t k = 0;
        for (int32_t high = b->n_pages - 1; k < room && high >= b->used; --high) {
            if (!b->count[high]) continue;
            const int32_t sharers = b->count[high], p = b->take();
            b->count[p] = sharers;
            from[k] = high; to[k] = p; tokens[k] = fill[high];
            ++k;
            there[high] = p;
            b->count[high] = 1;
            b->drop(high);
        }
        if (k)
            for (Book::Seq &s : b->seqs)
                for (int32_t &p : s.pages)
                    if (there[p] >= 0) p = there[p];
        *n_moves = k;
        return EBRL_OK;
    });
}

ebrl_status_t ebrl_pages_book_table(ebrl_pages_book_t b, int32_t n, const int32_t *seqs, int32_t *out, int64_t stride)
{
    return guarded([&]() -> ebrl_status_t {
        const ebrl_status_t st = check_seqs(b, n, seqs, false);
        if (st != EBRL_OK) return st;
        if (n && ((!out && stride) || stride < 0)) BAD("out is NULL or stride is negative");
        for (int i = 0; i < n; ++i)
            if ((int64_t)b->seqs[seqs[i]].pages.size() > stride) BAD("sequence %d has %d pages, the table's rows %lld entries", seqs[i], (int)b->seqs[seqs[i]].pages.size(), (long long)stride);
        for (int i = 0; i < n; ++i) {
            const std::vector<int32_t> &p = b->seqs[seqs[i]].pages;
            std::fill(std::copy(p.begin(), p.end(), out + i * stride), out + (i + 1) * stride, -1);
        }
        return EBRL_OK;
    });
}

int32_t ebrl_pages_book_len(ebrl_pages_book_t b, int32_t seq) { return b && seq >= 0 && (size_t)seq < b->seqs.size() ? b->seqs[seq].len : -1; }

int32_t ebrl_pages_book_used(ebrl_pages_book_t b) { return b ? b->used : -1; }

}  // extern "C"
