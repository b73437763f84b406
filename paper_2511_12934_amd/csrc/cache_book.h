// Which pages of the user cache belong to which sequence: host arithmetic only (include/aif_cache.h says what it means).
// What has to happen to the pages' contents is handed to the callers' functions.  Callers check numbers and room first;
// after init and set_pool nothing here allocates.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <vector>

namespace aif {

class CacheBook {
public:
    int32_t max_seqs = 0, max_len = 0, page_len = 1, pages_per_seq = 0;
    int32_t n_pages = 0, n_free = 0;

    void init(int32_t seqs, int32_t longest, int32_t rows_of_page, int32_t pages)
    {
        max_seqs = seqs;
        max_len = longest;
        page_len = rows_of_page;
        pages_per_seq = (int32_t)(((int64_t)longest + rows_of_page - 1) / rows_of_page);
        table_.assign((size_t)seqs * pages_per_seq, -1);
        len_.assign(seqs, 0);
        given_back_.reserve(seqs);
        set_pool(pages);
    }

    // The pool has n pages from now on; false, and nothing changed, where one in use lies beyond them.
    bool set_pool(int32_t n)
    {
        for (int32_t p = n; p < n_pages; ++p)
            if (refs_[p]) return false;
        std::vector<int32_t> refs((size_t)n, 0), moved((size_t)n, -1);
        std::vector<uint64_t> bits(((size_t)n + 63) / 64, 0);
        std::copy(refs_.begin(), refs_.begin() + std::min(n, n_pages), refs.begin());
        int32_t unused = 0;
        for (int32_t p = 0; p < n; ++p)
            if (!refs[p]) {
                bits[p / 64] |= 1ull << (p % 64);
                ++unused;
            }
        refs_.swap(refs);
        moved_.swap(moved);
        free_.swap(bits);
        hint_ = 0;
        n_pages = n;
        n_free = unused;
        return true;
    }

    int32_t len(int32_t seq) const { return len_[seq]; }
    int32_t pages(int32_t rows) const { return (int32_t)(((int64_t)rows + page_len - 1) / page_len); }
    int32_t page(int32_t seq, int32_t i) const { return table_[(size_t)seq * pages_per_seq + i]; }
    int32_t entry(int32_t seq, int32_t i) const { return (int32_t)((int64_t)seq * pages_per_seq + i); }

    // Pages that append(seq, rows) takes.
    int64_t append_needs(int32_t seq, int32_t rows) const
    {
        if (rows == 0) return 0;
        const int32_t have = len_[seq];
        return (int64_t)pages(have + rows) - pages(have) + (have % page_len && refs_[page(seq, have / page_len)] > 1);
    }
    // rows more rows, in runs of at most `most` that no page's and no multiple-of-most row of a page cuts:
    //   run(done, i, cow, row0, n): rows [done, done + n) are rows row0.. of page i of the sequence; cow >= 0: the page is a new
    //   one in the place of page cow, whose first row0 rows it has to get.
    // A page that several sequences hold when the call begins is copied by each that appends to it, also when the others of them do
    // so in the same call: nothing is written while another run reads it.  settle() ends the call.
    template <class F> void append(int32_t seq, int32_t rows, int32_t most, F &&run)
    {
        int32_t *pages_now = &table_[(size_t)seq * pages_per_seq];
        const int32_t have = len_[seq];
        for (int32_t done = 0; done < rows;) {
            const int32_t i = (have + done) / page_len, row0 = (have + done) % page_len;
            int32_t cow = -1;
            if (row0 == 0) {
                pages_now[i] = take();
            } else if (refs_[pages_now[i]] > 1) {
                cow = pages_now[i];
                given_back_.push_back(cow);
                pages_now[i] = take();
            }
            const int32_t n = std::min({most - row0 % most, page_len - row0, rows - done});
            run(done, i, cow, row0, n);
            done += n;
        }
        len_[seq] = have + rows;
    }
    void settle()
    {
        for (int32_t p : given_back_) drop(p);
        given_back_.clear();
    }

    // dst, which is empty, becomes src on the same pages.
    void fork(int32_t src, int32_t dst)
    {
        for (int32_t i = 0; i < pages(len_[src]); ++i) {
            const int32_t p = page(src, i);
            table_[(size_t)dst * pages_per_seq + i] = p;
            if (p >= 0) ++refs_[p];
        }
        len_[dst] = len_[src];
    }
    int64_t copy_needs(int32_t src) const
    {
        int64_t n = 0;
        for (int32_t i = 0; i < pages(len_[src]); ++i) n += page(src, i) >= 0;
        return n;
    }
    // ... on pages of its own: page(i, from, to), -1 for a dropped one.
    template <class F> void copy(int32_t src, int32_t dst, F &&each)
    {
        for (int32_t i = 0; i < pages(len_[src]); ++i) {
            const int32_t from = page(src, i), to = from >= 0 ? take() : -1;
            table_[(size_t)dst * pages_per_seq + i] = to;
            each(i, from, to);
        }
        len_[dst] = len_[src];
    }

    // The sequence's first rows stay; false, and nothing changed, where the last of them would lie in a dropped page.
    bool truncate(int32_t seq, int32_t rows)
    {
        if (rows % page_len && page(seq, rows / page_len) < 0) return false;
        for (int32_t i = pages(rows); i < pages(len_[seq]); ++i) drop(page(seq, i));
        len_[seq] = rows;
        return true;
    }

    // Drops the pages [lo, hi) behind the first sinks rows and before the last window rows; lo >= hi: none.
    void trim(int32_t seq, int32_t sinks, int32_t window, int32_t &lo, int32_t &hi)
    {
        lo = pages(sinks);
        hi = window < len_[seq] ? (len_[seq] - window) / page_len : 0;
        for (int32_t i = lo; i < hi; ++i) {
            drop(page(seq, i));
            table_[(size_t)seq * pages_per_seq + i] = -1;
        }
    }

    // Pages in use at n_pages - n_free and beyond go, in their order, to the free ones below, lowest first (as many of either):
    // move(from, to); then named(seq, i, to) for every table entry that changes.  out_of_place: their number beforehand.
    int64_t out_of_place() const
    {
        int64_t n = 0;
        for (int32_t p = n_pages - n_free; p < n_pages; ++p) n += refs_[p] > 0;
        return n;
    }
    template <class M, class N> void compact(M &&move, N &&named)
    {
        const int32_t used = n_pages - n_free;
        for (int32_t p = used; p < n_pages; ++p) {
            if (!refs_[p]) continue;
            const int32_t to = take();
            refs_[to] = refs_[p];
            refs_[p] = 1;
            drop(p);
            moved_[p] = to;
            move(p, to);
        }
        for (int32_t q = 0; q < max_seqs; ++q)
            for (int32_t i = 0; i < pages(len_[q]); ++i) {
                int32_t &p = table_[(size_t)q * pages_per_seq + i];
                if (p < used) continue;
                p = moved_[p];
                named(q, i, p);
            }
    }

private:
    // the lowest free page
    int32_t take()
    {
        while (!free_[hint_]) ++hint_;
        const int32_t p = (int32_t)(hint_ * 64) + __builtin_ctzll(free_[hint_]);
        free_[hint_] &= free_[hint_] - 1;
        refs_[p] = 1;
        --n_free;
        return p;
    }
    void drop(int32_t p)
    {
        if (p < 0 || --refs_[p]) return;
        free_[p / 64] |= 1ull << (p % 64);
        hint_ = std::min(hint_, (size_t)p / 64);
        ++n_free;
    }

    std::vector<int32_t> table_;        // [max_seqs, pages_per_seq]; entries behind a sequence's length mean nothing
    std::vector<int32_t> len_, refs_;   // refs_: sequences that hold a page
    std::vector<uint64_t> free_;        // a bit a page
    size_t hint_ = 0;                   // no word of free_ before it has a bit
    std::vector<int32_t> given_back_, moved_;
};

}  // namespace aif
