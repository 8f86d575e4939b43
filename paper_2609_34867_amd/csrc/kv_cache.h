// The paged key-value cache: where a key of a sequence lies.
//
// Keys and values are [num_pages][Hk][P][D] each, P = 2^shift rows per page, so
// that the rows of one head on a page are contiguous (a decode work-group reads
// P * D values in one piece).  Row b of the block table [B][max_pages] lists the
// pages of sequence b in order.  Everything here is plain arithmetic (constexpr:
// host and device), so the bounds can be tested without a GPU: a table entry
// outside [0, num_pages) or a key past the table is kNoPage, and nobody forms
// an address from it.
#pragma once

#include <stdint.h>

namespace p4q {

constexpr int kNoPage = -1;

// log2 of a page size the cache allows (a power of two from 16 to 4096), or -1
constexpr int page_shift(int page_size) {
    for (int s = 4; s <= 12; ++s)
        if (page_size == (1 << s)) return s;
    return -1;
}

// a table entry as a page of the cache, or kNoPage
constexpr int valid_page(int entry, int num_pages) {
    return (uint32_t)entry < (uint32_t)num_pages ? entry : kNoPage;
}

// the table column of `key`, or kNoPage if the table has none
constexpr int page_column(int64_t key, int shift, int max_pages) {
    return key >= 0 && (key >> shift) < max_pages ? (int)(key >> shift) : kNoPage;
}

// the table column that the rows from `key` on are fetched by, in a sequence whose first
// `keys` keys the table holds: a key past the last one (fetched ahead, never used) goes
// by the last one's, so that no entry past the sequence's keys is read; kNoPage
// without keys
constexpr int fetch_column(int key, int keys, int shift) {
    return keys > 0 ? (key < keys ? key : keys - 1) >> shift : kNoPage;
}

// element offset of row `slot` (0 .. P - 1) of head h on `page`, 64 bits: a cache
// of a few hundred thousand keys passes 2^31 elements
constexpr int64_t page_row(int page, int Hk, int h, int shift, int slot, int D) {
    return ((((int64_t)page * Hk + h) << shift) + slot) * D;
}

// keys that a sequence length stands for (a negative one: none)
constexpr int key_count(int len) { return len > 0 ? len : 0; }

// [first, last) of packed sequence b within rows [0, total): lists that do not
// ascend, or leave the buffer, are cut to it
struct Span {
    int first, last;
};
constexpr Span packed_span(int begin, int end, int total) {
    const int f = begin < 0 ? 0 : begin > total ? total : begin;
    const int l = end < f ? f : end > total ? total : end;
    return Span{f, l};
}

// n / G for n < 2^31 as (2 n m) >> (32 + s), with s = ceil(log2 G) and
// m = floor(2^(31 + s) / G) + 1 <= 2^32 - 1:  m G = 2^(31 + s) + e with 0 < e <= G <= 2^s,
// so n m / 2^(31 + s) exceeds n / G by less than n / 2^31 / G < 1 / G.
struct Magic {
    uint32_t m;
    int shift;
};
constexpr Magic magic_of(int G) {
    int s = 0;
    while ((1 << s) < G) ++s;
    return Magic{(uint32_t)(((uint64_t)1 << (31 + s)) / (uint32_t)G + 1), s};
}
constexpr int magic_div(int n, uint32_t m, int shift) {
    return (int)((uint32_t)(((uint64_t)(2u * (uint32_t)n) * m) >> 32) >> shift);
}

}  // namespace p4q
