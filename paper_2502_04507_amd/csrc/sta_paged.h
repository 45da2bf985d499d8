// A cache of keys and values in pages, as the kernels see it: key j of sequence s is slot j % page_size of page table[s][j / page_size].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_internal.h"
#include "sta_packed.h"
#include "sta_rows_check.h"

namespace {

// Strides in bytes.  Slots of a page and pages lie less than 2^32 bytes apart, so that a place is one product of 32 bits and one of 32 by 32 to 64.
struct PagedCache {
    char *k, *v;
    uint32_t page, token;
    int64_t head;
    const int32_t *table;
    int64_t table_row;              // entries
    const int32_t *used;
    sta::FastDiv by_page;           // page_size
    uint32_t pages;
    int32_t room;                   // keys that a row of the table has places for
};

// Where the numbers of a cache's keys stand.
struct KeyNumbers {
    uint32_t by_sequence;           // in rows, one for every sequence and key head; else beside the pages
    int64_t row;
};

// Entries of the table that are no pages of the pool are cut to what is there: what is read for them means nothing, and is inside the pool.
__device__ __forceinline__ uint32_t page_inside(int entry, const PagedCache &c) { return (uint32_t)bound_of(entry, 0, (int)c.pages - 1); }
__device__ __forceinline__ int used_of(uint32_t s, const PagedCache &c) { return bound_of(c.used[s], 0, c.room); }
// The place of a key in its page, in slots, and which entry of its sequence's row has the page.
__device__ __forceinline__ uint32_t entry_of(uint32_t key, const PagedCache &c, uint32_t *slot)
{
    const uint32_t n = sta::fast_div(key, c.by_page);
    *slot = key - n * c.by_page.d;
    return n;
}
__device__ __forceinline__ uint64_t place_of(uint32_t page, uint32_t slot, const PagedCache &c) { return (uint64_t)page * c.page + slot * c.token; }
// Where the number of a key stands, by floats: of key head h of Hkv, key `key` of sequence s, in a slot of a page.  Beside the pages one number is all keys' that a slot is, and so one sequence's
// alone where the page stands once in the table.
template <bool BY_SEQUENCE = true>          // false: by page in any case
__device__ __forceinline__ int64_t number_at(uint32_t s, uint32_t h, uint32_t Hkv, uint32_t key, uint32_t page, uint32_t slot, const PagedCache &c, const KeyNumbers &n)
{
    return BY_SEQUENCE && n.by_sequence ? ((int64_t)s * Hkv + h) * n.row + key : ((int64_t)page * Hkv + h) * c.by_page.d + slot;
}

// Whether the kernels can take a cache; written: its rows are.  S sequences of heads of D channels.
int paged_check(const sta_paged_cache *c, int S, int D, bool written)
{
    if (!c) return STA_ERR_NULL;
    if (c->numbers_by_sequence & ~1) return STA_ERR_UNSUPPORTED;
    if (c->pages < 0 || c->pages > 0x7fffffff || c->page_size < 1 || c->table_pages < 0 || c->table_row < 0 || c->table_row > kMostStride || S < 0) return STA_ERR_SHAPE;
    const sta_head_rows *rows[2] = {&c->k, &c->v};
    for (const sta_head_rows *r : rows) {
        sta_head_rows some = *r;
        if (c->pages == 0) some.data = reinterpret_cast<void *>(16);        // nothing is there to be read
        if (int rc = check_rows(&some, written, c->pages > 0 ? c->pages : 1, c->page_size, D)) return rc;
        if (r->dtype != STA_BF16) return STA_ERR_UNSUPPORTED;
        if (((uintptr_t)some.data & 15) || r->batch % 8 || r->token % 8 || r->head % 8) return STA_ERR_SHAPE;
    }
    const sta_head_rows &k = c->k, &v = c->v;
    if (k.batch != v.batch || k.token != v.token || k.head != v.head || k.heads != v.heads) return STA_ERR_SHAPE;
    // in bytes below 2^32; a slot inside a page, from its first, too, and a lane's rows of a group in 32 bits
    if (k.batch >= (int64_t)1 << 31 || k.token >= (int64_t)1 << 26 || (__int128)k.token * c->page_size >= (int64_t)1 << 31) return STA_ERR_SHAPE;
    if (S == 0) return STA_OK;
    if (!c->used || (!c->table && c->table_pages > 0)) return STA_ERR_NULL;
    if (((uintptr_t)c->table | (uintptr_t)c->used) & 3) return STA_ERR_SHAPE;
    return STA_OK;
}

// Keys that a row of the table has places for; none where the pool has no pages.
inline int64_t room_of(const sta_paged_cache &c)
{
    const int64_t room = (int64_t)c.table_pages * c.page_size;
    return c.pages == 0 ? 0 : room < kMostTokens ? room : kMostTokens;
}

// The keys' numbers of a cache of S sequences, all key heads; below 2^60 (else none of it is taken).
inline __int128 numbers_of(const sta_paged_cache &c, int S)
{
    return (c.numbers_by_sequence ? (__int128)S * c.table_pages : (__int128)c.pages) * c.page_size * c.k.heads;
}
inline bool numbers_fit(const sta_paged_cache &c, int S) { return numbers_of(c, S) <= (__int128)1 << 60; }
inline uint64_t number_bytes(const sta_paged_cache &c, int S) { return (uint64_t)numbers_of(c, S) * sizeof(float); }

inline KeyNumbers key_numbers_of(const sta_paged_cache &c) { return {(uint32_t)c.numbers_by_sequence, (int64_t)c.table_pages * c.page_size}; }

inline PagedCache paged_cache_of(const sta_paged_cache &c)
{
    PagedCache p = {};
    p.k = static_cast<char *>(c.k.data);
    p.v = static_cast<char *>(c.v.data);
    p.page = (uint32_t)(c.k.batch * 2);
    p.token = (uint32_t)(c.k.token * 2);
    p.head = c.k.head * 2;
    p.table = c.table;
    p.table_row = c.table_row;
    p.used = c.used;
    p.by_page = sta::fast_div_of(c.page_size);
    p.pages = (uint32_t)c.pages;
    p.room = (int32_t)room_of(c);
    return p;
}

// Bytes of the table and of the lengths of S sequences.
inline uint64_t table_bytes(const sta_paged_cache &c, int S) { return S > 0 && c.table_pages > 0 ? ((uint64_t)(S - 1) * c.table_row + c.table_pages) * sizeof(int32_t) : 0; }
inline uint64_t used_bytes(int S) { return (uint64_t)S * sizeof(int32_t); }

// Whether a range (or rows that are B x N tokens, where r is not null) meets the table or the lengths.
inline bool meets_table(const sta_paged_cache &c, int S, const sta_head_rows *r, int64_t B, int64_t N, int D, const void *at, uint64_t bytes)
{
    const void *from[2] = {c.table, c.used};
    const uint64_t size[2] = {table_bytes(c, S), used_bytes(S)};
    for (int i = 0; i < 2; ++i)
        if (size[i] && ((r && rows_meet(*r, B, N, D, from[i], size[i])) || ranges_meet(at, bytes, from[i], size[i]))) return true;
    return false;
}
// Whether a range meets the pages.
inline bool meets_pages(const sta_paged_cache &c, int D, const void *at, uint64_t bytes)
{
    return rows_meet(c.k, c.pages, c.page_size, D, at, bytes) || rows_meet(c.v, c.pages, c.page_size, D, at, bytes);
}
// Whether rows share a byte with the pages.  The pages' three strides and the rows' two are taken apart as those of tensors are.
inline bool rows_in_pages(const sta_paged_cache &c, int D, const sta_head_rows &r, int64_t tokens)
{
    if (tokens <= 0 || c.pages <= 0) return false;
    const sta_head_rows *pool[2] = {&c.k, &c.v};
    sta_head_rows one = r;
    one.batch = 0;
    for (const sta_head_rows *x : pool) {
        const uintptr_t a0 = (uintptr_t)one.data, b0 = (uintptr_t)x->data;
        if (a0 + extent_of(one, 1, tokens, D) <= b0 || b0 + extent_of(*x, c.pages, c.page_size, D) <= a0) continue;
        int visits = 512;
        if (sets_overlap(row_set_of(one, 1, tokens, D), 0, row_set_of(*x, c.pages, c.page_size, D), 0, (int64_t)(b0 - a0), &visits)) return true;
    }
    return false;
}

}  // namespace
