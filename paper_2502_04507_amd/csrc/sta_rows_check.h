// Host-side checks of sta_head_rows, shared by the entry points that take them.
#pragma once
#include <stdint.h>

#include "../../include/sta.h"

namespace {

inline bool valid_type(int dt) { return dt == STA_BF16 || dt == STA_F32; }
inline int64_t size_of(int dt) { return dt == STA_F32 ? 4 : 2; }

constexpr int64_t kMostStride = (int64_t)1 << 40;           // elements; products with 2^31 tokens or heads stay in 64 bits with room
inline int check_rows(const sta_head_rows *r, bool written, int64_t B, int64_t N, int D)
{
    if (!r || !r->data) return STA_ERR_NULL;
    if (r->heads < 1 || r->heads > 65536) return STA_ERR_SHAPE;
    if (!valid_type(r->dtype)) return STA_ERR_UNSUPPORTED;
    if ((uintptr_t)r->data % size_of(r->dtype)) return STA_ERR_SHAPE;
    int64_t stride[3] = {r->batch, r->token, r->head}, count[3] = {B, N, r->heads};
    long double last = D;
    for (int i = 0; i < 3; ++i) {
        if (stride[i] < 0 || stride[i] > kMostStride) return STA_ERR_SHAPE;
        last += (long double)(count[i] - 1) * stride[i];
    }
    if (last > 4.0e18L / 4) return STA_ERR_SHAPE;
    if (written) {                                          // from the smallest stride up: no row inside another
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2 - i; ++j)
                if (stride[j] > stride[j + 1]) {
                    const int64_t s = stride[j], c = count[j];
                    stride[j] = stride[j + 1]; count[j] = count[j + 1];
                    stride[j + 1] = s; count[j + 1] = c;
                }
        int64_t extent = D;
        for (int i = 0; i < 3; ++i) {
            if (count[i] == 1) continue;
            if (stride[i] < extent) return STA_ERR_SHAPE;
            extent += (count[i] - 1) * stride[i];
        }
    }
    return STA_OK;
}

// Bytes from the first to behind the last element.
inline uint64_t extent_of(const sta_head_rows &r, int64_t B, int64_t N, int D)
{
    return (uint64_t)((B - 1) * r.batch + (N - 1) * r.token + (r.heads - 1) * r.head + D) * size_of(r.dtype);
}

// The rows of a tensor as nested progressions, in bytes: the widest stride first, without those that do not move.
struct RowSet {
    int64_t stride[3], count[3], extent[4];         // extent[i]: from the first to behind the last byte of what dimensions i .. span
    int dims;
};
inline RowSet row_set_of(const sta_head_rows &r, int64_t B, int64_t N, int D)
{
    const int64_t size = size_of(r.dtype), stride[3] = {r.batch * size, r.token * size, r.head * size}, count[3] = {B, N, r.heads};
    RowSet s = {};
    for (int i = 0; i < 3; ++i) {
        if (count[i] <= 1 || stride[i] == 0) continue;
        int at = s.dims++;
        for (; at > 0 && s.stride[at - 1] < stride[i]; --at) {
            s.stride[at] = s.stride[at - 1];
            s.count[at] = s.count[at - 1];
        }
        s.stride[at] = stride[i];
        s.count[at] = count[i];
    }
    s.extent[s.dims] = D * size;
    for (int i = s.dims - 1; i >= 0; --i) s.extent[i] = s.extent[i + 1] + (s.count[i] - 1) * s.stride[i];
    return s;
}
inline int64_t floor_div(int64_t x, int64_t d) { return x / d - (x % d < 0); }

// Whether dimensions i .. of a and j .. of b, which begins `off` bytes behind a, share a byte.  The wider stride is taken apart (where both have it, only
// the difference of the two indices counts), and of its indices those alone are followed whose spans meet: one or two for tensors side by side in one
// allocation.  The answer is exact unless `visits` run out, and then it is yes.
inline bool sets_overlap(const RowSet &a, int i, const RowSet &b, int j, int64_t off, int *visits)
{
    if (off >= a.extent[i] || off + b.extent[j] <= 0) return false;
    if (i == a.dims && j == b.dims) return true;
    if (--*visits < 0) return true;
    const int64_t sa = i < a.dims ? a.stride[i] : 0, sb = j < b.dims ? b.stride[j] : 0, s = sa > sb ? sa : sb;
    const int ni = i + (sa == s), nj = j + (sb == s);
    // what is left of b begins at off + m s, and has to begin above -extent[nj] and below extent[ni]
    int64_t lo = floor_div(-b.extent[nj] - off, s) + 1, hi = -floor_div(off - a.extent[ni], s) - 1;
    const int64_t least = sa == s ? -(a.count[i] - 1) : 0, most = sb == s ? b.count[j] - 1 : 0;
    lo = lo > least ? lo : least;
    hi = hi < most ? hi : most;
    for (int64_t m = lo; m <= hi; ++m)
        if (sets_overlap(a, ni, b, nj, off + m * s, visits)) return true;
    return false;
}

// Whether a byte of a lies in b (not without tokens).
inline bool rows_overlap(const sta_head_rows &a, int64_t Na, const sta_head_rows &b, int64_t Nb, int64_t B, int D)
{
    if (Na <= 0 || Nb <= 0 || B <= 0) return false;
    const uintptr_t a0 = (uintptr_t)a.data, b0 = (uintptr_t)b.data;
    if (a0 + extent_of(a, B, Na, D) <= b0 || b0 + extent_of(b, B, Nb, D) <= a0) return false;
    int visits = 512;
    return sets_overlap(row_set_of(a, B, Na, D), 0, row_set_of(b, B, Nb, D), 0, (int64_t)(b0 - a0), &visits);
}
inline bool rows_overlap(const sta_head_rows &a, const sta_head_rows &b, int B, int N, int D) { return rows_overlap(a, N, b, N, B, D); }

// Whether `bytes` from `at` on (null: none) touch what the rows span.
inline bool rows_meet(const sta_head_rows &r, int64_t B, int64_t N, int D, const void *at, uint64_t bytes)
{
    const uintptr_t a = (uintptr_t)at, b = (uintptr_t)r.data;
    return at && B > 0 && N > 0 && a < b + extent_of(r, B, N, D) && b < a + bytes;
}
inline bool ranges_meet(const void *a, uint64_t a_bytes, const void *b, uint64_t b_bytes)
{
    return a && b && (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

// Whether what is written, rows (null: none) or a range, meets the steps or positions of a rotation (null: none) of B x N tokens.
inline bool meets_rotary(const sta_rotary *rotary, int64_t B, int64_t N, const sta_head_rows *r, int D, const void *at, uint64_t bytes)
{
    if (!rotary || rotary->channels < 2 || B < 1 || N < 1) return false;
    const __int128 last = (__int128)(B - 1) * rotary->position_batch + (__int128)(N - 1) * rotary->position_token + (rotary->pairs[1] || rotary->pairs[2] ? 3 : 1);
    const __int128 most = (__int128)1 << 60;
    const void *from[2] = {rotary->steps, rotary->positions};
    const uint64_t size[2] = {(uint64_t)rotary->channels / 2 * sizeof(int64_t), (uint64_t)(last < most ? last : most) * sizeof(int32_t)};
    for (int i = 0; i < 2; ++i)
        if ((r && rows_meet(*r, B, N, D, from[i], size[i])) || ranges_meet(at, bytes, from[i], size[i])) return true;
    return false;
}

// Whether what is written meets the bounds of S packed sequences: rows (null: none) or a range.
struct PackedBounds {
    const int32_t *cu_q, *cu_k, *k_used;
    int S;
    bool meet(const sta_head_rows *r, int64_t tokens, int D, const void *at, uint64_t bytes) const
    {
        const void *from[3] = {cu_q, cu_k, k_used};
        for (int i = 0; i < 3; ++i) {
            const uint64_t size = ((uint64_t)S + (i < 2)) * sizeof(int32_t);
            if ((r && rows_meet(*r, 1, tokens, D, from[i], size)) || ranges_meet(at, bytes, from[i], size)) return true;
        }
        return false;
    }
};

inline bool same_rows(const sta_head_rows &a, const sta_head_rows &b)
{
    return a.data == b.data && a.batch == b.batch && a.token == b.token && a.head == b.head && a.heads == b.heads && a.dtype == b.dtype;
}

}  // namespace
