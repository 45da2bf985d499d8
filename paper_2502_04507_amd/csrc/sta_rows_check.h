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

// Whether an element of a may lie in b (not without tokens).  Heads of one fused tensor interleave: same strides, other heads.
inline bool rows_overlap(const sta_head_rows &a, int64_t Na, const sta_head_rows &b, int64_t Nb, int64_t B, int D)
{
    if (Na <= 0 || Nb <= 0 || B <= 0) return false;
    const uintptr_t a0 = (uintptr_t)a.data, b0 = (uintptr_t)b.data;
    if (a0 + extent_of(a, B, Na, D) <= b0 || b0 + extent_of(b, B, Nb, D) <= a0) return false;
    if (a.dtype != b.dtype || a.token != b.token || a.token <= 0) return true;
    if (B > 1 && (a.batch != b.batch || a.batch % a.token)) return true;
    const int64_t size = size_of(a.dtype), period = a.token * size;
    const int64_t wide_a = ((a.heads - 1) * a.head + D) * size, wide_b = ((b.heads - 1) * b.head + D) * size;
    if (wide_a > period || wide_b > period) return true;
    const int64_t off = (int64_t)(((int64_t)(b0 - a0) % period + period) % period);        // where b's rows of a token begin
    return off < wide_a || off + wide_b > period;
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

inline bool same_rows(const sta_head_rows &a, const sta_head_rows &b)
{
    return a.data == b.data && a.batch == b.batch && a.token == b.token && a.head == b.head && a.heads == b.heads && a.dtype == b.dtype;
}

}  // namespace
