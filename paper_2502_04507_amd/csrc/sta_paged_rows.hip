// Rows of a cache in pages: new ones written into it.
//
// sta_paged_append_kernel  a row is D / 8 lanes of 16 bytes; a workgroup takes tokens of one sequence, which needs no search for it, and all their key and value heads.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_internal.h"
#include "sta_paged.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct AppendParams {
    PackedRows k, v;                    // strides in bytes
    const int32_t *cu;
    PagedCache c;
    float *weights;                     // or null
    sta::FastDiv by_chunks;             // lanes of a token: 2 Hkv D / 8
    uint32_t tokens, max_new, Hkv, each, per_seq;      // tokens of a workgroup at a time, workgroups of a sequence
};

// Eight channels of a row as bf16, rounded to nearest where they are float32.
template <bool F32>
__device__ __forceinline__ u32x4 eight_of(const char *at)
{
    if constexpr (!F32) return *reinterpret_cast<const u32x4 *>(at);
    const floatx4 a = *reinterpret_cast<const floatx4 *>(at), b = *reinterpret_cast<const floatx4 *>(at + 16);
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = static_cast<__bf16>(a[i]);
        r[4 + i] = static_cast<__bf16>(b[i]);
    }
    return __builtin_bit_cast(u32x4, r);
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void sta_paged_append_kernel(AppendParams p)
{
    constexpr uint32_t LPR = D / 8;
    constexpr int AT_ONCE = 4;
    const uint32_t s = blockIdx.y;
    const int first = bound_of(p.cu[s], 0, (int)p.tokens), all = bound_of(p.cu[s + 1], first, (int)p.tokens) - first;
    const int used = used_of(s, p.c), given = p.c.used[s], key0 = (given > 0 ? given : 0) - all;
    const uint32_t n = (uint32_t)all < p.max_new ? (uint32_t)all : p.max_new;
    const int32_t *row = p.c.table + (int64_t)s * p.c.table_row;
    for (uint32_t t0 = blockIdx.x * p.each; t0 < n; t0 += p.per_seq * p.each) {
        const uint32_t here = n - t0 < p.each ? n - t0 : p.each, lanes = here * p.by_chunks.d;
        for (uint32_t i0 = threadIdx.x; i0 < lanes; i0 += AT_ONCE * 256) {
            u32x4 x[AT_ONCE];
            char *to[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const uint32_t i = i0 + 256 * j;
                to[j] = nullptr;
                if (i >= lanes) continue;
                const uint32_t t = sta::fast_div(i, p.by_chunks), chunk = i - t * p.by_chunks.d, r = chunk / LPR, c = chunk % LPR;
                const bool value = r >= p.Hkv;
                const uint32_t h = value ? r - p.Hkv : r;
                const int key = key0 + (int)(t0 + t);
                if (key < 0 || key >= used) continue;
                uint32_t slot;
                const int page = row[entry_of((uint32_t)key, p.c, &slot)];
                if (page < 0 || page >= (int)p.c.pages) continue;
                const PackedRows &from = value ? p.v : p.k;
                x[j] = eight_of<F32>(from.data + (int64_t)(first + (int)(t0 + t)) * from.token + (int64_t)h * from.head + c * (F32 ? 32 : 16));
                to[j] = (value ? p.c.v : p.c.k) + place_of((uint32_t)page, slot, p.c) + (int64_t)h * p.c.head + 16 * c;
                if (p.weights && !value && c == 0) p.weights[((int64_t)page * p.Hkv + h) * p.c.by_page.d + slot] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (to[j]) *reinterpret_cast<u32x4 *>(to[j]) = x[j];
        }
    }
}

// Rows that are read 16 bytes at a time, of one of two types.
int new_rows_check(const sta_head_rows *r, int64_t tokens, int heads, int D)
{
    if (!r) return STA_ERR_NULL;
    sta_head_rows some = *r;
    if (tokens == 0) some.data = reinterpret_cast<void *>(16);
    some.batch = 0;
    if (int rc = check_rows(&some, false, 1, tokens > 0 ? tokens : 1, D)) return rc;
    const int64_t eight = 16 / size_of(r->dtype);
    if (r->heads != heads || ((uintptr_t)some.data & 15) || r->token % eight || r->head % eight) return STA_ERR_SHAPE;
    return STA_OK;
}

// Bytes of one number of 32 bits for every key of the pool and key head.
uint64_t weight_bytes(const sta_paged_cache &c) { return (uint64_t)c.pages * c.page_size * c.k.heads * sizeof(float); }

}  // namespace

extern "C" int sta_paged_append(const sta_head_rows *k, const sta_head_rows *v, int64_t tokens, const int32_t *cu, const sta_paged_cache *cache, int S,
                                int max_new, int D, float *weights, void *hip_stream)
{
    if (!k || !v || !cache) return STA_ERR_NULL;
    if (S < 0 || tokens < 0 || max_new < 0 || tokens > kMostTokens) return STA_ERR_SHAPE;
    if (D != 64 && D != 128) return STA_ERR_UNSUPPORTED;
    if (int rc = paged_check(cache, S, D, true)) return rc;
    const int Hkv = cache->k.heads;
    if (int rc = new_rows_check(k, tokens, Hkv, D)) return rc;
    if (int rc = new_rows_check(v, tokens, Hkv, D)) return rc;
    if (k->dtype != v->dtype) return STA_ERR_UNSUPPORTED;
    if ((__int128)cache->pages * cache->page_size * Hkv > (__int128)1 << 60) return STA_ERR_SHAPE;
    if (S == 0 || tokens == 0 || max_new == 0 || room_of(*cache) == 0) return STA_OK;
    if (!cu) return STA_ERR_NULL;
    if (((uintptr_t)cu | (uintptr_t)weights) & 3) return STA_ERR_SHAPE;
    if (S > 65535) return STA_ERR_SHAPE;
    if (rows_overlap(cache->k, cache->v, (int)cache->pages, cache->page_size, D)) return STA_ERR_ALIAS;
    const uint64_t w_bytes = weight_bytes(*cache), cu_bytes = ((uint64_t)S + 1) * sizeof(int32_t);
    const sta_head_rows *rows[2] = {k, v}, *pool[2] = {&cache->k, &cache->v};
    for (int i = 0; i < 2; ++i) {
        if (rows_in_pages(*cache, D, *rows[i], tokens) || rows_meet(*rows[i], 1, tokens, D, weights, w_bytes)) return STA_ERR_ALIAS;
        if (meets_table(*cache, S, pool[i], cache->pages, cache->page_size, D, nullptr, 0) ||
            rows_meet(*pool[i], cache->pages, cache->page_size, D, cu, cu_bytes))
            return STA_ERR_ALIAS;
    }
    if (meets_pages(*cache, D, weights, w_bytes) || meets_table(*cache, S, nullptr, 0, 0, D, weights, w_bytes) || ranges_meet(weights, w_bytes, cu, cu_bytes))
        return STA_ERR_ALIAS;
    AppendParams p = {};
    const int64_t size = size_of(k->dtype);
    p.k = {static_cast<char *>(k->data), k->token * size, k->head * size};
    p.v = {static_cast<char *>(v->data), v->token * size, v->head * size};
    p.cu = cu;
    p.c = paged_cache_of(*cache);
    p.weights = weights;
    p.by_chunks = sta::fast_div_of(2 * Hkv * (D / 8));
    p.tokens = (uint32_t)tokens;
    p.max_new = (uint32_t)max_new;
    p.Hkv = Hkv;
    // Four rounds of all lanes a workgroup; of a sequence as many workgroups as its longest may need, or as 16384 workgroups in all allow, which then go around.
    p.each = 1024 / p.by_chunks.d > 0 ? 1024 / p.by_chunks.d : 1;
    const int64_t longest = max_new < tokens ? max_new : tokens, want = (longest + p.each - 1) / p.each, most = S < 16384 ? 16384 / S : 1;
    p.per_seq = (uint32_t)(want < most ? want : most);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid(p.per_seq, S), block(256);
    hipError_t e;
    if (D == 64) e = k->dtype == STA_F32 ? sta::launch_kernel(sta_paged_append_kernel<64, true>, grid, block, stream, p) : sta::launch_kernel(sta_paged_append_kernel<64, false>, grid, block, stream, p);
    else e = k->dtype == STA_F32 ? sta::launch_kernel(sta_paged_append_kernel<128, true>, grid, block, stream, p) : sta::launch_kernel(sta_paged_append_kernel<128, false>, grid, block, stream, p);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}
