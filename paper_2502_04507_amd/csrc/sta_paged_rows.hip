// Rows of a cache in pages: new ones written into it, and those of the greatest weight taken over into other pages.
//
// sta_paged_append_kernel  a row is D / 8 lanes of 16 bytes; a workgroup takes tokens of one sequence, which needs no search for it, and all their key and value heads.
// sta_paged_select_kernel  a workgroup for each sequence and key head finds the smallest weight that stays, twelve, ten and ten bits of its place in the order of
//                          numbers at a time, by counting how many have which; then writes down in order which keys stay.
// sta_paged_move_kernel    takes the rows that stay, and their weights, to their new places.
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

// ---- eviction
struct EvictParams {
    PagedCache from, to;
    const float *weights;
    float *to_weights;                  // or null
    int32_t *kept, *to_used;
    uint32_t Hkv;
    int32_t keep, first, recent;
    sta::FastDiv by_Hkv, by_blocks;
};

// Numbers in an order of whole numbers: NaN above all others, 0 and -0 the same.
__device__ __forceinline__ uint32_t order_of(float w)
{
    uint32_t bits = __float_as_uint(w);
    asm volatile("" : "+v"(bits));                          // comparisons of numbers are compiled as if there were no NaN
    if ((bits & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if (bits == 0x80000000u) bits = 0;
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;

__global__ __launch_bounds__(kSelect) void sta_paged_select_kernel(EvictParams p)
{
    __shared__ uint32_t counts[4096];
    __shared__ uint32_t wave_sums[kSelectWaves], found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const uint32_t s = sta::fast_div(blockIdx.x, p.by_Hkv), h = blockIdx.x - s * p.Hkv;
    const int n = used_of(s, p.from), stay = n < p.keep ? n : p.keep;
    const int32_t *row = p.from.table + (int64_t)s * p.from.table_row;
    int32_t *kept = p.kept + (int64_t)blockIdx.x * p.keep;
    if (h == 0 && tid == 0) p.to_used[s] = stay;
    for (int j = stay + tid; j < p.keep; j += kSelect) kept[j] = -1;
    if (n <= p.keep) {
        for (int j = tid; j < n; j += kSelect) kept[j] = j;
        return;
    }
    auto order_at = [&](int j) {
        uint32_t slot;
        const uint32_t page = page_inside(row[entry_of((uint32_t)j, p.from, &slot)], p.from);
        return order_of(p.weights[((int64_t)page * p.Hkv + h) * p.from.by_page.d + slot]);
    };
    // what may go: keys lo .. hi - 1, of which `need` stay
    const int lo = p.first, hi = n - p.recent;
    uint32_t need = (uint32_t)(p.keep - p.first - p.recent), least = 0, known = 0;          // the bits of the least one that stays, those known so far
    for (int digit = 0; digit < 3 && need > 0; ++digit) {
        const int shift = digit == 0 ? 20 : digit == 1 ? 10 : 0, bins = digit == 0 ? 4096 : 1024;
        for (int b = tid; b < bins; b += kSelect) counts[b] = 0;
        __syncthreads();
#pragma unroll 4
        for (int j = lo + tid; j < hi; j += kSelect) {
            const uint32_t x = order_at(j);
            if ((x & known) == least) atomicAdd(&counts[(x >> shift) & (bins - 1)], 1u);
        }
        __syncthreads();
        // every thread has `each` bins, the first one the highest: how many stand in bins above
        const int each = bins / kSelect;
        uint32_t own = 0;
        for (int b = 0; b < each; ++b) own += counts[bins - 1 - (tid * each + b)];
        const uint32_t upto = scan64(own);
        if (lane == 63) wave_sums[wave] = upto;
        __syncthreads();
        uint32_t above = upto - own;
        for (int w = 0; w < wave; ++w) above += wave_sums[w];
        if (above < need && above + own >= need) {          // one thread: in its bins the number that still has to stay is reached
            int b = 0;
            for (; above + counts[bins - 1 - (tid * each + b)] < need; ++b) above += counts[bins - 1 - (tid * each + b)];
            found[0] = bins - 1 - (tid * each + b);
            found[1] = above;
        }
        __syncthreads();
        least |= found[0] << shift;
        known |= (uint32_t)(bins - 1) << shift;
        need -= found[1];
        __syncthreads();
    }
    // `need` of those equal to `least`, the first ones, stay, and all above it.  A wave has a run of keys: it counts them, and after those before it writes them down.
    if (p.keep == p.first + p.recent) least = 0xffffffffu;
    const int run = ((n + kSelectWaves - 1) / kSelectWaves + 63) & ~63, begin = wave * run, end = begin + run < n ? begin + run : n;
    auto look = [&](int j, bool *sure, bool *equal) {
        const bool inside = j >= lo && j < hi;
        const uint32_t x = j < end ? order_at(j) : 0;
        *sure = j < end && (!inside || x > least);
        *equal = j < end && inside && x == least;
    };
    uint32_t sure_before = 0, equal_before = 0;
    for (int j0 = begin; j0 < end; j0 += 64) {
        bool sure, equal;
        look(j0 + lane, &sure, &equal);
        sure_before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(sure));
        equal_before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(equal));
    }
    if (lane == 0) {
        counts[wave] = sure_before;
        counts[kSelectWaves + wave] = equal_before;
    }
    __syncthreads();
    sure_before = equal_before = 0;
    for (int w = 0; w < wave; ++w) {
        sure_before += counts[w];
        equal_before += counts[kSelectWaves + w];
    }
    for (int j0 = begin; j0 < end; j0 += 64) {
        bool sure, equal;
        look(j0 + lane, &sure, &equal);
        const uint64_t sures = __builtin_amdgcn_ballot_w64(sure), equals = __builtin_amdgcn_ballot_w64(equal), below = ((uint64_t)1 << lane) - 1;
        const uint32_t rank = equal_before + __builtin_popcountll(equals & below);
        const uint32_t equal_taken = rank < need ? rank : need;
        const uint32_t place = sure_before + __builtin_popcountll(sures & below) + equal_taken;
        if ((sure || (equal && rank < need)) && place < (uint32_t)p.keep) kept[place] = j0 + lane;
        sure_before += __builtin_popcountll(sures);
        equal_before += __builtin_popcountll(equals);
    }
}

template <int D>
__global__ __launch_bounds__(256) void sta_paged_move_kernel(EvictParams p)
{
    constexpr int LPR = D / 8, ROWS = 256 / LPR, AT_ONCE = 4;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_blocks), block = blockIdx.x - item * p.by_blocks.d;      // (sequence, key head), rows
    const uint32_t s = sta::fast_div(item, p.by_Hkv), h = item - s * p.Hkv;
    const int n = used_of(s, p.from), stay = n < p.keep ? n : p.keep, c = threadIdx.x % LPR;
    const int32_t *row = p.from.table + (int64_t)s * p.from.table_row, *to_row = p.to.table + (int64_t)s * p.to.table_row, *kept = p.kept + (int64_t)item * p.keep;
    u32x4 k[AT_ONCE], v[AT_ONCE];
    float w[AT_ONCE];
    int64_t to[AT_ONCE], to_weight[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        const int j = (int)block * ROWS * AT_ONCE + i * ROWS + (int)(threadIdx.x / LPR);
        to[i] = -1;
        if (j >= stay) continue;
        uint32_t slot, to_slot;
        const int to_page = to_row[entry_of((uint32_t)j, p.to, &to_slot)];
        if (to_page < 0 || to_page >= (int)p.to.pages) continue;
        const uint32_t page = page_inside(row[entry_of((uint32_t)bound_of(kept[j], 0, n - 1), p.from, &slot)], p.from);
        const uint64_t at = place_of(page, slot, p.from) + (int64_t)h * p.from.head + 16 * c;
        k[i] = *reinterpret_cast<const u32x4 *>(p.from.k + at);
        v[i] = *reinterpret_cast<const u32x4 *>(p.from.v + at);
        if (c == 0 && p.to_weights) w[i] = p.weights[((int64_t)page * p.Hkv + h) * p.from.by_page.d + slot];
        to[i] = (int64_t)(place_of((uint32_t)to_page, to_slot, p.to) + (int64_t)h * p.to.head + 16 * c);
        to_weight[i] = ((int64_t)to_page * p.Hkv + h) * p.to.by_page.d + to_slot;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
        if (to[i] < 0) continue;
        *reinterpret_cast<u32x4 *>(p.to.k + to[i]) = k[i];
        *reinterpret_cast<u32x4 *>(p.to.v + to[i]) = v[i];
        if (c == 0 && p.to_weights) p.to_weights[to_weight[i]] = w[i];
    }
}

// Whether two pools share memory without being one and the same.
bool pools_meet(const sta_paged_cache &a, const sta_paged_cache &b, int D)
{
    const sta_head_rows *x[2] = {&a.k, &a.v}, *y[2] = {&b.k, &b.v};
    const bool alike = a.pages == b.pages && a.page_size == b.page_size;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            if (i == j && alike && same_rows(*x[i], *y[j])) continue;
            if (a.pages <= 0 || b.pages <= 0) continue;
            const uintptr_t a0 = (uintptr_t)x[i]->data, b0 = (uintptr_t)y[j]->data;
            if (a0 + extent_of(*x[i], a.pages, a.page_size, D) <= b0 || b0 + extent_of(*y[j], b.pages, b.page_size, D) <= a0) continue;
            int visits = 512;
            if (sets_overlap(row_set_of(*x[i], a.pages, a.page_size, D), 0, row_set_of(*y[j], b.pages, b.page_size, D), 0, (int64_t)(b0 - a0), &visits)) return true;
        }
    return false;
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

extern "C" int sta_paged_evict(const sta_paged_cache *cache, const float *weights, const sta_paged_cache *into, float *into_weights, int32_t *kept, int S, int keep,
                               int first, int recent, int D, void *hip_stream)
{
    if (!cache || !into) return STA_ERR_NULL;
    if (S < 0 || keep < 0 || first < 0 || recent < 0 || (int64_t)first + recent > keep) return STA_ERR_SHAPE;
    if (D != 64 && D != 128) return STA_ERR_UNSUPPORTED;
    if (int rc = paged_check(cache, S, D, false)) return rc;
    if (int rc = paged_check(into, S, D, true)) return rc;
    const int Hkv = cache->k.heads;
    if (into->k.heads != Hkv || (int64_t)into->table_pages * into->page_size < keep || keep > kMostTokens) return STA_ERR_SHAPE;
    for (const sta_paged_cache *c : {cache, into})
        if ((__int128)c->pages * c->page_size * Hkv > (__int128)1 << 60) return STA_ERR_SHAPE;
    if (S == 0) return STA_OK;
    const uint64_t w_bytes = weight_bytes(*cache), to_bytes = into_weights ? weight_bytes(*into) : 0;
    if ((!weights && w_bytes > 0) || (!kept && keep > 0)) return STA_ERR_NULL;
    if (((uintptr_t)weights | (uintptr_t)into_weights | (uintptr_t)kept) & 3) return STA_ERR_SHAPE;
    const int64_t blocks = ((int64_t)keep + 4096 / (D / 2) - 1) / (4096 / (D / 2)), items = (int64_t)S * Hkv;
    constexpr int64_t most_selects = (1 << 22) - 1;         // of 1024 lanes
    if (items > most_selects || items * blocks > kMostWorkgroups) return STA_ERR_SHAPE;
    const uint64_t kept_bytes = (uint64_t)items * keep * sizeof(int32_t);
    if (rows_overlap(into->k, into->v, (int)into->pages, into->page_size, D) || pools_meet(*cache, *into, D)) return STA_ERR_ALIAS;
    const bool one = into_weights == weights && cache->pages == into->pages && cache->page_size == into->page_size;
    if (!one && ranges_meet(weights, w_bytes, into_weights, to_bytes)) return STA_ERR_ALIAS;
    const struct { const void *at; uint64_t bytes; } written[3] = {{into_weights, to_bytes}, {kept, kept_bytes}, {into->used, used_bytes(S)}};
    for (int i = 0; i < 3; ++i) {
        const auto &w = written[i];
        if (!w.at || !w.bytes) continue;
        if (meets_pages(*cache, D, w.at, w.bytes) || meets_pages(*into, D, w.at, w.bytes) || meets_table(*cache, S, nullptr, 0, 0, D, w.at, w.bytes) ||
            ranges_meet(w.at, w.bytes, into->table, table_bytes(*into, S)) || (i > 0 && ranges_meet(w.at, w.bytes, weights, w_bytes)))
            return STA_ERR_ALIAS;
        for (int j = 0; j < i; ++j)
            if (ranges_meet(w.at, w.bytes, written[j].at, written[j].bytes)) return STA_ERR_ALIAS;
    }
    const sta_head_rows *pool[2] = {&into->k, &into->v};
    for (const sta_head_rows *r : pool)
        if (meets_table(*cache, S, r, into->pages, into->page_size, D, nullptr, 0) || meets_table(*into, S, r, into->pages, into->page_size, D, nullptr, 0) ||
            rows_meet(*r, into->pages, into->page_size, D, weights, w_bytes))
            return STA_ERR_ALIAS;
    EvictParams p = {};
    p.from = paged_cache_of(*cache);
    p.to = paged_cache_of(*into);
    p.weights = weights;
    p.to_weights = into_weights;
    p.kept = kept;
    p.to_used = into->used;
    p.Hkv = Hkv;
    p.keep = keep;
    p.first = first;
    p.recent = recent;
    p.by_Hkv = sta::fast_div_of(Hkv);
    p.by_blocks = sta::fast_div_of(blocks > 0 ? (uint32_t)blocks : 1);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e = sta::launch_kernel(sta_paged_select_kernel, dim3((uint32_t)items), dim3(kSelect), stream, p);
    if (e == hipSuccess && keep > 0 && into->pages > 0 && cache->pages > 0) {
        const dim3 grid((uint32_t)(items * blocks)), block(256);
        e = D == 64 ? sta::launch_kernel(sta_paged_move_kernel<64>, grid, block, stream, p) : sta::launch_kernel(sta_paged_move_kernel<128>, grid, block, stream, p);
    }
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}
