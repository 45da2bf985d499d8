// Rows of a cache in pages: new ones written into it, and those of the greatest weight taken over into other pages.
//
// sta_paged_append_kernel  a row is D / 8 lanes of 16 bytes; a workgroup takes tokens of one sequence, which needs no search for it, and all their key and value heads.  Bound by memory: 12,366 tokens of 8 heads of 128
//                          channels from float32 24.4 us, 6.2 TB/s.
// sta_paged_select_kernel  a workgroup for each sequence and key head finds the smallest weight that stays, twelve, ten and ten bits of its place in the order of
//                          numbers at a time, by counting how many have which; then writes down in order which keys stay.  Bound by the instructions and LDS of the one CU that a head has:
//                          8 heads of 32,768 keys 23 us (2.5 to begin, 5 to bring the numbers, 4.5 the first digit, 3.5 the others, 2.5 to count and 5 to write down).  The
//                          counts of a thread's bins, 12 bytes, are in scratch, which is looked at by one thread for each digit.  More than 32,768 keys are looked up at every step:
//                          32,769 keys 11 us more, 131,072 80.
// sta_paged_move_kernel    takes the rows that stay, and their weights, to their new places.  Bound by memory: 24 sequences, 8 heads of 128 channels, 2048 rows each, 79 us, 5.0 TB/s
//                          (82 with stores through the caches).
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
    KeyNumbers numbers;
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

// 16 bytes of a row; STREAM: past the caches, where more is written than they hold.
constexpr int64_t kCaches = (int64_t)32 << 20;              // the L2 caches of the eight XCDs
template <bool STREAM>
__device__ __forceinline__ void store_row(char *to, u32x4 x)
{
    if (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(to));
    else *reinterpret_cast<u32x4 *>(to) = x;
}

template <int D, bool F32, bool STREAM>
__global__ __launch_bounds__(256) void sta_paged_append_kernel(AppendParams p)
{
    constexpr uint32_t LPR = D / 8;
    constexpr int AT_ONCE = 2;
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
                if (p.weights && !value && c == 0) p.weights[number_at(s, h, p.Hkv, (uint32_t)key, (uint32_t)page, slot, p.c, p.numbers)] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (to[j]) store_row<STREAM>(to[j], x[j]);
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
    uint32_t page_weights;              // numbers of a page, of all key heads
    uint32_t row_lanes;                 // not 0: rows are moved by the kernel that selects them, so many lanes a row
    uint32_t fours;                     // pages of a multiple of four slots (by sequence: such rows), weights at a multiple of 16 bytes
    KeyNumbers from_numbers, to_numbers;
};

// Takes 16 bytes, chunk c, of key `key` of head h to key j of the other cache, and the weight with the first.  BY_SEQUENCE: the numbers of either cache may be by sequence (as a choice at every number
// by itself it costs evictions that know no such caches 1 to 5 %: 8 heads of 32,768 keys 36.7 -> 38.3 us).
template <bool STREAM, bool BY_SEQUENCE>
__device__ __forceinline__ void move_chunk(const EvictParams &p, uint32_t s, uint32_t h, uint32_t j, uint32_t key, uint32_t c)
{
    uint32_t slot, to_slot;
    const int to_page = p.to.table[(int64_t)s * p.to.table_row + entry_of(j, p.to, &to_slot)];
    const uint32_t page = page_inside(p.from.table[(int64_t)s * p.from.table_row + entry_of(key, p.from, &slot)], p.from);
    if (to_page < 0 || to_page >= (int)p.to.pages) return;
    const uint64_t at = place_of(page, slot, p.from) + (int64_t)h * p.from.head + 16 * c, to = place_of((uint32_t)to_page, to_slot, p.to) + (int64_t)h * p.to.head + 16 * c;
    const u32x4 k = *reinterpret_cast<const u32x4 *>(p.from.k + at), v = *reinterpret_cast<const u32x4 *>(p.from.v + at);
    store_row<STREAM>(p.to.k + to, k);
    store_row<STREAM>(p.to.v + to, v);
    if (c == 0 && p.to_weights) p.to_weights[number_at<BY_SEQUENCE>(s, h, p.Hkv, j, (uint32_t)to_page, to_slot, p.to, p.to_numbers)] = p.weights[number_at<BY_SEQUENCE>(s, h, p.Hkv, key, page, slot, p.from, p.from_numbers)];
}

// The bits of a number as a whole number in their order: NaN above all others, 0 and -0 the same.  On the bits throughout: comparisons of numbers are compiled as if
// there were no NaN.
__device__ __forceinline__ uint32_t order_of(uint32_t bits)
{
    if ((bits & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if (bits == 0x80000000u) bits = 0;
    return bits ^ ((uint32_t)((int)bits >> 31) | 0x80000000u);
}

constexpr int kSelect = 1024, kSelectWaves = kSelect / 64;
constexpr uint32_t kFewRows = 256;

// What a wave looks at: a run of keys, four adjacent ones a lane and 256 at a time, as whole numbers in the order of their weights.  Keys that stay or go in any case (the first, the
// recent ones, and places behind the last) count as 0, which no weight has, nor any up to 2^20.  A run of up to 256 * GROUPS keys stays in LDS from the first look on, of a longer one every
// number is looked up every time.
template <int GROUPS, bool BY_SEQUENCE>
struct Run {
    u32x4 *own;                         // of the wave and lane, in LDS
    int begin, end, length, lo, hi;     // length: of a run
    bool kept;
    const int32_t *row;
    const uint32_t *weights;            // of the key head, by sequence of the sequence
    __device__ __forceinline__ u32x4 look(const EvictParams &p, int j) const
    {
        u32x4 w = {0, 0, 0, 0};
        if (p.fours) {
            uint32_t slot;
            if (j >= end) return w;
            if (BY_SEQUENCE && p.from_numbers.by_sequence) return *reinterpret_cast<const u32x4 *>(weights + j);
            const int entry = row[entry_of((uint32_t)j, p.from, &slot)];
            return *reinterpret_cast<const u32x4 *>(weights + ((uint64_t)page_inside(entry, p.from) * p.page_weights + slot));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (j + e >= end) return w;
            if (BY_SEQUENCE && p.from_numbers.by_sequence) {
                w[e] = weights[j + e];
                continue;
            }
            uint32_t slot;
            const uint32_t page = page_inside(row[entry_of((uint32_t)(j + e), p.from, &slot)], p.from);
            w[e] = weights[(uint64_t)page * p.page_weights + slot];
        }
        return w;
    }
    // j0: the first lane's first key.  Numbers from 0 up to infinity, as weights are, have a short way.
    __device__ __forceinline__ u32x4 order(int j0, int lane, u32x4 w) const
    {
        bool other = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) other = other || w[e] > 0x7f800000u;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(other) == 0, 1)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] |= 0x80000000u;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = order_of(w[e]);
        }
        if (!inside(j0)) {
            const int j = j0 + 4 * lane;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = j + e >= lo && j + e < hi ? w[e] : 0;
        }
        return w;
    }
    // whether no key of 256 stays or goes in any case
    __device__ __forceinline__ bool inside(int j0) const { return j0 >= lo && hi - j0 >= 256; }
    __device__ __forceinline__ void start(const EvictParams &p, int n, int wave, int lane, uint32_t s, uint32_t h, u32x4 *numbers)
    {
        length = ((n + kSelectWaves - 1) / kSelectWaves + 255) & ~255;
        kept = length <= 256 * GROUPS;
        begin = (int64_t)wave * length < n ? wave * length : n;             // (n may be a few thousand below 2^31)
        end = n - begin < length ? n : begin + length;
        const int all = n - p.recent;
        lo = p.first > begin ? p.first : begin;
        hi = all < end ? all : end;
        row = p.from.table + (int64_t)s * p.from.table_row;
        weights = reinterpret_cast<const uint32_t *>(p.weights) + number_at<BY_SEQUENCE>(s, h, p.Hkv, 0, 0, 0, p.from, p.from_numbers);
        own = numbers + wave * (64 * GROUPS) + lane;
        if (!kept) return;
        constexpr int AT_ONCE = GROUPS < 4 ? GROUPS : 8;
#pragma unroll 1
        for (int j0 = begin; j0 < end; j0 += 256 * AT_ONCE) {
            u32x4 w[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) w[i] = look(p, j0 + 256 * i + 4 * lane);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (j0 + 256 * i < end) own[(j0 - begin) / 4 + 64 * i] = order(j0 + 256 * i, lane, w[i]);
        }
    }
    // f(the first lane's first key, the numbers of four) of every lane, 256 keys at a time in ascending order.
    template <typename F>
    __device__ __forceinline__ void each(const EvictParams &p, int lane, F &&f) const
    {
        if (kept) {
#pragma unroll 1
            for (int j0 = begin; j0 < end; j0 += 256) f(j0, own[(j0 - begin) / 4]);
        } else {
#pragma unroll 1
            for (int j0 = begin; j0 < end; j0 += 256) f(j0, order(j0, lane, look(p, j0 + 4 * lane)));
        }
    }
};

// Workgroup: a sequence and key head, runs of up to 256 * GROUPS keys in LDS.
template <int GROUPS, bool BY_SEQUENCE>
__global__ __launch_bounds__(kSelect) void sta_paged_select_kernel(EvictParams p)
{
    __shared__ u32x4 numbers[kSelect * GROUPS];
    __shared__ __attribute__((aligned(16))) uint32_t counts[4096];
    __shared__ uint32_t wave_sums[kSelectWaves], found[2], totals[2][kSelectWaves], few[kFewRows];
    const uint32_t s = sta::fast_div(blockIdx.x, p.by_Hkv), h = blockIdx.x - s * p.Hkv;
    const int n = uniform(used_of(s, p.from)), stay = n < p.keep ? n : p.keep, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    int32_t *kept = p.kept + (int64_t)blockIdx.x * p.keep;
    if (h == 0 && tid == 0) p.to_used[s] = stay;
    for (int j = stay + tid; j < p.keep; j += kSelect) kept[j] = -1;
    // Few rows are moved here, by the workgroup that knows which.
    const uint32_t lanes = p.row_lanes, shift = 31 - __builtin_clz(lanes | 1);
    if (n <= p.keep) {
        for (int j = tid; j < n; j += kSelect) kept[j] = j;
        if (lanes)
            for (uint32_t i = tid; i < (uint32_t)n << shift; i += kSelect) move_chunk<false, BY_SEQUENCE>(p, s, h, i >> shift, i >> shift, i & (lanes - 1));
        return;
    }
    auto stays = [&](uint32_t at, int j) __attribute__((always_inline)) {
        if (at >= (uint32_t)p.keep) return;
        kept[at] = j;
        if (lanes && at < kFewRows) few[at] = (uint32_t)j;
    };
    Run<GROUPS, BY_SEQUENCE> run;
    run.start(p, n, wave, lane, s, h, numbers);
    uint32_t need = (uint32_t)(p.keep - p.first - p.recent);        // of those that may go so many stay
    uint32_t least = need > 0 ? 0 : 0xffffffffu;                    // the bits that are known of the least one that does
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
        if (need == 0) break;
        const int shift = digit == 0 ? 20 : digit == 1 ? 10 : 0, bins = digit == 0 ? 4096 : 1024;
        if (digit == 0) *reinterpret_cast<u32x4 *>(&counts[4 * tid]) = u32x4{0, 0, 0, 0};
        else counts[tid] = 0;
        __syncthreads();
        run.each(p, lane, [&](int, u32x4 x) {
            if (digit > 0) {                                        // most groups have none, of the last digit above all
                bool any = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) any = any || (x[e] ^ least) >> (shift + 10) == 0;
                if (__builtin_amdgcn_ballot_w64(any) == 0) return;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (digit == 0) atomicAdd(&counts[x[e] >> 20], 1u);
                else if ((x[e] ^ least) >> (shift + 10) == 0) atomicAdd(&counts[(x[e] >> shift) & (bins - 1)], 1u);
            }
        });
        __syncthreads();
        // a thread has four bins or one, the first thread the highest: how many stand in those above?
        uint32_t own[4] = {0, 0, 0, 0};                             // the highest first
        if (digit == 0) {
            const u32x4 all = *reinterpret_cast<const u32x4 *>(&counts[4 * (kSelect - 1 - tid)]);
#pragma unroll
            for (int e = 0; e < 4; ++e) own[e] = all[3 - e];
        } else {
            own[0] = counts[kSelect - 1 - tid];
        }
        const uint32_t sum = own[0] + own[1] + own[2] + own[3], upto = scan64(sum);
        if (lane == 63) wave_sums[wave] = upto;
        __syncthreads();
        const uint32_t before = sum64(lane < wave ? wave_sums[lane] : 0);
        uint32_t above = before + upto - sum;
        if (above < need && above + sum >= need) {                  // one thread: in its bins the number that still has to stay is reached
            int at = 0;
            uint32_t there = own[0];
#pragma unroll
            for (int e = 1; e < 4; ++e)
                if (at == e - 1 && above + there < need) {
                    above += there;
                    there = own[e];
                    at = e;
                }
            found[0] = digit == 0 ? 4 * (kSelect - 1 - tid) + 3 - at : kSelect - 1 - tid;
            found[1] = above;
        }
        __syncthreads();
        least |= found[0] << shift;
        need -= found[1];
    }
    // `need` of those equal to `least`, the first ones, stay, and all above it.  A wave counts its own, and after those before it writes them down.
    auto always = [&](int j) { return j < run.end && (j < p.first || j >= n - p.recent); };
    uint32_t sures = 0, equals = 0;
    run.each(p, lane, [&](int j0, u32x4 x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sures += x[e] > least;
            equals += x[e] == least;
        }
        if (!run.inside(j0)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sures += always(j0 + 4 * lane + e);
        }
    });
    sures = sum64(sures);
    equals = sum64(equals);
    if (lane == 0) {
        totals[0][wave] = sures;
        totals[1][wave] = equals;
    }
    __syncthreads();
    uint32_t sures_before = sum64(lane < wave ? totals[0][lane] : 0), equals_before = sum64(lane < wave ? totals[1][lane] : 0);
    run.each(p, lane, [&](int j0, u32x4 x) {
        const int j = j0 + 4 * lane;
        const bool even = __builtin_amdgcn_ballot_w64(x[0] == least || x[1] == least || x[2] == least || x[3] == least) != 0;
        if (run.inside(j0) && !even) {
            uint32_t mine = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += x[e] > least;
            const uint32_t upto = scan64(mine);
            uint32_t place = sures_before + (equals_before < need ? equals_before : need) + upto - mine;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[e] > least) {
                    stays(place, j + e);
                    ++place;
                }
            sures_before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
            return;
        }
        bool sure[4], equal[4];
        uint32_t mine = 0;                                          // counts of both, at most 256 each
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sure[e] = x[e] > least || always(j + e);
            equal[e] = x[e] == least;
            mine += (sure[e] ? 1u : 0u) + (equal[e] ? 1u << 16 : 0u);
        }
        const uint32_t upto = scan64(mine), all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63), until = upto - mine;
        uint32_t place = sures_before + (until & 0xffff), rank = equals_before + (until >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t at = place + (rank < need ? rank : need);
            if (sure[e] || (equal[e] && rank < need)) stays(at, j + e);
            place += sure[e];
            rank += equal[e];
        }
        sures_before += all & 0xffff;
        equals_before += all >> 16;
    });
    if (!lanes) return;
    __syncthreads();
    for (uint32_t i = tid; i < (uint32_t)p.keep << shift; i += kSelect) move_chunk<false, BY_SEQUENCE>(p, s, h, i >> shift, (uint32_t)bound_of((int)few[i >> shift], 0, n - 1), i & (lanes - 1));
}

// One row a lane: two and four at once, whose addresses and data leave room for fewer waves, took 86 and 96 us where one takes 81 (24 sequences, 8 heads, 2048 rows each).
template <int D, bool STREAM, bool BY_SEQUENCE>
__global__ __launch_bounds__(256) void sta_paged_move_kernel(EvictParams p)
{
    constexpr int LPR = D / 8, ROWS = 256 / LPR;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_blocks), block = blockIdx.x - item * p.by_blocks.d;      // (sequence, key head), rows
    const uint32_t s = sta::fast_div(item, p.by_Hkv), h = item - s * p.Hkv;
    const int n = used_of(s, p.from), stay = n < p.keep ? n : p.keep, j = (int)block * ROWS + (int)(threadIdx.x / LPR);
    if (j >= stay) return;
    move_chunk<STREAM, BY_SEQUENCE>(p, s, h, (uint32_t)j, (uint32_t)bound_of(p.kept[(int64_t)item * p.keep + j], 0, n - 1), threadIdx.x % LPR);
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
    if (!numbers_fit(*cache, S)) return STA_ERR_SHAPE;
    if (S == 0 || tokens == 0 || max_new == 0 || room_of(*cache) == 0) return STA_OK;
    if (!cu) return STA_ERR_NULL;
    if (((uintptr_t)cu | (uintptr_t)weights) & 3) return STA_ERR_SHAPE;
    if (S > 65535) return STA_ERR_SHAPE;
    if (rows_overlap(cache->k, cache->v, (int)cache->pages, cache->page_size, D)) return STA_ERR_ALIAS;
    const uint64_t w_bytes = number_bytes(*cache, S), cu_bytes = ((uint64_t)S + 1) * sizeof(int32_t);
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
    p.numbers = key_numbers_of(*cache);
    p.weights = weights;
    p.by_chunks = sta::fast_div_of(2 * Hkv * (D / 8));
    p.tokens = (uint32_t)tokens;
    p.max_new = (uint32_t)max_new;
    p.Hkv = Hkv;
    // Two rounds of all lanes a workgroup (four: 5.2 us where two take 4.3, four sequences of 512 tokens, 8 heads); of a sequence as many workgroups as its longest may need, or as 16384
    // workgroups in all allow, which then go around.
    p.each = 512 / p.by_chunks.d > 0 ? 512 / p.by_chunks.d : 1;
    const int64_t longest = max_new < tokens ? max_new : tokens, want = (longest + p.each - 1) / p.each, most = S < 16384 ? 16384 / S : 1;
    p.per_seq = (uint32_t)(want < most ? want : most);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    // What does not fit the caches goes past them: 12,366 tokens of 8 heads from float32 29.8 -> 24.4 us.  What fits is read from there by the attention that follows: 2048 tokens and their
    // attention, 32 heads over 8, 63.6 us, 67.1 with stores past the caches.
    const bool past = 4 * tokens * Hkv * D > kCaches;
    auto launch = [&](auto d, auto f32, auto streamed) {
        return sta::launch_kernel(sta_paged_append_kernel<decltype(d)::value, decltype(f32)::value, decltype(streamed)::value>, dim3(p.per_seq, S), dim3(256), stream, p);
    };
    auto by_type = [&](auto d, auto streamed) { return k->dtype == STA_F32 ? launch(d, std::true_type{}, streamed) : launch(d, std::false_type{}, streamed); };
    auto by_size = [&](auto d) { return past ? by_type(d, std::true_type{}) : by_type(d, std::false_type{}); };
    const hipError_t e = D == 64 ? by_size(std::integral_constant<int, 64>{}) : by_size(std::integral_constant<int, 128>{});
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
        if ((int64_t)c->page_size * Hkv > 0xffffffff || !numbers_fit(*c, S)) return STA_ERR_SHAPE;
    if (S == 0) return STA_OK;
    const uint64_t w_bytes = number_bytes(*cache, S), to_bytes = into_weights ? number_bytes(*into, S) : 0;
    if ((!weights && w_bytes > 0) || (!kept && keep > 0)) return STA_ERR_NULL;
    if (((uintptr_t)weights | (uintptr_t)into_weights | (uintptr_t)kept) & 3) return STA_ERR_SHAPE;
    const int64_t rows = 2048 / D, blocks = (keep + rows - 1) / rows, items = (int64_t)S * Hkv;
    constexpr int64_t most_selects = (1 << 22) - 1;         // of 1024 lanes
    if (items > most_selects || items * blocks > kMostWorkgroups) return STA_ERR_SHAPE;
    const uint64_t kept_bytes = (uint64_t)items * keep * sizeof(int32_t);
    if (rows_overlap(into->k, into->v, (int)into->pages, into->page_size, D) || pools_meet(*cache, *into, D)) return STA_ERR_ALIAS;
    // by page a number moves with its row, to where none is read; by sequence the numbers of a row of one array would move to where others are still to be read
    const bool one = into_weights == weights && cache->pages == into->pages && cache->page_size == into->page_size && same_rows(cache->k, into->k) && same_rows(cache->v, into->v) &&
                     !cache->numbers_by_sequence && !into->numbers_by_sequence;
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
    p.from_numbers = key_numbers_of(*cache);
    p.to_numbers = key_numbers_of(*into);
    p.weights = weights;
    p.to_weights = into_weights;
    p.kept = kept;
    p.to_used = into->used;
    p.Hkv = Hkv;
    p.keep = keep;
    p.first = first;
    p.recent = recent;
    p.by_Hkv = sta::fast_div_of(Hkv);
    // Up to 64 KB of a head's rows: three sequences, 4 heads of 64, 128 rows 7.0 us in one launch, 8.8 in two.
    const bool pools = into->pages > 0 && cache->pages > 0, here = pools && (int64_t)keep * D <= 64 * (int64_t)kFewRows;
    p.row_lanes = here ? D / 8 : 0;
    p.page_weights = (uint32_t)cache->page_size * Hkv;
    p.fours = (cache->numbers_by_sequence ? p.from_numbers.row : (int64_t)cache->page_size) % 4 == 0 && ((uintptr_t)weights & 15) == 0;
    p.by_blocks = sta::fast_div_of(blocks > 0 ? (uint32_t)blocks : 1);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto launch = [&](auto by) {
        constexpr bool BY = decltype(by)::value;
        // Up to 8192 keys two workgroups fit a CU, up to 32,768 one.  By the table's room, as the lengths stand on the device: short sequences in wide tables take 0 to 4 % longer (128 sequences
        // of 500 keys, 8 heads of 64, to 100 keys 28.0 and 29.2 us; 24 of 8000 to 500 25.2 both).
        hipError_t e = p.from.room <= 8 * kSelect ? sta::launch_kernel(sta_paged_select_kernel<2, BY>, dim3((uint32_t)items), dim3(kSelect), stream, p)
                                                  : sta::launch_kernel(sta_paged_select_kernel<8, BY>, dim3((uint32_t)items), dim3(kSelect), stream, p);
        if (e != hipSuccess || keep == 0 || !pools || here) return e;
        const dim3 grid((uint32_t)(items * blocks)), block(256);
        const bool past = (__int128)4 * items * keep * D > kCaches;
        if (D == 64) return past ? sta::launch_kernel(sta_paged_move_kernel<64, true, BY>, grid, block, stream, p) : sta::launch_kernel(sta_paged_move_kernel<64, false, BY>, grid, block, stream, p);
        return past ? sta::launch_kernel(sta_paged_move_kernel<128, true, BY>, grid, block, stream, p) : sta::launch_kernel(sta_paged_move_kernel<128, false, BY>, grid, block, stream, p);
    };
    const hipError_t e = cache->numbers_by_sequence || into->numbers_by_sequence ? launch(std::true_type{}) : launch(std::false_type{});
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}
