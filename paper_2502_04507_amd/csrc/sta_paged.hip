// Softmax attention over a cache in pages: the kernels of sta_packed_forward.h with keys that are looked up in a table.
//
// A lane looks up one row of the next stage while the present one is on its way (where that costs the walk registers, places wait in LDS: TileKeys): the entry of the table, as a load into
// a register, is older than the stage's DMA, so the wait for a stage covers it.  Where every group of rows of a DMA instruction (4 rows of 128 channels, 8 of 64) lies in one page, its place goes from
// the lane that has it into scalar registers, two v_readlane a group, and the DMA is as that of packed sequences; where a page ends inside a group, or the keys inside a
// stage, every lane gets its row's place from the lane that has it.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_paged.h"
#include "sta_packed_forward.h"

namespace {

struct PagedParams : PackedParams {     // k and v: the pool; k.token and k.head as there
    PagedCache c;
    uint32_t whole_groups;              // no page ends inside a group of rows
    sta::FastDiv by_slots;
    uint32_t at_once;                   // not 0: how many workgroups of tiles of 128 rows are there at once, where such are cut
};

// The keys of a sequence have no first row: its number stands in k0.
__device__ __forceinline__ PackedSeq seq_of(uint32_t s, const PagedParams &p)
{
    PackedSeq q;
    q.q0 = bound_of(p.cu_q[s], 0, (int)p.tokens_q);
    q.lq = bound_of(p.cu_q[s + 1], q.q0, (int)p.tokens_q) - q.q0;
    q.k0 = (int)s;
    q.lk = used_of(s, p.c);
    return q;
}

// Where tiles of 128 rows are cut, the size of the parts is chosen here, from the lengths: such that as many parts as there may be at once, three a CU, take all walks, or nearly so.  The launch has up to twice as many
// workgroups.  Those that find nothing to do are the last ones, part after part: between the others they leave some CUs with three and others with none (544 tokens below 208 us).  us,
// parts of the launch's size, about six a CU | this; 32 heads over 8 of 128 channels, one chunk of 416, 544, 640, 960 tokens on 16,384 keys 143, 170, 180, 271 | 126, 162, 188, 253; two of 256 on
// 32,768 and 20,001  248 | 236; 100, 60 and 350 on 9000, 16,000 and 30,000  242 | 238; 15 heads over 5, 700 on 20,001  156 | 127; 40 over 8, 300 and 200 on 12,000 and 9000  149 | 129; of 64
// channels, two of 256 as above 146 | 144, 24 heads, 333 on 20,000  74 | 73.
__device__ __forceinline__ uint32_t rank_of(uint32_t item, const PagedParams &p, uint32_t *part)
{
    if (p.at_once == 0) return rank_of(item, static_cast<const PackedParams &>(p), part);
    *part = sta::fast_div(item, p.by_slots);
    return item - *part * p.by_slots.d;
}
__device__ __forceinline__ uint32_t part_subs_of(const PagedParams &p, int lane)
{
    constexpr uint32_t MOST = 1 << 19;          // products with a part's number stay in 32 bits, whatever the lengths are
    if (p.at_once == 0) return p.part_subs;
    uint32_t tiles = 0, subs = 0;
    if (lane < (int)p.S) {
        const PackedSeq seq = seq_of((uint32_t)lane, p);
        tiles = ((uint32_t)seq.worked(p) * p.g + 127) / 128 * p.Hkv;
        subs = ((uint32_t)seq.lk + kSub - 1) / kSub;
        subs = subs < MOST ? subs : MOST;
    }
    uint32_t each = ((sum64(tiles * subs) + p.at_once - 1) / p.at_once + 1) & ~1u;      // (whole stages of two sub-blocks)
    each = each < MOST ? each : MOST;
    each = each > p.part_subs ? each : p.part_subs;
#pragma unroll 1
    for (int i = 0; i < 16 && sum64(tiles * ((subs + each - 1) / each)) > p.at_once; ++i) each += (each / 32 + 2) & ~1u;
    return each;
}

template <int D>
struct KeysOf<PagedParams, D> {
    static constexpr int LPR = D / 8, GR = Staged<D>::GroupRows;
    const char *kh, *vh;
    const int32_t *row;                 // of the table
    PackedDma<D, true> k_dma;
    PackedDma<D, false> v_dma;
    int entry;                          // of the lane's row of the next stage, and its place in the page, in bytes
    uint32_t slot;
    __device__ __forceinline__ void start(const PagedParams &p, const PackedSeq &seq, uint32_t kv, int lane)
    {
        kh = p.c.k + (int64_t)kv * p.c.head;
        vh = p.c.v + (int64_t)kv * p.c.head;
        row = p.c.table + (int64_t)seq.k0 * p.c.table_row;
        k_dma.start(lane, p.c.token);
        v_dma.start(lane, p.c.token);
        entry = 0;
        slot = 0;
    }
    // The entries for the rows from sub-block `sub` on; rows beyond the last key have the last key's.  There are keys.
    template <int SUBS>
    __device__ __forceinline__ void look_up(const PagedParams &p, const PackedSeq &seq, int sub)
    {
        if (seq.lk <= 0) return;
        const int key = sub * kSub + (SUBS == 1 ? fresh_lane() & 31 : fresh_lane()), last = seq.lk - 1;
        uint32_t at;
        const uint32_t n = entry_of((uint32_t)(key < last ? key : last), p.c, &at);
        slot = at * p.c.token;
        entry = row[n];
    }
    template <int SUBS, int COUNT, int K_GROUP, int V_GROUP>
    __device__ __forceinline__ void bring(const PagedParams &p, const PackedSeq &seq, int sub, int next, int from, char *to, int v_at, int apart)
    {
        const uint64_t place = (uint64_t)page_inside(entry, p.c) * p.c.page + slot;
        const uint32_t lo = (uint32_t)place, hi = (uint32_t)(place >> 32);
        look_up<SUBS>(p, seq, next);
        if (__builtin_expect((sub + SUBS) * kSub <= seq.lk && p.whole_groups, 1)) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int i = 0; i < COUNT; ++i) {
                    const int r = u * kSub + (from + i) * GR;
                    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, r) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, r);
                    k_dma.bring_whole(kh + at, to + u * apart + (from + i) * K_GROUP);
                    v_dma.bring_whole(vh + at, to + u * apart + v_at + (from + i) * V_GROUP);
                }
            asm volatile("; whole" ::: "memory");
        } else {
            const int lane = fresh_lane();
#pragma unroll 1
            for (int u = 0; u < SUBS; ++u)
#pragma unroll 1
                for (int i = 0; i < COUNT; ++i) {
                    const int r = u * kSub + (from + i) * GR + lane / LPR;
                    const uint64_t at = (uint64_t)(uint32_t)__shfl((int)hi, r) << 32 | (uint32_t)__shfl((int)lo, r);
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(kh + at + k_dma.chunk_of(lane)),
                                                     STA_LDS_PTR(to + u * apart + (from + i) * K_GROUP), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(vh + at + v_dma.chunk_of(lane)),
                                                     STA_LDS_PTR(to + u * apart + v_at + (from + i) * V_GROUP), 16, 0, 0);
                }
            asm volatile("; part" ::: "memory");
        }
    }
    // Behind a wait that covers the entries: from here on the compiler has nothing to wait for at their use, where stages are on their way.
    __device__ __forceinline__ void settle() { asm volatile("" : "+v"(entry)); }
    __device__ __forceinline__ void bring_values(const PagedParams &p, const PackedSeq &seq, int first, char *dst) const
    {
        const int lane = fresh_lane(), key = first + lane / LPR, last = seq.lk - 1;
        uint32_t at;
        const uint32_t n = entry_of((uint32_t)(key < last ? key : last), p.c, &at);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(vh + place_of(page_inside(row[n], p.c), at, p.c) + v_dma.chunk_of(lane)),
                                         STA_LDS_PTR(dst), 16, 0, 0);
    }
};

// Tiles of 128 rows of 128 channels: a wave works out the places of what it brings in the next stages together and keeps them in LDS, those of groups of rows where no page ends inside one, else of every row.
// In registers, looked up a stage ahead as above, they cost the walk its own, whose reloads wait for the stage that is on its way: prompts of 8192 and 4097 tokens, 32 heads over 8, 684 us where
// packed keys take 554; this way 564 where those take 538.
// Where groups of waves take stages in turn registers are left, and a look into LDS before each stage costs more than it saves (12 heads over 4, 500, 1, 65, 1 and 578 tokens on 77 to 7097: 69 us, 73 this
// way; 8 heads of 128, four of 480 on 2200: 33.6 and 34.6), and with 64 channels there is nothing between them.
template <>
struct TileKeys<PagedParams, 128, 1> : KeysOf<PagedParams, 128> {
    using Base = KeysOf<PagedParams, 128>;
    static constexpr int PLACES = 512, WAVES = 4, OF_STAGE = kSub / GR / WAVES, AT_ONCE = 4;        // of a wave, and its groups of a stage
    static_assert(PLACES % (64 * AT_ONCE) == 0 && PLACES % (OF_STAGE * GR) == 0, "");
    uint64_t *places;                           // a wave's own: no other looks at them
    int shift;                                  // log2 of its places of a stage
    __device__ __forceinline__ void start(const PagedParams &p, const PackedSeq &seq, uint32_t kv, int lane)
    {
        __shared__ uint64_t all[WAVES * PLACES];
        Base::start(p, seq, kv, lane);
        places = all + uniform(threadIdx.x >> 6) * PLACES;
        shift = __builtin_ctz(p.whole_groups ? OF_STAGE : OF_STAGE * GR);
    }
    template <int SUBS>
    __device__ __forceinline__ void look_up(const PagedParams &, const PackedSeq &, int) {}
    // Those of the wave's groups, the first of which is `from` in every stage, from sub-block `sub` on, as far as the keys go; behind the last key they are its own or its group's.  There are keys.
    __device__ __forceinline__ void fill(const PagedParams &p, const PackedSeq &seq, int sub, int from)
    {
        const int rows = p.whole_groups ? GR : 1, last = (seq.lk - 1) & -rows, lane = fresh_lane();       // rows of a place; the first of the last one's
#pragma unroll 1
        for (int x0 = 0; x0 < PLACES && ((int64_t)sub + (x0 >> shift)) * kSub < seq.lk; x0 += 64 * AT_ONCE) {
            int entry[AT_ONCE];
            uint32_t slot[AT_ONCE];
#pragma unroll
            for (int y = 0; y < AT_ONCE; ++y) {
                const int x = x0 + 64 * y + lane, stage = x >> shift;
                const int64_t r = ((int64_t)sub + stage) * kSub + from * GR + (x - (stage << shift)) * rows;
                const uint32_t n = entry_of((uint32_t)(r < last ? r : last), p.c, &slot[y]);
                entry[y] = row[n];
            }
#pragma unroll
            for (int y = 0; y < AT_ONCE; ++y) places[x0 + 64 * y + lane] = place_of(page_inside(entry[y], p.c), slot[y], p.c);
        }
    }
    // A place, from LDS at byte address at.
    static __device__ __forceinline__ uint64_t read_place(uint32_t at)
    {
        uint64_t x;
        asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(x) : "v"(at) : "memory");
        return x;
    }
    template <int SUBS, int COUNT, int K_GROUP, int V_GROUP>
    __device__ __forceinline__ void bring_turn(const PagedParams &p, const PackedSeq &seq, int sub, int i, int from, char *to, int v_at, int)
    {
        static_assert(SUBS == 1 && COUNT == OF_STAGE, "");
        const int turn = i & ((PLACES >> shift) - 1);
        if (turn == 0) fill(p, seq, sub, from);
        const uint32_t first = (uint32_t)(uintptr_t)places + (uint32_t)(turn << shift) * 8;
        const int lane = fresh_lane();
        if (__builtin_expect((sub + 1) * kSub <= seq.lk && p.whole_groups, 1)) {
            // the wave's groups' places, one in each of the first lanes
            const uint64_t mine = read_place(first + (uint32_t)(lane % COUNT) * 8);
            const int lo = (int)(uint32_t)mine, hi = (int)(mine >> 32);
            PackedDma<128, true> k_dma;         // worked out again, for registers
            PackedDma<128, false> v_dma;
            k_dma.start(lane, p.c.token);
            v_dma.start(lane, p.c.token);
#pragma unroll
            for (int n = 0; n < COUNT; ++n) {
                const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, n) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, n);
                k_dma.bring_whole(kh + at, to + (from + n) * K_GROUP);
                v_dma.bring_whole(vh + at, to + v_at + (from + n) * V_GROUP);
            }
            asm volatile("; whole" ::: "memory");
        } else {
#pragma unroll 1
            for (int n = 0; n < COUNT; ++n) {
                const int r = lane / LPR, inside = (from + n) * GR + r, left = seq.lk - 1 - sub * kSub;
                // rows beyond the last key: its
                const uint64_t at = p.whole_groups ? read_place(first + (uint32_t)n * 8) + (uint32_t)(inside < left ? r : left % GR) * p.c.token
                                                   : read_place(first + (uint32_t)(n * GR + r) * 8);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(kh + at + k_dma.chunk_of(lane)), STA_LDS_PTR(to + (from + n) * K_GROUP), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(vh + at + v_dma.chunk_of(lane)), STA_LDS_PTR(to + v_at + (from + n) * V_GROUP), 16, 0, 0);
            }
            asm volatile("; part" ::: "memory");
        }
    }
};

// As launches of packed sequences are cut, but where those are tiles of 64 rows by two groups that are not cut along the keys, and some walks are likely to be much longer than others (three quarters at
// most of the tokens that S sequences of max_q would have, and 96 sub-blocks of keys or more), or a CU has less than one of them (and 64 sub-blocks): then tiles of 32 rows by four groups, which walk half
// as long.  us, two groups | four | two, cut after 48 sub-blocks; heads / key heads x channels, new tokens on keys:
//   15/5 x 64, 333, 1, 2048, 65, 1, 578 on 1333, 4097, 2048, 3001, 77, 578   45 | 38 | 43       32/8 x 128, 100, 1, 1, 1, 700 on 2000, 5000, 3000, 8000, 700   100 | 55 | 49
//   16/16 x 64, 333, 1, 65, 1, 578 on 6333, 7097, 6001, 77, 3578             67 | 49 | 55       12/4 x 128, 500, 1, 65, 1, 578 on 6333, 7097, 6001, 77, 3578   87 | 68 | 74
//   8/8 x 128, three of 512 on 512, 1000, 3000                               42 | 26 | 31
// and where they stay: 40/8 x 128, 40 of 1 on 1000 and 300 on 1300  34 | 49 | 35; 32/8 x 128, four of 256 on 4096  80 | 124 | 117; 16 of 64 on 3000  64 | 128 | 97; 2048 on 4096  122 | 196 | 169.
bool paged_plan_of(int Hq, int Hkv, int D, int S, int64_t tokens_q, int max_q, int max_k, bool cut, PackedPlan *plan)
{
    if (!plan_of(Hq, Hkv, D, S, tokens_q, max_q, max_k, cut, plan)) return false;
    if (plan->few || plan->waves != 2 || plan->parts > 1) return true;
    const int64_t subs = ((int64_t)max_k + kSub - 1) / kSub, items = (int64_t)plan->slots * Hkv;
    const bool uneven = subs >= 96 && 4 * tokens_q <= 3 * (int64_t)S * max_q, sparse = subs >= 64 && items < sta::compute_units();
    if (!uneven && !sparse) return true;
    const int64_t slots = tiles_of(tokens_q, Hq / Hkv, S, max_q, 32);
    if (slots * Hkv > kMostWorkgroups) return true;
    plan->waves = 1;
    plan->slots = (uint32_t)slots;
    return true;
}

}  // namespace

extern "C" {

size_t sta_paged_workspace_bytes(int Hq, int Hkv, int D, int S, int64_t tokens_q, int max_q, int max_k)
{
    return sta_packed_workspace_bytes(Hq, Hkv, D, S, tokens_q, max_q, max_k);       // what is not cut there is not cut here
}

int sta_paged_forward(const sta_head_rows *q, const sta_head_rows *o, float *lse, int64_t tokens_q, const int32_t *cu_q, const sta_paged_cache *cache, int S,
                      int max_q, int max_k, int D, int causal, float scale, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!q || !o || !cache) return STA_ERR_NULL;
    if (S < 0 || tokens_q < 0 || max_q < 0 || max_k < 0 || tokens_q > kMostTokens) return STA_ERR_SHAPE;
    if ((D != 64 && D != 128) || !scale_of(scale, D, false, &scale)) return STA_ERR_UNSUPPORTED;
    if (int rc = sta::packed_check(q, tokens_q, 0, D, false)) return rc;
    if (int rc = sta::packed_check(o, tokens_q, q->heads, D, true)) return rc;
    if (int rc = paged_check(cache, S, D, false)) return rc;
    const int Hkv = cache->k.heads;
    if (q->heads % Hkv || tokens_q * q->heads > kMostTokens) return STA_ERR_SHAPE;
    if (S == 0 || tokens_q == 0 || max_q == 0) return STA_OK;
    if (!cu_q) return STA_ERR_NULL;
    if (((uintptr_t)cu_q | (uintptr_t)lse) & 3) return STA_ERR_SHAPE;
    const size_t lse_bytes = (size_t)tokens_q * q->heads * sizeof(float);
    if (rows_overlap(*o, tokens_q, *q, tokens_q, 1, D) || rows_in_pages(*cache, D, *o, tokens_q)) return STA_ERR_ALIAS;
    PackedPlan plan;
    if (!paged_plan_of(q->heads, Hkv, D, S, tokens_q, max_q, max_k, workspace != nullptr, &plan)) return STA_ERR_SHAPE;
    if (workspace && (((uintptr_t)workspace & 15) || workspace_bytes < plan.workspace() * sizeof(float))) return STA_ERR_WORKSPACE;
    const struct { const void *at; uint64_t bytes; } ranges[2] = {{workspace, workspace_bytes}, {lse, lse_bytes}};
    const PackedBounds bounds = {cu_q, nullptr, nullptr, S};
    for (const auto &w : ranges)
        if (rows_meet(*q, 1, tokens_q, D, w.at, w.bytes) || rows_meet(*o, 1, tokens_q, D, w.at, w.bytes) || meets_pages(*cache, D, w.at, w.bytes) ||
            bounds.meet(o, tokens_q, D, w.at, w.bytes) || meets_table(*cache, S, o, 1, tokens_q, D, w.at, w.bytes))
            return STA_ERR_ALIAS;
    if (ranges_meet(lse, lse_bytes, workspace, workspace_bytes)) return STA_ERR_ALIAS;
    PagedParams p = {};
    p.q = packed_rows_of(*q);
    p.o = packed_rows_of(*o);
    p.lse = lse;
    p.cu_q = cu_q;
    p.S = S;
    p.tokens_q = (uint32_t)tokens_q;
    p.max_q = max_q;
    p.max_k = max_k;
    p.Hkv = Hkv;
    p.g = q->heads / Hkv;
    p.by_g = sta::fast_div_of(p.g);
    p.by_Hkv = sta::fast_div_of(p.Hkv);
    p.by_parts = sta::fast_div_of(plan.parts);
    p.causal = causal != 0;
    p.scale = scale;
    p.scale_log2e = scale * 1.4426950408889634f;
    p.parts = plan.parts;
    p.part_subs = plan.part_subs;
    p.ws = static_cast<float *>(workspace);
    p.at_once = plan.parts > 1 && !plan.few && plan.waves == 4 && S <= 64 ? 3 * (uint32_t)sta::compute_units() : 0;
    p.by_slots = sta::fast_div_of(plan.slots > 0 ? plan.slots : 1);
    p.c = paged_cache_of(*cache);
    p.whole_groups = cache->page_size % (D == 128 ? Staged<128>::GroupRows : Staged<64>::GroupRows) == 0;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (D == 64) e = lse ? launch_packed<64, true>(p, plan, stream) : launch_packed<64, false>(p, plan, stream);
    else e = lse ? launch_packed<128, true>(p, plan, stream) : launch_packed<128, false>(p, plan, stream);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}

}  // extern "C"
