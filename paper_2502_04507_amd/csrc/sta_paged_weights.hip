// The attention weight that every key of a cache in pages gathers: w_j = decay before_j + sum over the rows that see j of exp(scale q . k_j - lse).
//
// S = Q K^T on v_mfma_f32_16x16x32_bf16 with the keys as columns, so that a lane owns a key: it adds up what it has of the key's column row block after
// row block, and the four lanes of a key are joined once, at the end.  The log sums are given, so there is no running maximum, no order among workgroups and nothing to
// join between them: a workgroup has all rows of its keys.  64 keys a wave stay in registers.
//
// Roundings.  Products of bf16 numbers are exact, scores, exponents and sums fp32: the sum of a stage's eight values is a tree, sixteen stages go into one sum, and
// those into the key's.
//
// sta_paged_few_weights_kernel   at most 16 or 32 rows per sequence and key head: rows and keys straight from memory to registers, no LDS.
// sta_paged_weights_kernel       more: stages of 32 rows go through LDS, shared by the waves along the keys; small launches cut the rows among a workgroup's waves.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_paged.h"
#include "sta_staged.h"

namespace {

constexpr int kKeys = 64;               // of a wave: four columns of 16

struct WeightsParams {
    PackedRows q;
    const float *lse;                   // [Hq, tokens]
    const int32_t *cu;
    PagedCache c;
    const float *before;                // or null
    float *weights;
    float decay, scale_log2e;
    uint32_t S, tokens, Hkv, g;
    int32_t max_q, max_k;
    sta::FastDiv by_g, by_Hkv, by_tiles;
    uint32_t causal;
};

struct WeightsSeq {
    int q0, lq, lk, rows;               // rows: of a key head, token after token
    // keys that the rows of token t see: the first keys_of(t)
    __device__ __forceinline__ int keys_of(int t, uint32_t causal) const
    {
        if (!causal) return lk;
        const int n = t + 1 + lk - lq;
        return n < 0 ? 0 : n < lk ? n : lk;
    }
};
__device__ __forceinline__ WeightsSeq weights_seq(uint32_t s, const WeightsParams &p)
{
    WeightsSeq q;
    q.q0 = bound_of(p.cu[s], 0, (int)p.tokens);
    q.lq = bound_of(p.cu[s + 1], q.q0, (int)p.tokens) - q.q0;
    q.lk = used_of(s, p.c);
    q.rows = (int)((uint32_t)(q.lq < p.max_q ? q.lq : p.max_q) * p.g);
    return q;
}

// The pages and slots of a lane's keys key0 + 16 col, and the fragments of their rows; keys that are not there are read as the last one.
template <int D>
__device__ __forceinline__ void load_keys(const WeightsParams &p, const int32_t *row, uint32_t kv, int key0, int lk, int lane, bf16x8 (&K)[4][D / 32])
{
    uint64_t at[4];
#pragma unroll
    for (int col = 0; col < 4; ++col) {
        const int key = key0 + 16 * col + (lane & 15);
        uint32_t slot;
        const uint32_t n = entry_of((uint32_t)(key < lk ? key : lk - 1), p.c, &slot);
        at[col] = place_of(page_inside(row[n], p.c), slot, p.c);
    }
    const char *head = p.c.k + (int64_t)kv * p.c.head + 16 * (lane >> 4);
#pragma unroll
    for (int col = 0; col < 4; ++col)
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) K[col][ks] = *reinterpret_cast<const bf16x8 *>(head + at[col] + 64 * ks);
}

// Row R of a key head: its token inside the sequence, and where its query row and its log sum are.
struct WeightRow {
    int token;
    const char *q;
    const float *lse;
};
__device__ __forceinline__ WeightRow weight_row(uint32_t R, const WeightsSeq &seq, uint32_t kv, const WeightsParams &p)
{
    const uint32_t t = sta::fast_div(R, p.by_g), h = kv * p.g + (R - t * p.g);
    const int64_t token = seq.q0 + (int64_t)t;
    return {(int)t, p.q.data + token * p.q.token + (int64_t)h * p.q.head, p.lse + (int64_t)h * p.tokens + token};
}
// What is taken from a row's exponents: infinity, which leaves 0 of every score, where it saw no key.  The bits are looked at, and kept from becoming a comparison of
// numbers again, which is compiled as if there were no NaN.
__device__ __forceinline__ float offset_of(float lse)
{
    uint32_t bits = __float_as_uint(lse);
    asm volatile("" : "+v"(bits));
    return bits == 0xff800000u ? INFINITY : lse * 1.4426950408889634f;
}

// A lane's key among the wave's 64 is 16 (lane / 16) + lane % 16: its sum goes to its place.
__device__ __forceinline__ void store_weights(const WeightsParams &p, const int32_t *row, uint32_t kv, int key0, int lk, int lane, const float (&sum)[4])
{
    float mine = 0.f;
#pragma unroll
    for (int col = 0; col < 4; ++col) {
        const float all = quad_lane_sum(sum[col]);
        mine = lane >> 4 == col ? all : mine;
    }
    const int key = key0 + lane;
    if (key >= lk || key >= p.max_k) return;
    uint32_t slot;
    const int page = row[entry_of((uint32_t)key, p.c, &slot)];
    if (page < 0 || page >= (int)p.c.pages) return;
    const int64_t at = ((int64_t)page * p.Hkv + kv) * p.c.by_page.d + slot;
    p.weights[at] = p.before ? fmaf(p.before[at], p.decay, mine) : mine;
}

// Workgroup (sequence, 256 keys, key head).
template <int D, int RB>
__global__ __launch_bounds__(256) void sta_paged_few_weights_kernel(WeightsParams p)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g4 = lane >> 4;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t s = sta::fast_div(item, p.by_tiles), tile = item - s * p.by_tiles.d;
    const WeightsSeq seq = weights_seq(s, p);
    const int key0 = ((int)tile * 4 + wave) * kKeys;
    if (key0 >= seq.lk) return;
    const int32_t *row = p.c.table + (int64_t)s * p.c.table_row;
    bf16x8 K[4][D / 32], Q[RB][D / 32];
    float offset[RB][4], sum[4] = {0.f, 0.f, 0.f, 0.f};
    int sees[RB][4];
    load_keys<D>(p, row, kv, key0, seq.lk, lane, K);
    const int rows = seq.rows < 16 * RB ? seq.rows : 16 * RB;
    if (rows > 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int R = 16 * rb + (lane & 15);
            const char *from = weight_row((uint32_t)(R < rows ? R : rows - 1), seq, kv, p).q + 16 * g4;
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) Q[rb][ks] = *reinterpret_cast<const bf16x8 *>(from + 64 * ks);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int mine = 16 * rb + 4 * g4 + r;
                const WeightRow w = weight_row((uint32_t)(mine < rows ? mine : rows - 1), seq, kv, p);
                offset[rb][r] = offset_of(*w.lse);
                sees[rb][r] = mine < rows ? seq.keys_of(w.token, p.causal) : 0;
            }
        }
#pragma unroll
        for (int col = 0; col < 4; ++col)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                floatx4 S = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < D / 32; ++ks) S = mfma_16x16x32(Q[rb][ks], K[col][ks], S);
                const int key = key0 + 16 * col + (lane & 15);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(S[r], p.scale_log2e, -offset[rb][r]));
                    sum[col] += key < sees[rb][r] ? e : 0.f;
                }
            }
    }
    store_weights(p, row, kv, key0, seq.lk, lane, sum);
}

// Workgroup (sequence, KW * 64 keys, key head): KW waves next to each other along the keys, RG = 4 / KW groups of them that take the stages of 32 rows in turn.
template <int D, int KW>
__global__ __launch_bounds__(256, 2) void sta_paged_weights_kernel(WeightsParams p)
{
    constexpr int RG = 4 / KW, KEYS = KW * kKeys, FOLD = 16;
    using L = StagedRows<D>;
    constexpr int PER_WAVE = L::Groups / KW > 0 ? L::Groups / KW : 1;       // DMA instructions of a wave for a stage
    constexpr int ROWS_AT = L::Tile, STAGE = L::Tile + 2 * kSub * 4;        // rows, their offsets, how many keys they see
    __shared__ __attribute__((aligned(1024))) char smem[RG * 2 * STAGE];
    __shared__ float joined[RG > 1 ? RG : 1][KEYS][4];
    const int lane = threadIdx.x & 63, all_waves = uniform(threadIdx.x >> 6), g4 = lane >> 4;
    const int rg = all_waves / KW, wave = all_waves % KW;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t s = sta::fast_div(item, p.by_tiles), tile = item - s * p.by_tiles.d;
    WeightsSeq seq = weights_seq(s, p);
    seq.q0 = uniform(seq.q0);
    seq.lq = uniform(seq.lq);
    seq.lk = uniform(seq.lk);
    seq.rows = uniform(seq.rows);
    const int tile0 = (int)tile * KEYS, key0 = tile0 + wave * kKeys;
    if (tile0 >= seq.lk) return;
    const int32_t *row = p.c.table + (int64_t)s * p.c.table_row;
    // the rows before token first_token see no key of the tile, those from whole_token on see all
    const int last = (tile0 + KEYS < seq.lk ? tile0 + KEYS : seq.lk) - 1, ahead = seq.lk - seq.lq;
    const int first_token = !p.causal || tile0 <= ahead ? 0 : tile0 - ahead, whole_token = !p.causal || last <= ahead ? 0 : last - ahead;
    const int step0 = (int)((int64_t)first_token * p.g < seq.rows ? first_token * (int)p.g / kSub : (seq.rows + kSub - 1) / kSub);
    const int steps_end = (seq.rows + kSub - 1) / kSub;
    const int64_t whole_row = (int64_t)whole_token * p.g;
    const int masked_end = (int)(whole_row < seq.rows ? (whole_row + kSub - 1) / kSub : steps_end);

    char *own = smem + rg * 2 * STAGE;
    float lse_next = 0.f;
    int sees_next = 0;
    auto issue = [&](int stage, int step) __attribute__((always_inline)) {
        if (step >= steps_end) return;
        const int first = step * kSub;
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int group = PER_WAVE * wave + i;
            if (L::Groups / KW == 0 && group >= L::Groups) break;
            const int R = first + group * L::GroupRows + lane / (D / 8);
            const char *from = weight_row((uint32_t)(R < seq.rows ? R : seq.rows - 1), seq, kv, p).q;
            const int pos = lane % (D / 8), r = lane / (D / 8);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + ((pos ^ L::turn(r)) << 4)), STA_LDS_PTR(own + stage * STAGE + group * L::Group), 16,
                                             0, 0);
        }
        if (wave == 0 && lane < kSub) {
            const int R = first + lane;
            const WeightRow w = weight_row((uint32_t)(R < seq.rows ? R : seq.rows - 1), seq, kv, p);
            lse_next = R < seq.rows ? *w.lse : -INFINITY;
            sees_next = R < seq.rows ? seq.keys_of(w.token, p.causal) : 0;
        }
    };
    issue(0, step0 + rg);
    bf16x8 K[4][D / 32];
    load_keys<D>(p, row, kv, key0, seq.lk, lane, K);
    const uint32_t base = (uint32_t)(uintptr_t)own, q_addr = L::address(base, lane), row_addr = base + ROWS_AT + 16 * g4;
    const float c = p.scale_log2e;
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, part[4] = {0.f, 0.f, 0.f, 0.f};
    int folded = 0;
    auto step = [&](auto stage_c, int at) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage_c)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (wave == 0 && lane < kSub) {
            *reinterpret_cast<float *>(own + ST * STAGE + ROWS_AT + 4 * lane) = offset_of(lse_next);
            *reinterpret_cast<int *>(own + ST * STAGE + ROWS_AT + 4 * kSub + 4 * lane) = sees_next;
        }
        __syncthreads();
        issue(ST ^ 1, at + RG);
        if (at < steps_end && key0 < seq.lk) {
            floatx4 S[2][4];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int col = 0; col < 4; ++col) S[rb][col] = floatx4{0.f, 0.f, 0.f, 0.f};
            bf16x8 o0 = ds_read_b128_at<ST * STAGE>(row_addr), o1 = ds_read_b128_at<ST * STAGE + 64>(row_addr);
            bf16x8 l0 = ds_read_b128_at<ST * STAGE + 4 * kSub>(row_addr), l1 = ds_read_b128_at<ST * STAGE + 4 * kSub + 64>(row_addr);
            rows_times_resident<D, ST * STAGE, 4, 4>(q_addr, K, S);
            lds_wait2<0>(o0, o1);
            lds_wait2<0>(l0, l1);
            typedef int intx4 __attribute__((ext_vector_type(4)));
            const floatx4 offset[2] = {__builtin_bit_cast(floatx4, o0), __builtin_bit_cast(floatx4, o1)};
            const intx4 sees[2] = {__builtin_bit_cast(intx4, l0), __builtin_bit_cast(intx4, l1)};
            const bool masked = at < masked_end;
#pragma unroll
            for (int col = 0; col < 4; ++col) {
                float e[2][4];
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) e[rb][r] = __builtin_amdgcn_exp2f(fmaf(S[rb][col][r], c, -offset[rb][r]));
                if (masked) {
                    const int key = key0 + 16 * col + (lane & 15);
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) e[rb][r] = key < sees[rb][r] ? e[rb][r] : 0.f;
                }
                part[col] += ((e[0][0] + e[0][1]) + (e[0][2] + e[0][3])) + ((e[1][0] + e[1][1]) + (e[1][2] + e[1][3]));
            }
            if (++folded == FOLD) {
                folded = 0;
#pragma unroll
                for (int col = 0; col < 4; ++col) {
                    sum[col] += part[col];
                    part[col] = 0.f;
                }
            }
        }
    };
    const int n_steps = (steps_end - step0 + RG - 1) / RG;          // of every group
#pragma unroll 1
    for (int i = 0; i < n_steps; i += 2) {
        step(std::integral_constant<int, 0>{}, step0 + rg + RG * i);
        if (i + 1 < n_steps) step(std::integral_constant<int, 1>{}, step0 + rg + RG * (i + 1));
    }
#pragma unroll
    for (int col = 0; col < 4; ++col) sum[col] += part[col];
    if constexpr (RG > 1) {                                         // the groups' sums, in ascending order
#pragma unroll
        for (int col = 0; col < 4; ++col) joined[rg][wave * kKeys + 16 * col + (lane & 15)][g4] = sum[col];
        __syncthreads();
        if (rg > 0) return;
#pragma unroll
        for (int col = 0; col < 4; ++col) {
            sum[col] = 0.f;
#pragma unroll
            for (int g = 0; g < RG; ++g) sum[col] += joined[g][wave * kKeys + 16 * col + (lane & 15)][g4];
        }
    }
    if (key0 < seq.lk) store_weights(p, row, kv, key0, seq.lk, lane, sum);
}

struct WeightsPlan {
    int few;                            // blocks of 16 rows, 0: stages
    int along;                          // waves of a workgroup along the keys
    int64_t tiles, workgroups;
};
WeightsPlan weights_plan(int S, int Hkv, int64_t rows, int max_k)
{
    const int64_t cus = sta::compute_units(), heads = (int64_t)S * Hkv;
    auto tiles = [&](int64_t keys) { return (max_k + keys - 1) / keys; };
    WeightsPlan plan = {};
    plan.workgroups = heads;
    if (heads > kMostWorkgroups) return plan;               // too many whatever the tiles are
    plan.few = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
    plan.along = plan.few || tiles(256) * heads >= 2 * cus ? 4 : tiles(128) * heads >= 2 * cus ? 2 : 1;
    plan.tiles = tiles(64 * plan.along);
    plan.workgroups = plan.tiles * heads;
    return plan;
}

template <int D>
hipError_t launch_weights(const WeightsParams &p, const WeightsPlan &plan, hipStream_t stream)
{
    const dim3 grid((uint32_t)plan.workgroups), block(256);
    if (plan.few == 1) return sta::launch_kernel(sta_paged_few_weights_kernel<D, 1>, grid, block, stream, p);
    if (plan.few == 2) return sta::launch_kernel(sta_paged_few_weights_kernel<D, 2>, grid, block, stream, p);
    if (plan.along == 4) return sta::launch_kernel(sta_paged_weights_kernel<D, 4>, grid, block, stream, p);
    if (plan.along == 2) return sta::launch_kernel(sta_paged_weights_kernel<D, 2>, grid, block, stream, p);
    return sta::launch_kernel(sta_paged_weights_kernel<D, 1>, grid, block, stream, p);
}

}  // namespace

extern "C" int sta_paged_weights(const sta_head_rows *q, const float *lse, int64_t tokens_q, const int32_t *cu_q, const sta_paged_cache *cache, int S, int max_q,
                                 int max_k, int D, int causal, float scale, const float *before, float decay, float *weights, void *hip_stream)
{
    if (!q || !cache) return STA_ERR_NULL;
    if (S < 0 || tokens_q < 0 || max_q < 0 || max_k < 0 || tokens_q > kMostTokens) return STA_ERR_SHAPE;
    const uint32_t decay_bits = __builtin_bit_cast(uint32_t, decay);
    if ((D != 64 && D != 128) || !scale_of(scale, D, false, &scale) || (decay_bits & 0x7fffffffu) >= 0x7f800000u) return STA_ERR_UNSUPPORTED;
    if (int rc = sta::packed_check(q, tokens_q, 0, D, false)) return rc;
    if (int rc = paged_check(cache, S, D, false)) return rc;
    const int Hkv = cache->k.heads;
    if (q->heads % Hkv || tokens_q * q->heads > kMostTokens) return STA_ERR_SHAPE;
    if ((__int128)cache->pages * cache->page_size * Hkv > (__int128)1 << 60) return STA_ERR_SHAPE;
    const int64_t room = room_of(*cache);
    if (max_k > room) max_k = (int)room;
    if (S == 0 || max_k == 0) return STA_OK;
    if (!cu_q || !weights || (!lse && tokens_q > 0)) return STA_ERR_NULL;
    if (((uintptr_t)cu_q | (uintptr_t)lse | (uintptr_t)before | (uintptr_t)weights) & 3) return STA_ERR_SHAPE;
    const WeightsPlan plan = weights_plan(S, Hkv, (int64_t)max_q * (q->heads / Hkv), max_k);
    if (plan.workgroups > kMostWorkgroups) return STA_ERR_SHAPE;
    const uint64_t w_bytes = (uint64_t)cache->pages * cache->page_size * Hkv * sizeof(float), lse_bytes = (uint64_t)tokens_q * q->heads * sizeof(float);
    if (rows_meet(*q, 1, tokens_q, D, weights, w_bytes) || meets_pages(*cache, D, weights, w_bytes) || meets_table(*cache, S, nullptr, 0, 0, D, weights, w_bytes) ||
        ranges_meet(weights, w_bytes, lse, lse_bytes) || ranges_meet(weights, w_bytes, cu_q, ((uint64_t)S + 1) * sizeof(int32_t)))
        return STA_ERR_ALIAS;
    if (decay_bits << 1 == 0) before = nullptr;             // what it holds then is not looked at
    if (before != weights && ranges_meet(weights, w_bytes, before, w_bytes)) return STA_ERR_ALIAS;
    WeightsParams p = {};
    p.q = packed_rows_of(*q);
    p.lse = lse;
    p.cu = cu_q;
    p.c = paged_cache_of(*cache);
    p.before = before;
    p.weights = weights;
    p.decay = decay;
    p.scale_log2e = scale * 1.4426950408889634f;
    p.S = S;
    p.tokens = (uint32_t)tokens_q;
    p.Hkv = Hkv;
    p.g = q->heads / Hkv;
    p.max_q = max_q;
    p.max_k = max_k;
    p.by_g = sta::fast_div_of(p.g);
    p.by_Hkv = sta::fast_div_of(p.Hkv);
    p.causal = causal != 0;
    p.by_tiles = sta::fast_div_of((uint32_t)plan.tiles);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = D == 64 ? launch_weights<64>(p, plan, stream) : launch_weights<128>(p, plan, stream);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}
