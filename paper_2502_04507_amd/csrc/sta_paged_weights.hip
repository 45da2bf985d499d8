// The attention weight that every key of a cache in pages gathers: w_j = decay before_j + sum over the rows that see j of exp(scale q . k_j - lse).
//
// S = Q K^T on v_mfma_f32_16x16x32_bf16 with the keys as columns, so that a lane owns a key: it adds up what it has of the key's column row block after
// row block, and the four lanes of a key are joined once, at the end.  The log sums are given, so there is no running maximum, no order among workgroups and nothing to
// join between them: a workgroup has all rows of its keys.  64 keys a wave stay in registers.
//
// Roundings.  Products of bf16 numbers are exact, scores, exponents and sums fp32: four values of a lane are a tree, those of 512 rows go into one sum, and those into the key's.
//
// sta_paged_few_weights_kernel   at most 16 or 32 rows per sequence and key head: rows and keys straight from memory to registers, no LDS.  Bound by memory: 48 tokens of 32 heads over 8
//                                on 1 to 16,384 keys 184 us, 4.7 TB/s (155 where nothing is written, though that is 12 of 870 MB; a kernel that only reads as much 125).  Numbers before are asked for behind the keys'
//                                rows and in a branch of their own: before them 190, inside the branch that finds their place 188, behind the sums 190.  Sums of 16 tiles held back and written
//                                together by workgroups that stay: 180, but 53 in place of 45 with 64 channels.
// sta_paged_weights_kernel       (and sta_paged_weights_rounds_kernel, its tiles in another order, the last ones halved)
//                                more: stages of 32 or 64 rows go through LDS, shared by the waves along the keys; small launches cut the rows among a workgroup's waves.  Bound by
//                                vector and matrix instructions, which hardly overlap (per 64 rows and 64 keys of a wave 1024 cycles of the matrix pipe, 64 exponentials of 8 cycles, as
//                                many multiply-adds and sums of 4): 2048 tokens of 32 heads over 8 of 128 channels on 16,384 keys 260 us, 990 TFLOP/s.  With stages of 32 rows 294 us, two stages
//                                in place of three 265, 32 keys a wave 315, 128 keys a workgroup 274 to 296; the order of the instructions in a stage changes nothing.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_paged.h"
#include "sta_staged.h"

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));


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
    uint32_t round;                     // tiles of a key head that are there at once, two a CU
    uint32_t even, g_shift;             // whether g is a power of two up to 32, and which
    KeyNumbers numbers;
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

// A wave's 16 NC keys from key0 on.  A lane has one of them, key0 + lane, to look up and to write; its number before and the fragments of the rows, 16 keys a column block, are asked for at once.
// Keys that are not there are read as the last one.
struct OwnKey {
    int64_t at;                         // of its number; below 0: none is written
    float before;
};
template <int D, int NC>
__device__ __forceinline__ OwnKey load_keys(const WeightsParams &p, uint32_t s, uint32_t kv, int key0, int lk, int lane, bf16x8 (&K)[NC][D / 32])
{
    const int mine = key0 + (NC < 4 ? lane % (16 * NC) : lane), key = mine < lk ? mine : lk - 1;
    uint32_t slot;
    const int page = p.c.table[(int64_t)s * p.c.table_row + entry_of((uint32_t)key, p.c, &slot)];
    const uint64_t place = place_of(page_inside(page, p.c), slot, p.c);
    const char *head = p.c.k + (int64_t)kv * p.c.head + 16 * (lane >> 4);
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const int from = 16 * col + (lane & 15);
        const uint64_t at = (uint64_t)(uint32_t)__shfl((int)(place >> 32), from) << 32 | (uint32_t)__shfl((int)place, from);
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) K[col][ks] = *reinterpret_cast<const bf16x8 *>(head + at + 64 * ks);
    }
    const bool there = lane < 16 * NC && mine < lk && mine < p.max_k && page >= 0 && page < (int)p.c.pages;
    OwnKey own = {there ? number_at(s, kv, p.Hkv, (uint32_t)mine, (uint32_t)page, slot, p.c, p.numbers) : -1, 0.f};
    if (own.at >= 0 && p.before) own.before = p.before[own.at];
    return own;
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

template <int NC>
__device__ __forceinline__ void store_weights(const WeightsParams &p, const OwnKey &own, int lane, const float (&sum)[NC])
{
    float mine = 0.f;
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const float all = quad_lane_sum(sum[col]);
        mine = lane >> 4 == col ? all : mine;
    }
    if (own.at >= 0) p.weights[own.at] = p.before ? fmaf(own.before, p.decay, mine) : mine;
}

// Workgroup (sequence, 64 NC keys, key head).
template <int D, int NC, int RB>
__global__ __launch_bounds__(256) void sta_paged_few_weights_kernel(WeightsParams p)
{
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g4 = lane >> 4;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t s = sta::fast_div(item, p.by_tiles), tile = item - s * p.by_tiles.d;
    const WeightsSeq seq = weights_seq(s, p);
    const int key0 = ((int)tile * 4 + wave) * (16 * NC);
    if (key0 >= seq.lk) return;
    bf16x8 K[NC][D / 32], Q[RB][D / 32];
    float offset[RB][4], sum[NC] = {};
    int sees[RB][4];
    const OwnKey own = load_keys<D, NC>(p, s, kv, key0, seq.lk, lane, K);
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
        for (int col = 0; col < NC; ++col)
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
    store_weights(p, own, lane, sum);
}

// Up to 64 sequences, a lane each: those with at least half as many rows as there may be come first, so that no long walk begins among the last workgroups (32 new tokens on 32,768
// keys and 512 on 20,001, 32 heads over 8: 106 us, 119 in the order of the sequences).
__device__ __forceinline__ uint32_t sequence_of_turn(uint32_t turn, int lane, const WeightsParams &p)
{
    const bool there = lane < (int)p.S, many = there && 2 * (int64_t)weights_seq(there ? lane : 0, p).lq >= p.max_q;
    const uint64_t first = __builtin_amdgcn_ballot_w64(many);
    uint32_t left = turn;
    uint64_t from = first;
    if (turn >= (uint32_t)__builtin_popcountll(first)) {
        left -= __builtin_popcountll(first);
        from = ~first;                          // (turn is below S, so no lane without a sequence is reached)
    }
    while (left-- > 0) from &= from - 1;
    return (uint32_t)__builtin_ctzll(from);
}

// Exponentials of a block of 16 rows, a column block of 16 keys: what the lane has of it is added up.
template <bool MASKED>
__device__ __forceinline__ float sum_of(const floatx4 &S, const floatx4 &offset, float c, int key, const intx4 &sees)
{
    float e[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        e[r] = __builtin_amdgcn_exp2f(fmaf(S[r], c, -offset[r]));
        if (MASKED) e[r] = key < sees[r] ? e[r] : 0.f;
    }
    return (e[0] + e[1]) + (e[2] + e[3]);
}

template <int PENDING>
__device__ __forceinline__ void lds_wait1(bf16x8 &a)
{
    asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(a) : "n"(PENDING));
}

// part[col] += the exponentials of BLOCKS blocks of 16 rows in the stage at AT of the addresses: their offsets stand at INFO of row_addr, how many keys they see SEES
// behind.  The exponentials of one block stand between the matrix instructions of the next, which take about as long.
template <int D, int NC, int BLOCKS, bool MASKED, int AT, int INFO, int SEES>
__device__ __forceinline__ void add_rows(uint32_t q_addr, uint32_t row_addr, const bf16x8 (&K)[NC][D / 32], float c, int key0, float (&part)[NC])
{
    constexpr int KS = D / 32, EACH = NC / KS > 0 ? NC / KS : 1;     // column blocks whose exponentials go with a k-step
    bf16x8 a[2][KS], o[2], l[2];
    floatx4 S[2][NC];
    auto read_info = [&](auto bc) {
        constexpr int b = decltype(bc)::value;
        o[b % 2] = ds_read_b128_at<INFO + 64 * b>(row_addr);
        if constexpr (MASKED) l[b % 2] = ds_read_b128_at<INFO + SEES + 64 * b>(row_addr);
    };
    auto read = [&](auto bc, auto kc) {
        constexpr int b = decltype(bc)::value, ks = decltype(kc)::value;
        a[b % 2][ks] = ds_read_b128_at<AT + (b / 2) * StagedRows<D>::Tile + (b % 2) * StagedRows<D>::Rows16 + ks * 64>(q_addr);
    };
    auto exponentials = [&](int b, int col) __attribute__((always_inline)) {
        part[col] += sum_of<MASKED>(S[b % 2][col], __builtin_bit_cast(floatx4, o[b % 2]), c, key0 + 16 * col, __builtin_bit_cast(intx4, l[b % 2]));
    };
    read_info(std::integral_constant<int, 0>{});
    static_for<0, KS>([&](auto kc) { read(std::integral_constant<int, 0>{}, kc); });
    static_for<0, BLOCKS>([&](auto bc) {
        constexpr int b = decltype(bc)::value;
        static_for<0, KS>([&](auto kc) {
            constexpr int ks = decltype(kc)::value;
            if constexpr (b + 1 < BLOCKS) {
                read(std::integral_constant<int, b + 1>{}, kc);
                lds_wait1<KS>(a[b % 2][ks]);                // (KS reads of the next block at most, so by the block's end its offsets are there as well)
            } else {
                lds_wait1<KS - 1 - ks>(a[b % 2][ks]);
            }
#pragma unroll
            for (int col = 0; col < NC; ++col) S[b % 2][col] = mfma_16x16x32(a[b % 2][ks], K[col][ks], ks == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : S[b % 2][col]);
            if constexpr (b > 0) {
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (EACH * ks + i < NC) exponentials(b - 1, EACH * ks + i);
#pragma unroll
                for (int col = 0; col < NC; ++col) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, EACH * (MASKED ? 20 : 12) / NC, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (b + 1 < BLOCKS) read_info(std::integral_constant<int, b + 1>{});
    });
    if constexpr (MASKED) lds_wait2<0>(o[(BLOCKS - 1) % 2], l[(BLOCKS - 1) % 2]);
    else lds_wait1<0>(o[(BLOCKS - 1) % 2]);
#pragma unroll
    for (int col = 0; col < NC; ++col) exponentials(BLOCKS - 1, col);
}

// A workgroup's LDS: KW waves next to each other along the keys, RG = 4 / KW groups of them that take the stages of 32 * U rows in turn.
template <int D, int NC, int KW, int U>
struct WeightsLds {
    static constexpr int RG = 4 / KW, KEYS = KW * 16 * NC, ROWS = 32 * U;
    static constexpr int ROWS_AT = U * StagedRows<D>::Tile, STAGE = ROWS_AT + 2 * ROWS * 4;        // rows, their offsets, how many keys they see
    // stages: one that is read and two on their way, or one where the groups' stages would leave room for one workgroup a CU
    static constexpr int RING = RG == 1 ? 3 : 2;
    static constexpr int STAGES = RG * RING * STAGE, BYTES = STAGES + (RG > 1 ? RG * KEYS * 16 : 0);   // the groups' sums behind them
};

// The numbers of KW * 64 keys from tile0 on.
template <int D, int NC, int KW, int U>
__device__ __forceinline__ void weights_tile(const WeightsParams &p, uint32_t s, int tile0, uint32_t kv, char *smem)
{
    using Lds = WeightsLds<D, NC, KW, U>;
    constexpr int RG = Lds::RG, OWN = 16 * NC, KEYS = Lds::KEYS, ROWS = Lds::ROWS, FOLD = 16 / U, ROWS_AT = Lds::ROWS_AT, STAGE = Lds::STAGE, RING = Lds::RING;
    using L = StagedRows<D>;
    constexpr int PER_WAVE = U * L::Groups / KW;                            // DMA instructions of a wave for a stage
    float (*joined)[KEYS][4] = reinterpret_cast<float (*)[KEYS][4]>(smem + Lds::STAGES);
    const int lane = threadIdx.x & 63, all_waves = uniform(threadIdx.x >> 6), g4 = lane >> 4;
    const int rg = all_waves / KW, wave = all_waves % KW;
    WeightsSeq seq = weights_seq(s, p);
    seq.q0 = uniform(seq.q0);
    seq.lq = uniform(seq.lq);
    seq.lk = uniform(seq.lk);
    seq.rows = uniform(seq.rows);
    const int key0 = tile0 + wave * OWN;
    if (tile0 >= seq.lk) return;
    // the rows before token first_token see no key of the tile, those from whole_token on see all
    const int last = (tile0 + KEYS < seq.lk ? tile0 + KEYS : seq.lk) - 1, ahead = seq.lk - seq.lq;
    const int first_token = !p.causal || tile0 <= ahead ? 0 : tile0 - ahead, whole_token = !p.causal || last <= ahead ? 0 : last - ahead;
    const int steps_end = (seq.rows + ROWS - 1) / ROWS;
    const int step0 = (int64_t)first_token * p.g < seq.rows ? first_token * (int)p.g / ROWS : steps_end;
    const int64_t whole_row = (int64_t)whole_token * p.g;
    const int masked_end = (int)(whole_row < seq.rows ? (whole_row + ROWS - 1) / ROWS : steps_end);

    char *own = smem + rg * RING * STAGE;
    const bool describes = wave == 0 && lane < ROWS;                        // this lane brings what a row's offset is and how many keys it sees
    float lse_next = 0.f;
    int sees_next = 0;
    const int r = lane / (D / 8), pos = lane % (D / 8);                     // of a DMA instruction: the lane's row and place
    const uint32_t swizzled = (uint32_t)((pos ^ L::turn(r)) << 4);
    // Where the group's size is a power of two that divides 32, the rows of a DMA instruction follow each other alike whichever it is: their first one's place is worked out in scalar
    // registers.
    const char *q_head = p.q.data + (int64_t)seq.q0 * p.q.token + (int64_t)(kv * p.g) * p.q.head;
    const uint32_t even_off = p.even ? (uint32_t)((r >> p.g_shift) * (int)p.q.token + (r & (int)(p.g - 1)) * (int)p.q.head) + swizzled : 0;
    const float *even_lse = p.lse + (int64_t)(kv * p.g + (p.even ? lane & (int)(p.g - 1) : 0)) * p.tokens + seq.q0 + (lane >> p.g_shift);
    // What describes the rows comes into registers, older than the stage's DMA; a step later it is there and goes to LDS, where it is read a step after that.
    auto issue = [&](int stage, int step) __attribute__((always_inline)) {
        if (step >= steps_end) return;
        const bool even = p.even && (step + 1) * ROWS <= seq.rows;
        if (describes) {
            if (even) {
                lse_next = even_lse[(uint32_t)(step * ROWS) >> p.g_shift];
                if (step < masked_end) sees_next = seq.keys_of((step * ROWS + lane) >> p.g_shift, p.causal);
            } else {
                const int R = step * ROWS + lane;
                const WeightRow w = weight_row((uint32_t)(R < seq.rows ? R : seq.rows - 1), seq, kv, p);
                lse_next = R < seq.rows ? *w.lse : -INFINITY;
                sees_next = R < seq.rows ? seq.keys_of(w.token, p.causal) : 0;
            }
        }
        if (even) {
#pragma unroll
            for (int i = 0; i < PER_WAVE; ++i) {
                const int group = PER_WAVE * wave + i, R = step * ROWS + group * L::GroupRows;
                const char *from = q_head + (int64_t)(R >> p.g_shift) * p.q.token + (int64_t)(R & (int)(p.g - 1)) * p.q.head;
                uint32_t o = even_off;
                asm volatile("" : "+v"(o));                                 // a 32-bit lane offset next to a scalar base
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from + o), STA_LDS_PTR(own + stage * STAGE + group * L::Group), 16, 0, 0);
            }
            asm volatile("; even" ::: "memory");
        } else {
#pragma unroll
            for (int i = 0; i < PER_WAVE; ++i) {
                const int group = PER_WAVE * wave + i, R = step * ROWS + group * L::GroupRows + r;
                const char *from = weight_row((uint32_t)(R < seq.rows ? R : seq.rows - 1), seq, kv, p).q + swizzled;       // rows beyond the last one are read as it
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, STA_LDS_PTR(own + stage * STAGE + group * L::Group), 16, 0, 0);
            }
            asm volatile("; any" ::: "memory");
        }
    };
    auto describe = [&](int stage) __attribute__((always_inline)) {
        if (!describes) return;
        *reinterpret_cast<float *>(own + stage * STAGE + ROWS_AT + 4 * lane) = offset_of(lse_next);
        *reinterpret_cast<int *>(own + stage * STAGE + ROWS_AT + 4 * ROWS + 4 * lane) = sees_next;
    };
    const int n_steps = (steps_end - step0 + RG - 1) / RG;                  // of every group
    issue(0, step0 + rg);
    describe(0);
    if (RING == 3) issue(1, step0 + rg + RG);
    bf16x8 K[NC][D / 32];
    const OwnKey own_key = load_keys<D, NC>(p, s, kv, key0, seq.lk, lane, K);
    // Waited for here: at their first use in the loop the compiler would wait for all that is on its way, stages among it, every time.
#pragma unroll
    for (int col = 0; col < NC; ++col)
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) asm volatile("" : "+v"(K[col][ks]));
    const uint32_t base = (uint32_t)(uintptr_t)own, q_addr = L::address(base, lane), row_addr = base + ROWS_AT + 16 * g4;
    const float c = p.scale_log2e;
    float sum[NC] = {}, part[NC] = {};
    int folded = 0;
    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < n_steps; ++i) {
        const int at = step0 + rg + RG * i, next = stage + 1 < RING ? stage + 1 : 0, after = next + 1 < RING ? next + 1 : 0;
        // This wave's part of the stage has landed, the next one's may be on its way; what describes that is older than its DMA.
        if (RING == 3 && at + RG < steps_end) {
            wait_dma<PER_WAVE>();
            asm volatile("" : "+v"(lse_next));
        } else {
            wait_dma<0>();
            asm volatile("" : "+v"(lse_next));
        }
        if (RING == 3) describe(next);                      // (where there is no next stage nobody reads it)
        else if (i > 0) describe(stage);
        __syncthreads();                                    // ... and everyone's, and nobody reads the stage before any more
        issue(RING == 3 ? after : next, at + (RING - 1) * RG);
        if (at < steps_end && key0 < seq.lk) {
            const uint32_t q_now = q_addr + (uint32_t)(stage * STAGE), row_now = row_addr + (uint32_t)(stage * STAGE);
            if (at < masked_end) add_rows<D, NC, 2 * U, true, 0, 0, 4 * ROWS>(q_now, row_now, K, c, key0 + (lane & 15), part);
            else add_rows<D, NC, 2 * U, false, 0, 0, 4 * ROWS>(q_now, row_now, K, c, key0 + (lane & 15), part);
            if (++folded == FOLD) {
                folded = 0;
#pragma unroll
                for (int col = 0; col < NC; ++col) {
                    sum[col] += part[col];
                    part[col] = 0.f;
                }
            }
        }
        stage = next;
    }
#pragma unroll
    for (int col = 0; col < NC; ++col) sum[col] += part[col];
    if constexpr (RG > 1) {                                         // the groups' sums, in ascending order
#pragma unroll
        for (int col = 0; col < NC; ++col) joined[rg][wave * OWN + 16 * col + (lane & 15)][g4] = sum[col];
        __syncthreads();
        if (rg > 0) return;
#pragma unroll
        for (int col = 0; col < NC; ++col) {
            sum[col] = 0.f;
#pragma unroll
            for (int g = 0; g < RG; ++g) sum[col] += joined[g][wave * OWN + 16 * col + (lane & 15)][g4];
        }
    }
    if (key0 < seq.lk) store_weights(p, own_key, lane, sum);
}

// Workgroup (sequence, KW * 64 keys, key head).
template <int D, int NC, int KW, int U>
__global__ __launch_bounds__(256, 2) void sta_paged_weights_kernel(WeightsParams p)
{
    __shared__ __attribute__((aligned(1024))) char smem[WeightsLds<D, NC, KW, U>::BYTES];
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t turn = sta::fast_div(item, p.by_tiles), tile = item - turn * p.by_tiles.d;
    const uint32_t s = p.S <= 64 ? sequence_of_turn(turn, threadIdx.x & 63, p) : turn;
    weights_tile<D, NC, KW, U>(p, s, (int)(tile * WeightsLds<D, NC, KW, U>::KEYS), kv, smem);
}

// Up to 64 sequences, a lane each: the tiles of 256 keys that there are, those of the sequences of many rows first.  What these leave behind whole rounds of workgroups over the chip, where it is a quarter of a
// round at most, are two workgroups' of 128 keys each, so that every CU has one at most: us, 32 heads over 8, tiles alone | this, 512 tokens on 20,001 keys 97 | 81, 128 on 20,001  31 | 28, 2048 on 20,001  348 | 290;
// and where more is left (always | this): 512 on 21,700  103 | 95, on 24,000  104 | 98.
template <int D>
__global__ __launch_bounds__(256, 2) void sta_paged_weights_rounds_kernel(WeightsParams p)
{
    constexpr int WHOLE = WeightsLds<D, 4, 4, 2>::BYTES, HALF = WeightsLds<D, 4, 2, 1>::BYTES;
    __shared__ __attribute__((aligned(1024))) char smem[WHOLE > HALF ? WHOLE : HALF];
    const int lane = threadIdx.x & 63;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    uint32_t own = 0;
    bool many = false;
    if (lane < (int)p.S) {
        const WeightsSeq seq = weights_seq((uint32_t)lane, p);
        const uint32_t there = ((uint32_t)seq.lk + 255) / 256;
        own = there < p.by_tiles.d ? there : p.by_tiles.d;
        many = 2 * (int64_t)seq.lq >= p.max_q;
    }
    const uint32_t upto_many = scan64(many ? own : 0), all_many = (uint32_t)__builtin_amdgcn_readlane((int)upto_many, 63);
    const uint32_t left = all_many % p.round, whole = 4 * left <= p.round ? all_many - left : all_many, with_halves = 2 * all_many - whole;
    const bool few = item >= with_halves;
    const uint32_t rank = few ? item - with_halves : item < whole ? item : whole + (item - whole) / 2;
    const uint32_t upto = few ? scan64(many ? 0 : own) : upto_many;
    const uint64_t at = __builtin_amdgcn_ballot_w64(upto > rank);
    if (at == 0) return;
    const int s = __builtin_ctzll(at);
    const int tile0 = (int)((rank - (uint32_t)__builtin_amdgcn_readlane((int)(upto - own), s)) * 256);
    if (!few && item >= whole) weights_tile<D, 4, 2, 1>(p, (uint32_t)s, tile0 + (int)((item - whole) % 2) * 128, kv, smem);
    else weights_tile<D, 4, 4, 2>(p, (uint32_t)s, tile0, kv, smem);
}

// Four waves along the keys where that makes two workgroups a CU, two waves by two groups where that does, or where walks are of 512 rows at most and three quarters of the CUs
// have one, else one wave by four groups.  us, four | two | one along the keys, new tokens on keys of heads / key heads x channels:
//   512 on 20,001, 32/8 x 128 (632 | 1256 | 2504 workgroups)  107 | 105 | 142       2048 on 16,384, 32/8 x 128 (512 | 1024 | 2048)  259 | 287 | 353
//   300 on 1300 and 1000 on 5000, 8/8 x 128 (320 | 640 | 1264)  25.6 | 23.5 | 27.9  four of 200 on 3000, 40/8 x 64 (384 | 768 | 1504)  37 | 31 | 35
//   512 on 4000, 32/8 x 128 (128 | 256 | 504)  49 | 35 | 31       300 on 9000, 16/2 x 128 (72 | 142 | 282)  65 | 40 | 34
//   eight of 64 on 1300, 40/5 x 128 (240 | 440 | 840)  18.8 | 18.1 | 24.6       50 on 30,000, 8/1 x 128 (118 | 235 | 469)  15.2 | 11.3 | 13.0
// With 64 channels, where a stage is half the work, two waves by two groups with stages of 64 rows are the better ones for more than 512 rows, whatever the launch: us, four | two along the keys,
//   512 on 20,001, 32/8  76 | 61       2048 on 8192, 16/16  58 | 50       2048 on 30,000, 8/8  90 | 83       four of 2048, 16/16  56 | 50       four of 1000 on 4000, 16/16  50 | 49
//   (as far as a launch has workgroups for tiles of 128 keys) and not for fewer: eight of 64 on 1300, 12/12  8.2 | 10.4; sixteen of 500 on 2048, 16/16  54.5 | 55.3       (stages of 32 rows: four of 200 on 3000, 40/8  29.5, 28.1 with 64; 1, 5 and 33 on 65 to 578, 16/16  4.3, 4.8;
//   with 128 channels four of 200 38.6, 42)
struct WeightsPlan {
    int few;                            // blocks of 16 rows, 0: stages
    int along;                          // waves of a workgroup along the keys
    bool deep;                          // stages of 64 rows for two waves by two groups
    int64_t tiles, workgroups;
};
WeightsPlan weights_plan(int S, int Hkv, int D, int64_t rows, int max_k)
{
    const int64_t cus = sta::compute_units(), heads = (int64_t)S * Hkv;
    auto tiles = [&](int64_t keys) { return (max_k + keys - 1) / keys; };
    WeightsPlan plan = {};
    plan.workgroups = heads;
    if (heads > kMostWorkgroups) return plan;               // too many whatever the tiles are
    plan.few = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
    plan.along = plan.few || tiles(256) * heads >= 2 * cus ? 4 : tiles(128) * heads >= (rows <= 512 ? 3 * cus / 4 : 2 * cus) ? 2 : 1;
    plan.deep = D == 64 && rows > 512;
    if (plan.deep && plan.along == 4 && tiles(128) * heads <= kMostWorkgroups) plan.along = 2;
    plan.tiles = tiles(64 * plan.along);
    plan.workgroups = plan.tiles * heads;
    return plan;
}

template <int D, int NC, int KW, int U>
hipError_t launch_stages(const WeightsParams &p, uint32_t workgroups, hipStream_t stream)
{
    return sta::launch_kernel(sta_paged_weights_kernel<D, NC, KW, U>, dim3(workgroups), dim3(256), stream, p);
}

template <int D>
hipError_t launch_weights(const WeightsParams &p, const WeightsPlan &plan, hipStream_t stream)
{
    const uint32_t n = (uint32_t)plan.workgroups;
    if (plan.few == 1) return sta::launch_kernel(sta_paged_few_weights_kernel<D, 4, 1>, dim3(n), dim3(256), stream, p);
    if (plan.few == 2) return sta::launch_kernel(sta_paged_few_weights_kernel<D, 4, 2>, dim3(n), dim3(256), stream, p);
    if constexpr (D == 128)
        if (plan.along == 4 && p.S <= 64 && plan.workgroups + p.round * p.Hkv <= kMostWorkgroups)
            return sta::launch_kernel(sta_paged_weights_rounds_kernel<D>, dim3(n + p.round * p.Hkv), dim3(256), stream, p);
    if constexpr (D == 64)
        if (plan.deep && plan.along == 2) return launch_stages<D, 4, 2, 2>(p, n, stream);
    return plan.along == 4 ? launch_stages<D, 4, 4, 2>(p, n, stream) : plan.along == 2 ? launch_stages<D, 4, 2, 1>(p, n, stream) : launch_stages<D, 4, 1, 1>(p, n, stream);
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
    if (!numbers_fit(*cache, S)) return STA_ERR_SHAPE;
    const int64_t room = room_of(*cache);
    if (max_k > room) max_k = (int)room;
    if (S == 0 || max_k == 0) return STA_OK;
    if (!cu_q || !weights || (!lse && tokens_q > 0)) return STA_ERR_NULL;
    if (((uintptr_t)cu_q | (uintptr_t)lse | (uintptr_t)before | (uintptr_t)weights) & 3) return STA_ERR_SHAPE;
    const WeightsPlan plan = weights_plan(S, Hkv, D, (int64_t)max_q * (q->heads / Hkv), max_k);
    if (plan.workgroups > kMostWorkgroups) return STA_ERR_SHAPE;
    const uint64_t w_bytes = number_bytes(*cache, S), lse_bytes = (uint64_t)tokens_q * q->heads * sizeof(float);
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
    p.numbers = key_numbers_of(*cache);
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
    p.even = (p.g & (p.g - 1)) == 0 && p.g <= 32 && q->head < (int64_t)1 << 25;
    p.g_shift = p.even ? (uint32_t)__builtin_ctz(p.g) : 0;
    p.by_tiles = sta::fast_div_of((uint32_t)plan.tiles);
    p.round = (2 * (uint32_t)sta::compute_units() + Hkv - 1) / Hkv;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = D == 64 ? launch_weights<64>(p, plan, stream) : launch_weights<128>(p, plan, stream);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}
