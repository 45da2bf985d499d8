// Gradients of the attention over packed sequences.
//
//   P_ij = exp(S_ij - lse_i),  dV_j = sum_i P_ij dO_i,  dP_ij = dO_i . V_j,  dS_ij = P_ij (dP_ij - delta_i),  delta_i = dO_i . O_i
//   dQ_i = scale sum_j dS_ij K_j,  dK_j = scale sum_i dS_ij Q_i       (i: the rows of all heads of a group)
//
// Two or three kernels, no atomics:
//   sta_packed_dq_kernel      four waves of 32 rows walk the keys they see: three products per block.  It also forms -delta_i and -lse_i / scale of
//                             its rows and leaves them, in the order of the rows, for the second kernel;
//   sta_packed_dkv_kernel     waves of 32 keys walk the rows that see them: four products per block;
//   sta_packed_join_kernel    where few keys are seen by many rows, workgroups walk parts of them, and this one adds the parts' sums.
// The heads of a group are rows like any others, so their gradients of K and V are summed in the accumulators.
//
// Roundings.  P and dS go into the matrix instructions as bf16, the only type that those take next to bf16 operands, and delta is formed from O as
// it was rounded.  Of the errors against 64 bits (relative, whole tensors of N(0,1) inputs) 1.7e-3 is the results' own rounding, which a computation
// in fp32 has as well; with dS rounded, and O in delta where rows see few keys, dQ and dK have 2.5e-3 to 3.2e-3 (dS in
// two bf16 parts would be a product more of three, of four); where a softmax is nearly one key's, dP - delta cancels and more of O's rounding is
// left (Q and K of 4 N(0,1): 1e-2).  Everything else, sums and statistics included, is fp32.
//
// What bounds them: the matrix pipe and, where workgroups are few, latencies.  32,768 tokens of 32 heads over 8 of 128 channels, causal: both kernels
// 1330 TFLOP/s of the seven products that they run (949 of the five that have to be), the rate of a large library product on this chip; 4 * 4096 tokens 1200; [2048, 1999, 77, 1023, 949] dQ 128 us, dK/dV 187
// (977 and 892 TFLOP/s; matrix pipe busy 41 and 36 %): a wave's 64 matrix instructions of a sub-block of dK/dV read 32 KB of LDS, what it can give in that
// time, with two waves a SIMD (accumulators 128 registers, K and V 128) that wait for one another's stages.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <utility>

#include "../../include/sta.h"
#include "sta_packed.h"
#include "sta_rows_check.h"

namespace {

struct BackwardParams {
    PackedParams p;                 // q, k, v, o and the bounds
    PackedRows d_o, d_q, d_k, d_v;
    const float *lse;               // [Hq, tokens_q]
    float *neg_lse, *neg_delta;     // [Hkv, tokens_q, g], in raw scores
    float inv_scale;
};

// Columns of a wave out of their accumulators: [channel block][column block] of the transposed result.
template <int D, int NC>
__device__ __forceinline__ void store_column(const floatx4 (&acc)[D / 16][NC], int col, float factor, char *row, int g4)
{
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) {
        bf16x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = static_cast<__bf16>(acc[cb][col][r] * factor);
        *reinterpret_cast<bf16x4 *>(row + 32 * cb + 8 * g4) = v;
    }
}

// The first group's accumulators += those of the others, in ascending order.
template <int D, int KW, int G, int NC>
__device__ __forceinline__ void join_groups(char *smem, int walk, int wave, int lane, floatx4 (&acc)[D / 16][NC])
{
    constexpr int WAVE = D / 16 * NC * 1024;
    __syncthreads();                                        // the stages, or the operand before, have been read
    if (walk > 0) {
        char *to = smem + ((walk - 1) * KW + wave) * WAVE + lane * 16;
#pragma unroll
        for (int cb = 0; cb < D / 16; ++cb)
#pragma unroll
            for (int col = 0; col < NC; ++col) *reinterpret_cast<floatx4 *>(to + (cb * NC + col) * 1024) = acc[cb][col];
    }
    __syncthreads();
    if (walk == 0)
#pragma unroll
        for (int other = 0; other < G - 1; ++other)
#pragma unroll
            for (int cb = 0; cb < D / 16; ++cb)
#pragma unroll
                for (int col = 0; col < NC; ++col)
                    acc[cb][col] += *reinterpret_cast<const floatx4 *>(smem + (other * KW + wave) * WAVE + (cb * NC + col) * 1024 + lane * 16);
}

// RW waves of 32 rows; KG groups of them take the sub-blocks of keys in turn, each with stages of its own, and the groups' sums are joined at the end.
template <int D, int RW, int KG>
__global__ __launch_bounds__(RW * KG * 64, KG > 2 ? D == 64 ? 2 : 1 : D == 64 ? 3 : 2) void sta_packed_dq_kernel(BackwardParams b)
{
    const PackedParams &p = b.p;
    constexpr int NC = 2, KS = D / 32, CB = D / 16, TILE = 32 * RW;
    using LK = Staged<D>;
    using LV = StagedRows<D>;
    constexpr int STAGE = LK::Tile + LV::Tile, V_AT = LK::Tile, PER_WAVE = LK::Groups / RW;
    constexpr int MERGE = (KG - 1) * RW * CB * NC * 1024;
    __shared__ __attribute__((aligned(1024))) char smem[2 * KG * STAGE > MERGE ? 2 * KG * STAGE : MERGE];
    const int lane = threadIdx.x & 63, all_waves = uniform(threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int walk = all_waves / RW, wave = all_waves % RW;
    char *own = smem + 2 * walk * STAGE;
    const uint32_t rank = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - rank * p.Hkv;
    PackedTile tile;
    if (!find_tile<TILE, false>(rank, p, lane, &tile)) return;
    const PackedSeq seq = tile.seq;
    const uint32_t rows = (uint32_t)seq.lq * p.g, row0 = tile.index * TILE;
    const uint32_t last_row = row0 + TILE < rows ? row0 + TILE - 1 : rows - 1;
    const int n_keys = uniform(seq.keys_of((int)sta::fast_div(last_row, p.by_g), p));
    const int n_sub = (n_keys + kSub - 1) / kSub;

    const uint32_t wave_row = row0 + 32 * wave;
    const bool idle = wave_row >= rows;
    int token[NC], lim[NC];
    int64_t head[NC];
    bool on[NC];
    float neg_lse[NC], neg_delta[NC];
    bf16x8 Q[NC][KS], G[NC][KS];
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const uint32_t row = wave_row + 16 * col + c16;
        on[col] = row < rows;
        const uint32_t r = on[col] ? row : rows - 1, t = sta::fast_div(r, p.by_g);
        token[col] = (int)t;
        head[col] = (int64_t)kv * p.g + (r - t * p.g);
        lim[col] = seq.keys_of((int)t, p);
        const char *q = p.q.data + (int64_t)(seq.q0 + token[col]) * p.q.token + head[col] * p.q.head;
        const char *g = b.d_o.data + (int64_t)(seq.q0 + token[col]) * b.d_o.token + head[col] * b.d_o.head;
        const char *o = p.o.data + (int64_t)(seq.q0 + token[col]) * p.o.token + head[col] * p.o.head;
        float delta = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Q[col][ks] = *reinterpret_cast<const bf16x8 *>(q + 64 * ks + 16 * g4);
            G[col][ks] = *reinterpret_cast<const bf16x8 *>(g + 64 * ks + 16 * g4);
            const bf16x8 O = *reinterpret_cast<const bf16x8 *>(o + 64 * ks + 16 * g4);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = fmaf((float)O[e], (float)G[col][ks][e], delta);
        }
        neg_delta[col] = -quad_lane_sum(delta);
        neg_lse[col] = -b.lse[head[col] * p.tokens_q + seq.q0 + token[col]] * b.inv_scale;
        if (on[col] && g4 == 0 && walk == 0) {
            const size_t stat = ((size_t)kv * p.tokens_q + seq.q0) * p.g + r;
            b.neg_lse[stat] = neg_lse[col];
            b.neg_delta[stat] = neg_delta[col];
        }
    }
    const uint32_t wave_last = wave_row + 31 < rows ? wave_row + 31 : rows - 1;
    const int lim_lo = idle ? 0 : uniform(seq.keys_of((int)sta::fast_div(wave_row, p.by_g), p));
    const int lim_hi = idle ? 0 : uniform(seq.keys_of((int)sta::fast_div(wave_last, p.by_g), p));

    const char *kh = p.k.data + (int64_t)seq.k0 * p.k.token + (int64_t)kv * p.k.head;
    const char *vh = p.v.data + (int64_t)seq.k0 * p.v.token + (int64_t)kv * p.v.head;
    PackedDma<D, false> k_dma;
    PackedDma<D, true> v_dma;
    k_dma.start(lane, p.k.token);
    v_dma.start(lane, p.v.token);
    auto issue = [&](int stage, int sub) __attribute__((always_inline)) {
        if (sub < n_sub)
            bring_stage<1, PER_WAVE, LK::Group, LV::Group>(k_dma, v_dma, kh, vh, p.k.token, p.v.token, sub, seq.lk, PER_WAVE * wave, own + stage * STAGE, V_AT, 0);
    };
    issue(0, walk);
    const uint32_t base = (uint32_t)(uintptr_t)own;
    uint32_t k_addr[KS], k_tr[4];
    LK::addresses(base, lane, k_addr, k_tr);
    const uint32_t v_addr = LV::address(base + V_AT, lane);
    floatx4 acc[CB][NC];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int col = 0; col < NC; ++col) acc[cb][col] = floatx4{0.f, 0.f, 0.f, 0.f};
    const float c = p.scale_log2e;
    auto step = [&](auto stage_c, int sub) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage_c)::value * STAGE;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (RW > 1) __syncthreads();
        issue(decltype(stage_c)::value ^ 1, sub + KG);
        const int first = sub * kSub;
        if (first >= lim_hi) return;                        // (and sub-blocks that the other groups alone still have)
        floatx4 S[2][NC], dP[2][NC];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    S[kb][col][r] = neg_lse[col];
                    dP[kb][col][r] = neg_delta[col];
                }
        staged_rows_times_resident<D, ST, NC>(k_addr, Q, S);                        // K Q^T - lse / scale
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[kb][col][r] = __builtin_amdgcn_exp2f(S[kb][col][r] * c);
        rows_times_resident<D, ST, NC>(v_addr, G, dP);                              // V dO^T - delta
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[kb][col][r] *= dP[kb][col][r];
        if (first + kSub > lim_lo) {                                                // a select, whatever the product is
#pragma unroll
            for (int col = 0; col < NC; ++col) {
                const int left = lim[col] - first - 4 * g4;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[kb][col][r] = 16 * kb + r < left ? S[kb][col][r] : 0.f;
            }
        }
        // (reads on their way are not carried over a branch: the compiler, which does not know that they are, may move their registers there)
        StagedTransposedProduct<D, ST> product;
        product.prefetch(k_tr);
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 dS[NC];
#pragma unroll
        for (int col = 0; col < NC; ++col)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) dS[col][4 * kb + r] = static_cast<__bf16>(S[kb][col][r]);
        product.template run<NC>(k_tr, dS, acc);                                    // dQ^T += K^T dS^T
    };
#pragma unroll 1
    for (int sub = 0; sub < n_sub; sub += 2 * KG) {         // the same number of barriers for every group
        step(std::integral_constant<int, 0>{}, sub + walk);
        if (sub + KG < n_sub) step(std::integral_constant<int, 1>{}, sub + KG + walk);
    }
    if constexpr (KG > 1) {
        join_groups<D, RW, KG>(smem, walk, wave, lane, acc);
        if (walk != 0) return;
    }
#pragma unroll
    for (int col = 0; col < NC; ++col)
        if (on[col]) store_column<D, NC>(acc, col, p.scale, b.d_q.data + (int64_t)(seq.q0 + token[col]) * b.d_q.token + head[col] * b.d_q.head, g4);
}

// Where a tile's walk of rows is cut into parts: n sub-blocks, `each` a part, the last one less.
struct RowParts {
    int parts, each;
};
__device__ __forceinline__ RowParts row_parts_of(int n, const PackedParams &p)
{
    const int each = max((n + (int)p.parts - 1) / (int)p.parts, 1);
    return {max((n + each - 1) / each, 1), each};
}
// A part's sums of dV, then dK: [key of the tile][D].  Tiles are counted by rank, as the launch and the workspace are.
template <int D, int TILE>
__device__ __forceinline__ float *row_part_at(const PackedParams &p, uint32_t rank, uint32_t kv, int part)
{
    return p.ws + (((size_t)rank * p.Hkv + kv) * p.parts + part) * (2 * TILE * D);
}

// KW waves of 32 keys; G groups of them take the sub-blocks of rows in turn, each with stages of its own, and the groups' sums are joined at the end.
// CUT: workgroups take parts of a tile's rows and leave their sums in memory, which sta_packed_join_kernel adds up.
template <int D, int KW, int G, bool CUT>
__global__ __attribute__((amdgpu_flat_work_group_size(KW * G * 64, KW * G * 64), amdgpu_waves_per_eu((D == 64 ? 3 : 2) - (G > 2))))
void sta_packed_dkv_kernel(BackwardParams b)
{
    const PackedParams &p = b.p;
    constexpr int NC = 2, KS = D / 32, CB = D / 16, TILE = 32 * KW;
    using L = Staged<D>;
    constexpr int STATS = 2 * L::Tile, STAGE = STATS + 1024, G_AT = L::Tile, PER_WAVE = L::Groups / KW, LPR = D / 8;
    constexpr int MERGE = G > 1 ? (G - 1) * KW * CB * NC * 1024 : 0;           // accumulators of one operand, of all groups but the first
    __shared__ __attribute__((aligned(1024))) char smem[2 * G * STAGE > MERGE ? 2 * G * STAGE : MERGE];
    const int lane = threadIdx.x & 63, all_waves = uniform(threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int walk = all_waves / KW, wave = all_waves % KW;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t rank = CUT ? sta::fast_div(item, p.by_parts) : item;
    const int part = CUT ? (int)(item - rank * p.parts) : 0;
    PackedTile tile;
    if (!find_tile<TILE, true>(rank, p, lane, &tile)) return;
    const PackedSeq seq = tile.seq;
    const int worked = seq.worked(p), rows = worked * (int)p.g, key0 = (int)tile.index * TILE, ahead = seq.lk - seq.lq;
    // key j is seen by the rows from first_row(j) on
    auto first_row = [&](int j) {
        const int t = j - ahead;
        return !p.causal || t <= 0 ? 0 : t < worked ? t * (int)p.g : rows;
    };
    int sub0 = uniform(first_row(key0) / kSub), n_sub = (rows + kSub - 1) / kSub;
    if constexpr (CUT) {
        const RowParts cut = row_parts_of(n_sub - sub0, p);
        if (part >= cut.parts) return;
        sub0 += part * cut.each;
        n_sub = min(sub0 + cut.each, n_sub);
    }
    const int wave_key = key0 + 32 * wave;
    const int see_lo = uniform(first_row(wave_key)), see_hi = uniform(first_row(wave_key + 31));        // of the wave's first and last key
    bf16x8 K[NC][KS], V[NC][KS];
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const int key = wave_key + 16 * col + c16, j = key < seq.lk ? key : seq.lk - 1;
        const char *k = p.k.data + (int64_t)(seq.k0 + j) * p.k.token + (int64_t)kv * p.k.head;
        const char *v = p.v.data + (int64_t)(seq.k0 + j) * p.v.token + (int64_t)kv * p.v.head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            K[col][ks] = *reinterpret_cast<const bf16x8 *>(k + 64 * ks + 16 * g4);
            V[col][ks] = *reinterpret_cast<const bf16x8 *>(v + 64 * ks + 16 * g4);
        }
    }
    // DMA: row -> (token, head); its 16-byte chunk at this lane's place.  All of it is worked out again for every stage: registers that are free
    // then are not in the loop.
    const char *qh = p.q.data + (int64_t)seq.q0 * p.q.token + (int64_t)kv * p.g * p.q.head;
    const char *gh = b.d_o.data + (int64_t)seq.q0 * b.d_o.token + (int64_t)kv * p.g * b.d_o.head;
    // what 24-bit products and 32-bit offsets hold: of 32 + g rows
    const int64_t most = (int64_t)1 << 24;
    const bool small = p.g <= 64 && p.q.token < most && p.q.head < most && b.d_o.token < most && b.d_o.head < most;
    const uint32_t magic = (65535u + p.g) / p.g;            // n / g = n * magic >> 16 for n < 32 + g <= 96
    const size_t stat0 = ((size_t)kv * p.tokens_q + seq.q0) * p.g;
    // The walk goes from the last rows, which all keys' walks begin with, towards the first that see the tile: workgroups of a sequence read the
    // same rows at about the same time.
    const int ends = sub0 + n_sub - 1;
    auto issue = [&](int stage, int at_walk) __attribute__((always_inline)) {
        if (at_walk >= n_sub) return;
        const int sub = ends - at_walk;
        char *to = smem + (2 * walk + stage) * STAGE;
        const int at = fresh_lane(), r_in = at / LPR, first = sub * kSub;
        const uint32_t chunk = PackedDma<D, false>::chunk_of(at);
        if (__builtin_expect(small && first + kSub <= rows, 1)) {
            // rows relative to the stage's first token, in 24-bit products: 8 instructions for a row of Q and dO where whole addresses take 24,
            // 10 of them at a quarter of the rate
            const uint32_t t0 = sta::fast_div((uint32_t)first, p.by_g), h0 = (uint32_t)first - t0 * p.g;
            const char *q0 = qh + (int64_t)t0 * p.q.token, *g0 = gh + (int64_t)t0 * b.d_o.token;
#pragma unroll
            for (int i = 0; i < PER_WAVE; ++i) {
                const int group = PER_WAVE * wave + i;
                const uint32_t n = h0 + (uint32_t)(group * L::GroupRows + r_in), t = __umul24(n, magic) >> 16, h = n - __umul24(t, p.g);
                uint32_t oq = __umul24(t, (uint32_t)p.q.token) + __umul24(h, (uint32_t)p.q.head) + chunk;
                uint32_t og = __umul24(t, (uint32_t)b.d_o.token) + __umul24(h, (uint32_t)b.d_o.head) + chunk;
                asm volatile("" : "+v"(oq), "+v"(og));
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(q0 + oq), STA_LDS_PTR(to + group * L::Group), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(g0 + og), STA_LDS_PTR(to + G_AT + group * L::Group), 16, 0, 0);
            }
            asm volatile("; whole" ::: "memory");
        } else {
#pragma unroll 1
            for (int i = 0; i < PER_WAVE; ++i) {
                const int group = PER_WAVE * wave + i, row = first + group * L::GroupRows + r_in;
                const uint32_t r = (uint32_t)(row < rows ? row : rows - 1), t = sta::fast_div(r, p.by_g), h = r - t * p.g;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(qh + ((int64_t)t * p.q.token + (int64_t)h * p.q.head + chunk)),
                                                 STA_LDS_PTR(to + group * L::Group), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gh + ((int64_t)t * b.d_o.token + (int64_t)h * b.d_o.head + chunk)),
                                                 STA_LDS_PTR(to + G_AT + group * L::Group), 16, 0, 0);
            }
            asm volatile("; part" ::: "memory");
        }
        if (wave == KW - 1) {
            const int row = sub * kSub + (at & (kSub - 1));
            const float *stats = (at < kSub ? b.neg_lse : b.neg_delta) + stat0;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(stats + (row < rows ? row : rows - 1)),
                                             STA_LDS_PTR(to + STATS), 4, 0, 0);
        }
    };
    issue(0, sub0 + walk);
    const uint32_t base = (uint32_t)(uintptr_t)smem + 2 * walk * STAGE;
    uint32_t row_addr[KS], tr_addr[4];
    L::addresses(base, lane, row_addr, tr_addr);
    const uint32_t stat_addr = base + STATS + 16 * g4;
    floatx4 dK[CB][NC], dV[CB][NC];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int col = 0; col < NC; ++col) dK[cb][col] = dV[cb][col] = floatx4{0.f, 0.f, 0.f, 0.f};
    const float c = p.scale_log2e;
    auto step = [&](auto stage_c, int at_walk) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage_c)::value * STAGE;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if constexpr (KW > 1) __syncthreads();              // (one wave a group: its stages are its own; [774] of 40 heads over 8 54 us with, 47 without)
        issue(decltype(stage_c)::value ^ 1, at_walk + G);
        const int first = (ends - at_walk) * kSub;
        if (at_walk >= n_sub || first + kSub <= see_lo || wave_key >= seq.lk) return;
        auto start = [&](auto off_c) {                      // four rows' statistics for every register of a row block
            floatx4 x[2];
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            u32x4 a, d;
            asm volatile("ds_read_b128 %0, %2 offset:%3\n\tds_read_b128 %1, %2 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(a), "=&v"(d)
                         : "v"(stat_addr), "n"(ST + decltype(off_c)::value), "n"(ST + decltype(off_c)::value + 64));
            x[0] = __builtin_bit_cast(floatx4, a);
            x[1] = __builtin_bit_cast(floatx4, d);
            return std::pair<floatx4, floatx4>(x[0], x[1]);
        };
        floatx4 S[2][NC];
        {
            const auto x = start(std::integral_constant<int, 0>{});
#pragma unroll
            for (int col = 0; col < NC; ++col) { S[0][col] = x.first; S[1][col] = x.second; }
        }
        staged_rows_times_resident<D, ST, NC>(row_addr, K, S);                      // Q K^T - lse / scale
        StagedTransposedProduct<D, ST + G_AT, D == 64 ? 4 : 2> for_v;
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[qb][col][r] = __builtin_amdgcn_exp2f(S[qb][col][r] * c);
        if (first < see_hi || first + kSub > rows) {        // a select, whatever the exponential is
            const int at = fresh_lane(), row0 = first + 4 * (at >> 4);
#pragma unroll
            for (int col = 0; col < NC; ++col) {
                const int from = first_row(wave_key + 16 * col + (at & 15));
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = row0 + 16 * qb + r;
                        S[qb][col][r] = row >= from && row < rows ? S[qb][col][r] : 0.f;
                    }
            }
        }
        for_v.prefetch(tr_addr);
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 packed[NC];
        auto pack = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int qb = 0; qb < 2; ++qb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) packed[col][4 * qb + r] = static_cast<__bf16>(S[qb][col][r]);
        };
        pack();
        for_v.template run<NC>(tr_addr, packed, dV);                                // dV^T += dO^T P
        floatx4 dP[2][NC];
        {
            const auto x = start(std::integral_constant<int, kSub * 4>{});
#pragma unroll
            for (int col = 0; col < NC; ++col) { dP[0][col] = x.first; dP[1][col] = x.second; }
        }
        staged_rows_times_resident<D, ST + G_AT, NC>(row_addr, V, dP);              // dO V^T - delta
        StagedTransposedProduct<D, ST, D == 64 ? 4 : 2> for_k;
        for_k.prefetch(tr_addr);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[qb][col][r] *= dP[qb][col][r];
        pack();
        for_k.template run<NC>(tr_addr, packed, dK);                                // dK^T += Q^T dS
    };
#pragma unroll 1
    for (int sub = sub0; sub < n_sub; sub += 2 * G) {       // the same number of barriers for every group
        step(std::integral_constant<int, 0>{}, sub + walk);
        if (sub + G < n_sub) step(std::integral_constant<int, 1>{}, sub + G + walk);
    }
    if constexpr (G > 1) {
        join_groups<D, KW, G>(smem, walk, wave, lane, dV);
        join_groups<D, KW, G>(smem, walk, wave, lane, dK);
        if (walk != 0) return;
    }
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const int key = wave_key + 16 * col + c16;
        if (key >= seq.lk) continue;
        if constexpr (CUT) {
            float *to = row_part_at<D, TILE>(p, rank, kv, part) + (size_t)(key - key0) * D + 4 * g4;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                *reinterpret_cast<floatx4 *>(to + 16 * cb) = dV[cb][col];
                *reinterpret_cast<floatx4 *>(to + TILE * D + 16 * cb) = dK[cb][col];
            }
            continue;
        }
        store_column<D, NC>(dV, col, 1.0f, b.d_v.data + (int64_t)(seq.k0 + key) * b.d_v.token + (int64_t)kv * b.d_v.head, g4);
        store_column<D, NC>(dK, col, p.scale, b.d_k.data + (int64_t)(seq.k0 + key) * b.d_k.token + (int64_t)kv * b.d_k.head, g4);
    }
}

// Sums the parts of a tile's keys in ascending order: workgroup (tile and key head, keys), D / 4 lanes a key.
template <int D, int TILE>
__global__ __launch_bounds__(256) void sta_packed_join_kernel(BackwardParams b)
{
    const PackedParams &p = b.p;
    constexpr int LPR = D / 4, KEYS = 256 / LPR;
    const uint32_t rank = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - rank * p.Hkv;
    PackedTile tile;
    if (!find_tile<TILE, true>(rank, p, threadIdx.x & 63, &tile)) return;
    const PackedSeq seq = tile.seq;
    const int key0 = (int)tile.index * TILE, in = (int)(blockIdx.y * KEYS + threadIdx.x / LPR), ch = 4 * (threadIdx.x % LPR);
    if (key0 + in >= seq.lk) return;
    // as in sta_packed_dkv_kernel
    const int worked = seq.worked(p), rows = worked * (int)p.g, t = key0 - (seq.lk - seq.lq), first = !p.causal || t <= 0 ? 0 : t < worked ? t * (int)p.g : rows;
    const int parts = row_parts_of((rows + kSub - 1) / kSub - first / kSub, p).parts;
    const float *from = row_part_at<D, TILE>(p, rank, kv, 0) + (size_t)in * D + ch;
    floatx4 v = floatx4{0.f, 0.f, 0.f, 0.f}, k = v;
    for (int j = 0; j < parts; ++j, from += 2 * TILE * D) {
        v += *reinterpret_cast<const floatx4 *>(from);
        k += *reinterpret_cast<const floatx4 *>(from + TILE * D);
    }
    const int64_t key = seq.k0 + key0 + in;
    bf16x4 dv, dk;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        dv[r] = static_cast<__bf16>(v[r]);
        dk[r] = static_cast<__bf16>(k[r] * p.scale);
    }
    *reinterpret_cast<bf16x4 *>(b.d_v.data + key * b.d_v.token + (int64_t)kv * b.d_v.head + 2 * ch) = dv;
    *reinterpret_cast<bf16x4 *>(b.d_k.data + key * b.d_k.token + (int64_t)kv * b.d_k.head + 2 * ch) = dk;
}

template <int D, int KW, int G>
hipError_t launch_dkv(const BackwardParams &b, int64_t tiles, hipStream_t stream)
{
    return sta::launch_kernel(sta_packed_dkv_kernel<D, KW, G, false>, dim3((uint32_t)tiles * b.p.Hkv), dim3(KW * G * 64), stream, b);
}

template <int D, int RW, int KG>
hipError_t launch_dq(const BackwardParams &b, int64_t tiles, hipStream_t stream)
{
    return sta::launch_kernel(sta_packed_dq_kernel<D, RW, KG>, dim3((uint32_t)tiles * b.p.Hkv), dim3(RW * KG * 64), stream, b);
}

template <int D>
hipError_t launch_gradients(const BackwardParams &b, int max_q, int max_k, int64_t slots, hipStream_t stream)
{
    const PackedParams &p = b.p;
    const int64_t row_tiles = tiles_of(p.tokens_q, p.g, p.S, max_q, 128), half_rows = tiles_of(p.tokens_q, p.g, p.S, max_q, 64), key_tiles = tiles_of(p.tokens_k, 1, p.S, max_k, 128),
                  half_tiles = tiles_of(p.tokens_k, 1, p.S, max_k, 64);
    const int64_t quarter_rows = tiles_of(p.tokens_q, p.g, p.S, max_q, 32), quarter_tiles = tiles_of(p.tokens_k, 1, p.S, max_k, 32);
    // Four waves of 32 rows (keys) share a stage where that makes workgroups for the chip (head dimension 128: two and a quarter a CU, 64: three); else
    // two waves by two groups that take the stages in turn, or, where these are fewer than a workgroup a CU (rows: half one, and walks worth it), one by
    // four.  Causal, heads / key heads x channels, us of dQ, dK/dV in that order:
    //   32/8 x 128, [1024] * 16         561 in all | 627 | -           4/4 x 128, 33 of 1 .. 2642   73, 104 | 52, 69 | -
    //   40/8 x 128, [774]               -, - | 24, 80 | 42, 47         16/2 x 128, [1500]           -, - | 33, 224 | 43, 119
    //   2/2 x 64, [2100, 300]           -, - | 23, 32 | 14, 19         5/5 x 64, [128] * 16         -, - | 6.9, 7.6 | 8.0, 8.1
    hipError_t e = hipSuccess;
    const int64_t cus = sta::compute_units(), full = (D == 64 ? 12 : 9) * cus / 4;
    if (p.tokens_q > 0 && row_tiles > 0)
        e = row_tiles * p.Hkv >= full ? launch_dq<D, 4, 1>(b, row_tiles, stream) :
            half_rows * p.Hkv >= cus / 2 || max_k < 256 ? launch_dq<D, 2, 2>(b, half_rows, stream) : launch_dq<D, 1, 4>(b, quarter_rows, stream);
    if (e != hipSuccess || key_tiles == 0) return e;
    // Few keys that many rows see (a video's queries against a prompt): parts of the rows, whose sums go through memory, 5 to 14 us.  Not causal, 24 heads
    // of 128 channels, 115,200 tokens on 512, 256 and 77 keys, us of dK/dV: 1318, 645, 300 with, 2345, 1090, 1087 by one wave by four groups; 12 heads of
    // 64, 27,648 tokens on 512 keys 106 + 7, 191; causal, 16/2 x 128, [1500] 74 + 6, 119; [774] of 40/8, shorter than that, 47 by groups.
    const int64_t items = key_tiles * p.Hkv, subs = ((int64_t)max_q * p.g + kSub - 1) / kSub;
    if (items < cus && subs >= 256) {
        const int64_t room = slots / items, long_enough = subs / 32, parts = room < long_enough ? room : long_enough;
        if (parts > 1) {
            BackwardParams cut = b;
            cut.p.parts = (uint32_t)parts;
            cut.p.by_parts = sta::fast_div_of((uint32_t)parts);
            if ((e = sta::launch_kernel(sta_packed_dkv_kernel<D, 4, 1, true>, dim3((uint32_t)(items * parts)), dim3(256), stream, cut)) != hipSuccess) return e;
            return sta::launch_kernel(sta_packed_join_kernel<D, 128>, dim3((uint32_t)items, D / 8), dim3(256), stream, cut);
        }
    }
    if (key_tiles * p.Hkv >= full) return launch_dkv<D, 4, 1>(b, key_tiles, stream);
    if (half_tiles * p.Hkv < cus) return launch_dkv<D, 1, 4>(b, quarter_tiles, stream);
    return launch_dkv<D, 2, 2>(b, half_tiles, stream);
}

constexpr size_t kStatPad = 64;     // floats behind either array

size_t stat_bytes(int Hq, int64_t tokens_q) { return (2 * ((size_t)Hq * tokens_q + kStatPad) * sizeof(float) + 15) & ~(size_t)15; }

// Parts of tiles of 128 keys that there is room for: two workgroups a CU, and a part for every 128 rows of all heads, so that small calls need little.
int64_t part_slots(int Hq, int64_t tokens_q)
{
    const int64_t most = 2 * sta::compute_units(), by_rows = (int64_t)Hq * tokens_q / 128;
    return by_rows < 64 ? 0 : by_rows < most ? by_rows : most;
}
constexpr size_t kPartBytes = 2 * 128 * 128 * sizeof(float);

}  // namespace

extern "C" {

size_t sta_packed_backward_workspace_bytes(int Hq, int64_t tokens_q)
{
    if (Hq < 1 || tokens_q < 0 || tokens_q > kMostTokens / Hq) return 0;
    return stat_bytes(Hq, tokens_q) + (size_t)part_slots(Hq, tokens_q) * kPartBytes;
}

int sta_packed_backward(const sta_head_rows *q, const sta_head_rows *k, const sta_head_rows *v, const sta_head_rows *o, const sta_head_rows *d_o,
                        const float *lse, const sta_head_rows *d_q, const sta_head_rows *d_k, const sta_head_rows *d_v, int64_t tokens_q,
                        int64_t tokens_k, const int32_t *cu_q, const int32_t *cu_k, int S, int max_q, int max_k, int D, int causal, float scale,
                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!q || !k || !v || !o || !d_o || (!lse && tokens_q > 0) || !d_q || !d_k || !d_v) return STA_ERR_NULL;
    if (S < 0 || tokens_q < 0 || tokens_k < 0 || max_q < 0 || max_k < 0 || tokens_q > kMostTokens || tokens_k > kMostTokens) return STA_ERR_SHAPE;
    if ((D != 64 && D != 128) || !scale_of(scale, D, true, &scale)) return STA_ERR_UNSUPPORTED;
    const sta_head_rows *in[5] = {q, k, v, o, d_o}, *out[3] = {d_q, d_k, d_v};
    const int64_t nq = tokens_q, nk = tokens_k, n_in[5] = {nq, nk, nk, nq, nq}, n_out[3] = {nq, nk, nk};
    for (int i = 0; i < 5; ++i)
        if (int rc = sta::packed_check(in[i], n_in[i], i == 0 || i == 1 ? 0 : i == 2 ? k->heads : q->heads, D, false)) return rc;
    for (int i = 0; i < 3; ++i)
        if (int rc = sta::packed_check(out[i], n_out[i], i == 0 ? q->heads : k->heads, D, true)) return rc;
    if (q->heads % k->heads || tokens_q * q->heads > kMostTokens) return STA_ERR_SHAPE;
    if (S == 0 || (tokens_q == 0 && tokens_k == 0)) return STA_OK;
    // (smaller tiles are for launches that tiles of 128 do not fill the chip with)
    const int64_t g = q->heads / k->heads;
    if (tiles_of(tokens_q, g, S, max_q, 128) * k->heads > kMostWorkgroups || tiles_of(tokens_k, 1, S, max_k, 128) * k->heads > kMostWorkgroups) return STA_ERR_SHAPE;
    if (!cu_q || !cu_k) return STA_ERR_NULL;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse) & 3) return STA_ERR_SHAPE;
    if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < sta_packed_backward_workspace_bytes(q->heads, tokens_q)) return STA_ERR_WORKSPACE;
    const size_t used = sta_packed_backward_workspace_bytes(q->heads, tokens_q), lse_bytes = (size_t)tokens_q * q->heads * sizeof(float);
    if (ranges_meet(workspace, used, lse, lse_bytes)) return STA_ERR_ALIAS;
    for (int j = 0; j < 3; ++j) {
        for (int i = 0; i < 5; ++i)
            if (rows_overlap(*in[i], n_in[i], *out[j], n_out[j], 1, D)) return STA_ERR_ALIAS;
        for (int i = 0; i < j; ++i)
            if (rows_overlap(*out[i], n_out[i], *out[j], n_out[j], 1, D)) return STA_ERR_ALIAS;
        if (rows_meet(*out[j], 1, n_out[j], D, workspace, used) || rows_meet(*out[j], 1, n_out[j], D, lse, lse_bytes)) return STA_ERR_ALIAS;
    }
    for (int i = 0; i < 5; ++i)
        if (rows_meet(*in[i], 1, n_in[i], D, workspace, used)) return STA_ERR_ALIAS;
    const PackedBounds bounds = {cu_q, cu_k, nullptr, S};
    for (int j = 0; j < 3; ++j)
        if (bounds.meet(out[j], n_out[j], D, workspace, used)) return STA_ERR_ALIAS;
    BackwardParams b = {};
    PackedParams &p = b.p;
    p.q = packed_rows_of(*q);
    p.k = packed_rows_of(*k);
    p.v = packed_rows_of(*v);
    p.o = packed_rows_of(*o);
    b.d_o = packed_rows_of(*d_o);
    b.d_q = packed_rows_of(*d_q);
    b.d_k = packed_rows_of(*d_k);
    b.d_v = packed_rows_of(*d_v);
    p.cu_q = cu_q;
    p.cu_k = cu_k;
    p.S = S;
    p.tokens_q = (uint32_t)tokens_q;
    p.tokens_k = (uint32_t)tokens_k;
    p.max_q = max_q;
    p.max_k = max_k;
    p.Hkv = k->heads;
    p.g = (uint32_t)g;
    p.by_g = sta::fast_div_of(p.g);
    p.by_Hkv = sta::fast_div_of(p.Hkv);
    p.by_parts = sta::fast_div_of(1);
    p.causal = causal != 0;
    p.scale = scale;
    p.scale_log2e = scale * 1.4426950408889634f;
    p.parts = 1;
    p.ws = reinterpret_cast<float *>(static_cast<char *>(workspace) + stat_bytes(q->heads, tokens_q));
    b.lse = lse;
    b.neg_lse = static_cast<float *>(workspace);
    b.neg_delta = b.neg_lse + (size_t)q->heads * tokens_q + kStatPad;
    b.inv_scale = 1.0f / scale;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const int64_t slots = part_slots(q->heads, tokens_q);
    const hipError_t e = D == 64 ? launch_gradients<64>(b, max_q, max_k, slots, stream) : launch_gradients<128>(b, max_q, max_k, slots, stream);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}

}  // extern "C"
