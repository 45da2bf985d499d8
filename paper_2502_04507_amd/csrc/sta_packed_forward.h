// The forward kernels of attention over packed sequences, for keys that lie one behind the other (sta_packed.hip) and for keys in pages
// (sta_paged.hip): Params says which, and KeysOf<Params, D> how a workgroup brings them to LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_packed.h"

namespace {

// By how much a score has to exceed a row's offset for the offset to move: 2^8 in the exponent.  Finite where the scale is next to nothing: an offset
// that no score was compared with is -infinity, and stays so only where no key is seen.
__device__ __forceinline__ float grow_above_of(float c) { return fminf(8.0f / c, 3.4028234663852886e38f); }

// Running softmax of a wave's columns: offsets in the units of the scores, sums, accumulators [channel block][column block] of O^T.
template <int D, int NC, bool LSE>
struct Softmax {
    static constexpr int CB = D / 16;
    floatx4 acc[CB][NC];
    float m[NC];                    // -infinity until a key is seen
    bool far;                       // an offset is so large (masks of the type's lowest number) that its product with the scale is too coarse
    uint32_t odd;                   // not 0: a masked sub-block of V held more than numbers
    using Sum = std::conditional_t<LSE, float, floatx4>;
    Sum l[NC];                      // LSE: this lane's share of the sum; otherwise all four are the whole sum of the rounded probabilities
    __device__ __forceinline__ void start()
    {
        far = false;
        odd = 0;
#pragma unroll
        for (int col = 0; col < NC; ++col) {
            m[col] = -INFINITY;
            l[col] = Sum{};
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) acc[cb][col] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // The sum of a column (over the lanes that share it).
    __device__ __forceinline__ float sum(int col) const
    {
        if constexpr (LSE) return quad_lane_sum(l[col]);
        else return l[col][0];
    }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Bit 15 of every half of the words of eight bf16 values: set where the value is an infinity or a NaN (the exponent of both is 0x7f80, and one
// more carries into that bit); and NaN alone.
__device__ __forceinline__ uint32_t no_numbers(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ uint32_t nans(uint32_t x) { return (((x & 0x007f007fu) + 0x007f007fu) << 8) & no_numbers(x); }

// O^T += V^T P^T with a zero in the place of every value of V that is no number: where a column does not see a key, its probability is 0, and 0
// times one of those would be no 0.  odd: whether there were any.  What columns get that see them, add_no_numbers adds.
template <int D, int NC, int V_OFF>
__device__ __forceinline__ void product_of_numbers(const uint32_t (&v_addr)[4], floatx4 (&acc)[D / 16][NC], const bf16x8 (&P)[NC], uint32_t &odd)
{
    using Product = StagedTransposedProduct<D, V_OFF>;
    Product pv;
    pv.template issue<0>(v_addr);
    static_for<0, Product::NG>([&](auto gc) {
        constexpr int g = decltype(gc)::value;
        if constexpr (g + 1 < Product::NG) {
            pv.template issue<g + 1>(v_addr);
            pv_wait<8>(pv.frag[g]);
        } else {
            pv_wait<0>(pv.frag[g]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 x = __builtin_bit_cast(u32x4, __builtin_shufflevector(pv.frag[g][i][0], pv.frag[g][i][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t at = no_numbers(x[w]);
                odd |= at;
                x[w] &= ~(at | (at - (at >> 15)));
            }
#pragma unroll
            for (int col = 0; col < NC; ++col) acc[4 * g + i][col] = mfma_16x16x32(__builtin_bit_cast(bf16x8, x), P[col], acc[4 * g + i][col]);
        }
        __builtin_amdgcn_sched_barrier(0);
    });
}

// How many infinities of either sign and NaN of a sub-block of V a column sees, a product each with ones in their places; a column that
// sees one gets it.  This runs behind the walk, and only where there are any.
template <int D, int NC>
__device__ __forceinline__ void add_no_numbers(const uint32_t (&v_addr)[4], floatx4 (&acc)[D / 16][NC], const int (&lim)[NC], int first, int g4)
{
    using Product = StagedTransposedProduct<D, 0>;
    Product pv;
    bf16x8 sees[NC];
#pragma unroll
    for (int col = 0; col < NC; ++col)
#pragma unroll
        for (int i = 0; i < 8; ++i) sees[col][i] = static_cast<__bf16>(first + 4 * g4 + (i < 4 ? i : 12 + i) < lim[col] ? 1.0f : 0.0f);
    static_for<0, Product::NG>([&](auto gc) {
        constexpr int g = decltype(gc)::value;
        pv.template issue<g>(v_addr);
        pv_wait<0>(pv.frag[g]);
        static_for<0, 12>([&](auto ic) {
            constexpr int i = decltype(ic)::value / 3, cb = 4 * g + i, kind = decltype(ic)::value % 3;       // +infinity, -infinity, NaN
            u32x4 x = __builtin_bit_cast(u32x4, __builtin_shufflevector(pv.frag[g][i][0], pv.frag[g][i][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t sign = x[w] & 0x80008000u, nan = nans(x[w]), inf = no_numbers(x[w]) & ~nan;
                const uint32_t at = kind == 0 ? inf & ~sign : kind == 1 ? inf & sign : nan;
                x[w] = (at >> 1) - (at >> 8);       // 1.0
            }
#pragma unroll
            for (int col = 0; col < NC; ++col) {
                const floatx4 n = mfma_16x16x32(__builtin_bit_cast(bf16x8, x), sees[col], floatx4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    // on the bits: floating-point sums of infinities may be folded by the compiler
                    const uint32_t o = __float_as_uint(acc[cb][col][r]), add = kind == 1 ? 0xff800000u : 0x7f800000u;
                    const bool against = (o & 0x7fffffffu) > 0x7f800000u || o == (add ^ 0x80000000u);       // NaN, the other infinity
                    acc[cb][col][r] = __uint_as_float(n[r] > 0.f ? (kind == 2 || against ? 0x7fc00000u : add) : o);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    });
}

// U sub-blocks of 32 keys, SUB bytes apart in LDS: K at OFF of k_addr in the layout StagedRows, V at OFF of v_addr in the layout Staged.  lim: how
// many keys a column sees; first: the first sub-block's first key.
// kFollow: every column sees all keys, and the offsets follow the largest scores.  kFixed: the same with the offsets as they are: probabilities, sums
// and accumulators have eight exponent bits, so an offset that is too low costs nothing until the sums near the end of that range, which is
// looked at behind the walk.  kMasked: some column may not see all keys; the offsets follow.  kCareful: so, and V may hold more than numbers.
constexpr int kFollow = 0, kFixed = 1, kMasked = 2, kCareful = 3;
template <int D, int NC, bool LSE, int MODE, int U, int SUB, int OFF>
__device__ __forceinline__ void softmax_sub_blocks(Softmax<D, NC, LSE> &st, uint32_t k_addr, const uint32_t (&v_addr)[4],
                                                   const bf16x8 (&Q)[NC][D / 32], float c, float grow_above, int first,
                                                   const int (&lim)[NC], int g4)
{
    constexpr bool MASKED = MODE >= kMasked;
    floatx4 S[U][2][NC];
    static_for<0, U>([&](auto uc) {
        constexpr int u = decltype(uc)::value;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int col = 0; col < NC; ++col) S[u][kb][col] = floatx4{0.f, 0.f, 0.f, 0.f};
        rows_times_resident<D, OFF + u * SUB, NC, 4>(k_addr, Q, S[u]);
        if constexpr (MASKED) {                             // a select, whatever the score is
#pragma unroll
            for (int col = 0; col < NC; ++col) {
                const int left = lim[col] - first - kSub * u - 4 * g4;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[u][kb][col][r] = 16 * kb + r < left ? S[u][kb][col][r] : -INFINITY;
            }
        }
    });
    if constexpr (MODE != kFixed) {
        // The offset only moves when a score exceeds it by more than grow_above.
        float mx[NC];
        bool grown = false;
#pragma unroll
        for (int col = 0; col < NC; ++col) {
            float m = S[0][0][col][0];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                m = max3(m, S[u][0][col][0], S[u][0][col][1]);
                m = max3(m, S[u][0][col][2], S[u][0][col][3]);
                m = max3(m, S[u][1][col][0], S[u][1][col][1]);
                m = max3(m, S[u][1][col][2], S[u][1][col][3]);
            }
            mx[col] = quad_lane_max(m);
            grown = grown || mx[col] > st.m[col] + grow_above;
        }
        if (__builtin_amdgcn_ballot_w64(grown) != 0) {
            bool far = false;
#pragma unroll
            for (int col = 0; col < NC; ++col) {
                const bool up = mx[col] > st.m[col] + grow_above;
                const float alpha = up ? __builtin_amdgcn_exp2f((st.m[col] - mx[col]) * c) : 1.f;
                st.m[col] = up ? mx[col] : st.m[col];
                st.l[col] *= alpha;
#pragma unroll
                for (int cb = 0; cb < D / 16; ++cb) st.acc[cb][col] *= alpha;
                far = far || (fabsf(st.m[col] * c) > 1024.f && st.m[col] != -INFINITY);
            }
            st.far = __builtin_amdgcn_ballot_w64(far) != 0;
        }
        if (__builtin_expect(st.far, 0)) {                      // the difference first, which is exact
#pragma unroll
            for (int col = 0; col < NC; ++col)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int r = 0; r < 4; ++r) S[u][kb][col][r] -= st.m[col] == -INFINITY ? 0.f : st.m[col];
        }
    }
    StagedTransposedProduct<D, OFF> pv;
    if constexpr (MODE != kCareful) {
        pv.prefetch(v_addr);
        __builtin_amdgcn_sched_barrier(0);
    }
    bf16x8 P[U][NC];
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const float mc = MODE == kFixed ? st.m[col] * c : st.far || st.m[col] == -INFINITY ? 0.f : st.m[col] * c;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(S[u][kb][col][r], c, -mc));
                    if constexpr (LSE) sum += e;
                    P[u][col][4 * kb + r] = static_cast<__bf16>(e);
                }
        if constexpr (LSE) {
            st.l[col] += sum;
            // Here, and not in the next stage: the compiler would keep the probabilities until then, and its registers run out in the loop, where
            // a reload waits for the stage that has just been asked for.
            asm volatile("" : "+v"(st.l[col]));
            __builtin_amdgcn_sched_barrier(0);              // one column's scores at a time: fewer registers
        }
    }
    if constexpr (!LSE) {
        bf16x8 ones;
#pragma unroll
        for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(1.0f);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int col = 0; col < NC; ++col) st.l[col] = mfma_16x16x32(ones, P[u][col], st.l[col]);
    }
    if constexpr (MODE == kCareful) {
        static_for<0, U>([&](auto uc) { product_of_numbers<D, NC, OFF + decltype(uc)::value * SUB>(v_addr, st.acc, P[decltype(uc)::value], st.odd); });
    } else {
        pv.template run<NC>(v_addr, P[0], st.acc);
        static_for<1, U>([&](auto uc) {
            StagedTransposedProduct<D, OFF + decltype(uc)::value * SUB> more;
            more.prefetch(v_addr);
            more.template run<NC>(v_addr, P[decltype(uc)::value], st.acc);
        });
    }
}

// ln of the denominator of a row whose offset is m (in scores) and whose sum is l: -infinity where no key was seen, which leaves the sum at 0.  NaN
// stays NaN; the bits are looked at, because the kernels are compiled as if comparisons met none.
__device__ __forceinline__ float lse_of(float m, float l, const PackedParams &p)
{
    uint32_t bits = __float_as_uint(l);
    asm volatile("" : "+v"(bits));
    return bits == 0 ? -INFINITY : fmaf(m, p.scale, __logf(l));
}

// What a part of a row whose offset is `own` counts where the row's is m.  Offsets are compared as scores: their products with the scale, in units of
// two to the one, may pass the largest number where they do not, and the smallest of those would be a part that has seen no key.
__device__ __forceinline__ float weight_of(float own, float m, float c) { return own == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((own - m) * c); }

// Where a column's row lies.
struct RowAt {
    int token, head;                // inside the sequence and the group
    bool on;
};
__device__ __forceinline__ RowAt row_at(uint32_t row, uint32_t rows, const PackedParams &p)
{
    const bool on = row < rows;
    const uint32_t r = on ? row : rows - 1;
    const uint32_t t = sta::fast_div(r, p.by_g);
    return {(int)t, (int)(r - t * p.g), on};
}

template <int D, int NC>
__device__ __forceinline__ void load_queries(const PackedParams &p, const PackedSeq &seq, uint32_t kv, uint32_t row0, uint32_t rows, int lane, bf16x8 (&Q)[NC][D / 32])
{
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const RowAt at = row_at(row0 + 16 * col + (lane & 15), rows, p);
        const char *row = p.q.data + (int64_t)(seq.q0 + at.token) * p.q.token + (int64_t)(kv * p.g + at.head) * p.q.head;
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) Q[col][ks] = *reinterpret_cast<const bf16x8 *>(row + 64 * ks + 16 * (lane >> 4));
    }
}

// How many keys the columns of a wave see.
template <int NC>
__device__ __forceinline__ void limits_of(const PackedParams &p, const PackedSeq &seq, uint32_t row0, uint32_t rows, int lane, int (&lim)[NC])
{
#pragma unroll
    for (int col = 0; col < NC; ++col) lim[col] = seq.keys_of(row_at(row0 + 16 * col + (lane & 15), rows, p).token, p);
}

// Partial sums of a tile's part: accumulators [R][D], then offsets (in scores) and sums of the rows.
template <int D, int R>
constexpr size_t part_floats() { return (size_t)R * D + 2 * R; }

// The tile's rank of a launch's item, and which part it is; sub-blocks of a part of a tile of 128 rows.
__device__ __forceinline__ uint32_t rank_of(uint32_t item, const PackedParams &p, uint32_t *part)
{
    const uint32_t rank = sta::fast_div(item, p.by_parts);
    *part = item - rank * p.parts;
    return rank;
}
__device__ __forceinline__ uint32_t part_subs_of(const PackedParams &p, int) { return p.part_subs; }

// How many parts of `each` a walk of n sub-blocks has, and where one ends: the last one takes what is left.
__device__ __forceinline__ int parts_of(int n, uint32_t each, const PackedParams &p)
{
    const int want = (n + (int)each - 1) / (int)each;
    return want < (int)p.parts ? want : (int)p.parts;
}
__device__ __forceinline__ int part_end(uint32_t part, int n, uint32_t each, const PackedParams &p)
{
    const int end = (int)((part + 1) * each);
    return part + 1 == p.parts || end > n ? n : end;
}

// slot: the tile's rank (few rows: the sequence), below what the launch and the workspace have, whatever the bounds on the device say.
__device__ __forceinline__ float *part_at(const PackedParams &p, size_t slot, uint32_t kv, uint32_t part, size_t floats)
{
    return p.ws + ((slot * p.Hkv + kv) * p.parts + part) * floats;
}

// The place of a workgroup in the order of the walks: every other round of workgroups over an XCD's CUs is turned around, so that the CU that has the
// longest walk of one round has the shortest of the next.  XCDs, and so the key heads on them, stay as they are.  Not where tiles are cut: parts of a
// tile are equal.  16 heads of 64 channels, [2048] * 4: 46.7 us, 50.0 without; 24 heads of 128, [1000] * 4: 38.8, 39.7; the chunk of 512 tokens, cut,
// 224 with, 210 without; and the gradients' kernels, 5 % faster to 8 % slower, are left as they are.
__device__ __forceinline__ uint32_t place_of_block(const PackedParams &p)
{
    constexpr uint32_t XCDS = 8, CUS = 32;
    const uint32_t b = blockIdx.x, round = b / (XCDS * CUS);
    return p.parts == 1 && (round & 1) && (round + 1) * XCDS * CUS <= gridDim.x ? (2 * round + 1) * XCDS * CUS - XCDS - b + 2 * (b % XCDS) : b;
}

// How a workgroup brings keys and values to LDS: start() for its sequence and key head; look_up() before the first of a walk's stages, which here needs nothing;
// bring() a stage (bring_stage says how), of which `next` is the following one of this wave; settle() behind the wait for an earlier stage; bring_values()
// one group of rows of V from row `first` on.
template <class Params, int D>
struct KeysOf;

template <int D>
struct KeysOf<PackedParams, D> {
    const char *kh, *vh;
    PackedDma<D, true> k_dma;
    PackedDma<D, false> v_dma;
    __device__ __forceinline__ void start(const PackedParams &p, const PackedSeq &seq, uint32_t kv, int lane)
    {
        kh = p.k.data + (int64_t)seq.k0 * p.k.token + (int64_t)kv * p.k.head;
        vh = p.v.data + (int64_t)seq.k0 * p.v.token + (int64_t)kv * p.v.head;
        k_dma.start(lane, p.k.token);
        v_dma.start(lane, p.v.token);
    }
    template <int SUBS>
    __device__ __forceinline__ void look_up(const PackedParams &, const PackedSeq &, int) {}
    template <int SUBS, int COUNT, int K_GROUP, int V_GROUP>
    __device__ __forceinline__ void bring(const PackedParams &p, const PackedSeq &seq, int sub, int, int from, char *to, int v_at, int apart)
    {
        bring_stage<SUBS, COUNT, K_GROUP, V_GROUP>(k_dma, v_dma, kh, vh, p.k.token, p.v.token, sub, seq.lk, from, to, v_at, apart);
    }
    __device__ __forceinline__ void settle() {}
    __device__ __forceinline__ void bring_values(const PackedParams &p, const PackedSeq &seq, int first, char *dst) const { v_dma.bring_part(vh, p.v.token, first, seq.lk, dst); }
};

// The same for the kernel of tiles, whose KG groups take stages of U sub-blocks in turn: bring_turn() brings the group's stage number i, which begins with sub-block `sub`.
template <class Params, int D, int KG>
struct TileKeys : KeysOf<Params, D> {
    template <int SUBS, int COUNT, int K_GROUP, int V_GROUP>
    __device__ __forceinline__ void bring_turn(const Params &p, const PackedSeq &seq, int sub, int, int from, char *to, int v_at, int apart)
    {
        this->template bring<SUBS, COUNT, K_GROUP, V_GROUP>(p, seq, sub, sub + SUBS * KG, from, to, v_at, apart);
    }
};

// RW waves of 32 rows; KG groups of them take the stages of U sub-blocks in turn, each with LDS of its own, and are joined at the end: small launches
// are cut that way inside the workgroups.
// The walk.  Of the stages that every row sees all of, the first sets the offsets and the others run without following the scores (20 of 83
// vector instructions a sub-block at head dimension 128 go with that, and the matrix pipe bounds it instead of them: prompts of 8192 and 4097 tokens, 32 heads over 8,
// us at best 706 and 623 at that step); the stages that some row does not see all of follow and mask.  At the end the results are looked at: sums beyond 2^96 or below
// 2^-64, offsets too large to be multiplied by the scale, or accumulators that are no numbers (a value that is none, seen or not), and the workgroup
// walks again with care.
template <class Params, int D, bool LSE, int U, int RW, int KG>
__global__ __launch_bounds__(RW * KG * 64, KG > 2 && D == 128 ? 1 : KG > 2 ? 2 : KG > 1 ? (D == 64 ? 4 : 2) : 3) void sta_packed_tile_kernel(Params p)
{
    constexpr int NC = 2, CB = D / 16, TILE = 32 * RW;
    using LK = StagedRows<D>;
    using LV = Staged<D>;
    constexpr int SUB = LK::Tile + LV::Tile, STAGE = U * SUB, V_AT = LK::Tile, PER_WAVE = LV::Groups / RW;
    constexpr int WAVE_ACC = CB * NC * 1024, MERGE = KG > 1 ? RW * KG * WAVE_ACC : 0;
    __shared__ __attribute__((aligned(1024))) char smem[2 * KG * STAGE > MERGE ? 2 * KG * STAGE : MERGE];
    __shared__ float2 stats[KG > 1 ? KG : 1][TILE];         // offset (in scores) and sum of a group's rows
    const int lane = threadIdx.x & 63, all_waves = uniform(threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    const int kg = all_waves / RW, wave = all_waves % RW;
    // key heads next to each other: workgroup ids go to the 8 XCDs in turn, and a head's keys stay in one L2 where Hkv is a multiple of 8
    const uint32_t place = place_of_block(p), item = sta::fast_div(place, p.by_Hkv), kv = place - item * p.Hkv;
    uint32_t part;
    const uint32_t rank = rank_of(item, p, &part);
    PackedTile tile;
    if (!find_tile<TILE, false>(rank, p, lane, &tile)) return;
    const PackedSeq seq = tile.seq;
    const uint32_t rows = (uint32_t)seq.lq * p.g, row0 = tile.index * TILE;
    const uint32_t last_row = row0 + TILE < rows ? row0 + TILE - 1 : rows - 1;
    const int n_keys = uniform(seq.keys_of((int)sta::fast_div(last_row, p.by_g), p));
    const int n_all = (n_keys + kSub - 1) / kSub;
    const uint32_t each = RW == 4 ? part_subs_of(p, lane) : p.part_subs;
    const int sub0 = (int)(part * each);
    const int sub1 = part_end(part, n_all, each, p);
    if (part > 0 && sub0 >= n_all) return;                  // the first part of a tile without keys writes its zeros

    const uint32_t wave_row = row0 + 32 * wave;
    const bool idle = wave_row >= rows;
    const uint32_t wave_last = wave_row + 31 < rows ? wave_row + 31 : rows - 1;
    const int n_whole = uniform(seq.keys_of((int)sta::fast_div(row0, p.by_g), p));          // keys that all rows see
    const int lim_hi = idle ? 0 : uniform(seq.keys_of((int)sta::fast_div(wave_last, p.by_g), p));

    TileKeys<Params, D, KG> keys;
    keys.start(p, seq, kv, lane);
    char *own = smem + 2 * kg * STAGE;
    // sub .. sub + U - 1; those of the last stage that nobody sees are brought as well, from the last key's row
    auto issue = [&](int stage, int i, int sub) __attribute__((always_inline)) {
        if (sub < sub1) keys.template bring_turn<U, PER_WAVE, LK::Group, LV::Group>(p, seq, sub, i, PER_WAVE * wave, own + stage * STAGE, V_AT, SUB);
    };
    // the group's stage number i begins with sub-block sub_of(i); all groups go around n_steps times
    auto sub_of = [&](int i) { return sub0 + U * (kg + KG * i); };
    const int n_steps = (sub1 - sub0 + U * KG - 1) / (U * KG);
    keys.template look_up<U>(p, seq, sub_of(0));
    issue(0, 0, sub_of(0));

    bf16x8 Q[NC][D / 32];
    load_queries<D, NC>(p, seq, kv, wave_row, rows, lane, Q);
    const uint32_t base = (uint32_t)(uintptr_t)own;
    const uint32_t k_addr = LK::address(base, lane);
    uint32_t v_addr[4];
    LV::transposed_addresses(base + V_AT, lane, v_addr);
    Softmax<D, NC, LSE> st;
    const float c = p.scale_log2e, grow_above = grow_above_of(c);
    int lim[NC] = {};                                       // found where the tail begins
    auto step = [&](auto stage_c, auto mode_c, int i) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage_c)::value, MODE = decltype(mode_c)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wave's part of the stage has landed
        if constexpr (RW > 1) __syncthreads();              // ... and everyone's, and nobody reads the other stage any more (one wave: its own alone)
        issue(ST ^ 1, i + 1, sub_of(i + 1));
        const int sub = sub_of(i), first = sub * kSub;
        if (MODE < kMasked || (sub < sub1 && first < lim_hi))
            softmax_sub_blocks<D, NC, LSE, MODE, U, SUB, ST * STAGE>(st, k_addr, v_addr, Q, c, grow_above, first, lim, g4);
    };
    using Stage0 = std::integral_constant<int, 0>;
    using Stage1 = std::integral_constant<int, 1>;
    using Follow = std::integral_constant<int, kFollow>;
    using Fixed = std::integral_constant<int, kFixed>;
    using Masked = std::integral_constant<int, kMasked>;
    using Careful = std::integral_constant<int, kCareful>;
    // stages of all groups that every row of the tile sees all of
    const int seen_by_all = (n_whole / kSub < sub1 ? n_whole / kSub : sub1) - sub0, n_fixed = seen_by_all > 0 ? seen_by_all / (U * KG) : 0;
    int i = 0;
    st.start();
    if (n_fixed >= 2) {
        step(Stage0{}, Follow{}, 0);
        step(Stage1{}, Fixed{}, 1);
#pragma unroll 1
        for (i = 2; i + 2 <= n_fixed; i += 2) {
            step(Stage0{}, Fixed{}, i);
            step(Stage1{}, Fixed{}, i + 1);
        }
    }
    const bool fixed = i > 0;
    limits_of<NC>(p, seq, wave_row, rows, fresh_lane(), lim);
#pragma unroll 1
    for (; i < n_steps; i += 2) {                           // i is even
        step(Stage0{}, Masked{}, i);
        if (i + 1 < n_steps) step(Stage1{}, Masked{}, i + 1);
    }
    constexpr float kRedoAbove = 79228162514264337593543950336.f, kRedoBelow = 5.42101086242752217e-20f;     // 2^96, 2^-64
    bool bad = false;
    uint32_t most = 0;
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const float l = st.sum(col);
        bad = bad || (fixed && (st.far || !(l < kRedoAbove) || l < kRedoBelow));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int r = 0; r < 4; ++r) most = max(most, __float_as_uint(st.acc[cb][col][r]) & 0x7fffffffu);
    }
    if (__builtin_expect(__syncthreads_or(bad || most >= 0x7f800000u), 0)) {
        st.start();
        keys.template look_up<U>(p, seq, sub_of(0));
        issue(0, 0, sub_of(0));
#pragma unroll 1
        for (i = 0; i < n_steps; i += 2) {
            step(Stage0{}, Careful{}, i);
            if (i + 1 < n_steps) step(Stage1{}, Careful{}, i + 1);
        }
        if (__syncthreads_or(st.odd != 0)) {
#pragma unroll 1
            for (i = 0; i < n_steps; ++i) {
#pragma unroll 1
                for (int sub = sub_of(i); sub < sub_of(i) + U; ++sub) {
#pragma unroll 1
                    for (int j = 0; j < PER_WAVE; ++j)
                        keys.bring_values(p, seq, sub * kSub + (PER_WAVE * wave + j) * LV::GroupRows, own + V_AT + (PER_WAVE * wave + j) * LV::Group);
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                    if (sub < sub1 && sub * kSub < lim_hi) add_no_numbers<D, NC>(v_addr, st.acc, lim, sub * kSub, g4);
                    __syncthreads();
                }
            }
        }
    }

    // ---- the groups' sums are joined: a wave takes its rows' channel blocks of its group's share, the groups' parts in ascending order
    float m[NC], l[NC];
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        m[col] = st.m[col];
        l[col] = st.sum(col);
    }
    constexpr int OWN = CB / KG;                            // channel blocks that a wave writes
    const int cb0 = KG > 1 ? OWN * kg : 0;
    if constexpr (KG > 1) {
        __syncthreads();
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int col = 0; col < NC; ++col)
                *reinterpret_cast<floatx4 *>(smem + (kg * RW + wave) * WAVE_ACC + (cb * NC + col) * 1024 + lane * 16) = st.acc[cb][col];
        if (g4 == 0)
#pragma unroll
            for (int col = 0; col < NC; ++col) stats[kg][32 * wave + 16 * col + c16] = make_float2(m[col], l[col]);
        __syncthreads();
#pragma unroll
        for (int col = 0; col < NC; ++col) {
            float weight[KG];
            m[col] = -INFINITY;
            l[col] = 0.f;
#pragma unroll
            for (int g = 0; g < KG; ++g) m[col] = fmaxf(m[col], stats[g][32 * wave + 16 * col + c16].x);
#pragma unroll
            for (int g = 0; g < KG; ++g) {
                const float2 x = stats[g][32 * wave + 16 * col + c16];
                weight[g] = weight_of(x.x, m[col], c);
                l[col] += x.y * weight[g];
            }
#pragma unroll
            for (int j = 0; j < OWN; ++j) {
                floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int g = 0; g < KG; ++g) {
                    const floatx4 x = *reinterpret_cast<const floatx4 *>(smem + (g * RW + wave) * WAVE_ACC + ((cb0 + j) * NC + col) * 1024 + lane * 16);
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[r] = fmaf(x[r], weight[g], sum[r]);
                }
                st.acc[j][col] = sum;
            }
        }
    }
    if (idle) return;
    const int last_lane = fresh_lane(), last_g4 = last_lane >> 4;
    if (parts_of(n_all, each, p) > 1) {
        float *ws = part_at(p, rank, kv, part, part_floats<D, TILE>());
#pragma unroll
        for (int col = 0; col < NC; ++col) {
            const int r = 32 * wave + 16 * col + (last_lane & 15);
#pragma unroll
            for (int j = 0; j < OWN; ++j) *reinterpret_cast<floatx4 *>(ws + (size_t)r * D + 16 * (cb0 + j) + 4 * last_g4) = st.acc[j][col];
            if (last_g4 == 0 && kg == 0) {
                ws[(size_t)TILE * D + r] = m[col];
                ws[(size_t)TILE * D + TILE + r] = l[col];
            }
        }
        return;
    }
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const float inv = l[col] > 0.f ? 1.f / l[col] : 0.f;
        const RowAt at = row_at(wave_row + 16 * col + (last_lane & 15), rows, p);
        if (!at.on) continue;
        const int64_t token = seq.q0 + at.token, head = kv * p.g + at.head;
        char *row = p.o.data + token * p.o.token + head * p.o.head;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
            bf16x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = static_cast<__bf16>(st.acc[j][col][r] * inv);
            *reinterpret_cast<bf16x4 *>(row + 32 * (cb0 + j) + 8 * last_g4) = v;
        }
        if (LSE && p.lse && last_g4 == 0 && kg == 0) p.lse[head * p.tokens_q + token] = lse_of(m[col], l[col], p);
    }
}

// Rows of one sequence and key head: at most 16 * NC.  Workgroup (part, key head, sequence).
template <class Params, int D, int NC, bool LSE>
__global__ __launch_bounds__(256) void sta_packed_few_kernel(Params p)
{
    constexpr int CB = D / 16, R = 16 * NC;
    using LK = StagedRows<D>;
    using LV = Staged<D>;
    constexpr int STAGE = LK::Tile + LV::Tile, V_AT = LK::Tile, OPS = LK::Groups + LV::Groups;
    constexpr int WAVE = 2 * STAGE, MERGE = CB * NC * 1024;         // a wave's LDS; its accumulators at the end
    static_assert(MERGE <= WAVE, "LDS");
    __shared__ __attribute__((aligned(1024))) char smem[4 * WAVE];
    __shared__ float2 stats[4][R];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    const uint32_t s = sta::fast_div(item, p.by_parts), part = item - s * p.parts;
    PackedSeq seq = seq_of(s, p);
    const uint32_t all_rows = (uint32_t)seq.lq * p.g, rows = all_rows < R ? all_rows : R;
    if (rows == 0) return;
    const int n_keys = uniform(seq.keys_of((int)sta::fast_div(rows - 1, p.by_g), p));
    const int n_all = (n_keys + kSub - 1) / kSub;
    const int sub0 = (int)(part * p.part_subs);
    const int sub1 = part_end(part, n_all, p.part_subs, p);
    if (part > 0 && sub0 >= n_all) return;

    int lim[NC];
    limits_of<NC>(p, seq, 0, rows, lane, lim);
    const int n_whole = uniform(seq.keys_of(0, p));         // keys that all rows see

    KeysOf<Params, D> keys;
    keys.start(p, seq, kv, lane);
    char *own = smem + wave * WAVE;
    auto issue = [&](int stage, int sub) __attribute__((always_inline)) {
        keys.template bring<1, LK::Groups, LK::Group, LV::Group>(p, seq, sub, sub + 4, 0, own + stage * STAGE, V_AT, 0);
    };
    int sub = sub0 + wave;
    bf16x8 Q[NC][D / 32];
    load_queries<D, NC>(p, seq, kv, 0, rows, lane, Q);
    if (sub < sub1) {
        keys.template look_up<1>(p, seq, sub);
        issue(0, sub);
    }
    const uint32_t base = (uint32_t)(uintptr_t)own;
    const uint32_t k_addr = LK::address(base, lane);
    uint32_t v_addr[4];
    LV::transposed_addresses(base + V_AT, lane, v_addr);
    Softmax<D, NC, LSE> st;
    st.start();
    const float c = p.scale_log2e, grow_above = grow_above_of(c);
    auto step = [&](auto stage_c, auto masked_c, int sub) __attribute__((always_inline)) {
        constexpr int ST = decltype(stage_c)::value;
        __builtin_amdgcn_sched_barrier(0);                  // reads of the other stage are done: their values have been used
        if (sub + 4 < sub1) {
            issue(ST ^ 1, sub + 4);
            wait_dma<OPS>();
            keys.settle();
        } else {
            wait_dma<0>();
        }
        const int first = sub * kSub;
        softmax_sub_blocks<D, NC, LSE, decltype(masked_c)::value ? kCareful : kFollow, 1, STAGE, ST * STAGE>(st, k_addr, v_addr, Q, c, grow_above, first, lim, g4);
    };
    using Stage0 = std::integral_constant<int, 0>;
    using Stage1 = std::integral_constant<int, 1>;
#pragma unroll 1
    for (; sub + 4 < sub1 && (sub + 5) * kSub <= n_whole; sub += 8) {
        step(Stage0{}, std::false_type{}, sub);
        step(Stage1{}, std::false_type{}, sub + 4);
    }
    const int tail = sub;
#pragma unroll 1
    for (; sub < sub1; sub += 8) {
        step(Stage0{}, std::true_type{}, sub);
        if (sub + 4 < sub1) step(Stage1{}, std::true_type{}, sub + 4);
    }
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(st.odd != 0) != 0, 0)) {
#pragma unroll 1
        for (sub = tail; sub < sub1; sub += 4) {
            __builtin_amdgcn_sched_barrier(0);
            keys.template look_up<1>(p, seq, sub);
            issue(0, sub);
            wait_dma<0>();
            add_no_numbers<D, NC>(v_addr, st.acc, lim, sub * kSub, g4);
        }
    }

    // ---- merge of the four waves: every wave sums the parts of its channel blocks, in ascending order
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int col = 0; col < NC; ++col) *reinterpret_cast<floatx4 *>(own + (cb * NC + col) * 1024 + lane * 16) = st.acc[cb][col];
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        const float l = st.sum(col);
        if (g4 == 0) stats[wave][16 * col + c16] = make_float2(st.m[col], l);
    }
    __syncthreads();
    const bool whole = parts_of(n_all, p.part_subs, p) <= 1;
    float *ws = whole ? nullptr : part_at(p, s, kv, part, part_floats<D, R>());
#pragma unroll
    for (int col = 0; col < NC; ++col) {
        float m = -INFINITY, l = 0.f, weight[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, stats[w][16 * col + c16].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 x = stats[w][16 * col + c16];
            weight[w] = weight_of(x.x, m, c);
            l += x.y * weight[w];
        }
        const float inv = whole ? (l > 0.f ? 1.f / l : 0.f) : 1.f;
        const RowAt at = row_at(16 * col + c16, rows, p);
        const int64_t token = seq.q0 + at.token, head = kv * p.g + at.head;
#pragma unroll
        for (int j = 0; j < CB / 4; ++j) {
            const int cb = wave * (CB / 4) + j;
            floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(smem + w * WAVE + (cb * NC + col) * 1024 + lane * 16);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[r] = fmaf(x[r], weight[w], sum[r]);
            }
            if (!at.on) continue;
            if (whole) {
                bf16x4 v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = static_cast<__bf16>(sum[r] * inv);
                *reinterpret_cast<bf16x4 *>(p.o.data + token * p.o.token + head * p.o.head + 32 * cb + 8 * g4) = v;
            } else {
                *reinterpret_cast<floatx4 *>(ws + (size_t)(16 * col + c16) * D + 16 * cb + 4 * g4) = sum;
            }
        }
        if (wave == 0 && g4 == 0 && at.on) {
            if (!whole) {
                ws[(size_t)R * D + 16 * col + c16] = m;
                ws[(size_t)R * D + R + 16 * col + c16] = l;
            } else if (LSE && p.lse) {
                p.lse[head * p.tokens_q + token] = lse_of(m, l, p);
            }
        }
    }
}

// Joins the parts of the rows of a tile: O = sum_j 2^(m_j - m) O_j / sum_j 2^(m_j - m) l_j, in ascending order.  D / 4 lanes a row, four
// channels a lane.
template <class Params, int D, int R, bool TILES>
__global__ __launch_bounds__(256) void sta_packed_merge_kernel(Params p)
{
    constexpr int LPR = D / 4, ROWS = 256 / LPR;
    const int lane = threadIdx.x & 63;
    const uint32_t item = sta::fast_div(blockIdx.x, p.by_Hkv), kv = blockIdx.x - item * p.Hkv;
    PackedTile tile;
    if constexpr (TILES) {
        if (!find_tile<R, false>(item, p, lane, &tile)) return;
    } else {
        tile.seq = seq_of(item, p);
        tile.index = 0;
    }
    const PackedSeq seq = tile.seq;
    const uint32_t rows = (uint32_t)seq.lq * p.g, row0 = tile.index * R;
    const uint32_t in_tile = rows - row0 < (uint32_t)R ? rows - row0 : (uint32_t)R;
    if (rows == 0) return;
    const uint32_t r = blockIdx.y * ROWS + threadIdx.x / LPR;
    const int n_all = (seq.keys_of((int)sta::fast_div(row0 + in_tile - 1, p.by_g), p) + kSub - 1) / kSub;
    const int n = parts_of(n_all, TILES && R == 128 ? part_subs_of(p, lane) : p.part_subs, p), ch = 4 * (threadIdx.x % LPR);
    if (r >= in_tile || n <= 1) return;
    const size_t floats = part_floats<D, R>();
    const float *ws = part_at(p, item, kv, 0, floats);
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < n; ++j) m = fmaxf(m, ws[j * floats + (size_t)R * D + r]);
    floatx4 sum = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < n; ++j) {
        const float *part = ws + j * floats;
        const float w = weight_of(part[(size_t)R * D + r], m, p.scale_log2e);
        l = fmaf(part[(size_t)R * D + R + r], w, l);
        const floatx4 x = *reinterpret_cast<const floatx4 *>(part + (size_t)r * D + ch);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(x[i], w, sum[i]);
    }
    const RowAt at = row_at(row0 + r, rows, p);
    const int64_t token = seq.q0 + at.token, head = kv * p.g + at.head;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    bf16x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = static_cast<__bf16>(sum[i] * inv);
    *reinterpret_cast<bf16x4 *>(p.o.data + token * p.o.token + head * p.o.head + 2 * ch) = v;
    if (p.lse && ch == 0) p.lse[head * p.tokens_q + token] = lse_of(m, l, p);
}

// How a launch is cut.  Rows of one sequence and key head that fit 16 or 32 columns take the kernel for few rows.  Others: tiles of 128 rows that
// share every stage where they are two and a quarter a CU (head dimension 64: three) or more, else tiles of 64 rows by two groups that take the stages
// in turn, or of 32 by four.  Tiles are cut along the keys where that puts more of the chip to work than the sums in memory and their merge, 5 to
// 9 us, take.  us of a call, causal unless said, heads / key heads x channels (tiles of 128 rows | two groups | four groups):
//   32/8 x 128, [400] * 6              22 | 30 | -       24/24 x 128, [1000] * 4   40 | 50 | -       40/8 x 128, [774]         22 | 18.5 | 36
//   16/16 x 64, [2048] * 4             51 | 60 | -       333 .. 2048 (1088 tiles of 64, 576 of 128)  31 | 25 | -
//   2/2 x 64, [2100, 300]              28 | 19 | 14.6    8/8 x 128, five of 8 .. 819 (256 of 64)     22 | 16 | 18
// and cut: 32/8 x 128, 512 rows on 16384 keys: 280 | 188 | 272 whole, 148 in parts of 64 sub-blocks of tiles of 128; 24/24 x 64, 333 on 20000: 217 | 151 | 119
// whole, 67; 16/2 x 128, 200 on 4000: 74 | 47 | 34, 30 in parts of two groups; not worth it: 40/8 x 128, 300 on 1500 (24 whole, 32 cut), [774] (18.5, 27).
// Few rows, 48 single tokens on caches of 1 to 16384 keys, parts of a chip's 2, 4, 8, 16, 32 workgroups a CU, with the merge: 356, 323, 324, 316, 330.
struct PackedPlan {
    int few;                        // 0: tiles; 1, 2: blocks of 16 columns
    int waves;                      // tiles of 32 * waves rows by 4 / waves groups
    uint32_t slots;                 // tiles (few: sequences), an upper bound
    uint32_t parts, part_subs;
    size_t floats;                  // of the parts
    size_t workspace() const { return parts > 1 ? floats : 0; }
};

constexpr uint32_t kNoParts = 1u << 30;

bool plan_of(int Hq, int Hkv, int D, int S, int64_t tokens_q, int max_q, int max_k, bool cut, PackedPlan *plan)
{
    const int64_t g = Hq / Hkv, rows = g * max_q, cus = sta::compute_units(), subs = ((int64_t)max_k + kSub - 1) / kSub;
    auto tiles = [&](int64_t tile) { return tiles_of(tokens_q, g, S, max_q, tile); };
    plan->few = rows <= 16 ? 1 : rows <= 32 ? 2 : 0;
    plan->waves = 4;
    int64_t want = cut && plan->few ? 4 * cus : 0, least = 16;
    if (!plan->few && tiles(128) * Hkv < (D == 64 ? 12 : 9) * cus / 4) {
        const int64_t halves = tiles(64) * Hkv;
        plan->waves = 2;
        if (halves < 2 * cus && cut && subs >= 256) {
            plan->waves = 4;
            want = 6 * cus;
            least = 64;
        } else if (halves < cus / 4 && cut && subs >= 48) {
            want = 2 * cus;
        } else if (halves < 3 * cus / 4) {
            plan->waves = 1;
        }
    }
    const int R = plan->few ? 16 * plan->few : 32 * plan->waves;
    const int64_t slots = plan->few ? S : tiles(R);
    plan->parts = 1;
    plan->part_subs = kNoParts;
    const int64_t items = slots * Hkv;
    if (items > kMostWorkgroups) return false;
    plan->slots = (uint32_t)slots;
    if (items > 0 && items < want / 2) {
        int64_t parts = (want + items - 1) / items, each = (subs + parts - 1) / parts;
        each = each < least ? least : (each + 7) & ~(int64_t)7;          // whole stages of all groups end with a part
        parts = (subs + each - 1) / each;
        if (parts > 1 && items * parts <= kMostWorkgroups) {
            plan->parts = (uint32_t)parts;
            plan->part_subs = (uint32_t)each;
        }
    }
    plan->floats = (size_t)items * plan->parts * ((size_t)R * D + 2 * R);
    return true;
}

template <int D, bool LSE, int RW, class Params>
hipError_t launch_tiles(const Params &p, const PackedPlan &plan, hipStream_t stream)
{
    constexpr int KG = 4 / RW, U = D == 64 && KG < 2 ? 2 : 1, ROWS = 1024 / D;
    const uint32_t items = plan.slots * p.Hkv;
    const hipError_t e = sta::launch_kernel(sta_packed_tile_kernel<Params, D, LSE, U, RW, KG>, dim3(items * plan.parts), dim3(256), stream, p);
    if constexpr (RW == 1) return e;                       // (never cut)
    else if (e != hipSuccess || plan.parts == 1) return e;
    else return sta::launch_kernel(sta_packed_merge_kernel<Params, D, 32 * RW, true>, dim3(items, 32 * RW / ROWS), dim3(256), stream, p);
}

template <int D, bool LSE, int NC, class Params>
hipError_t launch_few(const Params &p, const PackedPlan &plan, hipStream_t stream)
{
    constexpr int ROWS = 1024 / D;
    const uint32_t items = plan.slots * p.Hkv;
    const hipError_t e = sta::launch_kernel(sta_packed_few_kernel<Params, D, NC, LSE>, dim3(items * plan.parts), dim3(256), stream, p);
    if (e != hipSuccess || plan.parts == 1) return e;
    return sta::launch_kernel(sta_packed_merge_kernel<Params, D, 16 * NC, false>, dim3(items, 16 * NC / ROWS), dim3(256), stream, p);
}

template <int D, bool LSE, class Params>
hipError_t launch_packed(const Params &p, const PackedPlan &plan, hipStream_t stream)
{
    if (plan.few) return plan.few == 1 ? launch_few<D, LSE, 1>(p, plan, stream) : launch_few<D, LSE, 2>(p, plan, stream);
    return plan.waves == 4 ? launch_tiles<D, LSE, 4>(p, plan, stream) : plan.waves == 2 ? launch_tiles<D, LSE, 2>(p, plan, stream) : launch_tiles<D, LSE, 1>(p, plan, stream);
}

}  // namespace
