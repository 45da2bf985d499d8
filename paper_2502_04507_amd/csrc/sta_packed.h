// Attention over packed sequences: what the forward and gradient kernels share.  Sequence s has the query tokens cu_q[s] .. cu_q[s + 1]
// and the key tokens from cu_k[s] on; query heads g n .. g n + g - 1 (a group) read key head n.
//
// The rows of one sequence and key head are its (token, head of the group) pairs, token after token: row R = token * g + head.  So a
// tile of rows shares its keys whatever g is, a single token fills g of its rows, and along a tile the keys that a causal row sees
// never shrink.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_device_util.h"
#include "sta_internal.h"
#include "sta_staged.h"

namespace sta {

// Whether a [tokens, heads, D] tensor can be read (written) 16 bytes at a time; heads_of: heads it must have, 0: any.
int packed_check(const sta_head_rows *r, int64_t tokens, int heads_of, int D, bool written);

}  // namespace sta

namespace {

// Strides in bytes.
struct PackedRows {
    char *data;
    int64_t token, head;
};
inline PackedRows packed_rows_of(const sta_head_rows &r) { return {static_cast<char *>(r.data), r.token * 2, r.head * 2}; }

// The scale that is meant by the caller's: 1 / sqrt(D) where that is 0 or negative.  False: NaN, or more than 2^100, or (gradients, which divide by it)
// less than 2^-100.  By the bits: comparisons are compiled as if there were no NaN.
inline bool scale_of(float given, int D, bool gradients, float *scale)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, given), size = bits & 0x7fffffffu;
    if (size > 0x7f800000u) return false;
    *scale = size == 0 || bits != size ? 1.0f / sqrtf((float)D) : given;
    return *scale <= 0x1p100f && !(gradients && *scale < 0x1p-100f);
}

// Tokens of a tensor, and rows of all query heads: the kernels count keys and rows in int, up to a few hundred beyond the last one.
constexpr int64_t kMostTokens = 0x7ffff000;
// Workgroups of 256 lanes of a launch: a grid holds fewer than 2^32 lanes along x.
constexpr int64_t kMostWorkgroups = (1 << 24) - 1;

// Upper bound of the tiles of S sequences that hold `tokens` x g rows, none of more than `longest` x g.
inline int64_t tiles_of(int64_t tokens, int64_t g, int64_t S, int64_t longest, int64_t tile)
{
    if (longest > tokens) longest = tokens;                 // no sequence is; and so all products stay below 2^58
    const int64_t by_tokens = tokens * g / tile + S, by_longest = (longest * g + tile - 1) / tile * S;
    return by_tokens < by_longest ? by_tokens : by_longest;
}

struct PackedParams {
    PackedRows q, k, v, o;
    float *lse;                     // [Hq, tokens_q] or null
    const int32_t *cu_q, *cu_k, *k_used;
    uint32_t S, tokens_q, tokens_k;
    int32_t max_q, max_k;           // what the caller says no sequence is longer than, and what launches are counted by
    uint32_t Hkv, g;                // key heads, query heads of each
    sta::FastDiv by_g, by_Hkv, by_parts;
    uint32_t causal;
    float scale_log2e, scale;
    // tiles of rows cut along the keys: part j takes the sub-blocks part_subs * j .. ; a tile of more than one part leaves partial sums
    // in ws
    uint32_t part_subs, parts;
    float *ws;
};

// One sequence; every wave finds it for itself, so all members are the same in all lanes.
struct PackedSeq {
    int32_t q0, lq, k0, lk;         // first query and key token, and how many
    // query tokens that are worked on: those beyond max_q have no tile.  Also what the gradients of the keys sum over, so that they use no row
    // whose statistics this call has not formed
    __device__ __forceinline__ int worked(const PackedParams &p) const { return lq < p.max_q ? lq : p.max_q; }
    // keys that a row of query token t sees: the first keys_of(t)
    __device__ __forceinline__ int keys_of(int t, const PackedParams &p) const
    {
        if (!p.causal) return lk;
        const int n = t + 1 + lk - lq;
        return n < 0 ? 0 : n < lk ? n : lk;
    }
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Bounds that do not follow each other, or leave the tensors, are cut to what is there: no access depends on the arrays being right.
__device__ __forceinline__ int bound_of(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ PackedSeq seq_of(uint32_t s, const PackedParams &p)
{
    PackedSeq q;
    q.q0 = bound_of(p.cu_q[s], 0, (int)p.tokens_q);
    q.lq = bound_of(p.cu_q[s + 1], q.q0, (int)p.tokens_q) - q.q0;
    q.k0 = bound_of(p.cu_k[s], 0, (int)p.tokens_k);
    q.lk = bound_of(p.cu_k[s + 1], q.k0, (int)p.tokens_k) - q.k0;
    if (p.k_used) q.lk = bound_of(p.k_used[s], 0, q.lk);
    return q;
}

// Sum over the lanes up to and including this one: inside the rows of 16 lanes, then over the rows.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ uint32_t scan64(uint32_t x)
{
    x += from_lane<0x111, 0xf>(x);          // the lane 1, 2, 4, 8 before, of the row
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);          // the last lane of the row before: rows 1 and 3
    x += from_lane<0x143, 0xc>(x);          // the last lane of row 1: rows 2 and 3
    return x;
}
__device__ __forceinline__ uint32_t or64(uint32_t x)
{
    x |= from_lane<0x111, 0xf>(x);
    x |= from_lane<0x112, 0xf>(x);
    x |= from_lane<0x114, 0xf>(x);
    x |= from_lane<0x118, 0xf>(x);
    x |= from_lane<0x142, 0xa>(x);
    x |= from_lane<0x143, 0xc>(x);
    return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ uint32_t sum64(uint32_t x) { return __builtin_amdgcn_readlane(scan64(x), 63); }

// A tile of a sequence: TILE rows, or keys (KEYS).  Launches have an upper bound of the tiles, which only the device can count.
struct PackedTile {
    PackedSeq seq;
    uint32_t index;                 // of the tile in its sequence
};

// The tile of a workgroup, the longest walks first: with up to 64 sequences, a lane each, in the order of how many tiles' walks a tile's is
// long (rows that see more keys stand later in a causal sequence, keys that more rows see stand earlier), which a search over that number finds;
// with more, sequence after sequence from the last, 64 bounds at a time (32 heads over 8 of 128 channels, 40 tokens each, forward and gradients: 64
// sequences 19 and 41 us, 256 60 and 175, 1024 343 and 863, 4096 2694 and 6651: from some thousand on the search outweighs the walks).  False: there are not so many tiles.  Every loop ends whatever the bounds are.
template <int TILE, bool KEYS, class Params>
__device__ __forceinline__ bool find_tile(uint32_t rank, const Params &p, int lane, PackedTile *out)
{
    // tiles, and by how many tiles' walks they are longer than those of a sequence without earlier keys
    auto tiles_of = [&](uint32_t s, uint32_t *longer) {
        *longer = 0;
        if (s >= p.S) return 0u;
        const PackedSeq q = seq_of(s, p);
        if (!KEYS && q.lk > q.lq) {
            const uint64_t more = (uint64_t)(q.lk - q.lq) * p.g / TILE;
            *longer = more < (1u << 24) ? (uint32_t)more : 1u << 24;
        }
        return ((KEYS ? (uint32_t)(q.lk < p.max_k ? q.lk : p.max_k) : (uint32_t)q.worked(p) * p.g) + TILE - 1) / TILE;
    };
    uint32_t longer;
    int at;                         // lane of the sequence
    uint32_t s0 = 0;
    if (p.S <= 64) {
        const uint32_t own = tiles_of(lane, &longer), upto = scan64(own);
        if (rank >= (uint32_t)__builtin_amdgcn_readlane(upto, 63)) return false;
        // the largest level that so many tiles reach that this one is among them
        auto reach = [&](uint32_t level) {
            const uint32_t below = level > longer ? level - longer : 0;
            return own > below ? own - below : 0;
        };
        uint32_t lo = 0;
        for (uint32_t step = 0x80000000u >> __builtin_clz(or64(longer + own)); step > 0; step >>= 1)         // (own is not 0 everywhere)
            if (sum64(reach(lo + step)) > rank) lo += step;
        uint32_t left = rank - sum64(reach(lo + 1));
        uint64_t here = __builtin_amdgcn_ballot_w64(own != 0 && longer <= lo && lo < longer + own);
        while (left-- > 0) here &= here - 1;
        at = __builtin_ctzll(here);
        const uint32_t level = lo - __builtin_amdgcn_readlane(longer, at), n = __builtin_amdgcn_readlane(own, at);
        out->index = KEYS ? n - 1 - level : level;
    } else {
        uint32_t total = 0;
        for (uint32_t s = 0; s < p.S; s += 64) total += sum64(tiles_of(s + lane, &longer));
        if (rank >= total) return false;
        const uint32_t idx = KEYS ? rank : total - 1 - rank;
        uint32_t before = 0, own, upto;
        for (;; s0 += 64) {
            if (s0 >= p.S) return false;                        // (idx < total, unless the bounds have changed since)
            own = tiles_of(s0 + lane, &longer);
            upto = scan64(own);
            const uint32_t all = __builtin_amdgcn_readlane(upto, 63);
            if (idx < before + all) break;
            before += all;
        }
        at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(before + upto > idx));
        out->index = idx - before - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(own, at));
    }
    out->seq = seq_of(s0 + at, p);
    out->seq.q0 = uniform(out->seq.q0);
    out->seq.lq = uniform(out->seq.lq);
    out->seq.k0 = uniform(out->seq.k0);
    out->seq.lk = uniform(out->seq.lk);
    // The bounds have been read twice.  A caller that writes them from another stream meanwhile gets results that mean nothing, but no walk without an end and
    // no access outside the tensors.
    return out->index * TILE < (KEYS ? (uint32_t)out->seq.lk : (uint32_t)out->seq.lq * p.g);
}

// The lane, counted again: neither it nor what is worked out from it behind a loop is kept in registers through it.
__device__ __forceinline__ int fresh_lane()
{
    uint32_t none = 0;
    asm volatile("" : "+s"(none));
    return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// DMA of rows into LDS: where a lane's 16 bytes of a group of rows come from, and the rows beyond the last one read as the last one.
template <int D, bool ROWS_ONLY>
struct PackedDma {
    static constexpr int LPR = D / 8;                               // lanes per row
    static constexpr int GroupRows = Staged<D>::GroupRows;
    uint32_t off;                                                   // from the group's first row
    static __device__ __forceinline__ uint32_t chunk_of(int lane)
    {
        const int r = lane / LPR, pos = lane % LPR;
        if constexpr (ROWS_ONLY) return (uint32_t)((pos ^ StagedRows<D>::turn(r)) << 4);
        else return (uint32_t)(D == 128 ? (pos ^ (r << 2)) << 4 : (pos ^ (((r >> 1) & 3) << 1)) << 4);
    }
    __device__ __forceinline__ void start(int lane, int64_t token) { off = (uint32_t)((lane / LPR) * (int)token) + chunk_of(lane); }
    // A group of rows that are there, from a scalar address, to LDS address dst: no vector arithmetic.
    __device__ __forceinline__ void bring_whole(const char *group, char *dst) const
    {
        uint32_t o = off;
        asm volatile("" : "+v"(o));                                 // a 32-bit lane offset next to a scalar base
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(group + o), STA_LDS_PTR(dst), 16, 0, 0);
    }
    // Rows `first` .. of base (already at the sequence's first row), of which only `rows` exist.
    static __device__ __forceinline__ void bring_part(const char *base, int64_t token, int first, int rows, char *dst)
    {
        const int lane = fresh_lane(), row = first + lane / LPR;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(base + (int64_t)(row < rows ? row : rows - 1) * token + chunk_of(lane)),
                                         STA_LDS_PTR(dst), 16, 0, 0);
    }
};

// Rows of K and V of `subs` sub-blocks from sub-block `sub` on to LDS: K at `to` in groups K::Group apart, V v_at behind it, sub-blocks `apart` bytes apart;
// the wave's share is COUNT groups of each from its group `from` on.  Two paths that the compiler is kept from joining: joined, the common one
// works addresses out in vector registers as the other has to, 336 cycles of a sub-block's 770 at head dimension 128.
template <int SUBS, int COUNT, int K_GROUP, int V_GROUP, int D, bool K_ROWS, bool V_ROWS>
__device__ __forceinline__ void bring_stage(const PackedDma<D, K_ROWS> &k_dma, const PackedDma<D, V_ROWS> &v_dma, const char *kh, const char *vh, int64_t k_token,
                                            int64_t v_token, int sub, int rows, int from, char *to, int v_at, int apart)
{
    constexpr int GR = Staged<D>::GroupRows;
    const int first = sub * kSub + from * GR;
    if (__builtin_expect((sub + SUBS) * kSub <= rows, 1)) {
        const char *k = kh + (int64_t)first * k_token, *v = vh + (int64_t)first * v_token;
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int64_t row = u * kSub + i * GR;
                k_dma.bring_whole(k + row * k_token, to + u * apart + (from + i) * K_GROUP);
                v_dma.bring_whole(v + row * v_token, to + u * apart + v_at + (from + i) * V_GROUP);
            }
        asm volatile("; whole" ::: "memory");
    } else {
#pragma unroll 1
        for (int u = 0; u < SUBS; ++u)
#pragma unroll 1
            for (int i = 0; i < COUNT; ++i) {
                const int row = first + u * kSub + i * GR;
                k_dma.bring_part(kh, k_token, row, rows, to + u * apart + (from + i) * K_GROUP);
                v_dma.bring_part(vh, v_token, row, rows, to + u * apart + v_at + (from + i) * V_GROUP);
            }
        asm volatile("; part" ::: "memory");
    }
}

}  // namespace
