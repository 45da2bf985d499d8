// Softmax attention over packed sequences of different lengths, causal or not, grouped heads: forward.
//
// O = softmax(scale Q K^T) V for every sequence, row of a query token and head by itself; the running maximum and sum of the softmax
// make it one pass over the keys.  Formulation as in the tile attention: S^T = K Q^T on v_mfma_f32_16x16x32_bf16, so that a lane owns a
// column (a row of queries) and its softmax needs exchanges only among four lanes; P, rounded to bf16, goes from the accumulators
// straight into O^T += V^T P^T.
//
// Roundings.  P goes into the matrix instructions as bf16, the only type that those take next to bf16 operands; without lse the sum is of the rounded
// probabilities, which takes their common part out of the quotient and costs no vector instruction, with lse of the unrounded ones.  Of O's
// errors against 64 bits (relative, whole tensors of N(0,1) inputs) 1.5e-3 to 1.7e-3 is the result's own rounding, which a computation in fp32 has as
// well; with P rounded prompts have 1.8e-3 to 2.0e-3, 256 tokens on 32,768 keys 2.4e-3, single tokens 4.1e-4 (fp32 3.0e-4).  P in two bf16
// parts would be a product more of two.  Scores, offsets, sums and accumulators are fp32.
//
// sta_packed_tile_kernel   four waves (small launches: two waves by two groups, one by four) of 32 rows share the staged keys and values: prompts.
//                          Bound by the matrix pipe, whose clock the chip's power sets: 32,768 tokens of 32 heads over 8 of 128 channels, causal, 6.6 ms =
//                          1340 TFLOP/s of the pairs that are seen; prompts of 8192 and 4097 tokens 560 to 600 us (67 % of the cycles with a
//                          matrix instruction); 16 * 1024 tokens 178 us, 770 (short walks: the first stage's way in and the masked end).
// sta_packed_few_kernel    at most 16 or 32 rows per sequence and key head (single tokens and a few more): four waves take sub-blocks of
//                          32 keys in turn, each with LDS of its own and no barrier, and merge at the end.  Bound by reading the keys and values: 48
//                          tokens of 32 heads over 8 on caches of 1 to 16384 keys 314 us, 5.4 TB/s.
// sta_packed_merge_kernel  joins the parts of tiles that were cut along the keys to fill the chip.  Bound by its reads: 512 tokens
//                          of 32 heads of 128 channels in 8 and 12 parts, 84 MB, 22 us.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_packed.h"
#include "sta_packed_forward.h"
#include "sta_rows_check.h"

namespace sta {

int packed_check(const sta_head_rows *r, int64_t tokens, int heads_of, int D, bool written)
{
    if (!r) return STA_ERR_NULL;
    sta_head_rows some = *r;
    if (tokens == 0) some.data = reinterpret_cast<void *>(16);              // nothing is there to be read
    some.batch = 0;                                         // whatever the caller left there
    if (int rc = check_rows(&some, written, 1, tokens > 0 ? tokens : 1, D)) return rc;
    if (r->dtype != STA_BF16) return STA_ERR_UNSUPPORTED;
    if (heads_of && r->heads != heads_of) return STA_ERR_SHAPE;
    if (((uintptr_t)some.data & 15) || r->token % 8 || r->head % 8 || r->token >= (int64_t)1 << 26) return STA_ERR_SHAPE;
    return STA_OK;
}

}  // namespace sta

extern "C" {

size_t sta_packed_workspace_bytes(int Hq, int Hkv, int D, int S, int64_t tokens_q, int max_q, int max_k)
{
    if (Hq < 1 || Hkv < 1 || Hq % Hkv || (D != 64 && D != 128) || S < 0 || tokens_q < 0 || max_q < 0 || max_k < 0 || tokens_q > kMostTokens / Hq) return 0;
    PackedPlan plan;
    return plan_of(Hq, Hkv, D, S, tokens_q, max_q, max_k, true, &plan) ? plan.workspace() * sizeof(float) : 0;
}

int sta_packed_forward(const sta_head_rows *q, const sta_head_rows *k, const sta_head_rows *v, const sta_head_rows *o, float *lse,
                       int64_t tokens_q, int64_t tokens_k, const int32_t *cu_q, const int32_t *cu_k, const int32_t *k_used, int S, int max_q,
                       int max_k, int D, int causal, float scale, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!q || !k || !v || !o) return STA_ERR_NULL;
    if (S < 0 || tokens_q < 0 || tokens_k < 0 || max_q < 0 || max_k < 0 || tokens_q > kMostTokens || tokens_k > kMostTokens) return STA_ERR_SHAPE;
    if ((D != 64 && D != 128) || !scale_of(scale, D, false, &scale)) return STA_ERR_UNSUPPORTED;
    if (int rc = sta::packed_check(q, tokens_q, 0, D, false)) return rc;
    if (int rc = sta::packed_check(k, tokens_k, 0, D, false)) return rc;
    if (int rc = sta::packed_check(v, tokens_k, k->heads, D, false)) return rc;
    if (int rc = sta::packed_check(o, tokens_q, q->heads, D, true)) return rc;
    if (q->heads % k->heads || tokens_q * q->heads > kMostTokens) return STA_ERR_SHAPE;
    if (S == 0 || tokens_q == 0 || max_q == 0) return STA_OK;
    if (!cu_q || !cu_k) return STA_ERR_NULL;
    if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)k_used | (uintptr_t)lse) & 3) return STA_ERR_SHAPE;
    if (rows_overlap(*o, tokens_q, *q, tokens_q, 1, D) || rows_overlap(*o, tokens_q, *k, tokens_k, 1, D) || rows_overlap(*o, tokens_q, *v, tokens_k, 1, D))
        return STA_ERR_ALIAS;
    PackedPlan plan;
    if (!plan_of(q->heads, k->heads, D, S, tokens_q, max_q, max_k, workspace != nullptr, &plan)) return STA_ERR_SHAPE;
    const struct { const sta_head_rows *r; int64_t n; } tensors[4] = {{q, tokens_q}, {k, tokens_k}, {v, tokens_k}, {o, tokens_q}};
    if (workspace) {
        if (((uintptr_t)workspace & 15) || workspace_bytes < plan.workspace() * sizeof(float)) return STA_ERR_WORKSPACE;
        for (const auto &t : tensors)
            if (rows_meet(*t.r, 1, t.n, D, workspace, workspace_bytes)) return STA_ERR_ALIAS;
    }
    const size_t lse_bytes = (size_t)tokens_q * q->heads * sizeof(float);
    for (const auto &t : tensors)
        if (rows_meet(*t.r, 1, t.n, D, lse, lse_bytes)) return STA_ERR_ALIAS;
    if (ranges_meet(lse, lse_bytes, workspace, workspace_bytes)) return STA_ERR_ALIAS;
    const PackedBounds bounds = {cu_q, cu_k, k_used, S};
    if (bounds.meet(o, tokens_q, D, lse, lse_bytes) || bounds.meet(nullptr, 0, D, workspace, workspace_bytes)) return STA_ERR_ALIAS;
    PackedParams p = {};
    p.q = packed_rows_of(*q);
    p.k = packed_rows_of(*k);
    p.v = packed_rows_of(*v);
    p.o = packed_rows_of(*o);
    p.lse = lse;
    p.cu_q = cu_q;
    p.cu_k = cu_k;
    p.k_used = k_used;
    p.S = S;
    p.tokens_q = (uint32_t)tokens_q;
    p.tokens_k = (uint32_t)tokens_k;
    p.max_q = max_q;
    p.max_k = max_k;
    p.Hkv = k->heads;
    p.g = q->heads / k->heads;
    p.by_g = sta::fast_div_of(p.g);
    p.by_Hkv = sta::fast_div_of(p.Hkv);
    p.by_parts = sta::fast_div_of(plan.parts);
    p.causal = causal != 0;
    p.scale = scale;
    p.scale_log2e = scale * 1.4426950408889634f;
    p.parts = plan.parts;
    p.part_subs = plan.part_subs;
    p.ws = static_cast<float *>(workspace);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e;
    if (D == 64) e = lse ? launch_packed<64, true>(p, plan, stream) : launch_packed<64, false>(p, plan, stream);
    else e = lse ? launch_packed<128, true>(p, plan, stream) : launch_packed<128, false>(p, plan, stream);
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}

}  // extern "C"
