// Rows of heads between a layer's projections and its attention: RMS norm and rotary positions of query and key rows and the move of
// queries, keys and values into the attention's order, in one pass; its gradients; the rotation alone.
//
// A row is the D channels of one head of one token.  Mathematics, per row x with weight w, root mean square factor
// r = 1 / sqrt(mean(x^2) + eps) and a rotation R (orthogonal times a magnitude m) that the token's position gives:
//   forward   y = R (w o x r)
//   backward  g = R^T dy;  dw += g o x r;  dx = r (g o w - x r mean(g o w o x r))
// All of it is a few dozen fp32 operations per 16 bytes, so HBM bounds it: every row is read once and written once, and what a
// token needs beyond its rows (position, cosines and sines) is computed once for all of its heads.
//
// Fast path: L lanes share a row and a lane holds two chunks of 8 channels, chosen so that both members of a pair are in one lane (half
// layout: channels 8c.. and rot/2 + 8c..): no exchange between lanes but for the two sums over a row.  A wave holds 64 / L
// tokens side by side and walks over heads; the four waves of a workgroup take its tokens' heads in turn.  Tokens go in the order of
// the outputs' places, so that a wave writes whole runs of a head (2 KB at D = 128), and the workgroup reads its tokens' heads from
// end to end.
// General path: two pairs a lane, single elements from any address; 16, 32 or 64 lanes a row.
//
// Measured, of the bytes that are read and written once: 115,200 tokens of 72 heads of 128 channels in bf16 into tile order 806 us, 5.3 TB/s (a large copy
// 4.8 to 5.4); 32,768 tokens of 40 heads, rotation alone, 121 us, 5.5; from float32, 27,648 tokens of 36 heads, 147 us, 5.2, and the gradients 245 and
// 4.7 us, 4.4 (575 MB of writes for 510); one to 100 tokens 3.5 to 4 us, the launch and two trips to memory one after the other.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/sta.h"
#include "sta_internal.h"
#include "sta_rows_check.h"

namespace {

using sta::fast_div;
using sta::fast_div_of;
using sta::FastDiv;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kHalf = 0, kInterleaved = 1, kGeneral = 2;      // paths

// Rows of one tensor as a kernel walks them; strides in bytes.
struct Rows {
    char *data;
    int64_t batch, token, head;
};
struct Tensor {
    Rows x, dy, out;            // input rows; gradients of the outputs (backward); what is written
    const void *weight;         // [D] or null: ones
    uint32_t heads;
    uint32_t norm, rotate;
};
// The workgroups of one tensor's gradients, and their units.
struct Share {
    uint32_t first, blocks, units;
    FastDiv splits;             // units of one group of tokens
};
struct Params {
    Tensor t[3];
    Share share[3];
    uint32_t n_tensors;
    uint32_t tokens;            // B * N
    uint32_t D, rot;            // channels, rotated channels
    uint32_t weight_f32;
    uint32_t interleaved;       // of the general path
    float inv_D, eps;
    // rotation
    const int64_t *steps;
    const int32_t *positions;
    int64_t position_batch, position_token;
    uint32_t axis1, axis2;      // first pairs of axes 1 and 2
    float magnitude, sign;      // sign: -1 turns back
    uint32_t turns;             // there is a rotation
    // places
    FastDiv by_N, by_P, by_nw, by_nh, by_Tw, by_Th, by_gw, by_gh;
    uint32_t N, tiled, has_grid, T_t, T_h, T_w, g_h, g_w;
    // backward
    float *partial;             // [workgroups][D] sums of the weight gradients of queries, then keys, or null
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x2 v;
    v[0] = static_cast<__bf16>(a);   // round to nearest even
    v[1] = static_cast<__bf16>(b);
    return __builtin_bit_cast(uint32_t, v);
}

// The raw bits of a lane's channels of one row.
template <int PATH, bool F32>
struct Raw {
    u32x4 w[F32 ? 4 : 2];       // chunks of 8 channels
};
template <bool F32>
struct Raw<kGeneral, F32> {
    uint32_t w[4];              // two pairs of channels
};

// Which channels of a row a lane holds.
struct Place {
    uint32_t a, b;              // fast paths: first channels of the two chunks
    bool turn_a, turn_b;        // ... and whether they are rotated
    uint32_t e[4];              // general path: the channels of two pairs
    bool in, in2;               // the lane (general path: its pairs) are inside the row
};
template <int PATH, int L>
__device__ __forceinline__ Place place_of(uint32_t c, const Params &p)
{
    Place at = {};
    if constexpr (PATH == kHalf) {
        at.in = 16 * c < p.D;
        at.turn_a = at.turn_b = 16 * c < p.rot;
        at.a = at.turn_a ? 8 * c : at.in ? 16 * c : 0;
        at.b = at.turn_a ? p.rot / 2 + 8 * c : at.in ? 16 * c + 8 : 0;
    } else if constexpr (PATH == kInterleaved) {
        at.in = 16 * c < p.D;
        at.a = at.in ? 8 * c : 0;
        at.b = at.in ? p.D / 2 + 8 * c : 0;
        at.turn_a = at.in && at.a < p.rot;
        at.turn_b = at.in && at.b < p.rot;
    } else {
        const uint32_t pairs = p.rot / 2;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t i = c + L * j;
            const bool turned = i < pairs;
            at.e[2 * j] = turned && !p.interleaved ? i : 2 * i;           // unrotated pairs are neighbours behind the rotated ones
            at.e[2 * j + 1] = turned && !p.interleaved ? i + pairs : 2 * i + 1;
            (j ? at.turn_b : at.turn_a) = turned;
        }
        at.in = 2 * c < p.D;
        at.in2 = 2 * (c + L) < p.D;
#pragma unroll
        for (int j = 0; j < 4; ++j) at.e[j] = (j < 2 ? at.in : at.in2) ? at.e[j] : 0;
    }
    return at;
}

// What a lane holds of a row.  A lane that holds nothing reads the row's first channels, without a branch, and its shares of the row's sums
// are left out (general path: zeros).
template <int PATH, bool F32>
__device__ __forceinline__ Raw<PATH, F32> load_row(const char *row, const Place &at, bool on)
{
    Raw<PATH, F32> r;
    constexpr int S = F32 ? 4 : 2;
    if constexpr (PATH == kGeneral) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (F32) r.w[j] = *reinterpret_cast<const uint32_t *>(row + at.e[j] * S);
            else r.w[j] = (uint32_t)*reinterpret_cast<const uint16_t *>(row + at.e[j] * S) << 16;
            r.w[j] = on && (j < 2 ? at.in : at.in2) ? r.w[j] : 0;
        }
    } else {
        const u32x4 *a = reinterpret_cast<const u32x4 *>(row + at.a * S), *b = reinterpret_cast<const u32x4 *>(row + at.b * S);
        if constexpr (F32) {
            r.w[0] = a[0]; r.w[1] = a[1]; r.w[2] = b[0]; r.w[3] = b[1];
        } else {
            r.w[0] = a[0]; r.w[1] = b[0];
        }
    }
    return r;
}

constexpr int pairs_of(int path) { return path == kGeneral ? 2 : 8; }

// The 16 (general path: 4) channels as pairs (x0[i], x1[i]).
template <int PATH, bool F32>
__device__ __forceinline__ void unpack(const Raw<PATH, F32> &r, float (&x0)[pairs_of(PATH)], float (&x1)[pairs_of(PATH)])
{
    if constexpr (PATH == kGeneral) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            x0[j] = __uint_as_float(r.w[2 * j]);
            x1[j] = __uint_as_float(r.w[2 * j + 1]);
        }
    } else {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (F32) v[i] = __uint_as_float(r.w[i / 4][i % 4]);
            else v[i] = i & 1 ? high_half(r.w[i / 8][(i % 8) / 2]) : low_half(r.w[i / 8][(i % 8) / 2]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x0[i] = PATH == kHalf ? v[i] : v[2 * i];
            x1[i] = PATH == kHalf ? v[8 + i] : v[2 * i + 1];
        }
    }
}

// 16-byte stores that leave no dirty line in L2, like those of the permutation: the next kernel reads these rows.
template <int PATH, bool F32>
__device__ __forceinline__ void store_row(char *row, const Place &at, bool on, const float (&x0)[pairs_of(PATH)], const float (&x1)[pairs_of(PATH)])
{
    constexpr int S = F32 ? 4 : 2;
    if (!on) return;
    if constexpr (PATH == kGeneral) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = j & 1 ? x1[j / 2] : x0[j / 2];
            if (j < 2 ? at.in : at.in2) {
                if constexpr (F32) *reinterpret_cast<float *>(row + at.e[j] * S) = v;
                else *reinterpret_cast<__bf16 *>(row + at.e[j] * S) = static_cast<__bf16>(v);
            }
        }
    } else if (at.in) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[PATH == kHalf ? i : 2 * i] = x0[i];
            v[PATH == kHalf ? 8 + i : 2 * i + 1] = x1[i];
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            u32x4 *to = reinterpret_cast<u32x4 *>(row + (half ? at.b : at.a) * S);
            const float *x = v + 8 * half;
            if constexpr (F32) {
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    __builtin_nontemporal_store(u32x4{__float_as_uint(x[4 * q]), __float_as_uint(x[4 * q + 1]), __float_as_uint(x[4 * q + 2]),
                                                      __float_as_uint(x[4 * q + 3])}, to + q);
            } else {
                __builtin_nontemporal_store(u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}, to);
            }
        }
    }
}

// Sum over the L lanes of a row.
template <int L>
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int m = L / 2; m > 0; m /= 2) x += __shfl_xor(x, m, 64);
    return x;
}

// Cosine and sine of x * step / 2^64 turns.  The upper 32 bits of the product are the angle to 2^-32 turns; the nearest quarter
// turn is taken off exactly and what is left, at most an eighth of a turn, goes into the Taylor polynomials (terms left out: below
// 2e-9 and 3e-8).
__device__ __forceinline__ void turn_of(int32_t x, int64_t step, float magnitude, float sign, float &c, float &s)
{
    const uint32_t lo = (uint32_t)step, hi = (uint32_t)((uint64_t)step >> 32), n = (uint32_t)x;
    const uint32_t turns = __umulhi(n, lo) + n * hi - (x < 0 ? lo : 0u);
    const uint32_t quarter = (turns + 0x20000000u) >> 30;
    const float a = (float)(int32_t)(turns - (quarter << 30)) * 1.4629180792671596e-9f;       // 2 pi / 2^32
    const float a2 = a * a;
    const float sn = fmaf(fmaf(fmaf(fmaf(2.7557319e-6f, a2, -1.9841270e-4f), a2, 8.3333333e-3f), a2, -1.6666667e-1f), a2 * a, a);
    const float cs = fmaf(fmaf(fmaf(fmaf(2.4801587e-5f, a2, -1.3888889e-3f), a2, 4.1666667e-2f), a2, -0.5f), a2, 1.0f);
    const bool odd = quarter & 1;
    const float c0 = odd ? sn : cs, s0 = odd ? cs : sn;
    c = ((quarter + 1) & 2 ? -c0 : c0) * magnitude;
    s = (quarter & 2 ? -s0 : s0) * (magnitude * sign);
}

// The token of a place: where its rows lie and where it is on the axes.
struct Token {
    uint32_t b, n, place;       // batch, index in the inputs' order, index in the outputs' order
    int32_t at0, at1, at2;
};
__device__ __forceinline__ Token token_of(uint32_t id, const Params &p)
{
    Token t;
    t.b = fast_div(id, p.by_N);
    t.place = id - t.b * p.N;
    t.n = t.place;
    t.at0 = (int32_t)t.n;
    t.at1 = t.at2 = 0;
    if (p.tiled) {
        const uint32_t tile = fast_div(t.place, p.by_P), in = t.place - tile * p.by_P.d;
        const uint32_t row = fast_div(tile, p.by_nw), tw = tile - row * p.by_nw.d;
        const uint32_t tt = fast_div(row, p.by_nh), th = row - tt * p.by_nh.d;
        const uint32_t line = fast_div(in, p.by_Tw), iw = in - line * p.by_Tw.d;
        const uint32_t it = fast_div(line, p.by_Th), ih = line - it * p.by_Th.d;
        t.at0 = (int32_t)(tt * p.T_t + it);
        t.at1 = (int32_t)(th * p.T_h + ih);
        t.at2 = (int32_t)(tw * p.T_w + iw);
        t.n = ((uint32_t)t.at0 * p.g_h + (uint32_t)t.at1) * p.g_w + (uint32_t)t.at2;
    } else if (p.has_grid) {
        const uint32_t line = fast_div(t.n, p.by_gw);
        t.at2 = (int32_t)(t.n - line * p.g_w);
        const uint32_t plane = fast_div(line, p.by_gh);
        t.at1 = (int32_t)(line - plane * p.g_h);
        t.at0 = (int32_t)plane;
    }
    return t;
}
__device__ __forceinline__ void load_positions(Token &t, const Params &p)
{
    if (!p.positions) return;
    const int32_t *x = p.positions + (int64_t)t.b * p.position_batch + (int64_t)t.n * p.position_token;
    t.at0 = x[0];
    if (p.axis1 < p.rot / 2) t.at1 = x[1];
    if (p.axis2 < p.rot / 2) t.at2 = x[2];
}

// The steps of a lane's pairs; 0 for those that are not rotated.
template <int PATH, int L>
__device__ __forceinline__ void load_steps(uint32_t lane_in_row, const Place &at, const Params &p, int64_t (&step)[pairs_of(PATH)], bool (&first)[pairs_of(PATH)],
                                           bool (&second)[pairs_of(PATH)])
{
#pragma unroll
    for (int i = 0; i < pairs_of(PATH); ++i) {
        const bool b = PATH == kGeneral ? i == 1 : PATH == kInterleaved && i >= 4;
        const uint32_t pair = PATH == kHalf ? at.a + i : PATH == kGeneral ? lane_in_row + L * i : b ? at.b / 2 + i - 4 : at.a / 2 + i;
        step[i] = p.steps[(b ? at.turn_b : at.turn_a) ? pair : 0];
        first[i] = pair < p.axis1;
        second[i] = pair < p.axis2;
    }
}

// Cosines and sines of a lane's pairs.
template <int PATH, bool FEW_REGISTERS>
__device__ __forceinline__ void turns_of(const Token &t, const int64_t (&step)[pairs_of(PATH)], const bool (&first)[pairs_of(PATH)],
                                         const bool (&second)[pairs_of(PATH)], const Params &p, float (&c)[pairs_of(PATH)], float (&s)[pairs_of(PATH)])
{
#pragma unroll
    for (int i = 0; i < pairs_of(PATH); ++i) {
        turn_of(first[i] ? t.at0 : second[i] ? t.at1 : t.at2, step[i], p.magnitude, p.sign, c[i], s[i]);
        if (FEW_REGISTERS && i % 2) __builtin_amdgcn_sched_barrier(0);        // two pairs at a time
    }
}

// (selects, not zeros and ones: what is not rotated is to stay what it is, whatever it is)
template <int PATH>
__device__ __forceinline__ void rotate(float (&x0)[pairs_of(PATH)], float (&x1)[pairs_of(PATH)], const float (&c)[pairs_of(PATH)],
                                       const float (&s)[pairs_of(PATH)], const Place &at, float turn_back)
{
#pragma unroll
    for (int i = 0; i < pairs_of(PATH); ++i) {
        const bool on = (PATH == kGeneral ? i == 1 : PATH == kInterleaved && i >= 4) ? at.turn_b : at.turn_a;
        const float a = x0[i], b = x1[i], sn = s[i] * turn_back;
        x0[i] = on ? a * c[i] - b * sn : a;
        x1[i] = on ? a * sn + b * c[i] : b;
    }
}

template <int PATH>
__device__ __forceinline__ void load_weights(const void *weight, const Params &p, const Place &at, float (&w0)[pairs_of(PATH)],
                                             float (&w1)[pairs_of(PATH)])
{
    auto one = [&](uint32_t e) {
        return p.weight_f32 ? static_cast<const float *>(weight)[e] : __uint_as_float((uint32_t)static_cast<const uint16_t *>(weight)[e] << 16);
    };
#pragma unroll
    for (int i = 0; i < pairs_of(PATH); ++i) {
        w0[i] = w1[i] = 1.f;
        const bool in = PATH == kGeneral && i ? at.in2 : at.in;
        if (!weight || !in) continue;
        if constexpr (PATH == kGeneral) {
            w0[i] = one(at.e[2 * i]);
            w1[i] = one(at.e[2 * i + 1]);
        } else if constexpr (PATH == kHalf) {
            w0[i] = one(at.a + i);
            w1[i] = one(at.b + i);
        } else {
            const uint32_t e = i < 4 ? at.a + 2 * i : at.b + 2 * (i - 4);
            w0[i] = one(e);
            w1[i] = one(e + 1);
        }
    }
}

__device__ __forceinline__ const char *row_at(const Rows &r, uint32_t b, uint32_t token) { return r.data + (int64_t)b * r.batch + (int64_t)token * r.token; }

// The tensor and head of a wave's row number u of all tensors' heads.
struct HeadAt {
    uint32_t tensor, head;
};
__device__ __forceinline__ HeadAt head_at(uint32_t u, const Params &p)
{
    const uint32_t h1 = p.t[0].heads, h2 = h1 + p.t[1].heads;           // (0 heads where there is no such tensor)
    return u < h1 ? HeadAt{0, u} : u < h2 ? HeadAt{1, u - h1} : HeadAt{2, u - h2};
}

constexpr int kGridShift = 23;                              // a grid holds fewer than 2^32 lanes along x

// Workgroup (x, y, z): tokens 64 / L * (z * 2^23 + x) .., heads y * kWaves + wave and every gridDim.y * kWaves after that, of all tensors one after the other.
// AHEAD rows are on their way while one is worked on; the first are asked for before the positions and steps.
template <int PATH, int L, bool SRC_F32, bool DST_F32>
__global__ __launch_bounds__(kThreads) void sta_rows_forward_kernel(Params p)
{
    constexpr int NP = pairs_of(PATH), AHEAD = SRC_F32 ? 1 : 2;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first_id = ((blockIdx.z << kGridShift) + blockIdx.x) * (64 / L);        // at most 2^31 + 2^27
    if (first_id >= p.tokens) return;
    const uint32_t c = lane % L, id = first_id + lane / L;
    const bool on = id < p.tokens;
    Token t = token_of(on ? id : 0, p);
    const Place at = place_of<PATH, L>(c, p);
    const uint32_t stride = gridDim.y * kWaves, total = p.t[0].heads + p.t[1].heads + p.t[2].heads;
    uint32_t u = blockIdx.y * kWaves + wave;
    if (u >= total) return;
    auto load = [&](uint32_t v) __attribute__((always_inline)) {
        const HeadAt h = head_at(v, p);
        const Rows &x = p.t[h.tensor].x;
        return load_row<PATH, SRC_F32>(row_at(x, t.b, t.n) + (int64_t)h.head * x.head, at, on);
    };
    Raw<PATH, SRC_F32> next[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i == 0 || u + i * stride < total) next[i] = load(u + i * stride);
    float cs[NP], sn[NP], w0[NP], w1[NP];
    uint32_t weights_of = head_at(u, p).tensor;
    if (p.t[weights_of].norm) load_weights<PATH>(p.t[weights_of].weight, p, at, w0, w1);
    if (p.turns) {
        int64_t step[NP];
        bool first[NP], second[NP];
        load_steps<PATH, L>(c, at, p, step, first, second);
        load_positions(t, p);
        turns_of<PATH, false>(t, step, first, second, p, cs, sn);
    }
    for (; u < total; u += AHEAD * stride) {
        Raw<PATH, SRC_F32> raw[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            raw[i] = next[i];
            const uint32_t v = u + (AHEAD + i) * stride;
            if (v < total) next[i] = load(v);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const uint32_t v = u + i * stride;
            if (i > 0 && v >= total) break;
            const HeadAt h = head_at(v, p);
            const Tensor &T = p.t[h.tensor];
            float x0[NP], x1[NP];
            unpack<PATH, SRC_F32>(raw[i], x0, x1);
            if (T.norm) {
                if (h.tensor != weights_of) {
                    weights_of = h.tensor;
                    load_weights<PATH>(T.weight, p, at, w0, w1);
                }
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < NP; ++j) sum = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], sum));
                const float r = rsqrtf(fmaf(row_sum<L>(at.in ? sum : 0.f), p.inv_D, p.eps));
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    x0[j] *= r * w0[j];
                    x1[j] *= r * w1[j];
                }
            }
            if (T.rotate) rotate<PATH>(x0, x1, cs, sn, at, 1.f);
            store_row<PATH, DST_F32>(const_cast<char *>(row_at(T.out, t.b, t.place)) + (int64_t)h.head * T.out.head, at, on, x0, x1);
        }
    }
}

// A workgroup works for one tensor: on units of 64 / L tokens by the heads split * kWaves + wave, and every splits * kWaves after that, in turn with
// the tensor's other workgroups.  So a lane sums one weight gradient, which goes from the registers over the workgroup into `partial`.
// (With all tensors in one workgroup, 168 registers and 236 bytes of scratch, or 183 registers and nothing asked for ahead: 378 and 252 us for a
// clip of 27,648 tokens by 12 heads of 128 from float32; now 244, 4.5 TB/s.)
template <int PATH, int L, bool SRC_F32, bool DST_F32>
__global__ __launch_bounds__(kThreads, 3) void sta_rows_backward_kernel(Params p)
{
    constexpr int NP = pairs_of(PATH);
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t c = lane % L;
    const Place at = place_of<PATH, L>(c, p);
    const uint32_t tensor = blockIdx.x < p.share[1].first ? 0 : blockIdx.x < p.share[2].first ? 1 : 2;
    const Tensor &T = p.t[tensor];
    const Share &share = p.share[tensor];
    const uint32_t stride = share.splits.d * kWaves;
    if (!T.norm) {                                          // values: moved back
#pragma unroll 1
        for (uint32_t unit = blockIdx.x - share.first; unit < share.units; unit += share.blocks) {
            const uint32_t group = fast_div(unit, share.splits), id = group * (64 / L) + lane / L;
            const bool on = id < p.tokens;
            const Token t = token_of(on ? id : 0, p);
            const char *dy = row_at(T.dy, t.b, t.place);
            char *out = const_cast<char *>(row_at(T.out, t.b, t.n));
#pragma unroll 2
            for (uint32_t h = (unit - group * share.splits.d) * kWaves + wave; h < T.heads; h += stride) {
                float x0[NP], x1[NP];
                unpack<PATH, DST_F32>(load_row<PATH, DST_F32>(dy + (int64_t)h * T.dy.head, at, on), x0, x1);
                store_row<PATH, SRC_F32>(out + (int64_t)h * T.out.head, at, on, x0, x1);
            }
        }
        return;
    }
    float w0[NP], w1[NP], dw0[NP], dw1[NP];
    load_weights<PATH>(T.weight, p, at, w0, w1);
#pragma unroll
    for (int j = 0; j < NP; ++j) dw0[j] = dw1[j] = 0.f;
#pragma unroll 1
    for (uint32_t unit = blockIdx.x - share.first; unit < share.units; unit += share.blocks) {
        const uint32_t group = fast_div(unit, share.splits), id = group * (64 / L) + lane / L;
        const bool in = id < p.tokens;
        Token t = token_of(in ? id : 0, p);
        const char *x = row_at(T.x, t.b, t.n), *dy = row_at(T.dy, t.b, t.place);
        char *out = const_cast<char *>(row_at(T.out, t.b, t.n));
        // all waves go around as often; one without a head left works on the last one and drops it
        const uint32_t first_head = (unit - group * share.splits.d) * kWaves;
        uint32_t h = first_head + wave;
        auto address = [&](uint32_t head) { return (int64_t)(head < T.heads ? head : T.heads - 1); };
        Raw<PATH, SRC_F32> next_x = load_row<PATH, SRC_F32>(x + address(h) * T.x.head, at, in);
        Raw<PATH, DST_F32> next_g = load_row<PATH, DST_F32>(dy + address(h) * T.dy.head, at, in);
        float cs[NP] = {}, sn[NP] = {};
        if (p.turns) {
            int64_t step[NP];
            bool first[NP], second[NP];
            load_steps<PATH, L>(c, at, p, step, first, second);
            load_positions(t, p);
            turns_of<PATH, true>(t, step, first, second, p, cs, sn);
        }
        uint32_t left = (T.heads - first_head + stride - 1) / stride;
#pragma unroll 1
        do {
            const bool on = in && h < T.heads;
            float x0[NP], x1[NP], g0[NP], g1[NP];
            unpack<PATH, SRC_F32>(next_x, x0, x1);
            unpack<PATH, DST_F32>(next_g, g0, g1);
            if (left > 1) {
                next_x = load_row<PATH, SRC_F32>(x + address(h + stride) * T.x.head, at, in);
                next_g = load_row<PATH, DST_F32>(dy + address(h + stride) * T.dy.head, at, in);
            }
            if (__builtin_amdgcn_ballot_w64(!on) != 0) {    // a row that is not there holds another's values, and 0 times an infinity would be no 0
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    g0[j] = on ? g0[j] : 0.f;
                    g1[j] = on ? g1[j] : 0.f;
                }
            }
            rotate<PATH>(g0, g1, cs, sn, at, -1.f);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < NP; ++j) sum = fmaf(x0[j], x0[j], fmaf(x1[j], x1[j], sum));
            // 0 where there is no row: it is then no term of the weights' gradient either
            const float r = on ? rsqrtf(fmaf(row_sum<L>(at.in ? sum : 0.f), p.inv_D, p.eps)) : 0.f;
            float dot = 0.f;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                x0[j] *= r;
                x1[j] *= r;
                dw0[j] = fmaf(g0[j], x0[j], dw0[j]);
                dw1[j] = fmaf(g1[j], x1[j], dw1[j]);
                g0[j] *= w0[j];
                g1[j] *= w1[j];
                dot = fmaf(g0[j], x0[j], fmaf(g1[j], x1[j], dot));
            }
            dot = row_sum<L>(at.in ? dot : 0.f) * p.inv_D;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                x0[j] = r * fmaf(-dot, x0[j], g0[j]);
                x1[j] = r * fmaf(-dot, x1[j], g1[j]);
            }
            store_row<PATH, SRC_F32>(out + address(h) * T.out.head, at, on, x0, x1);
            h += stride;
        } while (--left > 0);
    }
    if (!p.partial) return;
    // over the tokens of a wave, then over the waves; channels in their places
    __shared__ float sums[kWaves][256];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        float a = dw0[j], b = dw1[j];
#pragma unroll
        for (int m = L; m < 64; m *= 2) {
            a += __shfl_xor(a, m, 64);
            b += __shfl_xor(b, m, 64);
        }
        if (lane < L && (PATH == kGeneral && j ? at.in2 : at.in)) {
            uint32_t ea, eb;
            if constexpr (PATH == kGeneral) { ea = at.e[2 * j]; eb = at.e[2 * j + 1]; }
            else if constexpr (PATH == kHalf) { ea = at.a + j; eb = at.b + j; }
            else { ea = j < 4 ? at.a + 2 * j : at.b + 2 * (j - 4); eb = ea + 1; }
            sums[wave][ea] = a;
            sums[wave][eb] = b;
        }
    }
    __syncthreads();
    float *to = p.partial + (size_t)blockIdx.x * p.D;
    for (uint32_t e = threadIdx.x; e < p.D; e += kThreads) to[e] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
}

// d_weight = sum of the workgroups' sums: 16 columns a workgroup, 64 slices of the rows of which a lane has eight on their way, then the slices in
// order.
constexpr int kSlices = 64;
__global__ __launch_bounds__(16 * kSlices) void sta_rows_weights_kernel(const float *partial, uint32_t q_rows, uint32_t k_rows, uint32_t D, float *d_q, float *d_k)
{
    __shared__ float sums[kSlices][17];
    const uint32_t col = threadIdx.x & 15, slice = threadIdx.x >> 4, e = blockIdx.x * 16 + col, rows = blockIdx.y ? k_rows : q_rows;
    if (blockIdx.y) partial += (size_t)q_rows * D;
    const bool in = e < D;
    float sum = 0.f;
    for (uint32_t r = slice; r < rows; r += 8 * kSlices) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = in && r + i * kSlices < rows ? partial[(size_t)(r + i * kSlices) * D + e] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
    }
    sums[slice][col] = sum;
    __syncthreads();
    float *to = blockIdx.y ? d_k : d_q;
    if (slice == 0 && in && to) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kSlices; ++i) sum += sums[i][col];
        to[e] = sum;
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------------------
constexpr int kMostD = 256;

Rows rows_of(const sta_head_rows &r)
{
    const int64_t s = size_of(r.dtype);
    return {static_cast<char *>(r.data), r.batch * s, r.token * s, r.head * s};
}

bool chunked(const Rows &r) { return (((uintptr_t)r.data | (uintptr_t)r.batch | (uintptr_t)r.token | (uintptr_t)r.head) & 15) == 0; }

// What does not depend on the tensors.
int fill_params(Params *p, const sta_rotary *rotary, int B, int N, int D, const int *grid, const int *tile, float eps, int inverse)
{
    if (B < 0 || N < 0) return STA_ERR_SHAPE;
    if (D < 2 || D > kMostD || D % 2) return STA_ERR_UNSUPPORTED;
    if ((int64_t)B * N > 0x7fffffff) return STA_ERR_SHAPE;
    if (tile && !grid) return STA_ERR_NULL;
    p->tokens = (uint32_t)((int64_t)B * N);
    p->D = D;
    p->inv_D = 1.f / (float)D;
    p->eps = eps;
    p->N = N > 0 ? N : 1;
    p->by_N = fast_div_of(p->N);
    if (grid) {
        int64_t n = 1;
        for (int a = 0; a < 3; ++a) {
            if (grid[a] <= 0 || (tile && (tile[a] <= 0 || grid[a] % tile[a] != 0))) return STA_ERR_SHAPE;
            n *= grid[a];
            if (n > 0x7fffffff) return STA_ERR_SHAPE;
        }
        if (n != N) return STA_ERR_SHAPE;
        p->has_grid = 1;
        p->g_h = grid[1];
        p->g_w = grid[2];
        p->by_gw = fast_div_of(grid[2]);
        p->by_gh = fast_div_of(grid[1]);
        if (tile) {
            p->tiled = 1;
            p->T_t = tile[0]; p->T_h = tile[1]; p->T_w = tile[2];
            p->by_P = fast_div_of((uint32_t)(tile[0] * tile[1] * tile[2]));
            p->by_nw = fast_div_of(grid[2] / tile[2]);
            p->by_nh = fast_div_of(grid[1] / tile[1]);
            p->by_Tw = fast_div_of(tile[2]);
            p->by_Th = fast_div_of(tile[1]);
        }
    }
    p->sign = inverse ? -1.f : 1.f;
    if (rotary) {
        const int pairs = rotary->channels / 2;
        if (rotary->channels < 0 || rotary->channels % 2 || rotary->channels > D) return STA_ERR_SHAPE;
        int64_t sum = 0;
        for (int a = 0; a < 3; ++a) {
            if (rotary->pairs[a] < 0) return STA_ERR_SHAPE;
            sum += rotary->pairs[a];
        }
        if (sum != pairs) return STA_ERR_SHAPE;
        if (!rotary->positions && !grid && rotary->pairs[0] != pairs) return STA_ERR_SHAPE;        // a token index has one axis
        if (pairs > 0 && !rotary->steps) return STA_ERR_NULL;
        if (((uintptr_t)rotary->steps & 7) || ((uintptr_t)rotary->positions & 3)) return STA_ERR_SHAPE;
        if (rotary->position_batch < 0 || rotary->position_token < 0 || rotary->position_batch > kMostStride || rotary->position_token > kMostStride)
            return STA_ERR_SHAPE;
        p->rot = rotary->channels;
        p->steps = rotary->steps;
        p->positions = pairs > 0 ? rotary->positions : nullptr;
        p->position_batch = rotary->position_batch;
        p->position_token = rotary->position_token;
        p->axis1 = rotary->pairs[0];
        p->axis2 = rotary->pairs[0] + rotary->pairs[1];
        p->magnitude = rotary->magnitude == 0.f ? 1.f : rotary->magnitude;
        p->interleaved = rotary->interleaved != 0;
        p->turns = pairs > 0;
    }
    return STA_OK;
}

// Which kernel: the general one where a chunk of 8 channels is not 16 aligned bytes or would be split by the rotation (4000 tokens of 24 heads of 128
// channels, queries, keys and values: 32 us, gradients 47; fast 29, 37; the clip of 115,200: 897, 1795; 775, 1162), and for few rows, where its
// lanes, with 2 pairs each and not 8, are done sooner: up to 2^21 channels (12 heads of 128 in bf16, forward and backward alone: one token 3.8, 6.7 us
// against 5.2, 9.0; 200 tokens of 24 heads, at that bound, 5.3, 10.3 against 7.2, 10.9; 1000 tokens 12.8, 20.3 against 12.8, 16.5).
constexpr uint64_t kFewChannels = 1u << 21;
int path_of(const Params &p)
{
    uint64_t heads = 0;
    for (uint32_t i = 0; i < p.n_tensors; ++i) heads += p.t[i].heads;
    if (p.D % 16 || p.rot % (p.interleaved ? 8 : 16) || p.tokens * heads * p.D <= kFewChannels) return kGeneral;
    for (uint32_t i = 0; i < p.n_tensors; ++i)
        if (!chunked(p.t[i].x) || !chunked(p.t[i].out) || !chunked(p.t[i].dy)) return kGeneral;
    return p.interleaved ? kInterleaved : kHalf;
}

// Workgroups: forward, fast path: two a CU (2 x 2180 tokens of 16 heads of 128 11.6 us; four 13.6; 4000 tokens of 72 heads 28.0; four 28.8, eight 33.4,
// sixteen 39.6); general path, forward and backward: four (256 tokens of 36 heads 5.1 us; two 5.9, one 7.0); gradients: four (18,432 tokens of 24 heads,
// with the forward, 96 us; two 105, one 131).
constexpr uint32_t kWantBlocks = 512, kWantGeneral = 1024;
constexpr uint32_t kMostPartials = 1024;        // workgroups of the gradients

// Heads are dealt to gridDim.y workgroups where the tokens alone do not make enough of them.
uint32_t split_of(uint32_t groups, uint32_t heads, uint32_t blocks)
{
    const uint32_t most = (heads + kWaves - 1) / kWaves, want = (blocks + groups - 1) / groups;
    return want < 1 ? 1 : want < most ? want : most;
}

// The forward's grid: `per` tokens a workgroup.
dim3 forward_grid(uint32_t tokens, uint32_t per, uint32_t heads, uint32_t blocks)
{
    const uint32_t groups = (tokens + per - 1) / per;
    return dim3(groups >> kGridShift ? 1u << kGridShift : groups, split_of(groups, heads, blocks), ((groups - 1) >> kGridShift) + 1);
}

template <int PATH, int L, bool SRC_F32, bool DST_F32>
hipError_t launch(Params &p, bool backward, hipStream_t stream)
{
    const uint32_t per = 64 / L, groups = (p.tokens + per - 1) / per;
    uint32_t heads = 0;
    for (uint32_t i = 0; i < p.n_tensors; ++i) heads += p.t[i].heads;
    if (!backward)
        return sta::launch_kernel(sta_rows_forward_kernel<PATH, L, SRC_F32, DST_F32>, forward_grid(p.tokens, per, heads, PATH == kGeneral ? kWantGeneral : kWantBlocks), dim3(kThreads), stream, p);
    // workgroups by heads, units of as few heads a wave as it takes to have that many
    uint32_t first = 0;
    for (uint32_t i = 0; i < 3; ++i) {
        Share &s = p.share[i];
        const uint32_t h = i < p.n_tensors ? p.t[i].heads : 0;
        uint32_t blocks = (uint32_t)((uint64_t)(kMostPartials - 3) * h / heads) + (h > 0);
        const uint32_t most = (h + kWaves - 1) / kWaves, want = (blocks + groups - 1) / groups, splits = want < 1 ? 1 : want < most ? want : most;
        s.units = h > 0 ? groups * (splits > 0 ? splits : 1) : 0;
        s.splits = fast_div_of(splits > 0 ? splits : 1);
        s.blocks = blocks < s.units ? blocks : s.units;
        s.first = first;
        first += s.blocks;
    }
    return sta::launch_kernel(sta_rows_backward_kernel<PATH, L, SRC_F32, DST_F32>, dim3(first), dim3(kThreads), stream, p);
}

template <int PATH, int L>
hipError_t launch_types(Params &p, bool src_f32, bool dst_f32, bool backward, hipStream_t stream)
{
    if (src_f32) return dst_f32 ? launch<PATH, L, true, true>(p, backward, stream) : launch<PATH, L, true, false>(p, backward, stream);
    return dst_f32 ? launch<PATH, L, false, true>(p, backward, stream) : launch<PATH, L, false, false>(p, backward, stream);
}

template <int PATH>
hipError_t launch_lanes(Params &p, bool src_f32, bool dst_f32, bool backward, hipStream_t stream)
{
    if (p.D <= 64) return launch_types<PATH, 4>(p, src_f32, dst_f32, backward, stream);
    if (p.D <= 128) return launch_types<PATH, 8>(p, src_f32, dst_f32, backward, stream);
    return launch_types<PATH, 16>(p, src_f32, dst_f32, backward, stream);
}

hipError_t launch_rows(Params &p, bool src_f32, bool dst_f32, bool backward, hipStream_t stream)
{
    switch (path_of(p)) {
    case kHalf: return launch_lanes<kHalf>(p, src_f32, dst_f32, backward, stream);
    case kInterleaved: return launch_lanes<kInterleaved>(p, src_f32, dst_f32, backward, stream);
    default:                    // two pairs a lane; 32 and 64 lanes where 16 do: 4000 tokens of 72 heads of 48 19 us, 29, 53
        if (p.D <= 64) return launch_types<kGeneral, 16>(p, src_f32, dst_f32, backward, stream);
        if (p.D <= 128) return launch_types<kGeneral, 32>(p, src_f32, dst_f32, backward, stream);
        return launch_types<kGeneral, 64>(p, src_f32, dst_f32, backward, stream);
    }
}

}  // namespace

extern "C" {

// Not part of the ABI (include/sta.h), for the tests: the grid of a forward launch of `per` tokens a workgroup.
void sta_rows_grid(uint32_t tokens, uint32_t per, uint32_t heads, uint32_t grid[3])
{
    const dim3 g = forward_grid(tokens, per, heads, kWantGeneral);
    grid[0] = g.x; grid[1] = g.y; grid[2] = g.z;
}

// Nor this: whether the checks of arguments take a and b to overlap.
int sta_rows_overlap(const sta_head_rows *a, int64_t Na, const sta_head_rows *b, int64_t Nb, int64_t B, int D) { return rows_overlap(*a, Na, *b, Nb, B, D); }

int sta_rope_steps(int channels, double theta, int scaling, double factor, double original_positions, int64_t *steps, float *magnitude)
{
    if (!steps) return STA_ERR_NULL;
    if (channels < 2 || channels % 2 || channels > kMostD) return STA_ERR_SHAPE;
    if (scaling < STA_ROPE_NONE || scaling > STA_ROPE_YARN) return STA_ERR_UNSUPPORTED;
    if (!(theta >= 1.0) || !(theta <= 1e300)) return STA_ERR_SHAPE;
    if (scaling != STA_ROPE_NONE && (!(factor >= 1.0) || !(factor <= 1e9))) return STA_ERR_SHAPE;
    if (scaling == STA_ROPE_YARN && !(original_positions >= 1.0)) return STA_ERR_SHAPE;
    const long double two_pi = 6.283185307179586476925286766559L;
    const int pairs = channels / 2;
    long double base = theta;
    if (scaling == STA_ROPE_NTK && pairs > 1) base *= powl((long double)factor, (long double)channels / (channels - 2));
    for (int i = 0; i < pairs; ++i) {
        long double f = powl(base, -(long double)i / pairs);
        if (scaling == STA_ROPE_LINEAR) f /= factor;
        if (scaling == STA_ROPE_YARN) {
            long double keep = (original_positions * f / two_pi - 1.0L) / 31.0L;
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f = f * keep + f / factor * (1 - keep);
        }
        steps[i] = (int64_t)roundl(f / two_pi * 18446744073709551616.0L);          // f <= 1: below 2^62
    }
    if (magnitude) *magnitude = scaling == STA_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return STA_OK;
}

int sta_rope(const sta_head_rows *in, const sta_head_rows *out, int n_tensors, int B, int N, int D, const sta_rotary *rotary, int inverse,
             void *hip_stream)
{
    if (!in || !out || !rotary) return STA_ERR_NULL;
    if (n_tensors < 1 || n_tensors > 3) return STA_ERR_SHAPE;
    Params p = {};
    if (int rc = fill_params(&p, rotary, B, N, D, nullptr, nullptr, 0.f, inverse)) return rc;
    if (p.tokens == 0) return STA_OK;
    for (int i = 0; i < n_tensors; ++i) {
        if (int rc = check_rows(in + i, false, B, N, D)) return rc;
        if (int rc = check_rows(out + i, true, B, N, D)) return rc;
        if (in[i].heads != out[i].heads) return STA_ERR_SHAPE;
        if (in[i].dtype != in[0].dtype || out[i].dtype != out[0].dtype) return STA_ERR_UNSUPPORTED;
    }
    for (int i = 0; i < n_tensors; ++i)
        if (meets_rotary(rotary, B, N, out + i, D, nullptr, 0)) return STA_ERR_ALIAS;
    for (int i = 0; i < n_tensors; ++i)
        for (int j = 0; j < n_tensors; ++j) {
            if (!(i == j && same_rows(in[i], out[j])) && rows_overlap(in[i], out[j], B, N, D)) return STA_ERR_ALIAS;
            if (i < j && rows_overlap(out[i], out[j], B, N, D)) return STA_ERR_ALIAS;
        }
    p.n_tensors = n_tensors;
    for (int i = 0; i < n_tensors; ++i) {
        p.t[i].x = rows_of(in[i]);
        p.t[i].out = rows_of(out[i]);
        p.t[i].heads = in[i].heads;
        p.t[i].rotate = p.turns;
    }
    const hipError_t e = launch_rows(p, in[0].dtype == STA_F32, out[0].dtype == STA_F32, false, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}

int sta_qk_norm_rope(const sta_head_rows *q, const sta_head_rows *k, const sta_head_rows *v, const sta_head_rows *q_out,
                     const sta_head_rows *k_out, const sta_head_rows *v_out, const void *q_weight, const void *k_weight, int weight_dt,
                     float eps, const sta_rotary *rotary, int B, int N, int D, const int grid[3], const int tile[3], void *hip_stream)
{
    if (!q || !k || !q_out || !k_out || (v == nullptr) != (v_out == nullptr)) return STA_ERR_NULL;
    if (!valid_type(weight_dt)) return STA_ERR_UNSUPPORTED;
    Params p = {};
    if (int rc = fill_params(&p, rotary, B, N, D, grid, tile, eps, 0)) return rc;
    if (p.tokens == 0) return STA_OK;
    const sta_head_rows *in[3] = {q, k, v}, *out[3] = {q_out, k_out, v_out};
    p.n_tensors = v ? 3 : 2;
    p.weight_f32 = weight_dt == STA_F32;
    for (uint32_t i = 0; i < p.n_tensors; ++i) {
        if (int rc = check_rows(in[i], false, B, N, D)) return rc;
        if (int rc = check_rows(out[i], true, B, N, D)) return rc;
        if (in[i]->heads != out[i]->heads) return STA_ERR_SHAPE;
        if (in[i]->dtype != q->dtype || out[i]->dtype != q_out->dtype) return STA_ERR_UNSUPPORTED;
        p.t[i].x = rows_of(*in[i]);
        p.t[i].out = rows_of(*out[i]);
        p.t[i].heads = in[i]->heads;
        p.t[i].norm = i < 2;
        p.t[i].rotate = i < 2 && p.turns;
        p.t[i].weight = i == 0 ? q_weight : i == 1 ? k_weight : nullptr;
        if ((uintptr_t)p.t[i].weight % size_of(weight_dt)) return STA_ERR_SHAPE;
    }
    for (uint32_t i = 0; i < p.n_tensors; ++i)
        for (uint32_t j = 0; j < p.n_tensors; ++j) {
            if (!(i == j && !tile && same_rows(*in[i], *out[j])) && rows_overlap(*in[i], *out[j], B, N, D)) return STA_ERR_ALIAS;
            if (i < j && rows_overlap(*out[i], *out[j], B, N, D)) return STA_ERR_ALIAS;
            if (rows_meet(*out[i], B, N, D, p.t[j].weight, (uint64_t)D * size_of(weight_dt))) return STA_ERR_ALIAS;
        }
    for (uint32_t i = 0; i < p.n_tensors; ++i)
        if (meets_rotary(rotary, B, N, out[i], D, nullptr, 0)) return STA_ERR_ALIAS;
    const hipError_t e = launch_rows(p, q->dtype == STA_F32, q_out->dtype == STA_F32, false, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? STA_OK : STA_ERR_HIP;
}

size_t sta_qk_norm_rope_workspace_bytes(int D)
{
    return D < 2 || D > kMostD || D % 2 ? 0 : (size_t)kMostPartials * D * sizeof(float);
}

int sta_qk_norm_rope_backward(const sta_head_rows *q, const sta_head_rows *k, const sta_head_rows *d_q_out, const sta_head_rows *d_k_out,
                              const sta_head_rows *d_v_out, const sta_head_rows *d_q, const sta_head_rows *d_k, const sta_head_rows *d_v,
                              const void *q_weight, const void *k_weight, int weight_dt, float *d_q_weight, float *d_k_weight, float eps,
                              const sta_rotary *rotary, int B, int N, int D, const int grid[3], const int tile[3], void *workspace,
                              size_t workspace_bytes, void *hip_stream)
{
    if (!q || !k || !d_q_out || !d_k_out || !d_q || !d_k || (d_v_out == nullptr) != (d_v == nullptr)) return STA_ERR_NULL;
    if (!valid_type(weight_dt)) return STA_ERR_UNSUPPORTED;
    Params p = {};
    if (int rc = fill_params(&p, rotary, B, N, D, grid, tile, eps, 0)) return rc;
    const bool sums = d_q_weight || d_k_weight;
    if (sums && (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < sta_qk_norm_rope_workspace_bytes(D))) return STA_ERR_WORKSPACE;
    if (((uintptr_t)d_q_weight | (uintptr_t)d_k_weight) & 3) return STA_ERR_SHAPE;
    const size_t sum_bytes = D * sizeof(float);
    const float *sum_of[2] = {d_q_weight, d_k_weight};
    if (ranges_meet(d_q_weight, sum_bytes, d_k_weight, sum_bytes)) return STA_ERR_ALIAS;
    for (const float *s : sum_of) {
        if (sums && ranges_meet(s, sum_bytes, workspace, sta_qk_norm_rope_workspace_bytes(D))) return STA_ERR_ALIAS;
        for (const void *w : {q_weight, k_weight})
            if (ranges_meet(s, sum_bytes, w, (uint64_t)D * size_of(weight_dt))) return STA_ERR_ALIAS;
    }
    const sta_head_rows *x[3] = {q, k, nullptr}, *dy[3] = {d_q_out, d_k_out, d_v_out}, *dx[3] = {d_q, d_k, d_v};
    p.n_tensors = d_v ? 3 : 2;
    p.weight_f32 = weight_dt == STA_F32;
    p.partial = sums ? static_cast<float *>(workspace) : nullptr;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (p.tokens != 0) {
        for (uint32_t i = 0; i < p.n_tensors; ++i) {
            if (x[i])
                if (int rc = check_rows(x[i], false, B, N, D)) return rc;
            if (int rc = check_rows(dy[i], false, B, N, D)) return rc;
            if (int rc = check_rows(dx[i], true, B, N, D)) return rc;
            if (dy[i]->heads != dx[i]->heads || (x[i] && x[i]->heads != dx[i]->heads)) return STA_ERR_SHAPE;
            if (dx[i]->dtype != q->dtype || (x[i] && x[i]->dtype != q->dtype) || dy[i]->dtype != d_q_out->dtype) return STA_ERR_UNSUPPORTED;
            p.t[i].dy = rows_of(*dy[i]);
            p.t[i].out = rows_of(*dx[i]);
            if (x[i]) p.t[i].x = rows_of(*x[i]);
            p.t[i].heads = dx[i]->heads;
            p.t[i].norm = i < 2;
            p.t[i].rotate = i < 2 && p.turns;
            p.t[i].weight = i == 0 ? q_weight : i == 1 ? k_weight : nullptr;
            if ((uintptr_t)p.t[i].weight % size_of(weight_dt)) return STA_ERR_SHAPE;
        }
        for (uint32_t i = 0; i < p.n_tensors; ++i)
            for (uint32_t j = 0; j < p.n_tensors; ++j) {
                if ((x[i] && rows_overlap(*x[i], *dx[j], B, N, D)) || rows_overlap(*dy[i], *dx[j], B, N, D)) return STA_ERR_ALIAS;
                if (i < j && rows_overlap(*dx[i], *dx[j], B, N, D)) return STA_ERR_ALIAS;
                if (rows_meet(*dx[i], B, N, D, p.t[j].weight, (uint64_t)D * size_of(weight_dt))) return STA_ERR_ALIAS;
            }
        for (uint32_t i = 0; i < p.n_tensors; ++i)
            for (const sta_head_rows *r : {x[i], dy[i], dx[i]}) {
                if (!r) continue;
                if (sums && rows_meet(*r, B, N, D, workspace, sta_qk_norm_rope_workspace_bytes(D))) return STA_ERR_ALIAS;
                for (const float *s : sum_of)
                    if (rows_meet(*r, B, N, D, s, sum_bytes)) return STA_ERR_ALIAS;
            }
        for (uint32_t i = 0; i < p.n_tensors; ++i)
            if (meets_rotary(rotary, B, N, dx[i], D, nullptr, 0)) return STA_ERR_ALIAS;
        for (const float *s : sum_of)
            if (meets_rotary(rotary, B, N, nullptr, D, s, sum_bytes)) return STA_ERR_ALIAS;
        if (sums && meets_rotary(rotary, B, N, nullptr, D, workspace, sta_qk_norm_rope_workspace_bytes(D))) return STA_ERR_ALIAS;
        if (launch_rows(p, q->dtype == STA_F32, d_q_out->dtype == STA_F32, true, stream) != hipSuccess) return STA_ERR_HIP;
    }
    if (sums && sta::launch_kernel(sta_rows_weights_kernel, dim3((D + 15) / 16, 2), dim3(16 * kSlices), stream, p.partial, p.share[0].blocks,
                                  p.share[1].blocks, p.D, d_q_weight, d_k_weight) != hipSuccess)
        return STA_ERR_HIP;
    return STA_OK;
}

}  // extern "C"
