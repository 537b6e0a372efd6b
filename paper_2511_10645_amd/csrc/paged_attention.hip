// Attention of one new token of every sequence over a paged key-value cache:
//
//      o_h = sum_t p_t v_t / sum_t p_t,   p_t = 2^(x_t - m),   x_t = log2(e) scale q_h . k_t,   m = the running maximum
//
// Bound by HBM: 2 head_dim elements per token and key-value head are read once and used for q_heads / kv_heads
// queries, a few flops per byte.
//
// Work is cut into units of 32 tokens of one (sequence, key-value head, up to 16 of its query heads) - a segment being
// all units of such a head - numbered one sequence after the other, and every wave of the grid takes the same number of
// consecutive units, whatever the lengths are: it finds its place from a sum over the lengths.  A wave writes the
// results of segments that are all its own; shares of others go to LDS, where the block's waves join them, and
// segments that several blocks share leave fp32 partial results in the scratch, joined by the block that arrives last
// (a counter per segment; nobody waits) in the order of their units, so that results do not depend on timing.  More than
// kGroupParts of them are joined in groups first, each by the last block of its group.
//
// A wave multiplies on the matrix cores without LDS: keys are the A operand of S^T = K Q^T (the cache keeps them in
// that operand's order, so a request of 64 lanes is contiguous), and S^T leaves the instruction as the B operand
// of O^T = V^T P^T wants it, 8 tokens of one query in a lane, if that product's tokens are taken in the order
// 4 (lane/16) + (0..3) of the unit's first 16, then of its second 16.  Values are loaded as rows, whole cache lines, 8
// tokens by head_dim/16 channels to a lane, and transposed there by byte permutes.  For that product p is held as the sum
// of two fp16 numbers, which keeps 22 of its bits (one number would add as much error as the result's own rounding, and
// the matrix cores have nothing else to do), after a factor of 2^15 (the largest p is 2^15, so that 11 bits are kept
// down to 2^-29 of it); sums stay in fp32.
#include <cmath>
#include <type_traits>

#include "kv_common.h"

namespace paro {

constexpr int kUnit = 32;                        // tokens of a unit
constexpr int kAttnBlocks = 256;                 // most blocks of a launch: one for every compute unit
constexpr int kQueries = 16;                     // query heads of a unit: the N of the matrix instruction
constexpr uint32_t kLeastUnits = 4;              // of a block
constexpr uint32_t kGroupParts = 32;             // partial results that are joined at once
constexpr float kPShift = 15.0f;                 // p is held 2^15 times
constexpr int kRsrcRaw = 0x00020000;             // raw buffer, 32-bit data format
constexpr int kAgent = 16;                       // agent scope: past the L2 of the XCD
constexpr int kOnce = 2;                         // keys and values are read once: non-temporal (131071 tokens from memory: 90 us, 98 without)

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));

// waves of a block: two for every SIMD, one where a wave's registers are more than half of them
template <int D> constexpr int attn_waves() { return D == 256 ? 4 : 8; }

// Blocks for a head of one sequence of `units` units, if these are few: one where its waves can take a unit each, then at most as many
// as are joined in one round, and twice that for long ones.
__host__ __device__ constexpr uint32_t one_parts(uint32_t units, uint32_t waves)
{
    const uint32_t parts = (units + kLeastUnits - 1) / kLeastUnits, most = units <= 64 ? 8 : 16;
    return units <= waves ? 1 : parts < most ? parts : most;
}

struct AttnArgs {
    const uint8_t *k, *v, *ks, *vs;
    const _Float16 *q;
    const int32_t *table, *lengths;
    _Float16 *o;
    float *lse;
    uint32_t *arrived;                           // [2 * kAttnBlocks] of groups of parts, [batch][kv_heads * chunks] of segments
    float *partial;                              // [2 * kAttnBlocks][kQueries * (D + 4)]: m, l, then the row, of every query
    int64_t ldq, ldo, ld_table;
    int page_log, n_pages, kv_heads, group, chunks, width, batch, window;
    float per_block;                             // 1 / blocks
    float scale;                                 // with log2(e)
    Scores scores;
};

// The other three of the 4 lanes that hold one query are lanes n ^ 16, n ^ 32, n ^ 48: two exchanges of rows of lanes.
__device__ inline float max4(float x)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ inline float sum4(float x)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// Sums over lanes 0..lane.
__device__ inline uint32_t sums_upto(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);       // row_shr 1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);       // row_bcast 15 into rows 1 and 3
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);       // row_bcast 31 into rows 2 and 3
    return x;
}

// The tokens [lo, hi) that a sequence of length n attends to, and the units that cover them (at least one, so that
// every output is written).
struct Span { int lo, hi, unit0, units; };
__device__ inline Span span_of(const AttnArgs &a, int n)
{
    Span s;
    const int room = a.width << a.page_log;      // at most 2^30
    n = n < 0 ? 0 : n > room ? room : n;
    s.hi = n;
    s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
    s.unit0 = s.lo / kUnit;
    s.units = n > 0 ? (n - 1) / kUnit - s.unit0 + 1 : 1;
    return s;
}

// Walks the sequences with their lengths in the lanes, 64 of them at a time.
struct Place {
    int first, length;                           // the lanes' sequences first + lane, and their lengths
    int b;                                       // current sequence, the number of its first unit and its span
    uint32_t base;
    Span sp;
    __device__ void lanes(const AttnArgs &a, int i, int lane)
    {
        first = i;
        length = a.lengths[i + lane < a.batch ? i + lane : a.batch - 1];
    }
    __device__ void sequence(const AttnArgs &a, int i, int lane)
    {
        b = i;
        if (i - first >= 64) lanes(a, i, lane);
        sp = span_of(a, __builtin_amdgcn_readlane(length, i - first));
    }
    __device__ void next(const AttnArgs &a, int lane, uint32_t hc)
    {
        base += (uint32_t)sp.units * hc;
        sequence(a, b + 1, lane);
    }
    // Goes to the one of the lanes' sequences that holds unit `at`, given the sums of their units; false if it lies behind them.
    __device__ bool find(const AttnArgs &a, uint32_t at, uint32_t upto, uint32_t hc, int lane)
    {
        const int before = __popcll(__ballot(base + upto * hc <= at));
        if (before) base += (uint32_t)__builtin_amdgcn_readlane((int)upto, before - 1) * hc;
        if (before < 64) sequence(a, first + before, lane);
        return before < 64;
    }
};

// One wave's state over the units of one head.
template <int D>
struct Running {
    static constexpr int R = D / 16;             // channel tiles: tile r holds channels (0..15) * R + r
    F4 acc[R];
    float m, l;                                  // of query lane % 16; l over this lane's tokens only
    __device__ void clear()
    {
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r] = F4{0, 0, 0, 0};
        m = -INFINITY; l = 0;
    }
};

__device__ inline half8v f16_of_e4m3(uint32_t lo, uint32_t hi, float scale)
{
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
    const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ inline uint32_t f16x2_of_e4m3(uint32_t w, float scale, bool hi)
{
    union { half2v h; uint32_t u; } c;
    c.h = hi ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false);
    return c.u;
}

__device__ inline uint32_t f16x2_of_e2m1(uint32_t w, float scale, int pair)
{
    return __builtin_bit_cast(uint32_t, pair == 0 ? f16x2_of_e2m1<0>(w, scale) : pair == 1 ? f16x2_of_e2m1<1>(w, scale) : pair == 2 ? f16x2_of_e2m1<2>(w, scale) : f16x2_of_e2m1<3>(w, scale));
}

template <int D, int FMT>
struct Operand {
    static constexpr int kKeyBytes = row_bytes<FMT>(D) / 4 < 16 ? row_bytes<FMT>(D) / 4 : 16;   // of a request in a lane (8: MXFP4 heads of 64 channels)
    static constexpr int kKeyLoads = row_bytes<FMT>(D) / 4 / kKeyBytes;   // requests per 16 tokens
    static constexpr int kRowBytes = row_bytes<FMT>(D) / 16;              // of a value row in a lane
    static constexpr int kRowWords = (kRowBytes + 3) / 4;
};

// What a wave holds of a unit between its requests and its products.
template <int D, int FMT>
struct Keys {
    U4 k[2][Operand<D, FMT>::kKeyLoads];
    uint32_t scale[2][FMT == kMxfp4 ? Operand<D, FMT>::kKeyLoads : 1];    // E4M3: bytes of 4 tokens, MXFP4: of the request's 32 channels
};
template <int D, int FMT>
struct Values {
    uint32_t v[8][Operand<D, FMT>::kRowWords];
    uint32_t scale[2];                           // bytes of 4 tokens
};

// One (page, head) of the cache as a buffer: a request past `bytes` returns 0 and costs nothing, which keeps the requests of a
// loop unconditional and their number in flight known.
__device__ inline __amdgpu_buffer_rsrc_t attn_rsrc(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, kRsrcRaw);
}

struct Head {                                    // of the segment at hand
    int64_t page_bytes, at;                      // of a page, of this head in it
    uint32_t bytes;                              // of this head in a page
    int page_log, head, kv_heads;
};

// keys of 2 x 16 tokens: token lane % 16, units of channels lane / 16 + 4 s; pages pg[0], pg[1] (negative: none)
template <int D, int FMT>
__device__ inline void load_keys(Keys<D, FMT> &x, const AttnArgs &a, const Head &h, const int (&pg)[2], int t0, bool on, int lane)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t p = pg[i] < 0 ? 0 : pg[i];
        const int tok = (t0 + 16 * i) & ((1 << h.page_log) - 1);
        const __amdgpu_buffer_rsrc_t r = attn_rsrc(a.k + p * h.page_bytes + h.at, on ? h.bytes : 0);
#pragma unroll
        for (int s = 0; s < Operand<D, FMT>::kKeyLoads; ++s)
            if constexpr (Operand<D, FMT>::kKeyBytes == 16)
                x.k[i][s] = __builtin_bit_cast(U4, __builtin_amdgcn_raw_buffer_load_b128(r, (((s * 4 + (lane >> 4)) << h.page_log) + (lane & 15)) << 4, tok << 4, kOnce));
            else {
                const U2 y = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(r, ((((lane >> 5) << h.page_log) + (lane & 15)) << 4) + ((lane >> 4) & 1) * 8, tok << 4, kOnce));
                x.k[i][s] = U4{y[0], y[1], 0, 0};
            }
        if constexpr (FMT != kFp16) {
            constexpr int S = row_scales<FMT>(D);
            const __amdgpu_buffer_rsrc_t q = attn_rsrc(a.ks + (((p * h.kv_heads + h.head) * S) << h.page_log), on ? S << h.page_log : 0);
            if constexpr (FMT == kE4m3) x.scale[i][0] = __builtin_amdgcn_raw_buffer_load_b32(q, 4 * (lane >> 4), tok, kOnce);
            else
#pragma unroll
                for (int s = 0; s < Operand<D, FMT>::kKeyLoads; ++s)
                    x.scale[i][s] = __builtin_amdgcn_raw_buffer_load_b8(q, ((D == 64 ? lane >> 5 : s * 4 + (lane >> 4)) << h.page_log) + (lane & 15), tok, kOnce);
        }
    }
}
// rows of values: tokens 16 i + 4 (lane / 16) + j, channels (lane % 16) * D/16 ...
template <int D, int FMT>
__device__ inline void load_values(Values<D, FMT> &x, const AttnArgs &a, const Head &h, const int (&pg)[2], int t0, int lane)
{
    constexpr int W = Operand<D, FMT>::kRowWords, kRowBytes = row_bytes<FMT>(D);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t p = pg[i] < 0 ? 0 : pg[i];
        const int tok = (t0 + 16 * i) & ((1 << h.page_log) - 1);
        const __amdgpu_buffer_rsrc_t r = attn_rsrc(a.v + p * h.page_bytes + h.at, h.bytes);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int off = (4 * (lane >> 4) + j) * kRowBytes + (lane & 15) * Operand<D, FMT>::kRowBytes;
            uint32_t *v = x.v[4 * i + j];
            if constexpr (W % 4 == 0)
#pragma unroll
                for (int w = 0; w < W; w += 4) {
                    const U4 y = __builtin_bit_cast(U4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 4 * w, tok * kRowBytes, kOnce));
                    v[w] = y[0]; v[w + 1] = y[1]; v[w + 2] = y[2]; v[w + 3] = y[3];
                }
            else if constexpr (W == 2) {
                const U2 y = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(r, off, tok * kRowBytes, kOnce));
                v[0] = y[0]; v[1] = y[1];
            } else if constexpr (Operand<D, FMT>::kRowBytes == 4)
                v[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, tok * kRowBytes, kOnce);
            else
                v[0] = __builtin_amdgcn_raw_buffer_load_b16(r, off, tok * kRowBytes, kOnce);
        }
        if constexpr (FMT != kFp16) {            // MXFP4: of the 32 channels that the lane's are among
            constexpr int S = row_scales<FMT>(D);
            const __amdgpu_buffer_rsrc_t q = attn_rsrc(a.vs + (((p * h.kv_heads + h.head) * S) << h.page_log), S << h.page_log);
            const int group = FMT == kMxfp4 ? ((lane & 15) * (D / 16)) >> 5 : 0;
            x.scale[i] = __builtin_amdgcn_raw_buffer_load_b32(q, (group << h.page_log) + 4 * (lane >> 4), tok, kOnce);
        }
    }
}

// log2-scaled scores of a unit: x[8], token 16 (j / 4) + 4 (lane / 16) + j % 4, query lane % 16; RAW: without the scale
template <int D, int FMT, bool RAW>
__device__ inline void scores(float (&x)[8], const Keys<D, FMT> &k, const half8v (&q)[D / 32], float scale)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        F4 s4 = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < Operand<D, FMT>::kKeyLoads; ++s) {
            if constexpr (FMT == 0) {
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, k.k[i][s]), q[s], s4, 0, 0, 0);
            } else if constexpr (FMT == kMxfp4) {
                const float up = __uint_as_float(k.scale[i][s] << 23);
#pragma unroll
                for (int w = 0; w < Operand<D, FMT>::kKeyBytes / 4; ++w)
                    s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of_e2m1(k.k[i][s][w], up), q[Operand<D, FMT>::kKeyBytes / 4 * s + w], s4, 0, 0, 0);
            } else {
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of_e4m3(k.k[i][s][0], k.k[i][s][1], 1.0f), q[2 * s], s4, 0, 0, 0);
                s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of_e4m3(k.k[i][s][2], k.k[i][s][3], 1.0f), q[2 * s + 1], s4, 0, 0, 0);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[4 * i + j] = RAW ? s4[j] : s4[j] * scale;
            if constexpr (FMT == kE4m3) x[4 * i + j] *= __uint_as_float(((k.scale[i][0] >> (8 * j)) & 255) << 23);
        }
    }
}

// Scores q . k capped, scaled to log2 and lowered by their tokens' distance from the last one, `away0` for the lane's first.
__device__ inline void adjust(float (&x)[8], const AttnArgs &a, float slope, float away0)
{
    if (a.scores.cap > 0) {
        capped(x, a.scores);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= a.scale;
    }
    if (a.scores.slopes) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmaf(-slope, away0 - (16 * (j >> 2) + (j & 3)), x[j]);
    }
}

// The unit's tokens outside [lo, hi) or on pages that are not there: scores -inf, and values 0 (such places may hold NaN).
template <int D, int FMT>
__device__ inline void mask(float (&x)[8], Values<D, FMT> &v, const int (&pg)[2], int t0, int lo, int hi, int lane)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int t = t0 + 16 * (j >> 2) + 4 * (lane >> 4) + (j & 3);
        const bool in = t >= lo && t < hi && pg[j >> 2] >= 0;
        x[j] = in ? x[j] : -INFINITY;
#pragma unroll
        for (int w = 0; w < Operand<D, FMT>::kRowWords; ++w) v.v[j][w] = in ? v.v[j][w] : 0u;
        if constexpr (FMT != kFp16) if (!in) v.scale[j >> 2] = (v.scale[j >> 2] & ~(255u << (8 * (j & 3)))) | (127u << (8 * (j & 3)));
    }
}

// The running maximum, sum and result take in a unit.
template <int D, int FMT>
__device__ inline void take_in(Running<D> &st, const float (&x)[8], const Values<D, FMT> &v)
{
    constexpr int R = D / 16;
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(st.m, max4(top));
    if (__ballot(top > st.m)) {
        const float f = top > st.m ? __builtin_amdgcn_exp2f(st.m - top) : 1.0f;
        st.l *= f;
#pragma unroll
        for (int r = 0; r < R; ++r) st.acc[r] *= f;
        st.m = top;
    }
    // The shift goes onto the difference: off a maximum of 2^24 and more, 15 is rounded to 16, and 2^16 is not an fp16 number.
    const float ref = st.m == -INFINITY ? 0.0f : st.m;
    half8v p, rest;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float e = __builtin_amdgcn_exp2f((x[j] - ref) + kPShift);
        st.l += e;
        p[j] = (_Float16)e;
        rest[j] = (_Float16)(e - (float)p[j]);
    }
    // O^T += V^T P^T, one tile of 16 channels after the other
    if constexpr (FMT == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            U4 f;
#pragma unroll
            for (int y = 0; y < 4; ++y) f[y] = __builtin_amdgcn_perm(v.v[2 * y + 1][r / 2], v.v[2 * y][r / 2], r & 1 ? 0x07060302u : 0x05040100u);
            st.acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, f), p, st.acc[r], 0, 0, 0);
            st.acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, f), rest, st.acc[r], 0, 0, 0);
        }
    } else {
        float vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) vs[j] = __uint_as_float(((v.scale[j >> 2] >> (8 * (j & 3))) & 255) << 23);
#pragma unroll
        for (int r = 0; r < R; r += 2) {
            uint32_t c[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = FMT == kE4m3 ? f16x2_of_e4m3(v.v[j][r / 4 % Operand<D, FMT>::kRowWords], vs[j], (r / 2) & 1) : f16x2_of_e2m1(v.v[j][r / 8], vs[j], (r / 2) & 3);
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                U4 f;
#pragma unroll
                for (int y = 0; y < 4; ++y) f[y] = __builtin_amdgcn_perm(c[2 * y + 1], c[2 * y], z ? 0x07060302u : 0x05040100u);
                st.acc[r + z] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, f), p, st.acc[r + z], 0, 0, 0);
                st.acc[r + z] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, f), rest, st.acc[r + z], 0, 0, 0);
            }
        }
    }
}

__device__ inline float lse_of(float m, float sum) { return sum == 0.0f ? -INFINITY : (m - kPShift + __builtin_amdgcn_logf(sum)) * kLn2; }

// x / d for a quotient up to 2^20, inv = 1 / d to some units of fp32; up to 2^22 with an exact inv (units of a block: above 2^20 only
// where the grid is at its 256 blocks).
__device__ inline uint32_t quotient(uint32_t x, uint32_t d, float inv)
{
    const uint32_t q = (uint32_t)((float)x * inv), r = x - q * d;        // off by one at most
    return (int)r < 0 ? q - 1 : r >= d ? q + 1 : q;
}

// A segment that a wave has a share of: sequence, (head, chunk), its units.
struct Segment {
    int b, seg;
    uint32_t seg0, seg1;                         // seg1 0: none
    __device__ Segment of_lane(int i) const
    {
        return {__builtin_amdgcn_readlane(b, i), __builtin_amdgcn_readlane(seg, i), (uint32_t)__builtin_amdgcn_readlane((int)seg0, i),
                (uint32_t)__builtin_amdgcn_readlane((int)seg1, i)};
    }
};
struct Target {
    int head, first, queries;                    // key-value head, first query head, their number
    Target() = default;
    __device__ Target(const AttnArgs &a, int seg)
    {
        int chunk = 0;
        head = seg;
        if (a.chunks > 1) { head = seg / a.chunks; chunk = seg - head * a.chunks; }
        first = head * a.group + chunk * kQueries;
        queries = a.group - chunk * kQueries < kQueries ? a.group - chunk * kQueries : kQueries;
    }
    __device__ _Float16 *o(const AttnArgs &a, int b, int D) const { return a.o + (int64_t)b * a.ldo + (int64_t)first * D; }
    __device__ float *lse(const AttnArgs &a, int b) const { return a.lse + (int64_t)b * (a.kv_heads * a.group) + first; }
};

// The blocks that share a segment, and the group of them that block `me` is in.
struct Sharers {
    uint32_t first, last, group, group_last;
    bool in_groups;
    __device__ Sharers(const Segment &g, uint32_t share, float per_share, uint32_t me)
    {
        first = quotient(g.seg0, share, per_share);
        last = quotient(g.seg1 - 1, share, per_share);
        in_groups = last - first + 1 > kGroupParts;
        group = (me - first) / kGroupParts * kGroupParts + first;
        group_last = group + kGroupParts - 1 < last ? group + kGroupParts - 1 : last;
    }
};

// 4 channels of one query, with the maximum and sum that belong to them
struct Four {
    float m, l;
    F4 v;
    __device__ void clear() { m = -INFINITY; l = 0; v = F4{0, 0, 0, 0}; }
    // Takes in N results; read(k) gives -inf, 0 and anything finite for one that is not there, all before any is used.
    template <int N, class Read>
    __device__ void add(Read read)
    {
        float pm[N], pl[N], top = m;
        F4 pv[N];
#pragma unroll
        for (int k = 0; k < N; ++k) read(k, pm[k], pl[k], pv[k]);
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, pm[k]);
        const float ref = top == -INFINITY ? 0.0f : top, f = __builtin_amdgcn_exp2f(m - ref);
        l *= f;
        v *= f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float g = __builtin_amdgcn_exp2f(pm[k] - ref);
            l = fmaf(pl[k], g, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(pv[k][e], g, v[e]);
        }
        m = top;
    }
    __device__ void result(const AttnArgs &a, const Target &to, int b, int D, int query, int channel) const
    {
        const float inv = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
        *(half4v *)(to.o(a, b, D) + query * D + channel) = half4v{(_Float16)(v[0] * inv), (_Float16)(v[1] * inv), (_Float16)(v[2] * inv), (_Float16)(v[3] * inv)};
        if (a.lse && channel == 0) to.lse(a, b)[query] = lse_of(m, l);
    }
};

template <int D> constexpr int part_floats() { return kQueries * (D + 4); }
// Four of the partial result in slot `slot`, through memory that all XCDs see
template <int D>
__device__ inline void store_part(__amdgpu_buffer_rsrc_t r, uint32_t slot, int query, int channel, const Four &x)
{
    const uint32_t row = (slot * part_floats<D>() + query * (D + 4)) * 4u;
    typedef decltype(__builtin_amdgcn_raw_buffer_load_b128(r, 0, 0, 0)) B4;
    typedef decltype(__builtin_amdgcn_raw_buffer_load_b64(r, 0, 0, 0)) B2;
    if (channel == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(B2, U2{__float_as_uint(x.m), __float_as_uint(x.l)}), r, row, 0, kAgent);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(B4, x.v), r, row + (4 + channel) * 4u, 0, kAgent);
}

// Joins the partial results of blocks first, first + step, ... last of a segment, by the whole block: thread tid < items gets
// the Four of item0 + tid.  s: LDS of 6 floats per thread.
template <int D, int THREADS>
__device__ inline Four join_parts(__amdgpu_buffer_rsrc_t r, float *s, const Segment &g, uint32_t share, uint32_t first, uint32_t step, uint32_t last,
                                  int item0, int items, int tid)
{
    constexpr int kLots = 4;
    Four x;
    x.clear();
    // parts k0, k0 + by, ..., N of them or as many as there are, for item i
    const auto take = [&](auto n, uint32_t k0, uint32_t by, int i) {
        const int query = i / (D / 4), channel = (i % (D / 4)) * 4;
        x.add<decltype(n)::value>([&](int z, float &m, float &l, F4 &v) {
            const uint32_t k = k0 + z * by;
            // past the last one: a request beyond the buffer, which gives zeros
            const uint32_t row = k <= last ? ((2 * k + (g.seg0 >= k * share)) * part_floats<D>() + query * (D + 4)) * 4u : 0x80000000u;
            const U2 ml = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(r, row, 0, kAgent));
            v = __builtin_bit_cast(F4, __builtin_amdgcn_raw_buffer_load_b128(r, row + (4 + channel) * 4u, 0, kAgent));
            m = k <= last ? __uint_as_float(ml[0]) : -INFINITY;
            l = __uint_as_float(ml[1]);
        });
    };
    // Few parts: every thread reads all of its item.  More: `lots` groups of threads take every lots-th part and meet in LDS.
    int lots = 1;
    if (last - first < 4 * step) {
        if (tid < items) take(std::integral_constant<int, 4>(), first, step, item0 + tid);
    } else if (last - first < 8 * step) {
        if (tid < items) take(std::integral_constant<int, 8>(), first, step, item0 + tid);
    } else {
        lots = THREADS / items;
        lots = lots < kLots ? lots : kLots;
        const int lot = tid / items;
        if (lot < lots)
            for (uint32_t j = first + lot * step; j <= last; j += 8 * lots * step) take(std::integral_constant<int, 8>(), j, lots * step, item0 + tid - lot * items);
    }
    if (lots > 1) {
        F4 *sv = (F4 *)s;
        U2 *sm = (U2 *)(s + 4 * THREADS);
        sv[tid] = x.v;
        sm[tid] = U2{__float_as_uint(x.m), __float_as_uint(x.l)};
        __syncthreads();
        if (tid < items) {
            x.clear();
            x.add<kLots>([&](int k, float &m, float &l, F4 &v) {
                const int at = k < lots ? tid + k * items : tid;
                const U2 ml = sm[at];
                v = sv[at];
                m = k < lots ? __uint_as_float(ml[0]) : -INFINITY;
                l = __uint_as_float(ml[1]);
            });
        }
    }
    __syncthreads();                             // all parts are read, and LDS is free again
    return x;
}

// Counts an arrival; whether it was the last of `all`, after which the counter is 0 again.
__device__ inline bool arrives_last(uint32_t *counter, uint32_t all)
{
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (before != all - 1) return false;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}
// What this wave stored is where all XCDs see it.
__device__ inline void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <int D, int FMT, bool SCORED>
__global__ __launch_bounds__(64 * attn_waves<D>(), 1) void paged_attention_kernel(const AttnArgs a)
{
    constexpr int WAVES = attn_waves<D>(), THREADS = 64 * WAVES, R = D / 16;
    constexpr int kRow = D + 4;                  // floats of a row in LDS: rows of 16 queries fall on distinct banks
    extern __shared__ __attribute__((aligned(16))) float s_o[];          // [wave][2][rows][kRow], later the joins'
    __shared__ float s_m[WAVES * 2 * kQueries], s_l[WAVES * 2 * kQueries];
    __shared__ Segment s_seg[WAVES][2];
    __shared__ int s_last[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t hc = (uint32_t)(a.kv_heads * a.chunks);
    const int rows = a.group < kQueries ? a.group : kQueries;            // of a slot in LDS

    // the units of all sequences: lane i sums `per` consecutive ones
    Place pl;
    const int per = (a.batch + 63) >> 6;
    uint32_t upto = 0;
    if (per == 1) {
        pl.lanes(a, 0, lane);
        upto = lane < a.batch ? (uint32_t)span_of(a, pl.length).units : 0u;
    } else {
#pragma unroll 4
        for (int j = 0; j < per; ++j) {
            const int i = lane * per + j, n = a.lengths[i < a.batch ? i : a.batch - 1];
            upto += i < a.batch ? (uint32_t)span_of(a, n).units : 0u;
        }
    }
    upto = sums_upto(upto);
    uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * hc;
    // Units of a block and of a wave: all waves of the grid alike; where that would leave a block fewer than kLeastUnits, fewer blocks.
    uint32_t share = quotient(total + gridDim.x - 1, gridDim.x, a.per_block), mine = 1;
    if (share < kLeastUnits) share = kLeastUnits;
    // One sequence of some thousand tokens at most: every head begins with a block of its own (segments are numbered `pitch` apart), so that
    // its parts are as few and as even as can be, and a head of up to WAVES units stays in one block (200 tokens: 9.1 -> 6.8 us).  That ends
    // at two units a wave: few heads of a longer sequence are spread over all blocks (one of 32768 tokens: 26.5 us in 16 blocks, 12.3 in
    // 256; a limit of one unit a wave takes 8 heads of 6000 tokens from 13.3 to 14.1).
    const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)upto, 0);
    uint32_t pitch = 0, head_end = total;
    if (a.batch == 1) {
        const uint32_t parts = one_parts(one, WAVES);
        if (share <= WAVES && hc * parts <= gridDim.x && one <= 2 * WAVES * parts) {
            const float per_parts = __builtin_amdgcn_rcpf((float)parts);
            share = quotient(one + parts - 1, parts, per_parts);
            pitch = parts * share;
            total = pitch * hc;
            head_end = quotient(blockIdx.x, parts, per_parts) * pitch + one;
        }
    }
    if (share >= WAVES || pitch) mine = (share + WAVES - 1) / WAVES;
    if (share >= WAVES && !pitch) share = mine * WAVES;
    const uint32_t begin = blockIdx.x * share;
    if (begin >= total) return;
    const uint32_t end = begin + share < head_end ? begin + share : head_end;
    const uint32_t wbegin = begin + wave * mine, wend = wbegin + mine < end ? wbegin + mine : end;
    const float per_share = __builtin_amdgcn_rcpf((float)share);

    const int n = lane & 15, quarter = lane >> 4;
    if (lane < 2) s_seg[wave][lane].seg1 = 0;
    if (tid < 2) s_last[tid] = 0;
    const bool busy = wbegin < wend;
    if (busy) {
        pl.base = 0;
        if (pitch) {
            pl.sequence(a, 0, lane);
        } else if (per == 1) {
            pl.find(a, wbegin, upto, hc, lane);
        } else {                                 // the lane whose sequences hold unit wbegin, and these one to a lane
            const int before = __popcll(__ballot(upto * hc <= wbegin));
            if (before) pl.base = (uint32_t)__builtin_amdgcn_readlane((int)upto, before - 1) * hc;
            for (int i = before * per;; i += 64) {
                pl.lanes(a, i, lane);
                if (pl.find(a, wbegin, sums_upto(i + lane < a.batch ? (uint32_t)span_of(a, pl.length).units : 0u), hc, lane)) break;
            }
        }
    }
    Head h;
    h.page_log = a.page_log;
    h.kv_heads = a.kv_heads;
    h.bytes = (uint32_t)row_bytes<FMT>(D) << a.page_log;
    h.page_bytes = (int64_t)h.bytes * a.kv_heads;
    Segment g;                                   // the segment at hand: units u0..u1 of it, tokens lo..hi of its sequence
    int u0, u1, lo, hi, pages = 0;
    const int32_t *row;
    Target to;
    half8v q[D / 32];
    float slope = 0;                             // of query lane % 16
    // the pages of the next 32 units, two halves to a unit
    const auto turn = [&](int u) {
        int t = (u + (lane >> 1)) * kUnit + (lane & 1) * 16;
        t = t < hi ? t : hi - 1;
        pages = hi > 0 ? row[t >> a.page_log] : 0;
    };
    const auto locate = [&](uint32_t at) {
        if (!pitch)
            while (pl.base + (uint32_t)pl.sp.units * hc <= at) pl.next(a, lane, hc);
        lo = pl.sp.lo; hi = pl.sp.hi;
        row = a.table + (int64_t)pl.b * a.ld_table;
        const uint32_t units = (uint32_t)pl.sp.units, apart = pitch ? pitch : units;
        g.b = pl.b;
        g.seg = (int)quotient(at - pl.base, apart, __builtin_amdgcn_rcpf((float)apart));
        g.seg0 = pl.base + (uint32_t)g.seg * apart;
        g.seg1 = g.seg0 + units;
        u0 = pl.sp.unit0 + (int)(at - g.seg0);
        u1 = pl.sp.unit0 + (int)((g.seg1 < wend ? g.seg1 : wend) - g.seg0);
        turn(u0);
        to = Target(a, g.seg);
        h.head = to.head;
        h.at = (int64_t)h.bytes * h.head;
        const _Float16 *qp = a.q + (int64_t)g.b * a.ldq + (int64_t)(to.first + (n < to.queries ? n : 0)) * D;
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
            q[s] = *(const half8v *)(qp + (FMT == kFp16 ? s * 32 + quarter * 8 : FMT == kE4m3 ? ((s >> 1) * 4 + quarter) * 16 + (s & 1) * 8 :
                                           D == 64 ? quarter * 16 + s * 8 : ((s >> 2) * 4 + quarter) * 32 + (s & 3) * 8));
        if constexpr (SCORED) if (a.scores.slopes) slope = a.scores.slopes[to.first + (n < to.queries ? n : 0)] * kLog2e;
    };
    if (busy) locate(wbegin);
    __syncthreads();                             // every wave has asked for its pages before the first keys fill the way to memory
    if (busy) {
        for (uint32_t at = wbegin;;) {
            const uint32_t stop = g.seg1 < wend ? g.seg1 : wend;
            Running<D> st;
            st.clear();
            if (hi > 0) {
                const auto page_of = [&](int (&pg)[2], int i) {
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const int p = __builtin_amdgcn_readlane(pages, 2 * (i & 31) + z);
                        pg[z] = (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
                    }
                };
                int pg[2];
                page_of(pg, 0);
                Keys<D, FMT> k;
                load_keys<D, FMT>(k, a, h, pg, u0 * kUnit, true, lane);
                for (int u = u0; u < u1; ++u) {
                    Values<D, FMT> v;
                    load_values<D, FMT>(v, a, h, pg, u * kUnit, lane);
                    float x[8];
                    scores<D, FMT, SCORED>(x, k, q, a.scale);
                    if constexpr (SCORED) adjust(x, a, slope, (float)(hi - 1 - u * kUnit - 4 * quarter));
                    const int now[2] = {pg[0], pg[1]};
                    // the next unit's keys are on their way through this one's softmax and values
                    if (((u + 1 - u0) & 31) == 0) turn(u + 1);
                    page_of(pg, u + 1 - u0);
                    load_keys<D, FMT>(k, a, h, pg, (u + 1) * kUnit, u + 1 < u1, lane);
                    if (u * kUnit < lo || (u + 1) * kUnit > hi || now[0] < 0 || now[1] < 0) mask<D, FMT>(x, v, now, u * kUnit, lo, hi, lane);
                    take_in<D, FMT>(st, x, v);
                }
            }
            const float l = sum4(st.l);
            if (at == g.seg0 && stop == g.seg1) {        // all of the segment is here
                if (n < to.queries) {
                    const float inv = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
                    _Float16 *o = to.o(a, g.b, D) + n * D + quarter * 4 * R;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (R == 4) {
                            half4v y = {(_Float16)(st.acc[0][i] * inv), (_Float16)(st.acc[1][i] * inv), (_Float16)(st.acc[2][i] * inv), (_Float16)(st.acc[3][i] * inv)};
                            *(half4v *)(o + i * R) = y;
                        } else {
#pragma unroll
                            for (int r = 0; r < R; r += 8) {
                                half8v y;
#pragma unroll
                                for (int e = 0; e < 8; ++e) y[e] = (_Float16)(st.acc[r + e][i] * inv);
                                *(half8v *)(o + i * R + r) = y;
                            }
                        }
                    }
                    if (a.lse && quarter == 0) to.lse(a, g.b)[n] = lse_of(st.m, l);
                }
            } else {
                const int slot = 2 * wave + (g.seg0 >= wbegin);          // the segment that goes on from before, or the one that goes on after
                if (lane == 0) s_seg[wave][g.seg0 >= wbegin] = g;
                if (quarter == 0) { s_m[slot * kQueries + n] = st.m; s_l[slot * kQueries + n] = l; }
                if (n < to.queries) {
                    float *o = s_o + (slot * rows + n) * kRow + quarter * 4 * R;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int r = 0; r < R; r += 4) *(F4 *)(o + i * R + r) = F4{st.acc[r][i], st.acc[r + 1][i], st.acc[r + 2][i], st.acc[r + 3][i]};
                }
            }
            at = stop;
            if (at >= wend) break;
            locate(at);
        }
    }
    __syncthreads();

    // Lane 2 w + z has what slot z of wave w holds.  A chain is a segment's slots in this block: one that goes on after its wave
    // began it, or wave 0's from before, and the first slots of the waves behind.  The chains are dealt to teams of waves, a
    // thread for every item of a chain.
    const __amdgpu_buffer_rsrc_t parts = attn_rsrc(a.partial, 2 * kAttnBlocks * part_floats<D>() * 4);
    const Segment held = s_seg[lane / 2 % WAVES][lane & 1];
    const bool there = lane < 2 * WAVES && held.seg1 != 0;
    const uint32_t starts = (uint32_t)__ballot(there && (lane & 1 || lane == 0));
    const int team_waves = rows * (D / 4) <= 64 ? 1 : rows * (D / 4) <= 128 ? 2 : rows * (D / 4) <= 256 ? 4 : 8;
    const int teams = WAVES >= team_waves ? WAVES / team_waves : 1, team = wave / team_waves;
    int turn_of = 0;
    for (uint32_t left = starts; left; left &= left - 1) {
        if (turn_of++ % teams != team) continue;
        const int slot0 = __builtin_ctz(left);
        const Segment g = held.of_lane(slot0);
        const uint32_t behind = (uint32_t)__ballot(there && !(lane & 1) && lane > slot0 && held.seg0 == g.seg0);
        const int links = 1 + __builtin_popcount(behind);
        const Target to(a, g.seg);
        const bool whole = g.seg0 >= begin && g.seg1 <= end;
        for (int i = tid - team * team_waves * 64; i < to.queries * (D / 4); i += team_waves * 64 < THREADS ? team_waves * 64 : THREADS) {
            const int query = i / (D / 4), channel = (i % (D / 4)) * 4;
            Four x;
            x.clear();
            for (int k0 = 0; k0 < links; k0 += 4)
                x.add<4>([&](int k, float &m, float &l, F4 &v) {
                    // past the last link: the first one again, with no weight
                    const bool on = k0 + k < links;
                    const int slot = on && k0 + k ? (slot0 & ~1) + 2 * (k0 + k) : slot0;
                    m = s_m[slot * kQueries + query];
                    m = on ? m : -INFINITY;
                    l = s_l[slot * kQueries + query];
                    v = *(const F4 *)(s_o + (slot * rows + query) * kRow + channel);
                });
            if (whole) x.result(a, to, g.b, D, query, channel);
            else store_part<D>(parts, 2 * blockIdx.x + (g.seg0 >= begin), query, channel, x);
        }
    }
    if (!starts) return;

    // Segments shared with other blocks: the one from before this block and the one that goes on after it.
    const Segment from = held.of_lane(__builtin_ctz(starts)), on = held.of_lane(31 - __builtin_clz(starts));
    const bool from_before = from.seg0 < begin, goes_on = on.seg0 >= begin && on.seg1 > end;
    if (!from_before && !goes_on) return;
    stores_done();
    __syncthreads();
    if (tid == 0 ? from_before : tid == 64 && goes_on) {
        const Segment g = wave == 0 ? from : on;
        const Sharers by(g, share, per_share, blockIdx.x);
        uint32_t *counter = by.in_groups ? a.arrived + 2 * by.group + (g.seg0 >= by.group * share) : a.arrived + 2 * kAttnBlocks + (size_t)g.b * hc + g.seg;
        s_last[wave] = arrives_last(counter, by.in_groups ? by.group_last - by.group + 1 : by.last - by.first + 1);
    }
    __syncthreads();

    // those whose last share has now arrived
    for (int z = 0; z < 2; ++z) {
        if (!__builtin_amdgcn_readfirstlane(s_last[z])) continue;
        const Segment g = z == 0 ? from : on;
        const Target to(a, g.seg);
        const Sharers by(g, share, per_share, blockIdx.x);
        const int items = to.queries * (D / 4);
        bool final = !by.in_groups;
        if (by.in_groups) {                      // the group's result takes the place of its first part
            for (int i0 = 0; i0 < items; i0 += THREADS) {
                const int some = items - i0 < THREADS ? items - i0 : THREADS;
                const Four x = join_parts<D, THREADS>(parts, s_o, g, share, by.group, 1, by.group_last, i0, some, tid);
                if (tid < some) store_part<D>(parts, 2 * by.group + (g.seg0 >= by.group * share), (i0 + tid) / (D / 4), ((i0 + tid) % (D / 4)) * 4, x);
            }
            stores_done();
            __syncthreads();
            if (tid == 0) s_last[z] = arrives_last(a.arrived + 2 * kAttnBlocks + (size_t)g.b * hc + g.seg, (by.last - by.first) / kGroupParts + 1);
            __syncthreads();
            final = __builtin_amdgcn_readfirstlane(s_last[z]);
        }
        if (final)
            for (int i0 = 0; i0 < items; i0 += THREADS) {
                const int some = items - i0 < THREADS ? items - i0 : THREADS;
                const Four x = join_parts<D, THREADS>(parts, s_o, g, share, by.first, by.in_groups ? kGroupParts : 1, by.last, i0, some, tid);
                if (tid < some) x.result(a, to, g.b, D, (i0 + tid) / (D / 4), ((i0 + tid) % (D / 4)) * 4);
            }
    }
}

static int attn_chunks(const paro_kv_cache &c, int q_heads) { return (q_heads / c.kv_heads + kQueries - 1) / kQueries; }
static size_t attn_part_bytes(const paro_kv_cache &c) { return sizeof(float) * kQueries * (c.head_dim + 4); }
static size_t attn_scratch_bytes(const paro_kv_cache &c) { return ((size_t)2 * kAttnBlocks * attn_part_bytes(c) + 255) / 256 * 256; }

// Most units of a head whose sequence has up to `tokens` tokens, of which `window` (0: all) are attended to.
static constexpr int64_t units_seen(int64_t tokens, int32_t window)
{
    const int64_t within = (int64_t)window + 2 * kUnit;
    return ((window > 0 && within < tokens ? within : tokens) + kUnit - 1) / kUnit;
}
static_assert(units_seen(4096, INT32_MAX) == 128 && units_seen(4096, 0) == 128 && units_seen(4096, 1) == 3 && units_seen(1, 1) == 1,
              "any window that an int32 holds");

template <int D, int FMT, bool SCORED>
static hipError_t launch_attention(AttnArgs &a, int64_t units, hipStream_t s)
{
    constexpr int WAVES = attn_waves<D>();
    // no more blocks than the longest sequences could have units for, and a single one's heads blocks of their own
    int64_t most = (units + kLeastUnits - 1) / kLeastUnits;
    const int64_t heads = (int64_t)a.kv_heads * a.chunks;
    if (const int64_t apart = heads * one_parts((uint32_t)(units / heads), WAVES); a.batch == 1 && most < apart) most = apart;
    const unsigned blocks = (unsigned)(most < kAttnBlocks ? most : kAttnBlocks);
    a.per_block = 1.0f / (float)blocks;
    const int rows = a.group < kQueries ? a.group : kQueries;
    const size_t shares = sizeof(float) * WAVES * 2 * rows * (D + 4), joins = sizeof(float) * 6 * 64 * WAVES;
    static std::atomic<uint64_t> attr_done{0};
    if (const int dev = once_pending(attr_done); dev >= 0) {
        const hipError_t e = hipFuncSetAttribute((const void *)paged_attention_kernel<D, FMT, SCORED>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)(sizeof(float) * WAVES * 2 * kQueries * (D + 4)));
        if (e != hipSuccess) return e;
        once_done(attr_done, dev);
    }
    hipLaunchKernelGGL((paged_attention_kernel<D, FMT, SCORED>), dim3(blocks), dim3(64 * WAVES),
                       shares > joins ? shares : joins, s, a);
    return hipGetLastError();
}

template <int FMT, bool SCORED>
static hipError_t launch_attention(int head_dim, AttnArgs &a, int64_t units, hipStream_t s)
{
    return head_dim == 64 ? launch_attention<64, FMT, SCORED>(a, units, s) : head_dim == 128 ? launch_attention<128, FMT, SCORED>(a, units, s) :
                                                                                             launch_attention<256, FMT, SCORED>(a, units, s);
}

}  // namespace paro

extern "C" size_t paro_workspace_exchange_bytes_attention(const paro_kv_cache *cache, int32_t q_heads, int32_t batch)
{
    using namespace paro;
    if (!cache || cache->kv_heads <= 0 || q_heads <= 0 || q_heads % cache->kv_heads || batch <= 0) return 0;
    const size_t counters = (2 * kAttnBlocks + (size_t)batch * cache->kv_heads * attn_chunks(*cache, q_heads)) * sizeof(uint32_t);
    return kWsPartialOff + (counters + 255) / 256 * 256;
}

extern "C" size_t paro_workspace_bytes_attention(const paro_kv_cache *cache, int32_t q_heads, int32_t batch)
{
    const size_t e = paro_workspace_exchange_bytes_attention(cache, q_heads, batch);
    return e && cache->head_dim > 0 ? e + paro::attn_scratch_bytes(*cache) : 0;
}

extern "C" paro_status paro_paged_attention(const paro_kv_cache *cache, const paro_half_t *Q, int64_t ldq, int32_t q_heads,
                                            const int32_t *block_table, int64_t ld_table, int32_t table_width,
                                            const int32_t *lengths, int32_t batch, float scale, int32_t window,
                                            paro_half_t *O, int64_t ldo, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    return paro_paged_attention_scored(cache, Q, ldq, q_heads, block_table, ld_table, table_width, lengths, batch, scale, window, nullptr, O, ldo, lse, ws,
                                       ws_bytes, stream);
}

extern "C" paro_status paro_paged_attention_scored(const paro_kv_cache *cache, const paro_half_t *Q, int64_t ldq, int32_t q_heads,
                                                   const int32_t *block_table, int64_t ld_table, int32_t table_width,
                                                   const int32_t *lengths, int32_t batch, float scale, int32_t window,
                                                   const paro_scores_t *scores, paro_half_t *O, int64_t ldo, float *lse, void *ws,
                                                   size_t ws_bytes, void *stream)
{
    using namespace paro;
    if (const paro_status st = check_cache(cache); st != PARO_OK) return st;
    if (!Q || !O || !block_table || !lengths) return PARO_ERR_NULL;
    const paro_kv_cache &c = *cache;
    if (batch <= 0 || q_heads <= 0 || q_heads % c.kv_heads || table_width <= 0 || window < 0) return PARO_ERR_SHAPE;
    if ((ld_table != 0 && ld_table < table_width) || O == Q) return PARO_ERR_SHAPE;
    AttnArgs a;
    if (const paro_status st = check_scores(scores, scale, a.scores); st != PARO_OK) return st;
    if (const paro_status st = check_rows(Q, ldq, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (const paro_status st = check_rows(O, ldo, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (!aligned(block_table, 4) || !aligned(lengths, 4) || (lse && !aligned(lse, 4))) return PARO_ERR_ALIGN;
    // units are numbered with 32 bits, and so are a sequence's tokens
    const int64_t tokens = (int64_t)table_width * c.page;
    if (q_heads > 65535) return PARO_ERR_UNSUPPORTED;
    const int64_t units = (int64_t)batch * c.kv_heads * attn_chunks(c, q_heads);
    if (tokens > (int64_t)1 << 30 || units > (int64_t)1 << 30 || units * ((tokens + kUnit - 1) / kUnit) > (int64_t)1 << 30) return PARO_ERR_UNSUPPORTED;
    const size_t scratch = attn_scratch_bytes(c);
    if (!ws || ws_bytes < paro_workspace_bytes_attention(cache, q_heads, batch)) return PARO_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return PARO_ERR_ALIGN;

    a.k = (const uint8_t *)c.k; a.v = (const uint8_t *)c.v; a.ks = c.k_scale; a.vs = c.v_scale;
    a.q = (const _Float16 *)Q; a.table = block_table; a.lengths = lengths; a.o = (_Float16 *)O; a.lse = lse;
    a.arrived = (uint32_t *)((char *)ws + kWsPartialOff);
    a.partial = (float *)((char *)ws + (ws_bytes & ~(size_t)255) - scratch);
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.page_log = log2_of(c.page); a.n_pages = c.n_pages; a.kv_heads = c.kv_heads; a.group = q_heads / c.kv_heads;
    a.chunks = attn_chunks(c, q_heads); a.width = table_width; a.batch = batch; a.window = window;
    a.scale = scale * kLog2e;
    const int64_t most = units * units_seen(tokens, window);
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    const bool scored = a.scores.cap > 0 || a.scores.slopes;
    switch (2 * kernel_format(c.format) + scored) {
    case 0: e = launch_attention<kFp16, false>(c.head_dim, a, most, s); break;
    case 1: e = launch_attention<kFp16, true>(c.head_dim, a, most, s); break;
    case 2: e = launch_attention<kE4m3, false>(c.head_dim, a, most, s); break;
    case 3: e = launch_attention<kE4m3, true>(c.head_dim, a, most, s); break;
    case 4: e = launch_attention<kMxfp4, false>(c.head_dim, a, most, s); break;
    default: e = launch_attention<kMxfp4, true>(c.head_dim, a, most, s); break;
    }
    return e == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}
