// Attention of many new tokens of every sequence over a paged key-value cache:
//
//      o_i = sum_t p_t v_t / sum_t p_t,   p_t = 2^(x_t - m),   x_t = log2(e) scale q_i . k_t,   lo_i <= t < hi_i
//
// A row at position p sees an interval of tokens: [p - window + 1, p], cut at first, stretched to prefix.  Bound by the matrix
// cores for long prompts (4 head_dim flops per row, head and token), by HBM for a few rows of a long sequence.
//
// A block has 128 pairs (row, query head) of one key-value head, numbered row by row, so that a head's keys and values are read once
// for all of its query heads, and walks its tokens in tiles of 64: keys and values go through LDS as fp16 (whatever the cache
// holds), two tiles deep, each wave of the block filling a quarter and using all for its 32 pairs.  A wave computes S^T = K Q^T by
// 32 x 32 x 16 products: a lane then has scores of one pair only, half of a tile's, so that the softmax's maximum and sum need one
// exchange between two lanes, and S^T's registers are the B operand of O^T = V^T P^T as they are, if that product takes the tokens of a step
// in the order 4 (lane/32) + (0..3), then 8 more; values are read from LDS transposed in that order.  The cache's order of keys (16-byte units
// that interleave the tokens) is the first product's operand order: LDS keeps it, and no access has bank conflicts.
//
// p enters the second product as fp16 after a factor of 2^kShift (16 bits would otherwise end at 2^-24 of the maximum): each is off by
// 2^-12 of itself on average, independently, which adds about as much to a result as its own rounding to fp16.  Sums stay in fp32.
//
// Few tiles with long sequences: `splits` blocks share a tile's tokens; each leaves fp32 results in the scratch, and the one that arrives
// last joins all in their order, so that results do not depend on timing.  Nobody waits.
#include "kv_common.h"

namespace paro {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef float F16 __attribute__((ext_vector_type(16)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint32_t U2 __attribute__((ext_vector_type(2)));

constexpr int kPairs = 32;                       // of a wave: the N of the matrix instruction
constexpr int kWaves = 4, kTilePairs = kWaves * kPairs;
constexpr int kTokens = 64;                      // of a tile of keys and values
constexpr int kPromptThreads = 64 * kWaves;
constexpr int kMaxSplits = 32;
constexpr int kSplitBlocks = 512;                // splits make this many blocks, two for every compute unit
constexpr int kLeastTiles = 4;                   // tiles of tokens that a split has at least
constexpr float kShift = 10.0f;                  // p is held 2^10 times
constexpr float kFarMax = 65536.0f;              // |maximum| above which scores are rounded before it is taken off
constexpr int kPromptRaw = 0x00020000;           // raw buffer, 32-bit data format
constexpr int kPromptAgent = 16;                 // agent scope: past the L2 of the XCD

struct PromptArgs {
    const uint8_t *k, *v, *ks, *vs;
    const _Float16 *q;
    const int32_t *starts, *table, *lengths, *prefix, *first;
    _Float16 *o;
    float *lse;
    uint32_t *arrived;                           // [tiles][kv_heads]
    float *partial;                              // [tiles][kv_heads][splits] of part_floats
    int64_t ldq, ldo, ld_table;
    int page_log, n_pages, kv_heads, group, width, batch, window, T, tiles, splits;
    float scale;                                 // with log2(e)
    Scores scores;
};

template <int D> constexpr size_t prompt_part_floats() { return (size_t)kTilePairs * (D + 2); }

// Sums over lanes 0..lane.
__device__ inline int prompt_sums_upto(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);        // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);        // row_bcast 15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);        // row_bcast 31 into rows 2 and 3
    return x;
}
// Over the lanes n and n ^ 32, which hold one pair.
__device__ inline float max2(float x)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ inline float sum2(float x)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// A tile of pairs: of sequence b, whose rows are row0 .. row0 + rows - 1 and whose tokens are 0 .. n - 1; the tile's first pair.
struct Where { int b, row0, rows, n, pair0; };

// Tile `tile` of all sequences' tiles; false: there are fewer.  starts are taken as they come, within 0..T and not falling.
__device__ inline bool find_tile(Where &w, const PromptArgs &a, int tile, int lane)
{
    int before = 0;                              // tiles of the sequences seen
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int b = b0 + lane < a.batch ? b0 + lane : a.batch - 1;
        int s0 = a.starts[b], s1 = a.starts[b + 1];
        s0 = s0 < 0 ? 0 : s0 > a.T ? a.T : s0;
        s1 = s1 < s0 ? s0 : s1 > a.T ? a.T : s1;
        const int tiles = b0 + lane < a.batch ? (int)(((int64_t)(s1 - s0) * a.group + kTilePairs - 1) / kTilePairs) : 0;
        const int upto = prompt_sums_upto(tiles);
        const uint64_t behind = __ballot(before + upto > tile);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            w.b = b0 + at;
            w.row0 = __builtin_amdgcn_readlane(s0, at);
            w.rows = __builtin_amdgcn_readlane(s1, at) - w.row0;
            w.pair0 = (tile - before - __builtin_amdgcn_readlane(upto, at) + __builtin_amdgcn_readlane(tiles, at)) * kTilePairs;
            const int room = a.width << a.page_log, n = __builtin_amdgcn_readfirstlane(a.lengths[w.b]);
            w.n = n < 0 ? 0 : n > room ? room : n;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

__device__ inline __amdgpu_buffer_rsrc_t prompt_rsrc(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, kPromptRaw);
}

// How a wave moves the 16 tokens of its quarter of a tile: `Loads` requests of `Bytes` a lane, `Channels` channels each.
template <int D, int FMT>
struct Move {
    static constexpr int Bytes = row_bytes<FMT>(D) * 16 / 64 < 16 ? row_bytes<FMT>(D) * 16 / 64 : 16;
    static constexpr int Loads = row_bytes<FMT>(D) * 16 / 64 / Bytes;
    static constexpr int Channels = D / 4 / Loads;
    static constexpr int Words = Bytes / 4;
};
template <int D, int FMT>
struct Staged {
    U4 k[Move<D, FMT>::Loads], v[Move<D, FMT>::Loads];
    uint32_t ks[Move<D, FMT>::Loads], vs[Move<D, FMT>::Loads];   // scale bytes; E4M3 keys: ks[0]
    int t0;                                      // first of the 16 tokens
};
template <int BYTES>
__device__ inline U4 prompt_load(__amdgpu_buffer_rsrc_t r, int off, int base)
{
    if constexpr (BYTES == 16) return __builtin_bit_cast(U4, __builtin_amdgcn_raw_buffer_load_b128(r, off, base, 0));
    const U2 y = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(r, off, base, 0));
    return U4{y[0], y[1], 0, 0};
}

// Asks for 16 tokens from t0 on (a multiple of 16) of page `page`; one that is not there gives zeros.
template <int D, int FMT>
__device__ inline void ask(Staged<D, FMT> &x, const PromptArgs &a, int head, int page, int t0, int lane)
{
    typedef Move<D, FMT> M;
    const bool there = (uint32_t)page < (uint32_t)a.n_pages;
    const int64_t place = ((int64_t)(there ? page : 0) * a.kv_heads + head) << a.page_log;       // the page's first token
    const int tok = t0 & ((1 << a.page_log) - 1);
    const uint32_t bytes = there ? (uint32_t)row_bytes<FMT>(D) << a.page_log : 0;
    const __amdgpu_buffer_rsrc_t rk = prompt_rsrc(a.k + place * row_bytes<FMT>(D), bytes), rv = prompt_rsrc(a.v + place * row_bytes<FMT>(D), bytes);
    x.t0 = t0;
#pragma unroll
    for (int i = 0; i < M::Loads; ++i) {
        // keys: token lane % 16, run of channels lane / 16 + 4 i (8-byte runs: two to a unit)
        const int run = (lane >> 4) + 4 * i, unit = M::Bytes == 16 ? run : run >> 1;
        x.k[i] = prompt_load<M::Bytes>(rk, (((unit << a.page_log) + (lane & 15)) << 4) + (M::Bytes == 16 ? 0 : (run & 1) * 8), tok << 4);
        x.v[i] = prompt_load<M::Bytes>(rv, (lane + 64 * i) * M::Bytes, tok * row_bytes<FMT>(D));
    }
    if constexpr (FMT != kFp16) {
        constexpr int S = row_scales<FMT>(D);
        const uint32_t some = there ? (uint32_t)S << a.page_log : 0;
        const __amdgpu_buffer_rsrc_t qk = prompt_rsrc(a.ks + place * S, some), qv = prompt_rsrc(a.vs + place * S, some);
#pragma unroll
        for (int i = 0; i < M::Loads; ++i) {
            const int t = (lane + 64 * i) * M::Channels / D, c = (lane + 64 * i) * M::Channels % D;
            if (FMT == kMxfp4 || i == 0)
                x.ks[i] = __builtin_amdgcn_raw_buffer_load_b8(qk, ((FMT == kMxfp4 ? ((lane >> 4) + 4 * i) * M::Channels / 32 : 0) << a.page_log) + (lane & 15), tok, 0);
            x.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(qv, ((FMT == kMxfp4 ? c / 32 : 0) << a.page_log) + t, tok, 0);
        }
    }
}

// The channels of request i as fp16, 8 at a time.
template <int D, int FMT>
__device__ inline half8v eight(U4 x, uint32_t scale, int z)
{
    const float up = __uint_as_float(scale << 23);
    if constexpr (FMT == kFp16) return __builtin_bit_cast(half8v, x);
    if constexpr (FMT == kMxfp4) return f16_of_e2m1(x[z], up);
    const uint32_t lo = x[2 * z], hi = x[2 * z + 1];
    const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, up, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, up, true);
    const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, up, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, up, true);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ inline bool any_not_finite(half8v x)
{
    const U4 u = __builtin_bit_cast(U4, x);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (u[i] & 0x7c00u) == 0x7c00u || (u[i] & 0x7c000000u) == 0x7c000000u;
    return bad;
}

// LDS: keys [head_dim/8][64 tokens] of 16 bytes; values [64 tokens][head_dim] in blocks of 32 channels whose order in a row depends on
// the row, so that the transposed reads of 4 rows at once fall on distinct banks.
template <int D> __device__ inline int value_block(int t, int block) { return D == 64 ? block ^ ((t >> 1) & 1) : block ^ (t & 3); }
template <int D> __device__ inline int value_at(int t, int c) { return t * 2 * D + value_block<D>(t, c >> 5) * 64 + (c & 31) * 2; }
template <int D> constexpr int kTileBytes = kTokens * D * 2;         // of keys, and of values

// Puts the 16 tokens where the products read them.  Values of tokens past `end` are zeros (such places may hold NaN); true if `look` and a
// value is not finite.
template <int D, int FMT>
__device__ inline bool put(const Staged<D, FMT> &x, uint8_t *keys, uint8_t *values, int quarter, int end, bool look, int lane)
{
    typedef Move<D, FMT> M;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < M::Loads; ++i) {
        const int kc = ((lane >> 4) + 4 * i) * M::Channels, vt = (lane + 64 * i) * M::Channels / D, vc = (lane + 64 * i) * M::Channels % D;
#pragma unroll
        for (int z = 0; z < M::Channels / 8; ++z) {
            *(half8v *)(keys + ((kc / 8 + z) * kTokens + quarter * 16 + (lane & 15)) * 16) = eight<D, FMT>(x.k[i], FMT == kE4m3 ? x.ks[0] : x.ks[i], z);
            half8v y = eight<D, FMT>(x.v[i], x.vs[i], z);
            if (look) {
                if (x.t0 + vt >= end) y = half8v{};
                bad |= any_not_finite(y);
            }
            *(half8v *)(values + value_at<D>(quarter * 16 + vt, vc + 8 * z)) = y;
        }
    }
    return bad;
}

typedef __fp16 Tr4 __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) Tr4 LdsTr4;

template <int D, int FMT, bool SCORED>
__global__ __launch_bounds__(kPromptThreads, D == 256 ? 1 : 2) void prompt_attention_kernel(const PromptArgs a)
{
    constexpr int R = D / 32, KS = D / 16;       // channel tiles of the result, steps of the first product
    extern __shared__ __attribute__((aligned(16))) uint8_t s_tiles[];        // [2] of keys and values
    __shared__ int s_lo[kWaves][2], s_hi[kWaves][2];
    __shared__ int s_bad[2];                     // 1 + the tile in this half that has values that are not finite, where not all see them
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, n32 = lane & 31;

    // longest tiles first; the heads of a tile side by side, which puts a head on one XCD where there are 8 of them
    const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % a.splits, tile = a.tiles - 1 - rest / a.splits;
    Where w;
    if (!find_tile(w, a, tile, lane)) return;
    const int pairs = w.rows * a.group;

    // this lane's pair and what it sees
    const int pair = w.pair0 + wave * kPairs + n32, kept = pair < pairs ? pair : pairs - 1;
    const int row = kept / a.group, qhead = head * a.group + kept - row * a.group;
    const int pos = w.n - w.rows + row;
    int lo = 0, hi = pos + 1;
    if (a.window) lo = pos - a.window + 1;
    if (a.first) { const int f = a.first[w.row0 + row]; lo = lo > f ? lo : f; }
    if (a.prefix) { int f = a.prefix[w.b]; f = f < w.n ? f : w.n; hi = hi > f ? hi : f; }
    lo = lo > 0 ? lo : 0;
    const bool some = lo < hi;
    // of the wave: the least and largest lo and hi
    int least = some ? lo : INT32_MAX, most = some ? hi : 0;
    int lo_most = some ? lo : INT32_MAX, hi_least = some ? hi : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        least = min(least, __shfl_xor(least, d)); most = max(most, __shfl_xor(most, d));
        lo_most = max(lo_most, __shfl_xor(lo_most, d)); hi_least = min(hi_least, __shfl_xor(hi_least, d));
    }
    least = __builtin_amdgcn_readfirstlane(least); most = __builtin_amdgcn_readfirstlane(most);
    lo_most = __builtin_amdgcn_readfirstlane(lo_most); hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    if (lane == 0) { s_lo[wave][0] = least; s_lo[wave][1] = lo_most; s_hi[wave][0] = most; s_hi[wave][1] = hi_least; }
    if (tid < 2) s_bad[tid] = 0;

    // queries: channels 16 s + 8 h .. of pair n32.  A negative scale goes into their sign, a scale of 0 makes them 0: factors of maxima are positive.
    half8v q[KS];
    {
        const _Float16 *qp = a.q + (int64_t)(w.row0 + row) * a.ldq + (int64_t)qhead * D + 8 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = *(const half8v *)(qp + 16 * s);
            if constexpr (!SCORED) {
                if (a.scale < 0) q[s] = -q[s];
                if (a.scale == 0) q[s] *= (_Float16)0;
            }
        }
    }
    const float scale = SCORED ? 1.0f : a.scale == 0 ? 1.0f : fabsf(a.scale);
    float slope = 0;
    if constexpr (SCORED) if (a.scores.slopes) slope = a.scores.slopes[qhead] * kLog2e;
    __syncthreads();
    int begin = s_lo[0][0], end = s_hi[0][0], whole_lo = s_lo[0][1], whole_hi = s_hi[0][1];      // of the block
#pragma unroll
    for (int i = 1; i < kWaves; ++i) {
        begin = min(begin, s_lo[i][0]); end = max(end, s_hi[i][0]);
        whole_lo = max(whole_lo, s_lo[i][1]); whole_hi = min(whole_hi, s_hi[i][1]);
    }
    begin = __builtin_amdgcn_readfirstlane(begin); end = __builtin_amdgcn_readfirstlane(end);
    whole_lo = __builtin_amdgcn_readfirstlane(whole_lo); whole_hi = __builtin_amdgcn_readfirstlane(whole_hi);
    // tiles of tokens, and this split's share of them
    const int tile0 = begin < end ? begin / kTokens : 0, tiles = begin < end ? (end + kTokens - 1) / kTokens - tile0 : 0;
    int parts = tiles / kLeastTiles;
    parts = parts < 1 ? 1 : parts > a.splits ? a.splits : parts;
    if (split >= parts) return;
    const int per = (tiles + parts - 1) / parts;
    const int u0 = tile0 + split * per, u1 = min(u0 + per, tile0 + tiles);       // u0 may lie past u1: an empty share

    F16 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[r][j] = 0;
    float m = -INFINITY, l = 0;                  // of the pair; l over this lane's tokens only

    const int32_t *table = a.table + (int64_t)w.b * a.ld_table;
    // the page of this wave's quarter of tile u; -1 past the end
    const auto page_of = [&](int u) {
        const int t = u * kTokens + wave * 16;
        return t < end && u < u1 ? __builtin_amdgcn_readfirstlane(table[t >> a.page_log]) : -1;
    };
    // a tile that some pair does not see all of, or that has a page missing, which its quarter alone knows
    const auto at_edge = [&](int u) { return u * kTokens < whole_lo || (u + 1) * kTokens > whole_hi; };
    __shared__ int s_gone[2][kWaves];            // 1: the quarter's page is not there
    Staged<D, FMT> x;
    const auto fill = [&](int u, int page) {
        uint8_t *to = s_tiles + (u & 1) * 2 * kTileBytes<D>;
        const bool bad = put<D, FMT>(x, to, to + kTileBytes<D>, wave, end, at_edge(u), lane);
        if (at_edge(u) && __ballot(bad) && lane == 0) s_bad[u & 1] = u + 1;
        if (lane == 0) s_gone[u & 1][wave] = (uint32_t)page >= (uint32_t)a.n_pages;
    };
    int page = page_of(u0), next_page = page_of(u0 + 1);
    if (u0 < u1) {
        ask<D, FMT>(x, a, head, page, u0 * kTokens + wave * 16, lane);
        fill(u0, page);
        page = next_page;
        ask<D, FMT>(x, a, head, page, (u0 + 1) * kTokens + wave * 16, lane);
        next_page = page_of(u0 + 2);
    }
    __syncthreads();
    for (int u = u0; u < u1; ++u) {
        if (u + 1 < u1) {
            fill(u + 1, page);
            page = next_page;
            ask<D, FMT>(x, a, head, page, (u + 2) * kTokens + wave * 16, lane);
            next_page = page_of(u + 3);
        }
        uint8_t *keys = s_tiles + (u & 1) * 2 * kTileBytes<D>, *values = keys + kTileBytes<D>;
        const int t0 = u * kTokens;
        int gone = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) gone |= s_gone[u & 1][i] << i;
        gone = __builtin_amdgcn_readfirstlane(gone);
        if (__builtin_amdgcn_readfirstlane(s_bad[u & 1]) == u + 1) {
            // Values that are not finite, where some pair does not see them: a weight of 0 would not keep them out of the product.  Those that do see
            // them take them here (their results are not finite, whatever the weight is); then zeros take their place.
            for (int t = t0; t < t0 + kTokens && t < end; ++t) {
                const bool seen = t >= lo && t < hi;
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float y = (float)*(const _Float16 *)(values + value_at<D>(t - t0, 32 * r + 8 * (j >> 2) + 4 * h + (j & 3)));
                        if (seen && !is_finite(y)) acc[r][j] += y;
                    }
            }
            __syncthreads();
            for (int i = tid; i < kTileBytes<D> / 16; i += kPromptThreads) {
                half8v y = *(half8v *)(values + 16 * i);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = is_finite((float)y[e]) ? y[e] : (_Float16)0;
                *(half8v *)(values + 16 * i) = y;
            }
            __syncthreads();
        }
        if (t0 < most && t0 + kTokens > least) {
            float s[2][16];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                F16 z;
#pragma unroll
                for (int j = 0; j < 16; ++j) z[j] = 0;
#pragma unroll
                for (int i = 0; i < KS; ++i)
                    z = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(const half8v *)(keys + ((2 * i + h) * kTokens + 32 * b + n32) * 16), q[i], z, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] = z[j];
            }
            if constexpr (SCORED) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    if (a.scores.cap > 0) {
                        capped(s[b], a.scores);
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[b][j] *= a.scale;
                    }
                    if (a.scores.slopes) {
                        const float away = (float)(pos - t0 - 4 * h - 32 * b);
#pragma unroll
                        for (int j = 0; j < 16; ++j) s[b][j] = fmaf(-slope, fabsf(away - (8 * (j >> 2) + (j & 3))), s[b][j]);
                    }
                }
            }
            // token 32 b + 8 (j / 4) + 4 h + j % 4 of the tile
            if (t0 < lo_most || t0 + kTokens > hi_least || gone) {
                const int from = lo - t0 - 4 * h, to = hi - t0 - 4 * h;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int t = 32 * b + 8 * (j >> 2) + (j & 3);
                        const bool in = t >= from && t < to && !((gone >> (2 * b + (j >> 3))) & 1);
                        s[b][j] = in ? s[b][j] : -INFINITY;
                    }
            }
            float top = s[0][0];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) top = fmaxf(top, s[b][j]);
            top = fmaxf(m, max2(top) * scale);
            if (__ballot(top > m)) {
                const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
                l *= f;
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[r][j] *= f;
                m = top;
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            if (__ballot(fabsf(ref) > kFarMax)) {
                // product and difference as one would be off by up to half a unit of the maximum here, and p has to stay within fp16
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float y = s[b][j] * scale;
                        s[b][j] = __builtin_amdgcn_exp2f((y - ref) + kShift);
                        l += s[b][j];
                    }
            } else {
                const float off = kShift - ref;
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        s[b][j] = __builtin_amdgcn_exp2f(fmaf(s[b][j], scale, off));
                        l += s[b][j];
                    }
            }
            // O^T += V^T P^T, 16 tokens a step
            const int l16 = lane & 15;
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                half8v p;
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = (_Float16)s[st >> 1][8 * (st & 1) + e];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int t = 16 * st + 4 * h + (l16 >> 2), c = 32 * r + 16 * ((lane >> 4) & 1) + 4 * (l16 & 3);
                    const Tr4 one = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsTr4 *)(values + value_at<D>(t, c)));
                    const Tr4 two = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsTr4 *)(values + value_at<D>(t + 8, c)));
                    half8v f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) { f[e] = (_Float16)one[e]; f[4 + e] = (_Float16)two[e]; }
                    acc[r] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, p, acc[r], 0, 0, 0);
                }
            }
        }
        __syncthreads();
    }
    l = sum2(l);

    if (parts > 1) {
        // every part's m, l and sums where its lanes left them, through memory that all XCDs see
        const size_t tile_at = (size_t)(tile * a.kv_heads + head);
        const auto part_rsrc = [&](int p) { return prompt_rsrc(a.partial + (tile_at * a.splits + p) * prompt_part_floats<D>(), (uint32_t)(prompt_part_floats<D>() * 4)); };
        const int ml_at = (kTilePairs * D + 2 * (wave * kPairs + n32)) * 4;
        const auto sums_at = [&](int r, int i) { return (((wave * R + r) * 4 + i) * 64 + lane) * 16; };
        typedef decltype(__builtin_amdgcn_raw_buffer_load_b128(part_rsrc(0), 0, 0, 0)) B4;
        typedef decltype(__builtin_amdgcn_raw_buffer_load_b64(part_rsrc(0), 0, 0, 0)) B2;
        {
            const __amdgpu_buffer_rsrc_t to = part_rsrc(split);
            if (h == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(B2, U2{__float_as_uint(m), __float_as_uint(l)}), to, ml_at, 0, kPromptAgent);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(B4, F4{acc[r][4 * i], acc[r][4 * i + 1], acc[r][4 * i + 2], acc[r][4 * i + 3]}), to, sums_at(r, i), 0, kPromptAgent);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            uint32_t *counter = a.arrived + tile_at;
            const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)parts - 1;
            if (s_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!__builtin_amdgcn_readfirstlane(s_last)) return;
        float top = -INFINITY;
        for (int p = 0; p < parts; ++p) top = fmaxf(top, __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(part_rsrc(p), ml_at, 0, kPromptAgent)));
        const float ref = top == -INFINITY ? 0.0f : top;
        m = top;
        l = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][j] = 0;
        for (int p = 0; p < parts; ++p) {
            const __amdgpu_buffer_rsrc_t from = part_rsrc(p);
            const U2 ml = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(from, ml_at, 0, kPromptAgent));
            F4 y[R][4];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[r][i] = __builtin_bit_cast(F4, __builtin_amdgcn_raw_buffer_load_b128(from, sums_at(r, i), 0, kPromptAgent));
            const float f = __builtin_amdgcn_exp2f(__uint_as_float(ml[0]) - ref);
            l = fmaf(__uint_as_float(ml[1]), f, l);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][j] = fmaf(y[r][j >> 2][j & 3], f, acc[r][j]);
        }
    }

    if (pair < pairs) {
        const float inv = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
        _Float16 *o = a.o + (int64_t)(w.row0 + row) * a.ldo + (int64_t)qhead * D + 4 * h;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(half4v *)(o + 32 * r + 8 * i) = half4v{(_Float16)(acc[r][4 * i] * inv), (_Float16)(acc[r][4 * i + 1] * inv), (_Float16)(acc[r][4 * i + 2] * inv),
                                                       (_Float16)(acc[r][4 * i + 3] * inv)};
        if (a.lse && h == 0)
            a.lse[(int64_t)(w.row0 + row) * (a.kv_heads * a.group) + qhead] = l == 0.0f ? -INFINITY : (m - kShift + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// Tiles that T rows of `batch` sequences can have at most.
static int64_t prompt_tiles(int64_t T, int64_t group, int64_t batch)
{
    const int64_t all = T * group;
    return batch == 1 ? (all + kTilePairs - 1) / kTilePairs : all / kTilePairs + (batch < T ? batch : T);
}
// Blocks that share a tile: as many as make kSplitBlocks blocks.
static int64_t prompt_splits(int64_t tiles, int64_t kv_heads)
{
    const int64_t heads = tiles * kv_heads, n = (kSplitBlocks + heads - 1) / heads;
    return n < kMaxSplits ? n : kMaxSplits;
}

template <int D, int FMT, bool SCORED>
static hipError_t launch_prompt(const PromptArgs &a, hipStream_t s)
{
    constexpr int lds = 4 * kTileBytes<D>;
    static std::atomic<uint64_t> attr_done{0};
    if (const int dev = once_pending(attr_done); dev >= 0) {
        const hipError_t e = hipFuncSetAttribute((const void *)prompt_attention_kernel<D, FMT, SCORED>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        once_done(attr_done, dev);
    }
    hipLaunchKernelGGL((prompt_attention_kernel<D, FMT, SCORED>), dim3((unsigned)(a.tiles * a.kv_heads * a.splits)), dim3(kPromptThreads), lds, s, a);
    return hipGetLastError();
}
template <int FMT, bool SCORED>
static hipError_t launch_prompt(int head_dim, const PromptArgs &a, hipStream_t s)
{
    return head_dim == 64 ? launch_prompt<64, FMT, SCORED>(a, s) : head_dim == 128 ? launch_prompt<128, FMT, SCORED>(a, s) : launch_prompt<256, FMT, SCORED>(a, s);
}

// Scratch for the parts of any call of so many tiles or fewer (fewer tiles are split more often): heads * splits is below kSplitBlocks + heads.
static size_t prompt_scratch_bytes(const paro_kv_cache &c, int64_t tiles)
{
    const int64_t heads = tiles * c.kv_heads, parts = heads < 2 * kSplitBlocks / kMaxSplits ? heads * kMaxSplits : 2 * kSplitBlocks;
    return (sizeof(float) * kTilePairs * (c.head_dim + 2) * (size_t)parts + 255) / 256 * 256;
}

}  // namespace paro

extern "C" size_t paro_workspace_exchange_bytes_prompt(const paro_kv_cache *cache, int32_t q_heads, int32_t T, int32_t batch)
{
    using namespace paro;
    if (!cache || cache->kv_heads <= 0 || q_heads <= 0 || q_heads % cache->kv_heads || T <= 0 || batch <= 0) return 0;
    const size_t counters = (size_t)prompt_tiles(T, q_heads / cache->kv_heads, batch) * cache->kv_heads * sizeof(uint32_t);
    return kWsPartialOff + (counters + 255) / 256 * 256;
}

extern "C" size_t paro_workspace_bytes_prompt(const paro_kv_cache *cache, int32_t q_heads, int32_t T, int32_t batch)
{
    using namespace paro;
    const size_t e = paro_workspace_exchange_bytes_prompt(cache, q_heads, T, batch);
    return e && cache->head_dim > 0 ? e + prompt_scratch_bytes(*cache, prompt_tiles(T, q_heads / cache->kv_heads, batch)) : 0;
}

extern "C" paro_status paro_prompt_attention(const paro_kv_cache *cache, const paro_half_t *Q, int64_t ldq, int32_t q_heads, int32_t T,
                                             const int32_t *starts, const int32_t *block_table, int64_t ld_table, int32_t table_width,
                                             const int32_t *lengths, int32_t batch, float scale, int32_t window, const paro_scores_t *scores,
                                             const int32_t *prefix, const int32_t *first, paro_half_t *O, int64_t ldo, float *lse, void *ws,
                                             size_t ws_bytes, void *stream)
{
    using namespace paro;
    if (const paro_status st = check_cache(cache); st != PARO_OK) return st;
    if (!Q || !O || !starts || !block_table || !lengths) return PARO_ERR_NULL;
    const paro_kv_cache &c = *cache;
    if (T <= 0 || batch <= 0 || q_heads <= 0 || q_heads % c.kv_heads || table_width <= 0 || window < 0) return PARO_ERR_SHAPE;
    if ((ld_table != 0 && ld_table < table_width) || O == Q) return PARO_ERR_SHAPE;
    PromptArgs a;
    if (const paro_status st = check_scores(scores, scale, a.scores); st != PARO_OK) return st;
    if (const paro_status st = check_rows(Q, ldq, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (const paro_status st = check_rows(O, ldo, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (!aligned(starts, 4) || !aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(prefix, 4) || !aligned(first, 4) || !aligned(lse, 4)) return PARO_ERR_ALIGN;
    // a sequence's tokens and pairs, and the blocks of a launch, are numbered with 32 bits
    const int64_t tokens = (int64_t)table_width * c.page;
    if (q_heads > 65535 || tokens > (int64_t)1 << 30 || T > 1 << 24 || (int64_t)T * q_heads > (int64_t)1 << 30) return PARO_ERR_UNSUPPORTED;
    const int64_t tiles = prompt_tiles(T, q_heads / c.kv_heads, batch), splits = prompt_splits(tiles, c.kv_heads);
    if (tiles * c.kv_heads * splits > (int64_t)1 << 24) return PARO_ERR_UNSUPPORTED;       // a launch holds fewer than 2^32 threads
    if (!ws || ws_bytes < paro_workspace_bytes_prompt(cache, q_heads, T, batch)) return PARO_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return PARO_ERR_ALIGN;

    a.k = (const uint8_t *)c.k; a.v = (const uint8_t *)c.v; a.ks = c.k_scale; a.vs = c.v_scale;
    a.q = (const _Float16 *)Q; a.starts = starts; a.table = block_table; a.lengths = lengths; a.prefix = prefix; a.first = first;
    a.o = (_Float16 *)O; a.lse = lse;
    a.arrived = (uint32_t *)((char *)ws + kWsPartialOff);
    a.partial = (float *)((char *)ws + (ws_bytes & ~(size_t)255) - prompt_scratch_bytes(c, tiles));
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.page_log = log2_of(c.page); a.n_pages = c.n_pages; a.kv_heads = c.kv_heads; a.group = q_heads / c.kv_heads; a.width = table_width;
    a.batch = batch; a.window = window < 1 << 30 ? window : 0; a.T = T; a.tiles = (int)tiles; a.splits = (int)splits;
    a.scale = scale * kLog2e;
    hipStream_t s = (hipStream_t)stream;
    const bool scored = a.scores.cap > 0 || a.scores.slopes;
    hipError_t e;
    switch (2 * kernel_format(c.format) + scored) {
    case 0: e = launch_prompt<kFp16, false>(c.head_dim, a, s); break;
    case 1: e = launch_prompt<kFp16, true>(c.head_dim, a, s); break;
    case 2: e = launch_prompt<kE4m3, false>(c.head_dim, a, s); break;
    case 3: e = launch_prompt<kE4m3, true>(c.head_dim, a, s); break;
    case 4: e = launch_prompt<kMxfp4, false>(c.head_dim, a, s); break;
    default: e = launch_prompt<kMxfp4, true>(c.head_dim, a, s); break;
    }
    return e == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}
