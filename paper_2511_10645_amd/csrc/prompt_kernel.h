// Attention of many new tokens of every sequence over a paged key-value cache:
//
//      o_i = sum_t p_t v_t / sum_t p_t,   p_t = 2^(x_t - m),   x_t = log2(e) scale q_i . k_t,   lo_i <= t < hi_i
//
// A row at position p sees an interval of tokens: [p - window + 1, p], cut at first, stretched to prefix.  Bound by the matrix
// cores for long prompts (4 head_dim flops per row, head and token), by HBM for a few rows of a long sequence.
//
// A block has 128 pairs (row, query head) of one key-value head, numbered row by row, so that a head's keys and values are read once for
// all of its query heads, and walks its tokens in tiles of 64: keys and values go through LDS as fp16 (whatever the cache holds), two
// tiles deep, each wave of the block filling a quarter and using all for its 32 pairs.  Calls with few rows to a sequence have blocks of
// 32 or 64 pairs whose waves share a tile's tokens instead (prompt_common.h).  A wave computes S^T = K Q^T by 32 x 32 x 16 products: a
// lane then has scores of one pair only, half of a tile's, so that the softmax's maximum and sum need one exchange between two lanes, and
// S^T's registers are the B operand of O^T = V^T P^T as they are, if that product takes the tokens of a step in the order 4 (lane/32) +
// (0..3), then 8 more; values are read from LDS transposed in that order.  The cache's order of keys (16-byte units that interleave the
// tokens) is the first product's operand order: LDS keeps it, and no access has bank conflicts.
//
// p enters the second product as fp16 numbers after a factor of 2^kShift (16 bits would otherwise end at 2^-24 of the maximum): as two, p
// and what its rounding left, which together are off by 2^-22 of p or by 2^-35 of the largest, where that product is not what the time
// goes into: blocks for few rows (0 to 6 % over fp16 caches, 6 to 13 % over others), heads of 256 channels (8 to 13 %), scores with a cap
// or a bias (8 to 14 %). Otherwise as one, off by 2^-11 of itself at most, independently, which adds about as much to a result as its own
// rounding to fp16 (2.9e-4 of the 2-norm instead of 2.0e-4): a second one costs 512 rows behind 32256 tokens 375 us instead of 280, 8192
// rows 725 instead of 534, 2048 rows 65 instead of 53 (E4M3 71 and 58, MXFP4 69 and 58), 8 x 1024 rows of heads of 64 93 instead of 77.
// Sums stay in fp32.
//
// Few tiles with long sequences: `splits` blocks share a tile's tokens; each leaves fp32 results in the scratch, and the one that arrives
// last joins all in their order, so that results do not depend on timing.  Nobody waits.
//
// Measured (32 query and 8 key-value heads of 128 channels, fp16): 512 rows behind 32256 tokens 280 us (975 TFLOP/s; 1180 is what a large
// fp16 product of random numbers reaches on the card, whose clock falls to 1.5 GHz under either), 8192 rows alone 560 (980), 2048 rows
// alone 50 (685).  A round of a wave takes 2600 cycles alone and 3200 beside another, 1024 of them products: both waves of a SIMD need
// its vector unit for 1100 each (exponentials 8 cycles, products' issue 8, others 4).  What a block has besides: 11000 cycles to its
// first scores (arguments, starts, pages and keys are memory's latency one after the other), 8000 from the last.
#pragma once

#include <type_traits>
#include <utility>

#include "prompt_common.h"

namespace paro {

// f of the numbers FROM .. TO - 1, as constants.
template <int FROM, class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, FROM + I>()), ...); }
template <int FROM, int TO, class F>
__device__ __forceinline__ void each(F f) { each_of<FROM>(f, std::make_integer_sequence<int, (TO > FROM ? TO - FROM : 0)>()); }

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
// The largest of lanes 0..lane, of numbers from 0 on.
__device__ inline int prompt_most_upto(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return x;
}
// The largest of three, without the quieting of signalling NaN that fmaxf brings along (an instruction for every value).  The compiler keeps 12 states
// between a product and the first vector instruction that takes its result, but not in front of inline assembly, whose operands it does not look at:
// what goes in here is behind product_done() or behind several products more.
__device__ inline float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
// The 12 states.  The compiler is not relied on where a branch follows either: where two paths meet it may count along the longer one.
__device__ __forceinline__ void product_done()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 11");
    __builtin_amdgcn_sched_barrier(0);
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

// Tile `tile` of all sequences' tiles, and about how many tiles of tokens all of them have; false: there are fewer.  starts are taken within
// 0..T and none below one before it: no row has two tiles, and tiles are as many as prompt_tiles() says at most, whatever the starts are.
template <class S>
__device__ inline bool find_tile(Where &w, int &work, const PromptArgs &a, int tile, int lane)
{
    int before = 0, taken = 0;                   // tiles of the sequences seen, and where the rows of the last of them end
    bool found = false;
    work = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int b = b0 + lane < a.batch ? b0 + lane : a.batch - 1;
        int s0 = a.starts[b], s1 = a.starts[b + 1], n = a.lengths[b];
        const int room = a.width << a.page_log;
        n = n < 0 ? 0 : n > room ? room : n;
        s0 = prompt_most_upto(s0 < taken ? taken : s0 > a.T ? a.T : s0);
        s1 = s1 < s0 ? s0 : s1 > a.T ? a.T : s1;
        const int tiles = b0 + lane < a.batch ? (int)(((int64_t)(s1 - s0) * a.group + S::Pairs - 1) / S::Pairs) : 0;
        const int upto = prompt_sums_upto(tiles);
        if (a.splits > 1) {
            int seen = n - (s1 - s0) / 2;        // by a row, on average
            if (a.window && seen > a.window) seen = a.window;
            work += __builtin_amdgcn_readlane(prompt_sums_upto(tiles * (seen / S::Tokens + 1)), 63);
        }
        const uint64_t behind = __ballot(before + upto > tile);
        if (behind && !found) {
            const int at = __builtin_ctzll(behind);
            w.b = b0 + at;
            w.row0 = __builtin_amdgcn_readlane(s0, at);
            w.rows = __builtin_amdgcn_readlane(s1, at) - w.row0;
            w.n = __builtin_amdgcn_readlane(n, at);
            w.pair0 = (tile - before - __builtin_amdgcn_readlane(upto, at) + __builtin_amdgcn_readlane(tiles, at)) * S::Pairs;
            found = true;
            if (a.splits == 1) return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
        taken = __builtin_amdgcn_readlane(s1, 63);
    }
    return found;
}

__device__ inline __amdgpu_buffer_rsrc_t prompt_rsrc(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, kPromptRaw);
}

// How a wave moves 16 tokens of keys or of values: `Loads` requests of `Bytes` a lane, `Channels` channels each.
template <int D, int FMT>
struct Move {
    static constexpr int Bytes = row_bytes<FMT>(D) * 16 / 64 < 16 ? row_bytes<FMT>(D) * 16 / 64 : 16;
    static constexpr int Loads = row_bytes<FMT>(D) * 16 / 64 / Bytes;
    static constexpr int Channels = D / 4 / Loads;
};
template <int BYTES>
__device__ inline U4 prompt_load(__amdgpu_buffer_rsrc_t r, int off, int base)
{
    if constexpr (BYTES == 16) return __builtin_bit_cast(U4, __builtin_amdgcn_raw_buffer_load_b128(r, off, base, 0));
    const U2 y = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(r, off, base, 0));
    return U4{y[0], y[1], 0, 0};
}

// 16 bytes a lane to LDS, side by side from `lds` on (the same for all lanes).
typedef __attribute__((address_space(3))) void PromptLds;
__device__ inline void prompt_copy(__amdgpu_buffer_rsrc_t r, uint8_t *lds, int off, int base)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (PromptLds *)lds, 16, off, base, 0, 0);
}

// LDS: keys [tokens/16][head_dim/8][16 tokens] of 16 bytes; values [tokens][head_dim] in 16-byte units whose order in a row depends on
// the row: transposed reads take 64 bytes of 4 rows at once, writes of converted values every other or every 4th unit of a few rows, and both fall on
// distinct banks.
template <int D> __device__ inline int key_at(int t, int unit) { return ((t >> 4) * (D / 8) + unit) * 256 + (t & 15) * 16; }
template <int D> __device__ inline int value_unit(int t, int unit) { return D == 64 ? unit ^ (5 * ((t >> 1) & 1)) : unit ^ (5 * (t & 3)) ^ (D == 256 ? 2 * (unit >> 4) : 0); }
template <int D> __device__ inline int value_at(int t, int c) { return t * 2 * D + value_unit<D>(t, c >> 3) * 16 + (c & 7) * 2; }

// 16 tokens of keys or of values on a page, from the page's memory to LDS: fp16 caches' without a way through registers, others' through x.
template <int D, int FMT, bool KEYS>
struct Run {
    typedef Move<D, FMT> M;
    static constexpr int S = row_scales<FMT>(D);
    __amdgpu_buffer_rsrc_t r, scales;
    int tok;
    // of page `page`, tokens t0 (a multiple of 16) and on; a page below 0 is not there and gives zeros
    __device__ void at(const PromptArgs &a, int head, int page, int t0)
    {
        const int64_t place = ((int64_t)(page < 0 ? 0 : page) * a.kv_heads + head) << a.page_log;       // the page's first token
        tok = t0 & ((1 << a.page_log) - 1);
        r = prompt_rsrc((KEYS ? a.k : a.v) + place * row_bytes<FMT>(D), page < 0 ? 0 : (uint32_t)row_bytes<FMT>(D) << a.page_log);
        if constexpr (FMT != kFp16) scales = prompt_rsrc((KEYS ? a.ks : a.vs) + place * S, page < 0 ? 0 : (uint32_t)S << a.page_log);
    }
    // where request i of a lane lies behind the run's first byte: keys of token lane % 16, run of channels lane / 16 + 4 i (8-byte ones: two to a unit)
    __device__ static int from(int i, int lane, int page_log)
    {
        if constexpr (KEYS) {
            const int run = (lane >> 4) + 4 * i, unit = M::Bytes == 16 ? run : run >> 1;
            return (((unit << page_log) + (lane & 15)) << 4) + (M::Bytes == 16 ? 0 : (run & 1) * 8);
        }
        if constexpr (FMT == kFp16) {            // the 16 bytes that come to 16 (lane + 64 i) of the run in LDS
            const int to = (lane + 64 * i) * 16, t = to / (2 * D);
            return t * 2 * D + value_unit<D>(t, to % (2 * D) / 16) * 16;
        }
        return (lane + 64 * i) * M::Bytes;
    }
    __device__ int base() const { return KEYS ? tok << 4 : tok * row_bytes<FMT>(D); }
    __device__ void copy(uint8_t *lds, int i, int lane, int page_log) const
    {
        prompt_copy(r, lds + i * 1024, from(i, lane, page_log), base());
    }
    struct Held { U4 x; uint32_t scale; };
    __device__ void ask(Held &y, int i, int lane, int page_log) const
    {
        y.x = prompt_load<M::Bytes>(r, from(i, lane, page_log), base());
        const int c = KEYS ? ((lane >> 4) + 4 * i) * M::Channels : (lane + 64 * i) * M::Channels % D, t = KEYS ? lane & 15 : (lane + 64 * i) * M::Channels / D;
        y.scale = __builtin_amdgcn_raw_buffer_load_b8(scales, ((FMT == kMxfp4 ? c / 32 : 0) << page_log) + t, tok, 0);
    }
    __device__ static void put(const Held &y, uint8_t *lds, int i, int lane)
    {
        const float up = __uint_as_float(y.scale << 23);
#pragma unroll
        for (int z = 0; z < M::Channels / 8; ++z) {
            half8v f;
            if constexpr (FMT == kMxfp4) {
                f = f16_of_e2m1(y.x[z], up);
            } else {
                const uint32_t lo = y.x[2 * (z & 1)], hi = y.x[2 * (z & 1) + 1];
                const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, up, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, up, true);
                const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, up, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, up, true);
                f = half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
            }
            const int kc = ((lane >> 4) + 4 * i) * M::Channels + 8 * z, vt = (lane + 64 * i) * M::Channels / D, vc = (lane + 64 * i) * M::Channels % D + 8 * z;
            *(half8v *)(lds + (KEYS ? key_at<D>(lane & 15, kc / 8) : value_at<D>(vt, vc))) = f;
        }
    }
};
template <int N> __device__ __forceinline__ void prompt_wait_vm() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14)); }

// The larger magnitudes, as 16-bit numbers, of m's and of 8 fp16 values' (those that are not finite have 0x7c00 and more).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline u16x2 most_magnitude(u16x2 m, U4 x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
    return m;
}

typedef __fp16 Tr4 __attribute__((__vector_size__(8)));
typedef __attribute__((address_space(3))) Tr4 LdsTr4;

// Scores capped, scaled to log2, lowered by distance: tokens t0 + 8 (j / 4) + j % 4, `away` before the pair's position.
__device__ inline void adjust(F16 &s, const PromptArgs &a, float slope, int away)
{
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = s[j];
    if (a.scores.cap > 0) {
        capped(x, a.scores);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] *= a.scale;
    }
    if (a.scores.slopes) {
        const float from = (float)away;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = fmaf(-slope, fabsf(from - (8 * (j >> 2) + (j & 3))), x[j]);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) s[j] = x[j];
}

template <class S, int FMT, bool SCORED>
__global__ __launch_bounds__(kPromptThreads, S::Blocks) void prompt_attention_kernel(const PromptArgs a)
{
    constexpr int D = S::D, NB = S::NB, R = D / 32, KS = D / 16;       // channel tiles of the result, steps of the first product
    constexpr bool Two = S::WN > 1 || D == 256 || SCORED;              // numbers that a weight is, as above
    // Two tiles of keys and two of values; later the waves' results, one wave's to a tile's place.  They are objects of their own, and a round knows
    // which ones it reads and which it fills: the compiler makes a read wait for every copy to LDS that might be to the same object.
    __shared__ __attribute__((aligned(16))) uint8_t s_keys0[S::TileBytes], s_keys1[S::TileBytes], s_values0[S::TileBytes], s_values1[S::TileBytes];
    const auto place = [&](int i) __attribute__((always_inline)) { return i == 0 ? s_keys0 : i == 1 ? s_keys1 : i == 2 ? s_values0 : s_values1; };
    __shared__ int s_lo[kWaves][2], s_hi[kWaves][2];
    __shared__ int s_bad, s_last;                // s_bad: 1 + the tile that has values that are not finite, where not all see them
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int h = lane >> 5, n32 = lane & 31, wm = wave % S::WM, wn = wave / S::WM;

    // The heads of a tile side by side, which puts a head on one XCD where there are 8 of them; longest tiles first.  Where all blocks are on the chip
    // at once, those that come second to a compute unit begin with the shortest, so that it has a long and a short one.
    const int slots = kChip / a.kv_heads, all = a.tiles * a.splits;
    int rest = blockIdx.x / a.kv_heads;
    const int head = blockIdx.x - rest * a.kv_heads;
    if (S::Blocks == 2 && rest >= slots && all <= 2 * slots) rest = all - 1 - (rest - slots);
    // Last what may have no share, so that the shares fill the chip evenly (prefix and cap, 256 channels: 79 us, 83 with the parts of a tile side by side;
    // 16 sequences of 4 rows of 256 channels behind 4000 tokens 53 and 76; four drafts of 5 rows 18 either way, of 2 to 6 rows 22 and 21).
    const int split = rest / a.tiles, tile = a.tiles - 1 - (rest - split * a.tiles);
    Where w;
    int work;
    if (!find_tile<S>(w, work, a, tile, lane)) return;
    const int pairs = w.rows * a.group, pair = w.pair0 + wm * 32 + n32;
    // the pair's row and query head (the last pair's for lanes past it)
    const auto lo_of = [&](int p) __attribute__((always_inline)) { const int lo = a.window ? p - a.window + 1 : 0; return lo > 0 ? lo : 0; };
    int prefix = 0;
    if (a.prefix) { prefix = __builtin_amdgcn_readfirstlane(a.prefix[w.b]); prefix = prefix < w.n ? prefix : w.n; }
    const auto hi_of = [&](int p) __attribute__((always_inline)) { return p + 1 > prefix ? p + 1 : prefix; };
    const int row = (pair < pairs ? pair : pairs - 1) / a.group, qhead = head * a.group + (pair < pairs ? pair : pairs - 1) - row * a.group;

    // what the pair sees: lo <= t < hi, from position pos
    const int pos = w.n - w.rows + row;
    int lo = lo_of(pos), hi = hi_of(pos);
    if (a.first) { const int f = a.first[w.row0 + row]; lo = lo > f ? lo : f; }
    if (lo >= hi) { lo = INT32_MAX; hi = 0; }
    // The least and largest lo and hi of the block, and the largest lo and least hi of it and of the wave.  Both rise with the row, unless documents have it otherwise.
    int begin, end, whole_lo, whole_hi, lo_most, hi_least;
    if (!a.first) {
        const auto pos_at = [&](int p) __attribute__((always_inline)) { return w.n - w.rows + (p < pairs ? p : pairs - 1) / a.group; };
        const int p0 = pos_at(w.pair0), p1 = pos_at(w.pair0 + S::Pairs - 1), w0 = pos_at(w.pair0 + wm * 32), w1 = pos_at(w.pair0 + wm * 32 + 31);
        begin = lo_of(p0); end = hi_of(p1); whole_lo = lo_of(p1); whole_hi = hi_of(p0);
        lo_most = lo_of(w1); hi_least = hi_of(w0);
    } else {
        int least = lo, most = hi;
        lo_most = lo; hi_least = hi;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            least = min(least, __shfl_xor(least, d)); most = max(most, __shfl_xor(most, d));
            lo_most = max(lo_most, __shfl_xor(lo_most, d)); hi_least = min(hi_least, __shfl_xor(hi_least, d));
        }
        lo_most = __builtin_amdgcn_readfirstlane(lo_most); hi_least = __builtin_amdgcn_readfirstlane(hi_least);
        if (lane == 0) { s_lo[wave][0] = least; s_lo[wave][1] = lo_most; s_hi[wave][0] = most; s_hi[wave][1] = hi_least; }
        __syncthreads();
        begin = s_lo[0][0]; end = s_hi[0][0]; whole_lo = s_lo[0][1]; whole_hi = s_hi[0][1];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) {
            begin = min(begin, s_lo[i][0]); end = max(end, s_hi[i][0]);
            whole_lo = max(whole_lo, s_lo[i][1]); whole_hi = min(whole_hi, s_hi[i][1]);
        }
        begin = __builtin_amdgcn_readfirstlane(begin); end = __builtin_amdgcn_readfirstlane(end);
        whole_lo = __builtin_amdgcn_readfirstlane(whole_lo); whole_hi = __builtin_amdgcn_readfirstlane(whole_hi);
    }

    // its query: channels 16 s + 8 h ..  A negative scale goes into the queries' sign, a scale of 0 makes them 0: factors of maxima are positive.
    half8v q[KS];
    {
        const _Float16 *qp = a.q + (int64_t)(w.row0 + row) * a.ldq + (int64_t)qhead * D + 8 * h;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = *(const half8v *)(qp + 16 * s);
        if constexpr (!SCORED)
            if (a.scale <= 0)
#pragma unroll
                for (int s = 0; s < KS; ++s) q[s] = a.scale < 0 ? -q[s] : q[s] * (_Float16)0;
    }
    const float scale = SCORED ? 1.0f : a.scale == 0 ? 1.0f : fabsf(a.scale);
    float slope = 0;
    if constexpr (SCORED) if (a.scores.slopes) slope = a.scores.slopes[qhead] * kLog2e;
    // tiles of tokens, and this split's share of them: parts are as long as a block's share of all work
    const int tile0 = begin < end ? begin / S::Tokens : 0, tiles = begin < end ? (end + S::Tokens - 1) / S::Tokens - tile0 : 0;
    int parts = 1;
    if (a.splits > 1) {
        constexpr int Least = kLeastTokens / S::Tokens;
        const int64_t mean = ((int64_t)work * a.kv_heads + kChip * S::Blocks - 1) / (kChip * S::Blocks);
        const int part = mean < Least ? Least : mean < tiles ? (int)mean : tiles;
        parts = min(a.splits, part ? (tiles + part - 1) / part : 1);
        if (parts < 1) parts = 1;
    }
    if (split >= parts) return;
    const int per = (tiles + parts - 1) / parts;
    const int u0 = tile0 + split * per, u1 = min(u0 + per, tile0 + tiles);       // u0 may lie past u1: an empty share

    F16 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[r][j] = 0;
    bool far = false;                            // a maximum of the wave's is beyond kFarMax
    float m = -INFINITY, l = 0, up = scale, off = kShift;       // p = 2^(up s + off) of a score s is taken from the maximum m; l over this lane's tokens only

    // The pages of 64 runs of 16 tokens from run0 on, one to a lane (-1: not there, or past the part's tokens), and which of them are there.
    const int32_t *table = a.table + (int64_t)w.b * a.ld_table;
    constexpr int Runs = S::Tokens / 16;         // of a tile
    int run0 = u0 * Runs, pages = -1;
    uint64_t there = 0;
    const auto turn = [&](int run) __attribute__((always_inline)) {
        run0 = run;
        const int t = (run + lane) * 16;
        pages = -1;
        if (t < end && run + lane < u1 * Runs) {
            const int p = table[t >> a.page_log];
            pages = (uint32_t)p < (uint32_t)a.n_pages ? p : -1;
        }
        there = __ballot(pages >= 0);
    };
    struct Pages { int page[S::Quarters]; uint32_t gone; };      // of this wave's runs of a tile; a bit for every run of the tile that is not there
    const auto pages_of = [&](int u) __attribute__((always_inline)) {           // once turn() has got them
        Pages p;
#pragma unroll
        for (int i = 0; i < S::Quarters; ++i) p.page[i] = __builtin_amdgcn_readlane(pages, u * Runs - run0 + wave + 4 * i);
        p.gone = (uint32_t)(~(there >> (u * Runs - run0))) & ((1u << Runs) - 1);
        return p;
    };
    constexpr int Loads = Move<D, FMT>::Loads, Jobs = S::Quarters * Loads;       // requests of a wave for its share of a tile's keys, and of its values
    constexpr bool Copied = FMT == kFp16;
    Run<D, FMT, true> kr[S::Quarters];
    Run<D, FMT, false> vr[S::Quarters];
    typename Run<D, FMT, true>::Held kh[Copied ? 1 : Jobs];
    typename Run<D, FMT, false>::Held vh[Copied ? 1 : Jobs];
    const auto keys_at = [&](const Pages &p, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::Quarters; ++i) kr[i].at(a, head, p.page[i], u * S::Tokens + (wave + 4 * i) * 16);
    };
    const auto values_at = [&](const Pages &p, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::Quarters; ++i) vr[i].at(a, head, p.page[i], u * S::Tokens + (wave + 4 * i) * 16);
    };
    const auto run_in = [&](uint8_t *place, int job) __attribute__((always_inline)) { return place + (wave + 4 * (job / Loads)) * (16 * 2 * D); };

    // S^T of a tile: score j of block b is of token 32 (NB wn + b) + 8 (j / 4) + 4 h + j % 4
    F16 s[NB];
    const int key_lane = key_at<D>(32 * NB * wn + n32, h);
    const auto key_frag = [&](const uint8_t *keys, int i) __attribute__((always_inline)) { return *(const half8v *)(keys + key_lane + key_at<D>(32 * (i / KS), 2 * (i % KS))); };
    // 16 tokens i / R of this wave's, channels 32 (i % R) .., transposed; tokens 4 h + (0..3), then 8 more
    int value_lane[R];
#pragma unroll
    for (int r = 0; r < R; ++r) value_lane[r] = value_at<D>(32 * NB * wn + 4 * h + ((lane & 15) >> 2), 32 * r + 16 * ((lane >> 4) & 1) + 4 * (lane & 3));
    const auto value_frag = [&](const uint8_t *values, int i) __attribute__((always_inline)) {
        const uint8_t *from = values + value_lane[i % R] + 16 * (i / R) * 2 * D;
        const Tr4 one = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsTr4 *)from), two = __builtin_amdgcn_ds_read_tr16_b64_v4f16((LdsTr4 *)(from + 8 * 2 * D));
        half8v f;
#pragma unroll
        for (int e = 0; e < 4; ++e) { f[e] = (_Float16)one[e]; f[4 + e] = (_Float16)two[e]; }
        return f;
    };
    // what is done to scores before their maximum is taken: other scores, and the mask
    const auto finish = [&](F16 (&z)[NB], int u, uint32_t gone) __attribute__((always_inline)) {
        const int t0 = u * S::Tokens + 32 * NB * wn + 4 * h;
        if constexpr (SCORED) {
#pragma unroll
            for (int b = 0; b < NB; ++b) adjust(z[b], a, slope, pos - t0 - 32 * b);
        }
        if (u * S::Tokens < lo_most || (u + 1) * S::Tokens > hi_least || gone) {
            // a bit for every token of a block that the pair sees; a score keeps its bits or takes those of -inf
            const auto below = [](int n) __attribute__((always_inline)) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t away = gone >> (2 * (NB * wn + b)), there = (away & 1 ? 0u : 0xffffu) | (away & 2 ? 0u : 0xffff0000u);
                const uint32_t seen = below(hi - t0 - 32 * b) & ~below(lo - t0 - 32 * b) & (there >> (4 * h));
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int in = __builtin_amdgcn_sbfe((int)seen, 8 * (j >> 2) + (j & 3), 1);
                    z[b][j] = __uint_as_float((__float_as_uint(z[b][j]) & (uint32_t)in) | (0xff800000u & ~(uint32_t)in));
                }
            }
        }
    };
    // new scores z, the largest of this lane's `top`: the sums follow if the maximum has grown by more than kSlack
    const auto follow = [&](float top, F16 (&z)[NB]) __attribute__((always_inline)) {
        top = max2(top) * scale;
        if (__ballot(top > m + kSlack)) {
            const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;
            m = fmaxf(m, top);
            l *= f;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][j] *= f;
            const float ref = m == -INFINITY ? 0.0f : m;
            far = __ballot(fabsf(ref) > kFarMax) != 0;
            up = far ? 1.0f : scale;
            off = far ? kShift : kShift - ref;
        }
        if (far) {
            // product and difference as one would be off by up to half a unit of the maximum here, and p has to stay within fp16
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
#pragma clang fp contract(off)
                    const float y = z[b][j] * scale;
                    z[b][j] = y - ref;
                }
        }
    };

    if (u0 < u1) {
        if (tid == 0) s_bad = 0;
        turn(run0);
        // A round's requests are for keys of u + Lead and values of u + Lead - 1: at once on the way to LDS, or held for a round.
        constexpr int Lead = Copied ? 2 : 3;
        Pages p1 = pages_of(u0 + 1), p2 = pages_of(u0 + 2), p3 = pages_of(u0 + 3);
        {
            const Pages p0 = pages_of(u0);
            keys_at(p0, u0);
            values_at(p0, u0);
            if constexpr (Copied) {
#pragma unroll
                for (int i = 0; i < Jobs; ++i) kr[i / Loads].copy(run_in(s_keys0, i), i % Loads, lane, a.page_log);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) vr[i / Loads].copy(run_in(s_values0, i), i % Loads, lane, a.page_log);
                keys_at(p1, u0 + 1);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) kr[i / Loads].copy(run_in(s_keys1, i), i % Loads, lane, a.page_log);
                values_at(p1, u0 + 1);
                keys_at(p2, u0 + 2);
                prompt_wait_vm<0>();
            } else {
#pragma unroll
                for (int i = 0; i < Jobs; ++i) kr[i / Loads].ask(kh[i], i % Loads, lane, a.page_log);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) vr[i / Loads].ask(vh[i], i % Loads, lane, a.page_log);
                keys_at(p1, u0 + 1);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) {
                    kr[0].put(kh[i], run_in(s_keys0, i), i % Loads, lane);
                    kr[i / Loads].ask(kh[i], i % Loads, lane, a.page_log);
                }
                values_at(p1, u0 + 1);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) {
                    vr[0].put(vh[i], run_in(s_values0, i), i % Loads, lane);
                    vr[i / Loads].ask(vh[i], i % Loads, lane, a.page_log);
                }
                keys_at(p2, u0 + 2);
#pragma unroll
                for (int i = 0; i < Jobs; ++i) {
                    kr[0].put(kh[i], run_in(s_keys1, i), i % Loads, lane);
                    kr[i / Loads].ask(kh[i], i % Loads, lane, a.page_log);
                }
                values_at(p2, u0 + 2);
                keys_at(p3, u0 + 3);
            }
            __syncthreads();
            const uint8_t *keys = s_keys0;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 16; ++j) s[b][j] = 0;
#pragma unroll
            for (int i = 0; i < NB * KS; ++i) s[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_frag(keys, i), q[i % KS], s[i / KS], 0, 0, 0);
            product_done();
            finish(s, u0, p0.gone);
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int j = 0; j < 16; j += 2) top = max3(top, s[b][j], s[b][j + 1]);
            follow(top, s);
        }
        // A round has the scores of tile u.  It turns them into weights while the matrix cores compute those of u + 1, then multiplies the weights
        // with the values of u while it looks for the next maximum; keys of u + 2 and values of u + 1 go to LDS meanwhile.  What the vector units do is dealt
        // out over the matrix instructions evenly, 32 cycles of a matrix core to as many of a vector unit: 8 each for the issue and for an exponential, 4 for others.
        const auto round = [&](int u, uint8_t *free_keys, uint8_t *keys, uint8_t *values, uint8_t *free_values) __attribute__((always_inline)) {
            // operands on their way from LDS, which takes 130 cycles and more; fewer where registers are short (2048 rows, cap, E4M3: 101 us, 130 with 5)
            constexpr int Ahead = SCORED ? 3 : NB * KS < 5 ? NB * KS : 5;
            half8v f[Ahead + 1];
            each<0, Ahead>([&](auto at) __attribute__((always_inline)) { f[at] = key_frag(keys, at); });
            if (u * S::Tokens < whole_lo || (u + 1) * S::Tokens > whole_hi) {
                // A tile that some pair does not see all of: values that nobody sees become zeros, for such places may hold NaN, whose product with a weight
                // of 0 is not 0.  Others that are not finite are taken here by the pairs that see them (their results are not finite, whatever the
                // weight is) before zeros take their place.
                u16x2 bad = {0, 0};
#pragma unroll
                for (int k = 0; k < S::TileBytes / 16 / kPromptThreads; ++k) {
                    const int i = tid + k * kPromptThreads;
                    U4 *y = (U4 *)(values + 16 * i);
                    if (u * S::Tokens + i / (D / 8) >= end) *y = U4{0, 0, 0, 0};
                    else bad = most_magnitude(bad, *y);
                }
                if (__ballot(bad[0] >= 0x7c00 || bad[1] >= 0x7c00) && lane == 0) s_bad = u + 1;
                __syncthreads();
                if (__builtin_amdgcn_readfirstlane(s_bad) == u + 1) {
                    for (int i = 32 * NB * wn; i < 32 * NB * (wn + 1); ++i) {
                        const bool seen = u * S::Tokens + i >= lo && u * S::Tokens + i < hi;
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const float y = (float)*(const _Float16 *)(values + value_at<D>(i, 32 * r + 8 * (j >> 2) + 4 * h + (j & 3)));
                                if (seen && !is_finite(y)) acc[r][j] += y;
                            }
                    }
                    __syncthreads();
                    for (int i = tid; i < S::TileBytes / 16; i += kPromptThreads) {
                        half8v y = *(half8v *)(values + 16 * i);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = is_finite((float)y[e]) ? y[e] : (_Float16)0;
                        *(half8v *)(values + 16 * i) = y;
                    }
                    __syncthreads();
                }
            }
            const uint32_t gone = p1.gone;
            if ((u + 4) * Runs - run0 >= 64) turn((u + 4) * Runs);
            // the next round's requests; past the part's last tile there is nothing to read, and zeros come
            const auto advance = [&]() __attribute__((always_inline)) {
                values_at(Copied ? p2 : p3, u + Lead);
                p1 = p2;
                p2 = p3;
                p3 = pages_of(u + 4);
                keys_at(Copied ? p2 : p3, u + Lead + 1);
            };

            constexpr int All = NB * 8, Late = NB * 3;       // pairs of scores; those whose weights the second product does not need at once
            half8v p[2 * NB], low[2 * NB];
            const auto weigh = [&](auto at) __attribute__((always_inline)) {
                constexpr int c = at, b = c / 8, e = c % 8;
                const float one = __builtin_amdgcn_exp2f(fmaf(s[b][2 * e], up, off)), two = __builtin_amdgcn_exp2f(fmaf(s[b][2 * e + 1], up, off));
                l += one;
                l += two;
                half2v both = {(_Float16)one, (_Float16)two};
                asm volatile("" : "+v"(both), "+v"(l));      // here, not where they are needed
                p[c / 4][2 * (e & 3)] = both[0];
                p[c / 4][2 * (e & 3) + 1] = both[1];
                if constexpr (Two) {
                    half2v more = {(_Float16)(one - (float)both[0]), (_Float16)(two - (float)both[1])};
                    asm volatile("" : "+v"(more));
                    low[c / 4][2 * (e & 3)] = more[0];
                    low[c / 4][2 * (e & 3) + 1] = more[1];
                }
            };
            F16 next[NB];
            {
                constexpr int Steps = NB * KS;
                each<0, Steps>([&](auto at) __attribute__((always_inline)) {
                    constexpr int i = at;
                    if constexpr (i + Ahead < Steps) f[(i + Ahead) % (Ahead + 1)] = key_frag(keys, i + Ahead);
                    else f[(i + Ahead) % (Ahead + 1)] = value_frag(values, i + Ahead - Steps);
                    F16 z = next[i / KS];
                    if constexpr (i % KS == 0)
#pragma unroll
                        for (int j = 0; j < 16; ++j) z[j] = 0;
                    next[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[i % (Ahead + 1)], q[i % KS], z, 0, 0, 0);
                    if constexpr (Copied)
                        each<i * 2 * Jobs / Steps, (i + 1) * 2 * Jobs / Steps>([&](auto job) __attribute__((always_inline)) {
                            constexpr int k = job;
                            if constexpr (k < Jobs) kr[k / Loads].copy(run_in(free_keys, k), k % Loads, lane, a.page_log);
                            else vr[(k - Jobs) / Loads].copy(run_in(free_values, k - Jobs), (k - Jobs) % Loads, lane, a.page_log);
                        });
                    each<i *(All - Late) / Steps, (i + 1) * (All - Late) / Steps>(weigh);
                    if constexpr (!Copied)
                        each<i * Jobs / Steps, (i + 1) * Jobs / Steps>([&](auto job) __attribute__((always_inline)) {
                            constexpr int k = job;
                            kr[0].put(kh[k], run_in(free_keys, k), k % Loads, lane);
                            kr[k / Loads].ask(kh[k], k % Loads, lane, a.page_log);
                        });
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
            // with NB of 2 the second product has begun before the maximum takes the first block, and is half done before it takes the second
            if constexpr (NB == 1) product_done();
            finish(next, u + 1, gone);
            float top = -INFINITY;
            {
                constexpr int Steps = 2 * NB * R, Soon = NB * R, Before = NB * KS;      // of the first product, whose ring of operands goes on
                each<0, Steps>([&](auto at) __attribute__((always_inline)) {
                    constexpr int i = at;
                    if constexpr (i + Ahead < Steps) f[(Before + i + Ahead) % (Ahead + 1)] = value_frag(values, i + Ahead);
                    acc[i % R] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[(Before + i) % (Ahead + 1)], p[i / R], acc[i % R], 0, 0, 0);
                    if constexpr (Two) acc[i % R] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[(Before + i) % (Ahead + 1)], low[i / R], acc[i % R], 0, 0, 0);
                    if constexpr (i < Soon) each<All - Late + i * Late / Soon, All - Late + (i + 1) * Late / Soon>(weigh);
                    each<i * All / Steps, (i + 1) * All / Steps>([&](auto two) __attribute__((always_inline)) {
                        constexpr int c = two;
                        top = max3(top, next[c / 8][2 * (c % 8)], next[c / 8][2 * (c % 8) + 1]);
                    });
                    if constexpr (!Copied)
                        each<i * Jobs / Steps, (i + 1) * Jobs / Steps>([&](auto job) __attribute__((always_inline)) {
                            constexpr int k = job;
                            vr[0].put(vh[k], run_in(free_values, k), k % Loads, lane);
                            vr[k / Loads].ask(vh[k], k % Loads, lane, a.page_log);
                        });
                    if constexpr (i == Steps - 1) advance();
                    __builtin_amdgcn_sched_barrier(0);
                });
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = next[b];
            follow(top, s);
            if constexpr (Copied) prompt_wait_vm<0>();
            __syncthreads();
        };
        for (int u = u0; u < u1; u += 2) {
            round(u, s_keys0, s_keys1, s_values0, s_values1);
            if (u + 1 < u1) round(u + 1, s_keys1, s_keys0, s_values1, s_values0);
        }
    }
    l = sum2(l);

    if constexpr (S::WN > 1) {
        // the waves that share pairs: their results meet in LDS, and each finishes every WN-th run of 4 registers
        static_assert(R * 4 * 64 * 16 <= S::TileBytes, "a wave's results fit a tile's place");      // [R][4][64] of 4
        __shared__ float s_m[kWaves][32], s_l[kWaves][32];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(F4 *)(place(wave) + ((r * 4 + i) * 64 + lane) * 16) = F4{acc[r][4 * i], acc[r][4 * i + 1], acc[r][4 * i + 2], acc[r][4 * i + 3]};
        if (h == 0) { s_m[wave][n32] = m; s_l[wave][n32] = l; }
        __syncthreads();
        float f[S::WN];
        m = -INFINITY;
#pragma unroll
        for (int z = 0; z < S::WN; ++z) m = fmaxf(m, s_m[wm + z * S::WM][n32]);
        const float ref = m == -INFINITY ? 0.0f : m;
        l = 0;
#pragma unroll
        for (int z = 0; z < S::WN; ++z) {
            f[z] = __builtin_amdgcn_exp2f(s_m[wm + z * S::WM][n32] - ref);
            l = fmaf(s_l[wm + z * S::WM][n32], f[z], l);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= 4 / S::WN) continue;
                F4 y = {0, 0, 0, 0};
#pragma unroll
                for (int z = 0; z < S::WN; ++z) {
                    const F4 v = *(const F4 *)(place(wm + z * S::WM) + ((r * 4 + i * S::WN + wn) * 64 + lane) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = fmaf(v[e], f[z], y[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[r][4 * i + e] = y[e];
            }
    }
    // from here on a wave has runs i * WN + wn of the 4 registers of a channel tile, in registers 4 i ..
    if (parts > 1) {
        // every part's m, l and sums where its lanes left them, through memory that all XCDs see
        const size_t tile_at = (size_t)tile * a.kv_heads + head;
        const auto part_rsrc = [&](int p) __attribute__((always_inline)) { return prompt_rsrc(a.partial + (tile_at * a.splits + p) * S::PartFloats, (uint32_t)(S::PartFloats * 4)); };
        const int ml_at = (S::Pairs * D + 2 * (wm * 32 + n32)) * 4;
        const auto sums_at = [&](int r, int i) __attribute__((always_inline)) { return (((wm * R + r) * 4 + i) * 64 + lane) * 16; };
        typedef decltype(__builtin_amdgcn_raw_buffer_load_b128(part_rsrc(0), 0, 0, 0)) B4;
        typedef decltype(__builtin_amdgcn_raw_buffer_load_b64(part_rsrc(0), 0, 0, 0)) B2;
        const bool live = w.pair0 + wm * 32 < pairs;         // a wave without pairs has nothing to leave and nothing to join
        if (live) {
            const __amdgpu_buffer_rsrc_t to = part_rsrc(split);
            if (h == 0 && wn == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(B2, U2{__float_as_uint(m), __float_as_uint(l)}), to, ml_at, 0, kPromptAgent);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int i = 0; i < 4 / S::WN; ++i)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(B4, F4{acc[r][4 * i], acc[r][4 * i + 1], acc[r][4 * i + 2], acc[r][4 * i + 3]}), to,
                                                           sums_at(r, i * S::WN + wn), 0, kPromptAgent);
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
        // as many parts as registers hold at a time, all of their requests before the first use; a part that is not there gives zeros, and does not count
        constexpr int At = 8 * S::WN / R < 1 ? 1 : 8 * S::WN / R > 8 ? 8 : 8 * S::WN / R;
        m = -INFINITY;
        l = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][j] = 0;
        for (int p0 = 0; p0 < (live ? parts : 0); p0 += At) {
            U2 ml[At];
            F4 y[At][R][4 / S::WN];
            const auto from = [&](int z) __attribute__((always_inline)) { return prompt_rsrc(a.partial + (tile_at * a.splits + p0 + z) * S::PartFloats, p0 + z < parts ? (uint32_t)(S::PartFloats * 4) : 0); };
#pragma unroll
            for (int z = 0; z < At; ++z) ml[z] = __builtin_bit_cast(U2, __builtin_amdgcn_raw_buffer_load_b64(from(z), ml_at, 0, kPromptAgent));
#pragma unroll
            for (int z = 0; z < At; ++z)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < 4 / S::WN; ++i) y[z][r][i] = __builtin_bit_cast(F4, __builtin_amdgcn_raw_buffer_load_b128(from(z), sums_at(r, i * S::WN + wn), 0, kPromptAgent));
            float top = m;
#pragma unroll
            for (int z = 0; z < At; ++z) top = fmaxf(top, p0 + z < parts ? __uint_as_float(ml[z][0]) : -INFINITY);
            const float ref = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            l *= keep;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][j] *= keep;
#pragma unroll
            for (int z = 0; z < At; ++z) {
                const float f = p0 + z < parts ? __builtin_amdgcn_exp2f(__uint_as_float(ml[z][0]) - ref) : 0.0f;
                l = fmaf(__uint_as_float(ml[z][1]), f, l);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < 4 / S::WN; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[r][4 * i + e] = fmaf(y[z][r][i][e], f, acc[r][4 * i + e]);
            }
        }
    }

    if (pair < pairs && a.lse && h == 0 && wn == 0)
        a.lse[(int64_t)(w.row0 + row) * (a.kv_heads * a.group) + qhead] = l == 0.0f ? -INFINITY : (m - kShift + __builtin_amdgcn_logf(l)) * kLn2;
    // Results go by way of LDS, so that a row's channels are written side by side (as they lie in registers, 16 bytes of 32 rows at a time, a block
    // took up to 20000 cycles for them): [32 pairs][D], 8 bytes more a row so that rows fall on other banks.
    {
        const float inv = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
        constexpr int Row = 2 * D + 8;
        static_assert(32 * Row <= S::TileBytes, "32 pairs' results fit a tile's place");
        uint8_t *out = place(wm);
        __syncthreads();                         // LDS is free: the waves' sums have been read
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < 4 / S::WN; ++i)
                *(half4v *)(out + n32 * Row + (32 * r + 8 * (i * S::WN + wn) + 4 * h) * 2) =
                    half4v{(_Float16)(acc[r][4 * i] * inv), (_Float16)(acc[r][4 * i + 1] * inv), (_Float16)(acc[r][4 * i + 2] * inv), (_Float16)(acc[r][4 * i + 3] * inv)};
        __syncthreads();
        constexpr int Lanes = D / 4;             // of a row, 8 bytes each
#pragma unroll 4
        for (int i = tid; i < S::Pairs * Lanes; i += kPromptThreads) {
            const int p = i / Lanes, c = i % Lanes * 4;
            if (w.pair0 + p >= pairs) break;
            const int to = (w.pair0 + p) / a.group, of = head * a.group + w.pair0 + p - to * a.group;
            *(half4v *)(a.o + (int64_t)(w.row0 + to) * a.ldo + (int64_t)of * D + c) = *(const half4v *)(place(p >> 5) + (p & 31) * Row + c * 2);
        }
    }
}

template <class S, int FMT, bool SCORED>
static hipError_t launch_prompt(PromptArgs &a, hipStream_t s)
{
    a.tiles = (int)prompt_tiles(a.T, a.group, a.batch, S::Pairs);
    a.splits = (int)prompt_splits(a.tiles, a.kv_heads);
    hipLaunchKernelGGL((prompt_attention_kernel<S, FMT, SCORED>), dim3((unsigned)(a.tiles * a.kv_heads * a.splits)), dim3(kPromptThreads), 0, s, a);
    return hipGetLastError();
}
template <int D, int FMT, bool SCORED>
static hipError_t launch_prompt(PromptArgs &a, hipStream_t s)
{
    if ((int64_t)a.T * a.group <= (int64_t)kFewPairs * a.batch) return launch_prompt<typename Shapes<D>::Few, FMT, SCORED>(a, s);
    return launch_prompt<typename Shapes<D>::Many, FMT, SCORED>(a, s);
}
template <int FMT>
static hipError_t launch_prompt(int head_dim, bool scored, PromptArgs &a, hipStream_t s)
{
    switch (2 * head_dim + scored) {
    case 128: return launch_prompt<64, FMT, false>(a, s);
    case 129: return launch_prompt<64, FMT, true>(a, s);
    case 256: return launch_prompt<128, FMT, false>(a, s);
    case 257: return launch_prompt<128, FMT, true>(a, s);
    case 512: return launch_prompt<256, FMT, false>(a, s);
    default: return launch_prompt<256, FMT, true>(a, s);
    }
}

}  // namespace paro
