// Rotary positions, alone or on the way into a paged key-value cache:
//
//      (a, b) -> magnitude * (a cos p f_i - b sin p f_i, a sin p f_i + b cos p f_i)   for pair i of a token at position p
//
// Bound by HBM (every element read and written once) and at few tokens by latency.  A block has some consecutive tokens
// and some of their heads; it evaluates each (token, pair) angle once, in LDS, for all of them (64 sines a token next to some
// thousand channels).  The angle is reduced to a fraction of a turn in fp64: p f loses nothing at long positions, where an fp32
// product is off by 2^-24 p f.  A thread then has 16 channels of a head, both halves of 8 pairs in either layout (two 16-byte
// requests, no exchange between lanes), keeps their sines and cosines and takes one head after the other, the next one's
// channels on their way.  A prompt's tokens are taken several to a block because the cache interleaves the tokens of a page
// in its keys: neighbouring tokens then fill whole pieces of a cache line in one L2.
#include <cmath>

#include "kv_common.h"

namespace paro {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;                   // most tokens of a block
constexpr int kRopeMany = 1024;                  // tokens from which on a block has several
constexpr int kRopeBlocks = 1024;                // blocks that heads are spread over
constexpr int kRopeMost = 1 << 24;               // tokens of a call: a launch holds fewer than 2^32 threads
constexpr int kRopePairs = 256;                  // most pairs of a head

struct RopeArgs {
    const _Float16 *q, *k, *v;                   // k NULL: no cache
    _Float16 *qr;
    uint8_t *ck, *cv, *cks, *cvs;
    const float *inv_freq;
    const int32_t *positions;
    const int64_t *slots;
    int64_t ldq, ldk, ldv, ldqr, n_slots;
    int T, tokens, q_heads, kv_heads, D, pairs, page_log, rows;      // pairs 0: no rotation; rows: heads of a block
    float magnitude;
};

__device__ inline half8v rounded(const float (&x)[8])
{
    half8v h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
    return h;
}

// The exponent of a cache row from the largest finite |value|: the least e in -15..8 with most <= 448 * 2^e (448 = 1.75 * 2^8).
__device__ inline int e4m3_exponent(float most)
{
    const uint32_t u = __float_as_uint(most);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return e < kKvExponentLeast ? kKvExponentLeast : e > kKvExponentMost ? kKvExponentMost : e;
}
__device__ inline float finite_or(float x, float other) { return is_finite(x) ? x : other; }
__device__ inline uint2 e4m3_codes(const float (&x)[8], float up, float most)
{
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = is_finite(x[e]) ? fminf(fmaxf(x[e] * up, -most), most) : NAN;
    return uint2{e4m3_pack(q[0], q[1], q[2], q[3]), e4m3_pack(q[4], q[5], q[6], q[7])};
}

// The exponent of 32 channels of an MXFP4 cache from their largest |value|: floor(log2 most) - 2 (6 = 1.5 * 2^2 is the largest code).
__device__ inline int mx_exponent(float most)
{
    const int e = (int)(__float_as_uint(most) >> 23) - 127 - 2;
    return e < kMxExponentLeast ? kMxExponentLeast : e > kMxExponentMost ? kMxExponentMost : e;
}
__device__ inline uint32_t e2m1_codes(const float (&x)[8], float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}
// The largest |value| of 8 channels, infinite if one of them is not finite.
__device__ inline float most_or_infinite(const float (&x)[8])
{
    float m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(finite_or(x[e], INFINITY)));
    return m;
}

template <int LAYOUT, int FMT>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float s_cs[];     // [token][cos of the pairs, sin of the pairs]
    // MXFP4: a thread's two runs of 8 channels may belong to different groups of 32, and a group to four threads (halves are paired at
    // any multiple of 8): the largest values of a head's runs meet here.  A head's threads are lanes of one wave, whose LDS accesses keep their order.
    __shared__ __attribute__((aligned(16))) float s_most[FMT == kMxfp4 ? 2 * kRopeThreads : 4];
    const int t0 = blockIdx.x * a.tokens;
    const int tokens = a.T - t0 < a.tokens ? a.T - t0 : a.tokens;
    for (int i = threadIdx.x; i < tokens * a.pairs; i += kRopeThreads) {
        const int t = i / a.pairs, p = i - t * a.pairs;
        const double turns = (double)a.positions[t0 + t] * ((double)a.inv_freq[p] * 0.15915494309189533577);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_cs[t * 2 * a.pairs + p] = c * a.magnitude;
        s_cs[t * 2 * a.pairs + a.pairs + p] = s * a.magnitude;
    }
    __syncthreads();

    // A thread keeps its 16 channels c and its token t, sines and cosines with them, and takes every `step`-th head.
    const int lanes = a.D / 16;                  // of a head
    const int c = threadIdx.x % lanes, line = threadIdx.x / lanes, step = kRopeThreads / lanes / a.tokens;
    const int t = line % a.tokens;
    const int first = blockIdx.y * a.rows, all = a.q_heads + (a.k ? 2 * a.kv_heads : 0);
    const int last = first + a.rows < all ? first + a.rows : all;
    int row = first + line / a.tokens;
    if (t >= tokens || line / a.tokens >= step) return;
    const bool paired = 8 * c < a.pairs;
    const int pa = LAYOUT == 0 && paired ? 8 * c : 16 * c, pb = LAYOUT == 0 && paired ? a.pairs + 8 * c : 16 * c + 8;
    float cs[8], sn[8];
    if (paired) {
        const float *at = s_cs + t * 2 * a.pairs + 8 * c;
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = at[e]; sn[e] = at[a.pairs + e]; }
    }
    int64_t slot = -1;
    if (a.k) slot = a.slots[t0 + t];
    const bool kept = (uint64_t)slot < (uint64_t)a.n_slots;
    const int64_t page0 = ((slot >> a.page_log) * a.kv_heads) << a.page_log;       // the first token of the page's first head
    const int off = (int)slot & ((1 << a.page_log) - 1);
    const _Float16 *xq = a.q + (t0 + t) * a.ldq, *xk = a.k + (t0 + t) * a.ldk, *xv = a.v + (t0 + t) * a.ldv;
    const auto source = [&](int r) {
        return r < a.q_heads ? xq + r * a.D : r < a.q_heads + a.kv_heads ? xk + (r - a.q_heads) * a.D : xv + (r - a.q_heads - a.kv_heads) * a.D;
    };
    const auto place_a = [&](int r) { return r < a.q_heads + a.kv_heads ? pa : 16 * c; };       // values are not rotated
    const auto place_b = [&](int r) { return r < a.q_heads + a.kv_heads ? pb : 16 * c + 8; };
    half8v na = {}, nb = {};                     // the next head's channels
    if (row < last) { na = *(const half8v *)(source(row) + place_a(row)); nb = *(const half8v *)(source(row) + place_b(row)); }
    for (; row < last; row += step) {
        const bool is_q = row < a.q_heads, is_k = !is_q && row < a.q_heads + a.kv_heads;
        const int head = is_q ? row : is_k ? row - a.q_heads : row - a.q_heads - a.kv_heads;
        const int ca = place_a(row), cb = place_b(row);
        const half8v ha = na, hb = nb;
        if (row + step < last) {
            na = *(const half8v *)(source(row + step) + place_a(row + step));
            nb = *(const half8v *)(source(row + step) + place_b(row + step));
        }
        float fa[8], fb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { fa[e] = (float)ha[e]; fb[e] = (float)hb[e]; }
        if (paired && (is_q || is_k)) {
            if (LAYOUT == 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = fa[e], q = fb[e];
                    fa[e] = p * cs[e] - q * sn[e];
                    fb[e] = p * sn[e] + q * cs[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = fa[2 * e], q = fa[2 * e + 1], r = fb[2 * e], s = fb[2 * e + 1];
                    fa[2 * e] = p * cs[e] - q * sn[e];
                    fa[2 * e + 1] = p * sn[e] + q * cs[e];
                    fb[2 * e] = r * cs[4 + e] - s * sn[4 + e];
                    fb[2 * e + 1] = r * sn[4 + e] + s * cs[4 + e];
                }
            }
        }
        if (is_q) {
            _Float16 *y = a.qr + (t0 + t) * a.ldqr + (int64_t)head * a.D;
            *(half8v *)(y + ca) = rounded(fa);
            *(half8v *)(y + cb) = rounded(fb);
            continue;
        }
        const int64_t place = page0 + ((int64_t)head << a.page_log);       // this head's first token of the page
        if constexpr (FMT == kMxfp4) {
            float *of_head = s_most + line * 2 * lanes;
            of_head[ca / 8] = most_or_infinite(fa);
            of_head[cb / 8] = most_or_infinite(fb);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const auto of_group = [&](int channel) {
                const float *m = of_head + channel / 32 * 4;
                return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
            };
            const float ma = of_group(ca), mb = of_group(cb);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();         // the next head's go to the same place
            if (!kept) continue;
            uint8_t *y = (is_k ? a.ck : a.cv) + place * (a.D / 2), *scales = (is_k ? a.cks : a.cvs) + place * (a.D / 32);
            const auto put = [&](const float (&f)[8], int channel, float most) {
                const int e = mx_exponent(most);
                const uint32_t codes = e2m1_codes(f, __uint_as_float((uint32_t)(127 + e) << 23));
                *(uint32_t *)(y + (is_k ? ((int64_t)(channel / 32) << (a.page_log + 4)) + off * 16 + channel % 32 / 2 : (int64_t)off * (a.D / 2) + channel / 2)) = codes;
                if (channel % 32 == 0) scales[((channel / 32) << a.page_log) + off] = (uint8_t)(most == INFINITY ? kMxNan : 127 + e);
            };
            put(fa, ca, ma);
            put(fb, cb, mb);
        } else if constexpr (FMT == 0) {
            if (!kept) continue;
            if (is_k) {
                uint8_t *y = a.ck + place * a.D * 2 + off * 16;
                *(half8v *)(y + ((int64_t)(ca / 8) << (a.page_log + 4))) = rounded(fa);
                *(half8v *)(y + ((int64_t)(cb / 8) << (a.page_log + 4))) = rounded(fb);
            } else {
                uint8_t *y = a.cv + ((place + off) * a.D + ca) * 2;
                *(half8v *)y = rounded(fa);
                *(half8v *)(y + 16) = rounded(fb);
            }
        } else {
            float most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fmaxf(fabsf(finite_or(fa[e], 0)), fabsf(finite_or(fb[e], 0))));
            for (int d = 1; d < lanes; d <<= 1) most = fmaxf(most, __shfl_xor(most, d));   // a head's lanes are here together
            if (!kept) continue;
            const int e = e4m3_exponent(most);
            const float up = __uint_as_float((uint32_t)(127 - e) << 23), within = e == kKvExponentMost ? 240.0f : kE4m3Max;
            const uint2 qa = e4m3_codes(fa, up, within), qb = e4m3_codes(fb, up, within);
            uint8_t *y = is_k ? a.ck + place * a.D + off * 16 : a.cv + (place + off) * a.D;
            if (is_k) {
                *(uint2 *)(y + ((int64_t)(ca / 16) << (a.page_log + 4)) + (ca & 8)) = qa;
                *(uint2 *)(y + ((int64_t)(cb / 16) << (a.page_log + 4)) + (cb & 8)) = qb;
            } else {
                *(uint2 *)(y + ca) = qa;
                *(uint2 *)(y + cb) = qb;
            }
            if (c == 0) (is_k ? a.cks : a.cvs)[place + off] = (uint8_t)(127 + e);
        }
    }
}

static hipError_t launch_rope(RopeArgs &a, int layout, int format, hipStream_t s)
{
    const int all = a.q_heads + (a.k ? 2 * a.kv_heads : 0);
    // Few tokens: one to a block.  Many: 4, whose keys are 64 bytes side by side in the cache (2048 tokens to an E4M3 cache: 14.8 us,
    // 16.2 with one and 15.1 with 8, which take the interleaved layout from 15.6 to 18.7 us at 4095 tokens).  Heads are spread
    // over blocks while these are few, down to one for every thread.
    a.tokens = a.T >= kRopeMany ? kRopeTokens : 1;
    const int blocks = (a.T + a.tokens - 1) / a.tokens, step = kRopeThreads / (a.D / 16) / a.tokens;
    int split = (kRopeBlocks + blocks - 1) / blocks;
    const int most = (all + step - 1) / step;
    split = split < most ? split : most;
    a.rows = (all + split - 1) / split;
    const dim3 grid((unsigned)blocks, (unsigned)((all + a.rows - 1) / a.rows));
    const size_t lds = sizeof(float) * 2 * a.tokens * (a.pairs ? a.pairs : 1);
    if (layout == 0) {
        if (format == kFp16) hipLaunchKernelGGL((rope_kernel<0, kFp16>), grid, dim3(kRopeThreads), lds, s, a);
        else if (format == kE4m3) hipLaunchKernelGGL((rope_kernel<0, kE4m3>), grid, dim3(kRopeThreads), lds, s, a);
        else hipLaunchKernelGGL((rope_kernel<0, kMxfp4>), grid, dim3(kRopeThreads), lds, s, a);
    } else {
        if (format == kFp16) hipLaunchKernelGGL((rope_kernel<1, kFp16>), grid, dim3(kRopeThreads), lds, s, a);
        else if (format == kE4m3) hipLaunchKernelGGL((rope_kernel<1, kE4m3>), grid, dim3(kRopeThreads), lds, s, a);
        else hipLaunchKernelGGL((rope_kernel<1, kMxfp4>), grid, dim3(kRopeThreads), lds, s, a);
    }
    return hipGetLastError();
}

static paro_status check_rope(const paro_rope_t *r)
{
    if (!r || !r->inv_freq) return PARO_ERR_NULL;
    if (r->head_dim <= 0 || r->rot_dim <= 0 || r->rot_dim > r->head_dim || !std::isfinite(r->magnitude)) return PARO_ERR_SHAPE;
    if (r->layout != 0 && r->layout != 1) return PARO_ERR_UNSUPPORTED;
    if (r->head_dim % 16 || r->rot_dim % 16 || r->head_dim > 2 * kRopePairs) return PARO_ERR_UNSUPPORTED;
    return aligned(r->inv_freq, 4) ? PARO_OK : PARO_ERR_ALIGN;
}

}  // namespace paro

extern "C" paro_status paro_rope(const paro_rope_t *rope, const paro_half_t *X, int64_t ldx, const int32_t *positions, int32_t heads,
                                 int32_t T, paro_half_t *Y, int64_t ldy, void *stream)
{
    using namespace paro;
    if (const paro_status st = check_rope(rope); st != PARO_OK) return st;
    if (!positions) return PARO_ERR_NULL;
    if (T <= 0 || heads <= 0) return PARO_ERR_SHAPE;
    if (const paro_status st = check_rows(X, ldx, (int64_t)heads * rope->head_dim); st != PARO_OK) return st;
    if (const paro_status st = check_rows(Y, ldy, (int64_t)heads * rope->head_dim); st != PARO_OK) return st;
    if (X == Y && ldx != ldy) return PARO_ERR_SHAPE;
    if (!aligned(positions, 4)) return PARO_ERR_ALIGN;
    if (heads > 65535 || T > kRopeMost) return PARO_ERR_UNSUPPORTED;
    RopeArgs a = {};
    a.q = (const _Float16 *)X; a.ldq = ldx; a.qr = (_Float16 *)Y; a.ldqr = ldy;
    a.inv_freq = rope->inv_freq; a.positions = positions; a.magnitude = rope->magnitude;
    a.T = T; a.q_heads = heads; a.D = rope->head_dim; a.pairs = rope->rot_dim / 2;
    return launch_rope(a, rope->layout, 0, (hipStream_t)stream) == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}

extern "C" paro_status paro_kv_append(const paro_kv_cache *cache, const paro_rope_t *rope, const paro_half_t *K, int64_t ldk,
                                      const paro_half_t *V, int64_t ldv, const int64_t *slots, const int32_t *positions, int32_t T,
                                      const paro_half_t *Q, int64_t ldq, int32_t q_heads, paro_half_t *Qr, int64_t ldqr, void *stream)
{
    using namespace paro;
    if (const paro_status st = check_cache(cache); st != PARO_OK) return st;
    if (!K || !V || !slots || (rope && !positions) || (Q && !Qr)) return PARO_ERR_NULL;
    const paro_kv_cache &c = *cache;
    if (rope) {
        if (const paro_status st = check_rope(rope); st != PARO_OK) return st;
        if (rope->head_dim != c.head_dim) return PARO_ERR_SHAPE;
    }
    if (T <= 0 || (Q && q_heads <= 0)) return PARO_ERR_SHAPE;
    const int64_t width = (int64_t)c.kv_heads * c.head_dim;
    if (const paro_status st = check_rows(K, ldk, width); st != PARO_OK) return st;
    if (const paro_status st = check_rows(V, ldv, width); st != PARO_OK) return st;
    if (Q) {
        if (const paro_status st = check_rows(Q, ldq, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
        if (const paro_status st = check_rows(Qr, ldqr, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
        if (Q == Qr && ldq != ldqr) return PARO_ERR_SHAPE;
    }
    if (!aligned(slots, 8) || (positions && !aligned(positions, 4))) return PARO_ERR_ALIGN;
    if (c.kv_heads > 65535 || (Q && q_heads > 65535) || T > kRopeMost) return PARO_ERR_UNSUPPORTED;
    RopeArgs a = {};
    a.q = (const _Float16 *)Q; a.ldq = ldq; a.qr = (_Float16 *)Qr; a.ldqr = ldqr; a.q_heads = Q ? q_heads : 0;
    a.k = (const _Float16 *)K; a.ldk = ldk; a.v = (const _Float16 *)V; a.ldv = ldv; a.kv_heads = c.kv_heads;
    a.ck = (uint8_t *)c.k; a.cv = (uint8_t *)c.v; a.cks = c.k_scale; a.cvs = c.v_scale;
    a.slots = slots; a.n_slots = (int64_t)c.n_pages * c.page; a.page_log = log2_of(c.page);
    a.T = T; a.D = c.head_dim;
    if (rope) { a.inv_freq = rope->inv_freq; a.positions = positions; a.magnitude = rope->magnitude; a.pairs = rope->rot_dim / 2; }
    return launch_rope(a, rope ? rope->layout : 0, kernel_format(c.format), (hipStream_t)stream) == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}

extern "C" paro_status paro_rope_frequencies_host(int32_t rot_dim, double base, int32_t scaling, double factor, double trained,
                                                  double low, double high, float *inv_freq_host, float *magnitude_host)
{
    if (!inv_freq_host || !magnitude_host) return PARO_ERR_NULL;
    if (scaling < 0 || scaling > 4) return PARO_ERR_UNSUPPORTED;
    if (rot_dim < 2 || rot_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return PARO_ERR_SHAPE;
    if (scaling != 0 && (!(factor >= 1.0) || !std::isfinite(factor))) return PARO_ERR_SHAPE;
    if (scaling == 2 && rot_dim == 2) return PARO_ERR_SHAPE;
    if (scaling >= 3 && (!(trained >= 1.0) || !(low > 0.0) || !(high > low) || !std::isfinite(trained) || !std::isfinite(high))) return PARO_ERR_SHAPE;
    const double two_pi = 6.283185307179586476925;
    if (scaling == 2) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    double c_low = 0, c_high = 0;
    if (scaling == 4) {
        const auto channel = [&](double turns) { return rot_dim * std::log(trained / (two_pi * turns)) / (2 * std::log(base)); };
        const auto clamped = [&](double c) { return std::fmin(std::fmax(c, 0.0), rot_dim - 1.0); };
        c_low = clamped(std::floor(channel(high)));
        c_high = clamped(std::ceil(channel(low)));
        if (c_high - c_low < 0.001) c_high = c_low + 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double s = 1;                            // the part that stays as it is
        if (scaling == 1) s = 0;
        if (scaling == 3) s = std::fmin(std::fmax((trained * f / two_pi - low) / (high - low), 0.0), 1.0);
        if (scaling == 4) s = 1 - std::fmin(std::fmax((i - c_low) / (c_high - c_low), 0.0), 1.0);
        inv_freq_host[i] = (float)(s == 1 ? f : s * f + (1 - s) * (f / factor));
    }
    *magnitude_host = scaling == 4 ? (float)(0.1 * std::log(factor) + 1) : 1.0f;
    return PARO_OK;
}
