// Attention of one new token of every sequence over a paged key-value cache:
//
//      o_h = sum_t p_t v_t / sum_t p_t,   p_t = 2^(x_t - m),   x_t = log2(e) scale q_h . k_t,   m = the running maximum
//
// Bound by HBM: 2 head_dim elements per token and key-value head are read once and used for q_heads / kv_heads
// queries, a few flops per byte.
//
// Work is cut into units of 32 tokens of one (sequence, key-value head, 16 of its query heads), numbered one
// sequence after the other, and every block takes the same number of consecutive units, whatever the lengths are: a
// block finds its place from a sum over the lengths.  The 4 waves of a block take its units in turn, each with a
// running maximum of its own, and join through LDS where a sequence's head ends; heads that several blocks share leave
// fp32 partial results in the scratch, and the block that arrives last (a counter per head; nobody waits) joins them in
// the order of their units, so that results do not depend on timing.
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

#include "kv_common.h"

namespace paro {

constexpr int kUnit = 32;                        // tokens of a unit
constexpr int kAttnWaves = 4;
constexpr int kAttnBlocks = 512;                 // most blocks of a launch: 2 for every compute unit
constexpr int kQueries = 16;                     // query heads of a unit: the N of the matrix instruction
constexpr float kPShift = 15.0f;                 // p is held 2^15 times
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const uint8_t *k, *v, *ks, *vs;
    const _Float16 *q;
    const int32_t *table, *lengths;
    _Float16 *o;
    float *lse;
    uint32_t *arrived;                           // [batch][kv_heads * chunks]
    float *partial;                              // [2 * blocks][kQueries * (D + 2)]
    int64_t ldq, ldo, ld_table;
    int page_log, n_pages, kv_heads, group, chunks, width, batch, window;
    float scale;                                 // with log2(e)
};

__device__ inline void agent_store(float *p, float a, float b)
{
    union { float f[2]; uint64_t u; } w = {{a, b}};
    __hip_atomic_store((uint64_t *)p, w.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void agent_load(const float *p, float &a, float &b)
{
    union { uint64_t u; float f[2]; } w;
    w.u = __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    a = w.f[0]; b = w.f[1];
}

// maximum / sum over the 4 lanes that hold one query (lanes n, n + 16, n + 32, n + 48)
__device__ inline float max4(float x) { x = fmaxf(x, __shfl_xor(x, 16)); return fmaxf(x, __shfl_xor(x, 32)); }
__device__ inline float sum4(float x) { x += __shfl_xor(x, 16); return x + __shfl_xor(x, 32); }

// [first token, end) that sequence b attends to, and the units that cover it (at least one, so that every output is written)
struct Span { int lo, hi, unit0, units; };
__device__ inline Span span_of(const AttnArgs &a, int b)
{
    Span s;
    const int64_t room = (int64_t)a.width << a.page_log;
    int n = a.lengths[b];
    n = n < 0 ? 0 : n;
    if (n > room) n = (int)room;
    s.hi = n;
    s.lo = a.window > 0 && n > a.window ? n - a.window : 0;
    s.unit0 = s.lo / kUnit;
    s.units = n > 0 ? (n - 1) / kUnit - s.unit0 + 1 : 1;
    return s;
}

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

template <int D, int FMT>
struct Operand {
    static constexpr int kKeyLoads = FMT == 0 ? D / 32 : D / 64;          // 16-byte requests per 16 tokens
    static constexpr int kRowWords = D / 16 * (FMT == 0 ? 2 : 1) / 4;     // dwords of a value row in a lane
};

// 16 tokens of keys: token lane % 16, units of channels lane / 16 + 4 s
template <int D, int FMT>
__device__ inline void load_keys(U4 *k, const uint8_t *page, int page_log, int tok, int lane)
{
#pragma unroll
    for (int s = 0; s < Operand<D, FMT>::kKeyLoads; ++s)
        k[s] = *(const U4 *)(page + ((((s * 4 + (lane >> 4)) << page_log) + tok + (lane & 15)) << 4));
}
// 4 rows of values, tokens 4 (lane / 16) + i, channels (lane % 16) * D/16 ...
template <int D, int FMT>
__device__ inline void load_values(uint32_t *v, const uint8_t *page, int tok, int lane)
{
    constexpr int W = Operand<D, FMT>::kRowWords;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint8_t *p = page + (tok + 4 * (lane >> 4) + i) * (D * (FMT == 0 ? 2 : 1)) + (lane & 15) * (4 * W);
        if constexpr (W % 4 == 0)
#pragma unroll
            for (int x = 0; x < W; x += 4) { const U4 y = *(const U4 *)(p + 4 * x); v[i * W + x] = y[0]; v[i * W + x + 1] = y[1]; v[i * W + x + 2] = y[2]; v[i * W + x + 3] = y[3]; }
        else if constexpr (W == 2) { const uint2 y = *(const uint2 *)p; v[i * W] = y.x; v[i * W + 1] = y.y; }
        else v[i * W] = *(const uint32_t *)p;
    }
}

template <int D, int FMT>
__global__ __launch_bounds__(64 * kAttnWaves, D == 256 ? 1 : 2) void paged_attention_kernel(const AttnArgs a)
{
    using Op = Operand<D, FMT>;
    constexpr int R = D / 16, KL = Op::kKeyLoads, VW = Op::kRowWords, EB = FMT == 0 ? 2 : 1;
    constexpr int kRow = D + 4;                  // floats of a row in LDS: rows of 16 queries fall on distinct banks
    constexpr int kPart = kQueries * (D + 2);    // floats of a partial result
    __shared__ __attribute__((aligned(16))) float s_o[kAttnWaves * kQueries * kRow];
    __shared__ float s_m[256], s_l[256];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hc = a.kv_heads * a.chunks;

    // this block's place: lane i sums the units of `per` consecutive sequences
    const int per = (a.batch + 63) / 64;
    uint32_t mine = 0;
    for (int j = 0; j < per; ++j) {
        const int b = lane * per + j;
        if (b < a.batch) mine += (uint32_t)span_of(a, b).units;
    }
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    const uint32_t total = __shfl(upto, 63) * (uint32_t)hc;
    uint32_t share = (total + gridDim.x - 1) / gridDim.x;
    share = (share + kAttnWaves - 1) / kAttnWaves * kAttnWaves;
    const uint32_t begin = blockIdx.x * share;
    if (begin >= total) return;
    const uint32_t end = begin + share < total ? begin + share : total;

    // the sequence that `begin` lies in, and the number of its first unit
    const uint64_t before = __ballot(upto * (uint32_t)hc <= begin);
    const int l0 = __popcll(before);             // lanes whose sequences all lie before
    int b = l0 * per;
    uint32_t base = l0 ? __shfl(upto, l0 - 1) * (uint32_t)hc : 0;
    Span sp = span_of(a, b);
    while (base + (uint32_t)sp.units * hc <= begin) { base += (uint32_t)sp.units * hc; ++b; sp = span_of(a, b); }

    const int64_t head_bytes = (int64_t)D * EB << a.page_log, page_bytes = head_bytes * a.kv_heads;
    const int n = lane & 15, quarter = lane >> 4;

    uint32_t at = begin;
    while (at < end) {
        while (base + (uint32_t)sp.units * hc <= at) { base += (uint32_t)sp.units * hc; ++b; sp = span_of(a, b); }
        const int seg = (int)((at - base) / (uint32_t)sp.units);                  // which (head, chunk) of the sequence
        const uint32_t seg0 = base + (uint32_t)seg * sp.units, seg1 = seg0 + sp.units;
        const int head = seg / a.chunks, q0 = (seg - head * a.chunks) * kQueries;
        const int queries = a.group - q0 < kQueries ? a.group - q0 : kQueries;
        const uint32_t stop = seg1 < end ? seg1 : end;
        const int u0 = sp.unit0 + (int)(at - seg0), u1 = sp.unit0 + (int)(stop - seg0);

        Running<D> st;
        st.clear();
        half8v qf[D / 32];
        {
            const _Float16 *q = a.q + (int64_t)b * a.ldq + (int64_t)(head * a.group + q0 + (n < queries ? n : 0)) * D;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const int c = FMT == 0 ? s * 32 + quarter * 8 : ((s >> 1) * 4 + quarter) * 16 + (s & 1) * 8;
                qf[s] = *(const half8v *)(q + c);
            }
        }
        const int32_t *row = a.table + (int64_t)b * a.ld_table;
        int pages = 0;
        for (int u = u0 + wave, it = 0; u < u1 && sp.hi > 0; u += kAttnWaves, ++it) {
            if ((it & 31) == 0) {                // the pages of this wave's next 32 units, two halves to a unit
                int t = (u + (lane >> 1) * kAttnWaves) * kUnit + (lane & 1) * 16;
                t = t < sp.hi ? t : sp.hi - 1;
                pages = row[t >> a.page_log];
                if ((uint32_t)pages >= (uint32_t)a.n_pages) pages = -1;
            }
            const int t0 = u * kUnit, mask = (1 << a.page_log) - 1;
            int pg[2];
            const uint8_t *vp[2];
            U4 kf[2][KL];
            uint32_t vr[8][VW];
            uint32_t ksc[2], vsc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pg[h] = __builtin_amdgcn_readlane(pages, 2 * (it & 31) + h);
                const int64_t p = pg[h] < 0 ? 0 : pg[h];
                const int tok = (t0 + 16 * h) & mask;
                load_keys<D, FMT>(kf[h], a.k + p * page_bytes + head * head_bytes, a.page_log, tok, lane);
                vp[h] = a.v + p * page_bytes + head * head_bytes;
                if constexpr (FMT == 1) {
                    const int64_t so = ((p * a.kv_heads + head) << a.page_log) + tok + 4 * quarter;
                    ksc[h] = *(const uint32_t *)(a.ks + so);
                    vsc[h] = *(const uint32_t *)(a.vs + so);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) load_values<D, FMT>(vr[4 * h], vp[h], (t0 + 16 * h) & mask, lane);

            float x[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                F4 s4 = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KL; ++s) {
                    if constexpr (FMT == 0) {
                        union { U4 u; half8v h8; } c = {kf[h][s]};
                        s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(c.h8, qf[s], s4, 0, 0, 0);
                    } else {
                        s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of_e4m3(kf[h][s][0], kf[h][s][1], 1.0f), qf[2 * s], s4, 0, 0, 0);
                        s4 = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of_e4m3(kf[h][s][2], kf[h][s][3], 1.0f), qf[2 * s + 1], s4, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[h][i] = s4[i] * a.scale;
                    if constexpr (FMT == 1) x[h][i] *= __uint_as_float(((ksc[h] >> (8 * i)) & 255) << 23);
                }
            }
            // a unit that is not all there: scores -inf, and values 0 (what such places hold may be NaN)
            if (t0 < sp.lo || t0 + kUnit > sp.hi || pg[0] < 0 || pg[1] < 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int t = t0 + 16 * (j >> 2) + 4 * quarter + (j & 3);
                    const bool in = t >= sp.lo && t < sp.hi && pg[j >> 2] >= 0;
                    if (!in) x[j >> 2][j & 3] = -INFINITY;
#pragma unroll
                    for (int w = 0; w < VW; ++w) vr[j][w] = in ? vr[j][w] : 0u;
                    if constexpr (FMT == 1) if (!in) vsc[j >> 2] = (vsc[j >> 2] & ~(255u << (8 * (j & 3)))) | (127u << (8 * (j & 3)));
                }
            }
            float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            top = fmaxf(st.m, max4(top));
            if (__ballot(top > st.m)) {
                const float f = top > st.m ? __builtin_amdgcn_exp2f(st.m - top) : 1.0f;
                st.l *= f;
#pragma unroll
                for (int r = 0; r < R; ++r) st.acc[r] *= f;
                st.m = top;
            }
            const float off = (st.m == -INFINITY ? 0.0f : st.m) - kPShift;
            half8v p, rest;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(x[j >> 2][j & 3] - off);
                st.l += e;
                p[j] = (_Float16)e;
                rest[j] = (_Float16)(e - (float)p[j]);
            }
            // O^T += V^T P^T, one tile of 16 channels after the other
            if constexpr (FMT == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    union { half8v h; uint32_t u[4]; } f;
#pragma unroll
                    for (int y = 0; y < 4; ++y) f.u[y] = __builtin_amdgcn_perm(vr[2 * y + 1][r / 2], vr[2 * y][r / 2], r & 1 ? 0x07060302u : 0x05040100u);
                    st.acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h, p, st.acc[r], 0, 0, 0);
                    st.acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h, rest, st.acc[r], 0, 0, 0);
                }
            } else {
                float vs[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) vs[j] = __uint_as_float(((vsc[j >> 2] >> (8 * (j & 3))) & 255) << 23);
#pragma unroll
                for (int r = 0; r < R; r += 2) {
                    uint32_t c[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) c[j] = f16x2_of_e4m3(vr[j][r / 4], vs[j], (r / 2) & 1);
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        union { half8v h; uint32_t u[4]; } f;
#pragma unroll
                        for (int y = 0; y < 4; ++y) f.u[y] = __builtin_amdgcn_perm(c[2 * y + 1], c[2 * y], z ? 0x07060302u : 0x05040100u);
                        st.acc[r + z] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h, p, st.acc[r + z], 0, 0, 0);
                        st.acc[r + z] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h, rest, st.acc[r + z], 0, 0, 0);
                    }
                }
            }
        }

        // the waves' results side by side in LDS
        const float l = sum4(st.l);
        if (quarter == 0) { s_m[wave * kQueries + n] = st.m; s_l[wave * kQueries + n] = l; }
        if (n < queries) {
            float *o = s_o + (wave * kQueries + n) * kRow;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < R; r += 4)
                    *(F4 *)(o + (quarter * 4 + i) * R + r) = F4{st.acc[r][i], st.acc[r + 1][i], st.acc[r + 2][i], st.acc[r + 3][i]};
        }
        __syncthreads();
        const bool whole = at == seg0 && stop == seg1;
        const int items = queries * (D / 8);     // 8 channels of one query each
        const int64_t out_row = (int64_t)b * a.ldo + (int64_t)(head * a.group + q0) * D;
        const int64_t lse_row = (int64_t)b * a.kv_heads * a.group + head * a.group + q0;
        float *part = a.partial + (size_t)(2 * blockIdx.x + (seg0 >= begin)) * kPart;
        for (int i = tid; i < items; i += 64 * kAttnWaves) {
            const int qi = i / (D / 8), c = (i % (D / 8)) * 8;
            float m = s_m[qi], sum = 0, v[8] = {};
#pragma unroll
            for (int w = 1; w < kAttnWaves; ++w) m = fmaxf(m, s_m[w * kQueries + qi]);
            const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(s_m[w * kQueries + qi] - ref);
                sum += f * s_l[w * kQueries + qi];
                const float *o = s_o + (w * kQueries + qi) * kRow + c;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += f * o[e];
            }
            if (whole) {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                half8v h;
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = (_Float16)(v[e] * inv);
                *(half8v *)(a.o + out_row + (int64_t)qi * D + c) = h;
                if (a.lse && c == 0) a.lse[lse_row + qi] = sum == 0.0f ? -INFINITY : (m - kPShift + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
#pragma unroll
                for (int e = 0; e < 8; e += 2) agent_store(part + 2 * kQueries + qi * D + c + e, v[e], v[e + 1]);
                if (c == 0) agent_store(part + 2 * qi, m, sum);
            }
        }
        if (!whole) {
            // every store of this block is at the agent's point of coherence before its arrival is counted
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            const uint32_t first = seg0 / share, last = (seg1 - 1) / share;        // blocks that share this head
            if (tid == 0) {
                uint32_t *arrived = a.arrived + (size_t)b * hc + seg;
                const uint32_t before_me = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = before_me == last - first;
                if (before_me == last - first) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) {
                // `lots` groups of threads each take every lots-th part; a thread has 8 channels of one query
                const int lots = items < 256 ? 256 / items : 1;
                const int lot = tid / items;
                for (int i = lots > 1 ? tid - lot * items : tid; i < items && lot < (lots > 1 ? lots : 1 << 30); i += lots > 1 ? items : 256) {
                    const int qi = i / (D / 8), c = (i % (D / 8)) * 8;
                    float m = -INFINITY, sum = 0, v[8] = {};
                    constexpr int kBatch = 4;
                    const int my = lots > 1 ? lot : 0;
                    for (uint32_t j = first + my; j <= last; j += (uint32_t)(kBatch * lots)) {
                        float pm[kBatch], pl[kBatch], pv[kBatch][8];
#pragma unroll
                        for (int z = 0; z < kBatch; ++z) {
                            const uint32_t jj = j + z * lots <= last ? j + z * lots : j;
                            const float *pp = a.partial + (size_t)(2 * jj + (seg0 >= jj * share)) * kPart;
                            agent_load(pp + 2 * qi, pm[z], pl[z]);
#pragma unroll
                            for (int e = 0; e < 8; e += 2) agent_load(pp + 2 * kQueries + qi * D + c + e, pv[z][e], pv[z][e + 1]);
                        }
#pragma unroll
                        for (int z = 0; z < kBatch; ++z)
                            if (j + z * lots <= last) {
                                const float top = fmaxf(m, pm[z]), ref = top == -INFINITY ? 0.0f : top;
                                const float f = __builtin_amdgcn_exp2f(m - ref), g = __builtin_amdgcn_exp2f(pm[z] - ref);
                                sum = sum * f + pl[z] * g;
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = v[e] * f + pv[z][e] * g;
                                m = top;
                            }
                    }
                    if (lots > 1) {              // side by side in LDS again
                        float *o = s_o + (lot * items + i) * 8;
                        *(F4 *)o = F4{v[0], v[1], v[2], v[3]};
                        *(F4 *)(o + 4) = F4{v[4], v[5], v[6], v[7]};
                        s_m[lot * items + i] = m;
                        s_l[lot * items + i] = sum;
                    } else {
                        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                        half8v h;
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[e] = (_Float16)(v[e] * inv);
                        *(half8v *)(a.o + out_row + (int64_t)qi * D + c) = h;
                        if (a.lse && c == 0) a.lse[lse_row + qi] = sum == 0.0f ? -INFINITY : (m - kPShift + __builtin_amdgcn_logf(sum)) * kLn2;
                    }
                }
                if (lots > 1) {
                    __syncthreads();
                    if (tid < items) {
                        const int qi = tid / (D / 8), c = (tid % (D / 8)) * 8;
                        float m = -INFINITY, sum = 0, v[8] = {};
                        for (int g = 0; g < lots; ++g) m = fmaxf(m, s_m[g * items + tid]);
                        const float ref = m == -INFINITY ? 0.0f : m;
                        for (int g = 0; g < lots; ++g) {
                            const float f = __builtin_amdgcn_exp2f(s_m[g * items + tid] - ref);
                            sum += f * s_l[g * items + tid];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] += f * s_o[(g * items + tid) * 8 + e];
                        }
                        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                        half8v h;
#pragma unroll
                        for (int e = 0; e < 8; ++e) h[e] = (_Float16)(v[e] * inv);
                        *(half8v *)(a.o + out_row + (int64_t)qi * D + c) = h;
                        if (a.lse && c == 0) a.lse[lse_row + qi] = sum == 0.0f ? -INFINITY : (m - kPShift + __builtin_amdgcn_logf(sum)) * kLn2;
                    }
                }
            }
        }
        __syncthreads();                         // LDS is the next head's
        at = stop;
    }
}

static int attn_chunks(const paro_kv_cache &c, int q_heads) { return (q_heads / c.kv_heads + kQueries - 1) / kQueries; }
static size_t attn_part_bytes(const paro_kv_cache &c) { return sizeof(float) * kQueries * (c.head_dim + 2); }
static size_t attn_scratch_bytes(const paro_kv_cache &c) { return ((size_t)2 * kAttnBlocks * attn_part_bytes(c) + 255) / 256 * 256; }

template <int D, int FMT>
static hipError_t launch_attention(const AttnArgs &a, int blocks, hipStream_t s)
{
    hipLaunchKernelGGL((paged_attention_kernel<D, FMT>), dim3(blocks), dim3(64 * kAttnWaves), 0, s, a);
    return hipGetLastError();
}

}  // namespace paro

extern "C" size_t paro_workspace_exchange_bytes_attention(const paro_kv_cache *cache, int32_t q_heads, int32_t batch)
{
    using namespace paro;
    if (!cache || cache->kv_heads <= 0 || q_heads <= 0 || q_heads % cache->kv_heads || batch <= 0) return 0;
    const size_t counters = (size_t)batch * cache->kv_heads * attn_chunks(*cache, q_heads) * sizeof(uint32_t);
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
    using namespace paro;
    if (const paro_status st = check_cache(cache); st != PARO_OK) return st;
    if (!Q || !O || !block_table || !lengths) return PARO_ERR_NULL;
    const paro_kv_cache &c = *cache;
    if (batch <= 0 || q_heads <= 0 || q_heads % c.kv_heads || table_width <= 0 || window < 0) return PARO_ERR_SHAPE;
    if (ld_table != 0 && ld_table < table_width) return PARO_ERR_SHAPE;
    if (!std::isfinite(scale)) return PARO_ERR_SHAPE;
    if (const paro_status st = check_rows(Q, ldq, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (const paro_status st = check_rows(O, ldo, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (!aligned(block_table, 4) || !aligned(lengths, 4) || (lse && !aligned(lse, 4))) return PARO_ERR_ALIGN;
    // units are numbered with 32 bits, and so are a sequence's tokens
    const int64_t tokens = (int64_t)table_width * c.page;
    const int64_t units = (int64_t)batch * c.kv_heads * attn_chunks(c, q_heads);
    if (tokens > (int64_t)1 << 30 || units > (int64_t)1 << 30 || units * ((tokens + kUnit - 1) / kUnit) > (int64_t)1 << 30) return PARO_ERR_UNSUPPORTED;
    const size_t scratch = attn_scratch_bytes(c);
    if (!ws || ws_bytes < paro_workspace_bytes_attention(cache, q_heads, batch)) return PARO_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return PARO_ERR_ALIGN;

    AttnArgs a;
    a.k = (const uint8_t *)c.k; a.v = (const uint8_t *)c.v; a.ks = c.k_scale; a.vs = c.v_scale;
    a.q = (const _Float16 *)Q; a.table = block_table; a.lengths = lengths; a.o = (_Float16 *)O; a.lse = lse;
    a.arrived = (uint32_t *)((char *)ws + kWsPartialOff);
    a.partial = (float *)((char *)ws + (ws_bytes & ~(size_t)255) - scratch);
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.page_log = log2_of(c.page); a.n_pages = c.n_pages; a.kv_heads = c.kv_heads; a.group = q_heads / c.kv_heads;
    a.chunks = attn_chunks(c, q_heads); a.width = table_width; a.batch = batch; a.window = window;
    a.scale = scale * kLog2e;
    // no more blocks than the longest sequences could fill with a unit for every wave
    int64_t seen = tokens;
    if (window > 0 && window + 2 * kUnit < seen) seen = window + 2 * kUnit;
    const int64_t most = units * ((seen + kUnit - 1) / kUnit);
    const int blocks = (int)(most / kAttnWaves + 1 < kAttnBlocks ? most / kAttnWaves + 1 : kAttnBlocks);
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    switch (c.head_dim * 2 + c.format) {
    case 128: e = launch_attention<64, 0>(a, blocks, s); break;
    case 129: e = launch_attention<64, 1>(a, blocks, s); break;
    case 256: e = launch_attention<128, 0>(a, blocks, s); break;
    case 257: e = launch_attention<128, 1>(a, blocks, s); break;
    case 512: e = launch_attention<256, 0>(a, blocks, s); break;
    default: e = launch_attention<256, 1>(a, blocks, s); break;
    }
    return e == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}
