// What the kernels of the key-value cache share: the checks of its descriptor, its formats, the conversions to E4M3 and the scores of attention.
#pragma once

#include <cmath>

#include "paro_internal.h"

namespace paro {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr float kE4m3Max = 448.0f;
constexpr int kKvExponentLeast = -15, kKvExponentMost = 8;      // of an E4M3 cache row's scale (include/paro.h)
constexpr int kMxExponentLeast = -23, kMxExponentMost = 13;    // of an MXFP4 cache's scales: all values are fp16 values
constexpr uint32_t kMxNan = 255;                               // the scale byte of 32 channels one of which is not finite
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The cache's formats as the kernels number them.
constexpr int kFp16 = 0, kE4m3 = 1, kMxfp4 = 2;
inline int kernel_format(int format) { return format == 4 ? kMxfp4 : format; }
// Bytes of a token's row of D channels, scale bytes with it.
template <int FMT> __host__ __device__ constexpr int row_bytes(int D) { return FMT == kFp16 ? 2 * D : FMT == kE4m3 ? D : D / 2; }
template <int FMT> __host__ __device__ constexpr int row_scales(int D) { return FMT == kFp16 ? 0 : FMT == kE4m3 ? 1 : D / 32; }

inline bool aligned(const void *p, size_t n) { return (uintptr_t)p % n == 0; }

// The cache's own fields; what a call reads or writes through them is in bounds once this is PARO_OK.
inline paro_status check_cache(const paro_kv_cache *c)
{
    if (!c || !c->k || !c->v) return PARO_ERR_NULL;
    if (c->format != 0 && c->format != 1 && c->format != 4) return PARO_ERR_UNSUPPORTED;
    if (c->format != 0 && (!c->k_scale || !c->v_scale)) return PARO_ERR_NULL;
    if (c->n_pages <= 0 || c->kv_heads <= 0 || c->page <= 0) return PARO_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return PARO_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return PARO_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return PARO_ERR_ALIGN;
    if (c->format != 0 && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))) return PARO_ERR_ALIGN;
    return PARO_OK;
}

// fp16 rows of `width` channels
inline paro_status check_rows(const paro_half_t *p, int64_t ld, int64_t width)
{
    if (!p) return PARO_ERR_NULL;
    if (ld < width) return PARO_ERR_SHAPE;
    if (ld % 8 || !aligned(p, 16)) return PARO_ERR_ALIGN;
    return PARO_OK;
}

inline int log2_of(int n)
{
    int k = 0;
    while ((1 << k) < n) ++k;
    return k;
}

// (x - x == 0 is not that: the compiler may contract it with the product that x came from.)
__device__ inline bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Four fp32 values, within +-448 or NaN, as E4M3 bytes (round to nearest even).
__device__ inline uint32_t e4m3_pack(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Channels 2 SEL, 2 SEL + 1 of a dword of eight E2M1 codes; the scale's exponent counts (255: NaN).
template <int SEL> __device__ inline half2v f16x2_of_e2m1(uint32_t w, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL); }
__device__ inline half8v f16_of_e2m1(uint32_t w, float scale)
{
    const half2v a = f16x2_of_e2m1<0>(w, scale), b = f16x2_of_e2m1<1>(w, scale), c = f16x2_of_e2m1<2>(w, scale), d = f16x2_of_e2m1<3>(w, scale);
    return half8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What is done to scores (paro_scores_t), in units of log2: x = cap tanh(y), y = q . k * per_cap, where there is a cap.
struct Scores {
    float cap, per_cap;                          // 0: no cap
    const float *slopes;                         // by query head, NULL: none
};
inline paro_status check_scores(const paro_scores_t *s, float scale, Scores &to)
{
    to = {};
    if (!std::isfinite(scale * kLog2e)) return PARO_ERR_SHAPE;
    if (!s) return PARO_OK;
    if (!(s->cap >= 0.0f) || !std::isfinite(s->cap * kLog2e) || (s->cap > 0.0f && !std::isfinite(scale / s->cap))) return PARO_ERR_SHAPE;
    if (s->slopes && !aligned(s->slopes, 4)) return PARO_ERR_ALIGN;
    if (s->cap > 0.0f) {
        // Kept within 2^125: capped() takes it 2 log2(e) times, and infinity times a score of 0 would be NaN.  Others are 2^-48 and more, as products
        // of fp16 values are multiples of that, and their tanh is 1 either way.
        to.cap = s->cap * kLog2e;
        to.per_cap = std::fmin(std::fmax(scale / s->cap, -0x1p125f), 0x1p125f);
    }
    to.slopes = s->slopes;
    return PARO_OK;
}

// tanh, by its series below 0.4 (the first term left out is 6e-8 of it) and as 1 - 2 / (e^2y + 1) above (0.38 and more, off by 2^-23):
// the second alone would be off by 2^-24 of the cap however small the score is.
__device__ inline float tanh_series(float y)
{
    const float z = y * y;
    float p = fmaf(z, -1382.0f / 155925.0f, 62.0f / 2835.0f);
    p = fmaf(z, p, -17.0f / 315.0f);
    p = fmaf(z, p, 2.0f / 15.0f);
    p = fmaf(z, p, -1.0f / 3.0f);
    return fmaf(z * p, y, y);
}
__device__ inline float tanh_far(float y)
{
    const float e = __builtin_amdgcn_exp2f(2.0f * kLog2e * fabsf(y));
    return copysignf(fmaf(-2.0f, __builtin_amdgcn_rcpf(e + 1.0f), 1.0f), y);
}
constexpr float kTanhFar = 0.4f;
// N scores' q . k, capped in place.  Caps of up to 64 are taken as (1 - e^-2y) / (1 + e^-2y) alone, which is off by 2^-24 of the cap (2^-18 and less)
// besides 2^-22 of itself, with half the instructions (2048 rows of 32 heads of 128 channels, cap 30: 92 us, 107 with the two forms above; E4M3 102 and 154).  Others have those,
// the second where a lane of the wave needs it.
constexpr float kNearCap = 64.0f * kLog2e;
template <int N>
__device__ inline void capped(float (&x)[N], const Scores &s)
{
    if (s.cap <= kNearCap) {
        const float k = -2.0f * kLog2e * fabsf(s.per_cap), cap = s.per_cap < 0 ? -s.cap : s.cap;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float e = __builtin_amdgcn_exp2f(fabsf(x[j]) * k), y = (1.0f - e) * __builtin_amdgcn_rcpf(1.0f + e);
            x[j] = cap * copysignf(y, x[j]);
        }
        return;
    }
    float most = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) { x[j] *= s.per_cap; most = fmaxf(most, fabsf(x[j])); }
    if (__ballot(most >= kTanhFar)) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float near = tanh_series(x[j]), far = tanh_far(x[j]);
            x[j] = s.cap * (fabsf(x[j]) >= kTanhFar ? far : near);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = s.cap * tanh_series(x[j]);
    }
}

}  // namespace paro
