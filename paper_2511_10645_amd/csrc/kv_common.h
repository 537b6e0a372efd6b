// What the kernels of the key-value cache share: the checks of its descriptor and the conversions to E4M3.
#pragma once

#include "paro_internal.h"

namespace paro {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

constexpr float kE4m3Max = 448.0f;
constexpr int kKvExponentLeast = -15, kKvExponentMost = 8;      // of a cache row's scale (include/paro.h)

inline bool aligned(const void *p, size_t n) { return (uintptr_t)p % n == 0; }

// The cache's own fields; what a call reads or writes through them is in bounds once this is PARO_OK.
inline paro_status check_cache(const paro_kv_cache *c)
{
    if (!c || !c->k || !c->v) return PARO_ERR_NULL;
    if (c->format != 0 && c->format != 1) return PARO_ERR_UNSUPPORTED;
    if (c->format == 1 && (!c->k_scale || !c->v_scale)) return PARO_ERR_NULL;
    if (c->n_pages <= 0 || c->kv_heads <= 0 || c->page <= 0) return PARO_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return PARO_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return PARO_ERR_UNSUPPORTED;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return PARO_ERR_ALIGN;
    if (c->format == 1 && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))) return PARO_ERR_ALIGN;
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

}  // namespace paro
