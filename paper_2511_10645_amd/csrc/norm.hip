// Root-mean-square norm with the residual's addition, in fp16 or with an 8-bit result:
//
//      h = x + r,   y = h / sqrt(mean(h^2) + eps) * w;   E4M3: scale = max|y| / 448 of a row or of 128 channels
//
// Bound by HBM (x, r read, h, y written once: 8 bytes per element) and at few rows by latency.  A row stays in registers
// between the sum of its squares and its results; a row's lanes hold 8 consecutive channels per 16-byte request.  The
// 8-bit form needs no second pass: 1 / sqrt(.) is common to a row, so max|h w| is taken along with the sum of squares
// (rows) or of 16 lanes (128 channels), and code = h w (448 / max|h w|).
#include <cmath>

#include "kv_common.h"

namespace paro {

struct NormArgs {
    const _Float16 *x, *r, *w;
    _Float16 *h, *y;
    uint8_t *codes;
    float *scales;
    int64_t ldx, ldr, ldh, ldy;
    int T, C;
    float eps;
};

constexpr int kNormThreads = 256;
constexpr int kNormRows = 1 << 21;               // a launch holds fewer than 2^32 threads, up to 1024 of them for a row

enum NormOut { kNormF16, kNormRow, kNormGroup };

// LANES threads hold a row, NV x 8 channels each.  LANES < 256: rows of a block are independent (a wave or part of one
// per row); 256 and more: one row per block, sums joined in LDS.
template <int LANES, int NV, NormOut OUT>
__global__ __launch_bounds__(LANES < kNormThreads ? kNormThreads : LANES) void norm_kernel(const NormArgs a)
{
    constexpr int kRows = LANES < kNormThreads ? kNormThreads / LANES : 1;
    const int lane = threadIdx.x % LANES;
    const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const bool on = t < a.T;
    const int vectors = a.C / 8;
    half8v x[NV], r[NV], w[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * 8;
        x[k] = r[k] = w[k] = half8v{};
        if (on && k * LANES + lane < vectors) {
            x[k] = *(const half8v *)(a.x + t * a.ldx + c);
            if (a.r) r[k] = *(const half8v *)(a.r + t * a.ldr + c);
            w[k] = *(const half8v *)(a.w + c);
        }
    }
    float h[NV][8], sum = 0, most[OUT == kNormGroup ? NV : 1];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (k == 0 || OUT == kNormGroup) most[OUT == kNormGroup ? k : 0] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[k][e] = (float)x[k][e] + (float)r[k][e];
            sum = fmaf(h[k][e], h[k][e], sum);
            if constexpr (OUT != kNormF16) {
                float &m = most[OUT == kNormGroup ? k : 0];
                m = fmaxf(m, fabsf(h[k][e] * (float)w[k][e]));
            }
        }
    }
    if (a.h && on)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k * LANES + lane < vectors) {
                half8v o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (_Float16)h[k][e];
                *(half8v *)(a.h + t * a.ldh + (k * LANES + lane) * 8) = o;
            }
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d <<= 1) {
        sum += __shfl_xor(sum, d);
        if constexpr (OUT == kNormRow) most[0] = fmaxf(most[0], __shfl_xor(most[0], d));
    }
    if constexpr (LANES > 64) {
        constexpr int kWaves = (LANES < kNormThreads ? kNormThreads : LANES) / 64, kOfRow = LANES / 64;
        __shared__ float s_sum[kWaves], s_most[kWaves];
        const int wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0) { s_sum[wave] = sum; if constexpr (OUT == kNormRow) s_most[wave] = most[0]; }
        __syncthreads();
        const int first = wave / kOfRow * kOfRow;
        sum = 0;
#pragma unroll
        for (int i = 0; i < kOfRow; ++i) {
            sum += s_sum[first + i];
            if constexpr (OUT == kNormRow) most[0] = i ? fmaxf(most[0], s_most[first + i]) : s_most[first];
        }
    }
    if constexpr (OUT == kNormGroup)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) most[k] = fmaxf(most[k], __shfl_xor(most[k], d));
    if (!on) return;
    const float inv = 1.0f / sqrtf(sum / (float)a.C + a.eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int v = k * LANES + lane;
        if (v >= vectors) continue;
        if constexpr (OUT == kNormF16) {
            half8v o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (_Float16)(h[k][e] * inv * (float)w[k][e]);
            *(half8v *)(a.y + t * a.ldy + v * 8) = o;
        } else {
            const float m = most[OUT == kNormGroup ? k : 0];
            // a maximum below the floor of 1e-30 / 448 takes that scale
            const float scale = fmaxf(m * inv, 1e-30f) / kE4m3Max;
            const float least = inv * (kE4m3Max / 1e-30f);
            // no norm at all (a row of zeros without eps, or NaN in it): every code is NaN
            const float up = m * inv > 1e-30f ? kE4m3Max / m : is_finite(inv) ? fminf(least, 3e38f) : NAN;
            float q[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = h[k][e] * (float)w[k][e] * up;
                q[e] = is_finite(y) ? fminf(fmaxf(y, -kE4m3Max), kE4m3Max) : NAN;
            }
            uint2 o = {e4m3_pack(q[0], q[1], q[2], q[3]), e4m3_pack(q[4], q[5], q[6], q[7])};
            *(uint2 *)(a.codes + t * a.C + v * 8) = o;
            if (OUT == kNormGroup && (v & 15) == 0) a.scales[t * (a.C / 128) + v / 16] = scale;
            if (OUT == kNormRow && v == 0) a.scales[t] = scale;
        }
    }
}

template <int LANES, int NV, NormOut OUT>
static hipError_t launch_norm_as(const NormArgs &a, hipStream_t s)
{
    constexpr int kThreads = LANES < kNormThreads ? kNormThreads : LANES, kRows = kThreads / LANES;
    hipLaunchKernelGGL((norm_kernel<LANES, NV, OUT>), dim3(((unsigned)a.T + kRows - 1) / kRows), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// One 16-byte request for every lane of a row where that takes up to 512 lanes, more of them for longer rows.  Measured: 4096 rows of
// 1024 channels 7.3 us on 128 lanes, 7.8 on 256; one row of 4096 2.45 us on 512 lanes, 2.8 on 256, 3.3 on 128, 4.4 on 64; 2047 rows
// of 5120 13.7 us as 256 x 3, 14.2 as 256 x 4.  8-bit rows up to 4096 channels, whose lanes store 8 bytes at a time, stay on 256
// lanes (4096 of them 19.7 us, 20.4 on 512).  The number of rows plays no part: a row's result is the same in any batch.
template <NormOut OUT>
static hipError_t launch_norm(const NormArgs &a, hipStream_t s)
{
    const int v = a.C / 8;
    if (v <= 16) return launch_norm_as<16, 1, OUT>(a, s);
    if (v <= 64) return launch_norm_as<64, 1, OUT>(a, s);
    if (v <= 128) return launch_norm_as<128, 1, OUT>(a, s);
    if (v <= 256) return launch_norm_as<256, 1, OUT>(a, s);
    if (v <= 512) {
        if constexpr (OUT == kNormF16) return launch_norm_as<512, 1, OUT>(a, s);
        else return launch_norm_as<256, 2, OUT>(a, s);
    }
    if (v <= 768) return launch_norm_as<256, 3, OUT>(a, s);
    if (v <= 1024) return launch_norm_as<256, 4, OUT>(a, s);
    return launch_norm_as<1024, 4, OUT>(a, s);
}

static paro_status norm_checks(const paro_half_t *X, int64_t ldx, const paro_half_t *R, int64_t ldr, const paro_half_t *weight, float eps,
                               int32_t T, int32_t C, paro_half_t *H, int64_t ldh, NormArgs &a)
{
    if (!X || !weight) return PARO_ERR_NULL;
    if (T <= 0 || C <= 0 || !(eps >= 0.0f) || !std::isfinite(eps)) return PARO_ERR_SHAPE;
    if (C % 8) return PARO_ERR_ALIGN;
    if (C > 32768 || T > kNormRows) return PARO_ERR_UNSUPPORTED;
    if (const paro_status st = check_rows(X, ldx, C); st != PARO_OK) return st;
    if (R) if (const paro_status st = check_rows(R, ldr, C); st != PARO_OK) return st;
    if (H) if (const paro_status st = check_rows(H, ldh, C); st != PARO_OK) return st;
    if (!aligned(weight, 16)) return PARO_ERR_ALIGN;
    if (H && ((H == X && ldh != ldx) || (H == R && ldh != ldr))) return PARO_ERR_SHAPE;
    a = {(const _Float16 *)X, (const _Float16 *)R, (const _Float16 *)weight, (_Float16 *)H, nullptr, nullptr, nullptr, ldx, ldr, ldh, 0, T, C, eps};
    return PARO_OK;
}

}  // namespace paro

extern "C" paro_status paro_rms_norm(const paro_half_t *X, int64_t ldx, const paro_half_t *R, int64_t ldr, const paro_half_t *weight,
                                     float eps, int32_t T, int32_t C, paro_half_t *H, int64_t ldh, paro_half_t *Y, int64_t ldy, void *stream)
{
    using namespace paro;
    NormArgs a;
    if (const paro_status st = norm_checks(X, ldx, R, ldr, weight, eps, T, C, H, ldh, a); st != PARO_OK) return st;
    if (const paro_status st = check_rows(Y, ldy, C); st != PARO_OK) return st;
    if (Y == H || (Y == X && ldy != ldx) || (Y == R && ldy != ldr)) return PARO_ERR_SHAPE;
    a.y = (_Float16 *)Y;
    a.ldy = ldy;
    return launch_norm<kNormF16>(a, (hipStream_t)stream) == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}

extern "C" paro_status paro_rms_norm_quantize_e4m3(const paro_half_t *X, int64_t ldx, const paro_half_t *R, int64_t ldr,
                                                   const paro_half_t *weight, float eps, int32_t group, int32_t T, int32_t C,
                                                   paro_half_t *H, int64_t ldh, uint8_t *codes, float *scales, void *stream)
{
    using namespace paro;
    NormArgs a;
    if (!codes || !scales) return PARO_ERR_NULL;
    if (group != 0 && group != kGroup) return PARO_ERR_UNSUPPORTED;
    if (const paro_status st = norm_checks(X, ldx, R, ldr, weight, eps, T, C, H, ldh, a); st != PARO_OK) return st;
    if (group && C % group) return PARO_ERR_SHAPE;
    if (!aligned(codes, 8) || !aligned(scales, 4)) return PARO_ERR_ALIGN;
    a.codes = codes;
    a.scales = scales;
    const hipError_t e = group ? launch_norm<kNormGroup>(a, (hipStream_t)stream) : launch_norm<kNormRow>(a, (hipStream_t)stream);
    return e == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}
