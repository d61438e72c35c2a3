// RMS norm of every query and key head and its rotation, in one pass over the rows a QKV projection leaves.
//
//   h <- h / sqrt(mean(h^2) + eps) * g,   (h[j], h[j + hd/2]) <- (h[j] c - h[j + hd/2] s, h[j + hd/2] c + h[j] s)
//
// A head is held by a group of lanes (a power of two), up to four pairs (j, j + hd/2) a lane, so both partners of
// every pair and the whole sum of squares stay in registers.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>

namespace sd {

template <typename T, typename OT, int LPH>
__global__ __launch_bounds__(256) void head_norm_k(const HeadNormArgs a) {
    constexpr int GPB = 256 / LPH;
    const int nh = a.nq + a.nkv, half = a.hd >> 1;
    const int64_t item = (int64_t)blockIdx.x * GPB + threadIdx.x / LPH;
    const int l = threadIdx.x % LPH;
    const bool live = item < (int64_t)a.R * nh;
    const int r = live ? (int)(item / nh) : 0, hh = live ? (int)(item % nh) : 0;
    const bool is_q = hh < a.nq;
    const int h = is_q ? hh : hh - a.nq;
    const T *src = is_q ? reinterpret_cast<const T *>(a.q) + (int64_t)r * a.ldq : reinterpret_cast<const T *>(a.k) + (int64_t)r * a.ldk;
    OT *dst = is_q ? reinterpret_cast<OT *>(a.q_out) + (int64_t)r * a.ldqo : reinterpret_cast<OT *>(a.k_out) + (int64_t)r * a.ldko;
    const float *gw = is_q ? a.q_norm : a.k_norm;
    src += (int64_t)h * a.hd;
    dst += (int64_t)h * a.hd;
    const int pos = live ? a.pos[r] : -1;
    const bool on = pos >= 0 && pos < a.n_pos;
    float u[4], v[4];
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int j = l + e * LPH;
        u[e] = v[e] = 0.f;
        if (on && j < half) { u[e] = (float)src[j]; v[e] = (float)src[j + half]; }
        ss += u[e] * u[e] + v[e] * v[e];
    }
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, WAVE);
    const float inv = 1.f / sqrtf(ss / (float)a.hd + a.eps);
    if (!on) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int j = l + e * LPH;
        if (j >= half) continue;
        const float x = u[e] * inv * gw[j], y = v[e] * inv * gw[j + half];
        const float c = a.rope_cos[(int64_t)pos * half + j], s = a.rope_sin[(int64_t)pos * half + j];
        dst[j] = (OT)(x * c - y * s);
        dst[j + half] = (OT)(y * c + x * s);
    }
}

template <typename T, typename OT>
static hipError_t launch_head_norm_t(const HeadNormArgs &a, hipStream_t s) {
    const int need = (a.hd / 2 + 3) / 4;
    int lph = 4;
    while (lph < need) lph *= 2;
    const int64_t wgs = ((int64_t)a.R * (a.nq + a.nkv) + 256 / lph - 1) / (256 / lph);
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), block(256);
    switch (lph) {
        case 4: hipLaunchKernelGGL((head_norm_k<T, OT, 4>), grid, block, 0, s, a); break;
        case 8: hipLaunchKernelGGL((head_norm_k<T, OT, 8>), grid, block, 0, s, a); break;
        case 16: hipLaunchKernelGGL((head_norm_k<T, OT, 16>), grid, block, 0, s, a); break;
        case 32: hipLaunchKernelGGL((head_norm_k<T, OT, 32>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((head_norm_k<T, OT, 64>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

hipError_t launch_head_norm(const HeadNormArgs &a, hipStream_t s) {
    if (a.dtype == DT_F32) return a.out_dtype == DT_F32 ? launch_head_norm_t<float, float>(a, s) : launch_head_norm_t<float, __bf16>(a, s);
    return a.out_dtype == DT_F32 ? launch_head_norm_t<__bf16, float>(a, s) : launch_head_norm_t<__bf16, __bf16>(a, s);
}

}  // namespace sd
