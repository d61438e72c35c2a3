// RMS norm of every query and key head and its rotation, in one pass over the rows a QKV projection leaves.
//
//   h <- h / sqrt(mean(h^2) + eps) * g,   (h[j], h[j + hd/2]) <- (h[j] c - h[j + hd/2] s, h[j + hd/2] c + h[j] s)
//
// A head is held by a group of lanes (a power of two), four pairs (j, j + hd/2) a lane, so both partners of every pair
// and the whole sum of squares stay in registers and a head is read and written once.  What bounds the kernel is memory
// (large calls) or the launch (small ones).
#include "common.hpp"
#include "kv.hpp"
#include "params.hpp"

#include <algorithm>

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b4_t __attribute__((ext_vector_type(4)));

// pair index of element e of lane l: neighbours where whole vectors are loaded, a stride otherwise
template <int LPH, bool VEC> __device__ __forceinline__ int pair_of(int l, int e) { return VEC ? 4 * l + e : l + e * LPH; }

// four elements of one half of a head, zeros past its end
template <typename T, int LPH, bool VEC>
__device__ __forceinline__ f4_t load4(const T *p, int l, int half) {
    f4_t v = {0.f, 0.f, 0.f, 0.f};
    if constexpr (VEC) {
        if (4 * l < half) {
            if constexpr (sizeof(T) == 4) v = *reinterpret_cast<const f4_t *>(p + 4 * l);
            else v = __builtin_convertvector(*reinterpret_cast<const b4_t *>(p + 4 * l), f4_t);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l + e * LPH < half) v[e] = (float)p[l + e * LPH];
    }
    return v;
}

template <typename T, int LPH, bool VEC>
__device__ __forceinline__ void store4(T *p, int l, int half, const f4_t v) {
    if constexpr (VEC) {
        if (4 * l < half) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<f4_t *>(p + 4 * l) = v;
            else *reinterpret_cast<b4_t *>(p + 4 * l) = __builtin_convertvector(v, b4_t);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l + e * LPH < half) p[l + e * LPH] = (T)v[e];
    }
}

// One head: its norm and rotation; u, v hold this lane's elements of the two halves.
template <int LPH, bool VEC>
__device__ __forceinline__ void norm_rotate(f4_t &u, f4_t &v, const float *g, float eps, int hd, const f4_t c, const f4_t s, int l) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) ss += u[e] * u[e] + v[e] * v[e];
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, WAVE);
    const float inv = 1.f / sqrtf(ss / (float)hd + eps);
    const f4_t x = u * inv * load4<float, LPH, VEC>(g, l, hd >> 1);
    const f4_t y = v * inv * load4<float, LPH, VEC>(g + (hd >> 1), l, hd >> 1);
    u = x * c - y * s;
    v = y * c + x * s;
}

}  // namespace

// HB: heads of one row a group of lanes takes, one after the other (their loads are issued together, and the rotation
// factors of the row's position are read once).
template <typename T, typename OT, int LPH, bool VEC, int HB>
__global__ __launch_bounds__(256) void head_norm_k(const HeadNormArgs a) {
    constexpr int GPB = 256 / LPH;
    const uint32_t nh = a.nq + a.nkv, units = (nh + HB - 1) / HB;
    const int half = a.hd >> 1;
    const uint32_t item = blockIdx.x * GPB + threadIdx.x / LPH;  // below 2^31 + GPB: the host bounds R * nh
    const uint32_t r = item / units, h0 = (item % units) * HB;
    if (r >= (uint32_t)a.R) return;  // whole groups of lanes leave: the sums below stay inside a group
    const int l = threadIdx.x % LPH;
    const int pos = a.pos[r];
    if (pos < 0 || pos >= a.n_pos) return;
    const T *src[HB];
    f4_t u[HB], v[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        const int hh = min(h0 + i, nh - 1);
        src[i] = hh < a.nq ? reinterpret_cast<const T *>(a.q) + (int64_t)r * a.ldq + (int64_t)hh * a.hd
                           : reinterpret_cast<const T *>(a.k) + (int64_t)r * a.ldk + (int64_t)(hh - a.nq) * a.hd;
        u[i] = load4<T, LPH, VEC>(src[i], l, half);
        v[i] = load4<T, LPH, VEC>(src[i] + half, l, half);
    }
    const f4_t c = load4<float, LPH, VEC>(a.rope_cos + (int64_t)pos * half, l, half);
    const f4_t s = load4<float, LPH, VEC>(a.rope_sin + (int64_t)pos * half, l, half);
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (HB > 1 && h0 + i >= nh) break;
        const int hh = h0 + i;
        const bool is_q = hh < a.nq;
        const float *gw = is_q ? a.q_norm : a.k_norm;
        OT *dst = is_q ? reinterpret_cast<OT *>(a.q_out) + (int64_t)r * a.ldqo + (int64_t)hh * a.hd
                       : reinterpret_cast<OT *>(a.k_out) + (int64_t)r * a.ldko + (int64_t)(hh - a.nq) * a.hd;
        norm_rotate<LPH, VEC>(u[i], v[i], gw, a.eps, a.hd, c, s, l);
        store4<OT, LPH, VEC>(dst, l, half, u[i]);
        store4<OT, LPH, VEC>(dst + half, l, half, v[i]);
    }
}

template <typename T, typename OT, int LPH>
static hipError_t launch_head_norm_lanes(const HeadNormArgs &a, bool vec, hipStream_t s) {
    const int64_t heads = (int64_t)a.R * (a.nq + a.nkv);
    // four heads a group of lanes once that still leaves every compute unit its 2048 threads
    const bool many = vec && heads / 4 * LPH >= 256 * 2048;
    const int units = many ? (a.nq + a.nkv + 3) / 4 : a.nq + a.nkv;
    const dim3 grid((unsigned)(((int64_t)a.R * units + 256 / LPH - 1) / (256 / LPH))), block(256);
    if (many) hipLaunchKernelGGL((head_norm_k<T, OT, LPH, true, 4>), grid, block, 0, s, a);
    else if (vec) hipLaunchKernelGGL((head_norm_k<T, OT, LPH, true, 1>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((head_norm_k<T, OT, LPH, false, 1>), grid, block, 0, s, a);
    return hipGetLastError();
}

template <typename T, typename OT>
static hipError_t launch_head_norm_t(const HeadNormArgs &a, hipStream_t s) {
    if ((int64_t)a.R * (a.nq + a.nkv) > 0x7fffffff) return hipErrorInvalidValue;
    // whole vectors of four: every row, both halves of every head, the tables and the weights start on such a vector
    auto fits = [](const void *p, size_t size, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && ld % 4 == 0; };
    const bool vec = a.hd % 8 == 0 && fits(a.rope_cos, 4, 0) && fits(a.rope_sin, 4, 0) &&
                     (a.nq == 0 || (fits(a.q, sizeof(T), a.ldq) && fits(a.q_out, sizeof(OT), a.ldqo) && fits(a.q_norm, 4, 0))) &&
                     (a.nkv == 0 || (fits(a.k, sizeof(T), a.ldk) && fits(a.k_out, sizeof(OT), a.ldko) && fits(a.k_norm, 4, 0)));
    const int need = (a.hd / 2 + 3) / 4;  // lanes of a head
    if (need <= 4) return launch_head_norm_lanes<T, OT, 4>(a, vec, s);
    if (need <= 8) return launch_head_norm_lanes<T, OT, 8>(a, vec, s);
    if (need <= 16) return launch_head_norm_lanes<T, OT, 16>(a, vec, s);
    if (need <= 32) return launch_head_norm_lanes<T, OT, 32>(a, vec, s);
    return launch_head_norm_lanes<T, OT, 64>(a, vec, s);
}

hipError_t launch_head_norm(const HeadNormArgs &a, hipStream_t s) {
    if (a.dtype == DT_F32) return a.out_dtype == DT_F32 ? launch_head_norm_t<float, float>(a, s) : launch_head_norm_t<float, __bf16>(a, s);
    return a.out_dtype == DT_F32 ? launch_head_norm_t<__bf16, float>(a, s) : launch_head_norm_t<__bf16, __bf16>(a, s);
}

// The engine's form: the plain result of a layer's QKV projection -> queries (fp32 and two bf16 terms) and the paged
// cache, what the QKV epilogue writes for models without head norms.  A group of lanes per head, value heads included.
template <int LPH>
__global__ __launch_bounds__(256) void qkv_norm_k(const QkvNormArgs a) {
    if (a.active != nullptr && *a.active == 0) return;
    constexpr int GPB = 256 / LPH;
    const int half = a.hd >> 1, nh = a.nq + 2 * a.nkv;
    const int item = blockIdx.x * GPB + threadIdx.x / LPH, l = threadIdx.x % LPH;
    const int r = item / nh, hh = item % nh;
    if (r >= a.R) return;
    const int j = 4 * l, pos = a.row_pos[r], seq = a.row_seq[r];
    f4_t u = {0.f, 0.f, 0.f, 0.f}, v = u, c = u, s = u;
    if (j < half) {
        if (a.packed) {  // columns of the re-tiled matrix: eight first elements of pairs, then their eight partners
            const int P = hh * half + j;
            const float *p = a.q_in + (size_t)r * a.ldq + (P >> 3) * 16 + (P & 7);
            u = *reinterpret_cast<const f4_t *>(p);
            v = *reinterpret_cast<const f4_t *>(p + 8);
        } else {
            const float *p = hh < a.nq ? a.q_in + (size_t)r * a.ldq + hh * a.hd
                                       : (hh < a.nq + a.nkv ? a.k_in : a.v_in) + (size_t)r * a.ldkv + (hh - a.nq) % a.nkv * a.hd;
            u = *reinterpret_cast<const f4_t *>(p + j);
            v = *reinterpret_cast<const f4_t *>(p + half + j);
        }
    }
    if (hh < a.nq + a.nkv) {
        c = load4<float, LPH, true>(a.rope_cos + (size_t)pos * half, l, half);
        s = load4<float, LPH, true>(a.rope_sin + (size_t)pos * half, l, half);
        norm_rotate<LPH, true>(u, v, hh < a.nq ? a.q_norm : a.k_norm, a.eps, a.hd, c, s, l);
    }
    if (j >= half) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (hh < a.nq) {
            const size_t o = ((size_t)r * a.nq + hh) * a.hd + j + e;
            a.q[o] = u[e];
            a.q[o + half] = v[e];
            store_split_bf16(a.qb, o, a.qb_lo, u[e]);
            store_split_bf16(a.qb, o + half, a.qb_lo, v[e]);
        } else {
            const bool is_k = hh < a.nq + a.nkv;
            const int kvh = hh - a.nq - (is_k ? 0 : a.nkv);
            kv_store(a.kv, a.kv_dtype, is_k, seq, pos, kvh, j + e, u[e]);
            kv_store(a.kv, a.kv_dtype, is_k, seq, pos, kvh, j + e + half, v[e]);
        }
    }
}

hipError_t launch_qkv_norm(const QkvNormArgs &a, hipStream_t s) {
    if (a.hd % 8 || a.hd > 512 || (a.packed && a.hd % 16)) return hipErrorInvalidValue;
    const int need = (a.hd / 2 + 3) / 4, lph = need <= 8 ? 8 : (need <= 16 ? 16 : (need <= 32 ? 32 : 64));
    const int64_t wgs = ((int64_t)a.R * (a.nq + 2 * a.nkv) + 256 / lph - 1) / (256 / lph);
    if (wgs * (256 / lph) > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), block(256);
    switch (lph) {
        case 8: hipLaunchKernelGGL((qkv_norm_k<8>), grid, block, 0, s, a); break;
        case 16: hipLaunchKernelGGL((qkv_norm_k<16>), grid, block, 0, s, a); break;
        case 32: hipLaunchKernelGGL((qkv_norm_k<32>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((qkv_norm_k<64>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace sd
