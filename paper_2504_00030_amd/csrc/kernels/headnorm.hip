// RMS norm of every query and key head and its rotation, in one pass over the rows a QKV projection leaves.
//
//   h <- h / sqrt(mean(h^2) + eps) * g,   (h[j], h[j + hd/2]) <- (h[j] c - h[j + hd/2] s, h[j + hd/2] c + h[j] s)
//
// A head is held by a group of lanes (a power of two), four or eight pairs (j, j + hd/2) a lane, so both partners of every
// pair and the whole sum of squares stay in registers and a head is read and written once.  What bounds the kernel is
// memory (16384 rows x 40 heads of 128, bf16 to bf16 65 us, fp32 to fp32 117 us: 5.2 and 5.7 TB/s; a copy of such arrays
// reaches 6.0) or, for small calls, the launch (one row: 2.9 us).
#include "common.hpp"
#include "kv.hpp"
#include "params.hpp"

#include <algorithm>

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

// W vectors of four elements of one half of a head, zeros past its end: neighbours 4 W l .. where whole vectors are loaded,
// every LPH-th element otherwise (W = 1)
template <typename T, int LPH, bool VEC, int W>
__device__ __forceinline__ void load_w(const T *p, int l, int half, f4_t (&v)[W]) {
    if constexpr (VEC) {
        const bool in = 4 * W * l < half;
        if constexpr (sizeof(T) == 2 && W == 2) {
            b8_t x = {};
            if (in) x = *reinterpret_cast<const b8_t *>(p + 8 * l);
            v[0] = f4_t{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
            v[1] = f4_t{(float)x[4], (float)x[5], (float)x[6], (float)x[7]};
        } else {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                v[w] = f4_t{0.f, 0.f, 0.f, 0.f};
                if (in) {
                    if constexpr (sizeof(T) == 4) v[w] = *reinterpret_cast<const f4_t *>(p + 4 * (W * l + w));
                    else v[w] = __builtin_convertvector(*reinterpret_cast<const b4_t *>(p + 4 * (W * l + w)), f4_t);
                }
            }
        }
    } else {
        v[0] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l + e * LPH < half) v[0][e] = (float)p[l + e * LPH];
    }
}

template <typename T, int LPH, bool VEC, int W>
__device__ __forceinline__ void store_w(T *p, int l, int half, const f4_t (&v)[W]) {
    if constexpr (VEC) {
        if (4 * W * l >= half) return;
        if constexpr (sizeof(T) == 2 && W == 2) {
            b8_t x;
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = (__bf16)v[0][e]; x[4 + e] = (__bf16)v[1][e]; }
            *reinterpret_cast<b8_t *>(p + 8 * l) = x;
        } else {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<f4_t *>(p + 4 * (W * l + w)) = v[w];
                else *reinterpret_cast<b4_t *>(p + 4 * (W * l + w)) = __builtin_convertvector(v[w], b4_t);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (l + e * LPH < half) p[l + e * LPH] = (T)v[0][e];
    }
}

// One head: its norm and rotation; u, v hold this lane's elements of the two halves, gu, gv their weights.
template <int LPH, int W>
__device__ __forceinline__ void norm_rotate(f4_t (&u)[W], f4_t (&v)[W], const f4_t (&gu)[W], const f4_t (&gv)[W], float eps, int hd,
                                            const f4_t (&c)[W], const f4_t (&s)[W]) {
    float ss = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int e = 0; e < 4; ++e) ss += u[w][e] * u[w][e] + v[w][e] * v[w][e];
#pragma unroll
    for (int m = LPH / 2; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, WAVE);
    const float inv = 1.f / sqrtf(ss / (float)hd + eps);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const f4_t x = u[w] * inv * gu[w], y = v[w] * inv * gv[w];
        u[w] = x * c[w] - y * s[w];
        v[w] = y * c[w] + x * s[w];
    }
}

}  // namespace

// W: vectors of four pairs a lane holds.  One head a group of lanes: groups that take two, four or eight heads of a row, to
// read the rotation factors once, were slower at every size (16384 rows x 40 heads of 128, bf16: 66 us with one, 72 / 74 / 79
// with two / four / eight; the factors come from the caches either way).
template <typename T, typename OT, int LPH, bool VEC, int W>
__global__ __launch_bounds__(256) void head_norm_k(const HeadNormArgs a) {
    constexpr int GPB = 256 / LPH;
    const uint32_t nh = a.nq + a.nkv;
    const int half = a.hd >> 1;
    const uint32_t item = workgroup() * GPB + threadIdx.x / LPH;  // below 2^32: the host bounds R * nh
    const uint32_t r = item / nh;
    const int hh = (int)(item % nh);
    if (r >= (uint32_t)a.R) return;  // whole groups of lanes leave: the sums below stay inside a group
    const int l = threadIdx.x % LPH;
    const int pos = a.pos[r];
    if (pos < 0 || pos >= a.n_pos) return;
    const bool is_q = hh < a.nq;
    const int h = is_q ? hh : hh - a.nq;
    const T *src = (is_q ? reinterpret_cast<const T *>(a.q) + (int64_t)r * a.ldq : reinterpret_cast<const T *>(a.k) + (int64_t)r * a.ldk) + (int64_t)h * a.hd;
    OT *dst = (is_q ? reinterpret_cast<OT *>(a.q_out) + (int64_t)r * a.ldqo : reinterpret_cast<OT *>(a.k_out) + (int64_t)r * a.ldko) + (int64_t)h * a.hd;
    const float *gw = is_q ? a.q_norm : a.k_norm;
    f4_t u[W], v[W], c[W], s[W], gu[W], gv[W];
    load_w<T, LPH, VEC, W>(src, l, half, u);
    load_w<T, LPH, VEC, W>(src + half, l, half, v);
    load_w<float, LPH, VEC, W>(a.rope_cos + (int64_t)pos * half, l, half, c);
    load_w<float, LPH, VEC, W>(a.rope_sin + (int64_t)pos * half, l, half, s);
    load_w<float, LPH, VEC, W>(gw, l, half, gu);
    load_w<float, LPH, VEC, W>(gw + half, l, half, gv);
    norm_rotate<LPH, W>(u, v, gu, gv, a.eps, a.hd, c, s);
    store_w<OT, LPH, VEC, W>(dst, l, half, u);
    store_w<OT, LPH, VEC, W>(dst + half, l, half, v);
}

template <typename T, typename OT, int LPH, bool VEC, int W>
static hipError_t launch_one(const HeadNormArgs &a, hipStream_t s) {
    const int64_t wgs = ((int64_t)a.R * (a.nq + a.nkv) + 256 / LPH - 1) / (256 / LPH);
    hipLaunchKernelGGL((head_norm_k<T, OT, LPH, VEC, W>), grid_of(wgs), dim3(256), 0, s, a);
    return hipGetLastError();
}

// The group of lanes for heads of hd elements, 8 W of them a lane.
template <typename T, typename OT, bool VEC, int W>
static hipError_t launch_lanes(const HeadNormArgs &a, hipStream_t s) {
    const int need = (a.hd / 2 + 4 * W - 1) / (4 * W);
    if (need <= 4) return launch_one<T, OT, 4, VEC, W>(a, s);
    if (need <= 8) return launch_one<T, OT, 8, VEC, W>(a, s);
    if (need <= 16) return launch_one<T, OT, 16, VEC, W>(a, s);
    if constexpr (W == 1) {  // eight pairs a lane: 512 elements are 32 lanes
        if (need > 32) return launch_one<T, OT, 64, VEC, W>(a, s);
    }
    return launch_one<T, OT, 32, VEC, W>(a, s);
}

template <typename T, typename OT>
static hipError_t launch_head_norm_t(const HeadNormArgs &a, hipStream_t s) {
    if ((int64_t)a.R * (a.nq + a.nkv) > 0x7fffffff) return hipErrorInvalidValue;
    // whole vectors of n: every row, both halves of every head, the tables and the weights start on such a vector
    auto fits = [](const void *p, size_t bytes, int64_t ld, int n) { return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld % n == 0; };
    auto all_fit = [&](int n) {
        return a.hd % (2 * n) == 0 && fits(a.rope_cos, 16, 0, n) && fits(a.rope_sin, 16, 0, n) &&
               (a.nq == 0 || (fits(a.q, n * sizeof(T), a.ldq, n) && fits(a.q_out, n * sizeof(OT), a.ldqo, n) && fits(a.q_norm, 16, 0, n))) &&
               (a.nkv == 0 || (fits(a.k, n * sizeof(T), a.ldk, n) && fits(a.k_out, n * sizeof(OT), a.ldko, n) && fits(a.k_norm, 16, 0, n)));
    };
    // bf16 in and out: eight pairs a lane, so that its loads and stores are 16 bytes as well (16384 rows x 40 heads of 128:
    // 66 against 89 us, 5.1 TB/s)
    if constexpr (sizeof(T) == 2 && sizeof(OT) == 2) {
        if (all_fit(8)) return launch_lanes<T, OT, true, 2>(a, s);
    }
    return all_fit(4) ? launch_lanes<T, OT, true, 1>(a, s) : launch_lanes<T, OT, false, 1>(a, s);
}

hipError_t launch_head_norm(const HeadNormArgs &a, hipStream_t s) {
    if (a.dtype == DT_F32) return a.out_dtype == DT_F32 ? launch_head_norm_t<float, float>(a, s) : launch_head_norm_t<float, __bf16>(a, s);
    return a.out_dtype == DT_F32 ? launch_head_norm_t<__bf16, float>(a, s) : launch_head_norm_t<__bf16, __bf16>(a, s);
}

// The engine's form: the plain result of a layer's QKV projection -> queries (fp32 and two bf16 terms) and the paged
// cache, what the QKV epilogue writes for models without head norms.  A group of lanes per head, value heads included.
// A prompt of 1024 tokens, 48 heads of 128: 18.5 us, 3.4 TB/s (29.7 with every element stored by itself; the projection in
// front takes 159); nine rows of a verification pass: 5.0 us.
template <int LPH>
__global__ __launch_bounds__(256) void qkv_norm_k(const QkvNormArgs a) {
    if (a.active != nullptr && *a.active == 0) return;
    constexpr int GPB = 256 / LPH;
    const int half = a.hd >> 1, nh = a.nq + 2 * a.nkv;
    const int item = blockIdx.x * GPB + threadIdx.x / LPH, l = threadIdx.x % LPH;
    const int r = item / nh, hh = item % nh;
    if (r >= a.R) return;
    const int j = 4 * l, pos = a.row_pos[r], seq = a.row_seq[r];
    f4_t u[1] = {f4_t{0.f, 0.f, 0.f, 0.f}}, v[1] = {u[0]};
    if (j < half) {
        if (a.packed) {  // columns of the re-tiled matrix: eight first elements of pairs, then their eight partners
            const int P = hh * half + j;
            const float *p = a.q_in + (size_t)r * a.ldq + (P >> 3) * 16 + (P & 7);
            u[0] = *reinterpret_cast<const f4_t *>(p);
            v[0] = *reinterpret_cast<const f4_t *>(p + 8);
        } else {
            const float *p = hh < a.nq ? a.q_in + (size_t)r * a.ldq + hh * a.hd
                                       : (hh < a.nq + a.nkv ? a.k_in : a.v_in) + (size_t)r * a.ldkv + (hh - a.nq) % a.nkv * a.hd;
            u[0] = *reinterpret_cast<const f4_t *>(p + j);
            v[0] = *reinterpret_cast<const f4_t *>(p + half + j);
        }
    }
    if (hh < a.nq + a.nkv) {
        const float *gw = hh < a.nq ? a.q_norm : a.k_norm;
        f4_t c[1], s[1], gu[1], gv[1];
        load_w<float, LPH, true, 1>(a.rope_cos + (size_t)pos * half, l, half, c);
        load_w<float, LPH, true, 1>(a.rope_sin + (size_t)pos * half, l, half, s);
        load_w<float, LPH, true, 1>(gw, l, half, gu);
        load_w<float, LPH, true, 1>(gw + half, l, half, gv);
        norm_rotate<LPH, 1>(u, v, gu, gv, a.eps, a.hd, c, s);
    }
    if (j >= half) return;
    // a lane's four neighbours are stored together, except values: those lie across the page (j and hd are multiples of 4)
    auto four = [](bf16_t *p, const f4_t x) { *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])); };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f4_t x = h ? v[0] : u[0];
        const int at = j + h * half;
        if (hh < a.nq) {
            const size_t o = ((size_t)r * a.nq + hh) * a.hd + at;
            *reinterpret_cast<f4_t *>(a.q + o) = x;
            four(a.qb + o, x);
            if (a.qb_lo) {
                f4_t lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) lo[e] = x[e] - bf16_to_f32(f32_to_bf16(x[e]));
                four(a.qb + o + a.qb_lo, lo);
            }
        } else if (hh < a.nq + a.nkv) {
            const size_t o = kv_index_k(a.kv, seq, pos, hh - a.nq, at);
            if (a.kv_dtype == DT_BF16) four(reinterpret_cast<bf16_t *>(a.kv.k) + o, x);
            else *reinterpret_cast<f4_t *>(reinterpret_cast<float *>(a.kv.k) + o) = x;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) kv_store(a.kv, a.kv_dtype, false, seq, pos, hh - a.nq - a.nkv, at + e, x[e]);
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
