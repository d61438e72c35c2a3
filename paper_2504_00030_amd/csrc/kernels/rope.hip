// Rotary tables, and the rotation of a pass's rows with the writes of the paged cache.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

// V neighbouring elements as fp32
template <typename T, int V>
__device__ __forceinline__ void load_v(const T *p, float (&v)[V]) {
    if constexpr (V == 8 && sizeof(T) == 2) {
        const b8_t x = *reinterpret_cast<const b8_t *>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)x[e];
    } else if constexpr (V % 4 == 0) {
#pragma unroll
        for (int w = 0; w < V / 4; ++w) {
            f4_t x;
            if constexpr (sizeof(T) == 4) x = reinterpret_cast<const f4_t *>(p)[w];
            else x = __builtin_convertvector(reinterpret_cast<const b4_t *>(p)[w], f4_t);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * w + e] = x[e];
        }
    } else {
        v[0] = (float)p[0];
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_v(T *p, const float (&v)[V]) {
    if constexpr (V == 8 && sizeof(T) == 2) {
        b8_t x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (__bf16)v[e];
        *reinterpret_cast<b8_t *>(p) = x;
    } else if constexpr (V % 4 == 0) {
#pragma unroll
        for (int w = 0; w < V / 4; ++w) {
            const f4_t x = {v[4 * w], v[4 * w + 1], v[4 * w + 2], v[4 * w + 3]};
            if constexpr (sizeof(T) == 4) reinterpret_cast<f4_t *>(p)[w] = x;
            else reinterpret_cast<b4_t *>(p)[w] = __builtin_convertvector(x, b4_t);
        }
    } else {
        p[0] = (T)v[0];
    }
}

}  // namespace

// ---- tables --------------------------------------------------------------------------------------------------------
// cos(p f_j), sin(p f_j) of STRIP positions of one pair a thread: the first position's angle and the step's by the 64-bit
// functions, the others by the addition theorem in 64 bits (each of the fifteen steps adds less than 2^-51 to the error, 7e-15 together;
// the angle's own rounding is p f_j 2^-53).  Bound by the writes (131072 x 64: 12.8 us, 5.2 TB/s) or, for
// short tables, by two evaluations of sine and cosine (512 x 16: 3.1 us).
template <int STRIP>
__global__ __launch_bounds__(256) void rope_tables_k(const RopeTableArgs a) {
    const uint32_t strips = (uint32_t)((a.n_pos + STRIP - 1) / STRIP);
    const uint64_t t = (uint64_t)workgroup() * 256 + threadIdx.x;
    const uint32_t strip = (uint32_t)(t / (uint32_t)a.half);
    if (strip >= strips) return;
    const int j = (int)(t % (uint32_t)a.half);
    const double f = a.f[j];
    const int p0 = (int)strip * STRIP, n = min(STRIP, a.n_pos - p0);
    double c, s, cf, sf;
    sincos((double)p0 * f, &s, &c);
    sincos(f, &sf, &cf);
    float *co = a.rope_cos + (int64_t)p0 * a.half + j, *si = a.rope_sin + (int64_t)p0 * a.half + j;
#pragma unroll
    for (int i = 0; i < STRIP; ++i) {
        if (i < n) {
            co[(int64_t)i * a.half] = (float)(c * a.magnitude);
            si[(int64_t)i * a.half] = (float)(s * a.magnitude);
        }
        const double cn = c * cf - s * sf;
        s = s * cf + c * sf;
        c = cn;
    }
}

hipError_t launch_rope_tables(const RopeTableArgs &a, hipStream_t s) {
    constexpr int STRIP = 16;
    const int64_t threads = ((int64_t)a.n_pos + STRIP - 1) / STRIP * a.half;
    hipLaunchKernelGGL((rope_tables_k<STRIP>), grid_of((threads + 255) / 256), dim3(256), 0, s, a);
    return hipGetLastError();
}

// ---- rotation and cache --------------------------------------------------------------------------------------------
// A thread takes 2 V elements of a head: V pairs, first and second elements apart (half of the head) or neighbours
// (interleaved), or 2 V neighbours of the part that does not turn and of value heads, each read and written once.
// Nothing is shared between threads, so heads of any size fill the lanes: the units of a row are numbered through.  Bound by
// memory (16384 rows x 48 heads of 128, bf16: 72 us, 5.6 TB/s; a copy reaches 6.1) or by the launch (one row: 2.5 us).
template <typename T, typename OT, int V, bool INTER>
__global__ __launch_bounds__(256) void rope_cache_k(const RopeCacheArgs a, const int row0, const int rows) {
    const uint32_t per_head = (uint32_t)(a.hd + 2 * V - 1) / (2 * V), per_row = per_head * (uint32_t)(a.nq + 2 * a.nkv);
    const uint32_t t = workgroup() * 256 + threadIdx.x;  // below 2^32: the host hands out slabs of rows
    const uint32_t rr = t / per_row;
    if (rr >= (uint32_t)rows) return;
    const int r = row0 + (int)rr;
    const uint32_t rest = t % per_row;
    const int hh = (int)(rest / per_head), u = (int)(rest % per_head);
    const int pos = a.pos[r];
    if (pos < 0 || pos >= a.n_pos) return;
    const T *src;
    OT *dst;
    if (hh < a.nq) {
        src = reinterpret_cast<const T *>(a.q) + (int64_t)r * a.ldq + (int64_t)hh * a.hd;
        dst = reinterpret_cast<OT *>(a.q_out) + (int64_t)r * a.ldqo + (int64_t)hh * a.hd;
    } else {
        const int slot = a.slot[r];
        if (slot < 0 || slot >= a.slots) return;
        const bool value = hh >= a.nq + a.nkv;
        const int h = hh - a.nq - (value ? a.nkv : 0);
        const int64_t o = (((int64_t)(slot >> a.page_shift) * a.nkv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
        src = value ? reinterpret_cast<const T *>(a.v) + (int64_t)r * a.ldv : reinterpret_cast<const T *>(a.k) + (int64_t)r * a.ldk;
        src += (int64_t)h * a.hd;
        dst = reinterpret_cast<OT *>(value ? a.v_pages : a.k_pages) + o * a.hd;
    }
    const int rh = a.rot >> 1, turning = hh < a.nq + a.nkv ? a.rot / (2 * V) : 0;  // units of the head that turn
    if (u < turning) {
        float c[V], s[V];
        load_v<float, V>(a.rope_cos + (int64_t)pos * rh + V * u, c);
        load_v<float, V>(a.rope_sin + (int64_t)pos * rh + V * u, s);
        const int o1 = INTER ? 2 * V * u : V * u, o2 = INTER ? o1 + V : rh + V * u;
        float x[V], y[V];
        load_v<T, V>(src + o1, x);
        load_v<T, V>(src + o2, y);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            // interleaved: pair e of the unit is elements 2e and 2e + 1 of its 2 V
            float &h0 = INTER ? (2 * e < V ? x[2 * e % V] : y[2 * e % V]) : x[e];
            float &h1 = INTER ? (2 * e + 1 < V ? x[(2 * e + 1) % V] : y[(2 * e + 1) % V]) : y[e];
            const float p = h0, q = h1;
            h0 = p * c[e] - q * s[e];
            h1 = q * c[e] + p * s[e];
        }
        store_v<OT, V>(dst + o1, x);
        store_v<OT, V>(dst + o2, y);
    } else {
        const int o = (turning ? a.rot : 0) + 2 * V * (u - turning);
        float x[V], y[V];
        load_v<T, V>(src + o, x);
        const bool two = V > 1 || o + 1 < a.hd;  // (a head of odd size ends in a unit of one element)
        if (two) load_v<T, V>(src + o + V, y);
        store_v<OT, V>(dst + o, x);
        if (two) store_v<OT, V>(dst + o + V, y);
    }
}

template <typename T, typename OT, int V>
static hipError_t launch_rope_v(const RopeCacheArgs &a, hipStream_t s) {
    const int64_t per_row = (int64_t)((a.hd + 2 * V - 1) / (2 * V)) * (a.nq + 2 * a.nkv);
    const int64_t slab = std::max<int64_t>(1, ((int64_t)1 << 31) / per_row);
    for (int64_t row0 = 0; row0 < a.R; row0 += slab) {
        const int64_t rows = std::min<int64_t>(slab, a.R - row0);
        const dim3 grid = grid_of((rows * per_row + 255) / 256);
        if (a.interleaved) hipLaunchKernelGGL((rope_cache_k<T, OT, V, true>), grid, dim3(256), 0, s, a, (int)row0, (int)rows);
        else hipLaunchKernelGGL((rope_cache_k<T, OT, V, false>), grid, dim3(256), 0, s, a, (int)row0, (int)rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, typename OT>
static hipError_t launch_rope_t(const RopeCacheArgs &a, hipStream_t s) {
    auto fits = [](const void *p, size_t bytes, int64_t ld, int n) { return reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld % n == 0; };
    // whole vectors of n: units never cross the end of the turning part, and every head and table row starts on a vector
    auto all_fit = [&](int n) {
        const size_t vi = std::min<size_t>(16, n * sizeof(T)), vo = std::min<size_t>(16, n * sizeof(OT));
        return a.rot % (2 * n) == 0 && a.hd % (2 * n) == 0 && fits(a.rope_cos, 16, 0, n) && fits(a.rope_sin, 16, 0, n) &&
               (a.nq == 0 || (fits(a.q, vi, a.ldq, n) && fits(a.q_out, vo, a.ldqo, n))) &&
               (a.nkv == 0 || (fits(a.k, vi, a.ldk, n) && fits(a.v, vi, a.ldv, n)));
    };
    if constexpr (sizeof(T) == 2 && sizeof(OT) == 2) {
        if (all_fit(8)) return launch_rope_v<T, OT, 8>(a, s);
    }
    return all_fit(4) ? launch_rope_v<T, OT, 4>(a, s) : launch_rope_v<T, OT, 1>(a, s);
}

hipError_t launch_rope_cache(const RopeCacheArgs &a, hipStream_t s) {
    if (a.dtype == DT_F32) return a.out_dtype == DT_F32 ? launch_rope_t<float, float>(a, s) : launch_rope_t<float, __bf16>(a, s);
    return a.out_dtype == DT_F32 ? launch_rope_t<__bf16, float>(a, s) : launch_rope_t<__bf16, __bf16>(a, s);
}

}  // namespace sd
