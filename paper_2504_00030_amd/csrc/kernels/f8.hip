// e4m3 product with block scales, and the quantiser of its rows.
//
//   y[r][n] = sum_b xs[b][r] ws[n / 128][b] sum_{k in block b} x[r][k] w[n][k],   blocks of 128 columns
//
// v_mfma_f32_16x16x128_f8f6f4 multiplies exactly one block: its result, started from zero, is the inner sum of 16 rows
// of w by 16 rows of x, and one fused multiply-add per element adds it to the fp32 accumulators with the product of
// the two scales.  w is the first operand, so a lane's four results are four neighbouring columns of one row of y:
// they share one scale product, and they are stored together.  The instruction's k order inside a block is free as
// long as both operands use the same one: lane l holds row l % 16 and the 16-byte chunks l / 16 and l / 16 + 4 of the
// block's eight, so that each load of a wave covers whole halves of 128-byte lines of the row-major operands.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>

namespace sd {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef float f2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b4_t __attribute__((ext_vector_type(4)));
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

namespace {

constexpr int F8_BLOCK = 128;
constexpr float F8_MAX = 448.f;
constexpr float F8_LEAST = 0x1p-96f;  // least magnitude a block counts with: 448 / a and a / 448 stay normal numbers

__device__ __forceinline__ f4_t mfma_f8(const u4_t &a0, const u4_t &a1, const u4_t &b0, const u4_t &b1) {
    const v8i_t a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
    const v8i_t b = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
    const f4_t z = {0.f, 0.f, 0.f, 0.f};
    // formats 0 / 0: both operands e4m3; constant zero scales select the form without block exponents
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, z, 0, 0, 0, 0, 0, 0);
}

// eight e4m3 values as fp16, which holds each of them
__device__ __forceinline__ h8_t to_f16(uint32_t lo, uint32_t hi) {
    const h2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const h2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return h8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// four values scaled and rounded to e4m3
__device__ __forceinline__ uint32_t quant4(const float *v, float f) {
    int q = 0;
    q = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * f, v[1] * f, q, false);
    q = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * f, v[3] * f, q, true);
    return (uint32_t)q;
}

// four neighbouring columns of a row of y
template <typename OT>
__device__ __forceinline__ void store_y4(OT *y, const f4_t v, int n, int N, bool aligned) {
    if (aligned && n + 4 <= N) {
        if constexpr (sizeof(OT) == 4) *reinterpret_cast<f4_t *>(y + n) = v;
        else *reinterpret_cast<b4_t *>(y + n) = __builtin_convertvector(v, b4_t);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) y[n + i] = (OT)v[i];
}

}  // namespace

// ---- quantiser -------------------------------------------------------------------------------------------------
// Sixteen lanes per block of 128 columns, eight columns each.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_f8_k(const T *__restrict__ x, int64_t ldx, int R, int K, int KB,
                                                  uint8_t *__restrict__ q, float *__restrict__ scale) {
    const int64_t grp = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int sub = threadIdx.x & 15;
    if (grp >= (int64_t)R * KB) return;
    const int r = (int)(grp / KB), b = (int)(grp % KB);
    const int k = b * F8_BLOCK + sub * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (k < K) {
        const T *p = x + (int64_t)r * ldx + k;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
    }
    float a = F8_LEAST;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(v[i]));
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) a = fmaxf(a, __shfl_xor(a, m, WAVE));
    const float f = F8_MAX / a;
    if (k < K) {
        *reinterpret_cast<uint2 *>(q + (int64_t)r * K + k) = make_uint2(quant4(v, f), quant4(v + 4, f));
    }
    if (sub == 0) scale[(int64_t)b * R + r] = a / F8_MAX;
}

hipError_t launch_quant_f8(const void *x, int dtype, int64_t ldx, int R, int K, void *q, float *scale, hipStream_t s) {
    const int KB = (K + F8_BLOCK - 1) / F8_BLOCK;
    const int64_t wgs = ((int64_t)R * KB + 15) / 16;
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)wgs), block(256);
    uint8_t *qo = reinterpret_cast<uint8_t *>(q);
    if (dtype == DT_F32) hipLaunchKernelGGL((quant_f8_k<float, false>), grid, block, 0, s, reinterpret_cast<const float *>(x), ldx, R, K, KB, qo, scale);
    else hipLaunchKernelGGL((quant_f8_k<__bf16, false>), grid, block, 0, s, reinterpret_cast<const __bf16 *>(x), ldx, R, K, KB, qo, scale);
    return hipGetLastError();
}

// ---- product: the waves of a workgroup share K ------------------------------------------------------------------
// A workgroup computes 16 NG columns by 16 RB rows of y.  Its NW waves take the blocks of k in turn, each with fragments
// of its own straight from memory (w passes each compute unit once and needs no LDS), and their sums meet in LDS in a
// fixed order.  The e4m3 values enter v_mfma_f32_16x16x32_f16 as fp16, which holds every one of them.
// XIN: type of x: SPEC_F8's bytes with their scales, or fp32 / bf16 rows, which every wave quantises for itself (the
// fragment of one block is 32 values in each of four lanes, so the block's largest is two shuffles away).
enum { X_F8 = 0, X_F32 = 1, X_BF16 = 2 };

template <int XIN> struct RawX { u4_t v[XIN == X_F8 ? 2 : (XIN == X_F32 ? 8 : 4)]; };

// the 32 values of a lane as fp16 and the scale of its block; `dead0`, `dead1`: its first / second 16 lie past the row
template <int XIN>
__device__ __forceinline__ float take_x(const RawX<XIN> &raw, float sx, bool dead0, bool dead1, h8_t (&h)[4]) {
    if constexpr (XIN == X_F8) {
        const u4_t z = {0, 0, 0, 0};
        const u4_t c0 = dead0 ? z : raw.v[0], c1 = dead1 ? z : raw.v[1];
        h[0] = to_f16(c0[0], c0[1]); h[1] = to_f16(c0[2], c0[3]);
        h[2] = to_f16(c1[0], c1[1]); h[3] = to_f16(c1[2], c1[3]);
        return sx;
    } else {
        float v[32];
        if constexpr (XIN == X_F32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(raw.v[i / 4][i % 4]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = i % 2 ? bf16_hi(raw.v[i / 8][i / 2 % 4]) : bf16_lo(raw.v[i / 8][i / 2 % 4]);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (dead0) v[i] = 0.f;
            if (dead1) v[16 + i] = 0.f;
        }
        float m = F8_LEAST;
#pragma unroll
        for (int i = 0; i < 32; ++i) m = fmaxf(m, fabsf(v[i]));
        m = fmaxf(m, __shfl_xor(m, 16, WAVE));
        m = fmaxf(m, __shfl_xor(m, 32, WAVE));
        const float f = F8_MAX / m;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = to_f16(quant4(v + 8 * i, f), quant4(v + 8 * i + 4, f));
        return m / F8_MAX;
    }
}

template <typename OT, int NG, int RB, int NW, int D, int XIN>
__global__ __launch_bounds__(64 * NW) void f8_stream_k(const F8Args a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = lane & 15, g = lane >> 4;
    const int n_tiles = (a.N + 16 * NG - 1) / (16 * NG);
    const int n0 = (blockIdx.x % n_tiles) * 16 * NG, r0 = (blockIdx.x / n_tiles) * 16 * RB;
    const int K = a.K, KB = a.KB;
    constexpr int XB = XIN == X_F32 ? 4 : (XIN == X_BF16 ? 2 : 1);  // bytes of an element of x
    const uint8_t *wp[NG], *xp[RB];
    const float *sp[RB];
    // lanes past the last row or column repeat it; what they compute is not stored
#pragma unroll
    for (int i = 0; i < NG; ++i) wp[i] = a.w + (int64_t)min(n0 + 16 * i + sub, a.N - 1) * K + g * 16;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        const int r = min(r0 + 16 * j + sub, a.R - 1);
        xp[j] = reinterpret_cast<const uint8_t *>(a.x) + ((int64_t)r * a.ldx + g * 16) * XB;
        sp[j] = a.xs + r;
    }
    const float *wsp = a.ws + (int64_t)(n0 / F8_BLOCK) * KB;
    f4_t acc[NG][RB];
#pragma unroll
    for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[i][j] = f4_t{0.f, 0.f, 0.f, 0.f};

    struct Stage { u4_t w[NG][2]; RawX<XIN> x[RB]; float sx[RB], sw; };
    Stage st[D];
    // byte offsets of the lane's two chunks in block b of a row; a chunk past the end reads the row's beginning instead
    auto chunks = [&](int b, int &c0, int &c1) {
        c0 = b * F8_BLOCK; c1 = c0 + 64;
        if (c0 + F8_BLOCK > K) {
            if (c0 + g * 16 >= K) c0 = -g * 16;
            if (c1 + g * 16 >= K) c1 = -g * 16;
        }
    };
    auto load_w = [&](Stage &s, int b) {
        int c0, c1;
        chunks(b, c0, c1);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            s.w[i][0] = *reinterpret_cast<const u4_t *>(wp[i] + c0);
            s.w[i][1] = *reinterpret_cast<const u4_t *>(wp[i] + c1);
        }
        s.sw = wsp[b];
    };
    auto load_x = [&](Stage &s, int b, int j) {
        int c0, c1;
        chunks(b, c0, c1);
#pragma unroll
        for (int i = 0; i < XB; ++i) {
            s.x[j].v[i] = *reinterpret_cast<const u4_t *>(xp[j] + (int64_t)c0 * XB + 16 * i);
            s.x[j].v[XB + i] = *reinterpret_cast<const u4_t *>(xp[j] + (int64_t)c1 * XB + 16 * i);
        }
        if constexpr (XIN == X_F8) s.sx[j] = sp[j][(int64_t)b * a.R];
    };
#pragma unroll
    for (int d = 0; d < D; ++d) {
        const int b = min(wave + d * NW, KB - 1);
        load_w(st[d], b);
#pragma unroll
        for (int j = 0; j < RB; ++j) load_x(st[d], b, j);
    }
    for (int b0 = wave; b0 < KB; b0 += D * NW) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int b = b0 + d * NW;
            if (b >= KB) break;
            Stage &s = st[d];
            // each register set is reloaded as soon as its values have been converted
            const int nb = min(b + D * NW, KB - 1);
            h8_t hw[NG][4];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                hw[i][0] = to_f16(s.w[i][0][0], s.w[i][0][1]); hw[i][1] = to_f16(s.w[i][0][2], s.w[i][0][3]);
                hw[i][2] = to_f16(s.w[i][1][0], s.w[i][1][1]); hw[i][3] = to_f16(s.w[i][1][2], s.w[i][1][3]);
            }
            const float sw = s.sw;
            load_w(s, nb);
            const bool part = (b + 1) * F8_BLOCK > K;
            const bool dead0 = part && b * F8_BLOCK + g * 16 >= K, dead1 = part && b * F8_BLOCK + 64 + g * 16 >= K;
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                h8_t hx[4];
                const float sc = sw * take_x<XIN>(s.x[j], s.sx[j], dead0, dead1, hx);
                load_x(s, nb, j);
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    f4_t t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(hw[i][q], hx[q], t, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[e], sc, acc[i][j][e]);
                }
            }
        }
    }
    __shared__ f4_t red[NW][NG][64];
    OT *y = reinterpret_cast<OT *>(a.y);
    const bool aligned = a.ldy % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % (4 * sizeof(OT)) == 0;
#pragma unroll
    for (int j = 0; j < RB; ++j) {
        if (j > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < NG; ++i) red[wave][i][lane] = acc[i][j];
        __syncthreads();
        const int r = r0 + 16 * j + sub;
        for (int i = wave; i < NG; i += NW) {
            f4_t v = red[0][i][lane];
#pragma unroll
            for (int w = 1; w < NW; ++w) v += red[w][i][lane];
            if (r < a.R) store_y4(y + (int64_t)r * a.ldy, v, n0 + 16 * i + 4 * g, a.N, aligned);
        }
    }
}

template <typename OT, int NG, int RB, int NW, int D, int XIN>
static hipError_t launch_stream(const F8Args &a, hipStream_t s) {
    const int64_t wgs = (int64_t)((a.N + 16 * NG - 1) / (16 * NG)) * ((a.R + 16 * RB - 1) / (16 * RB));
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((f8_stream_k<OT, NG, RB, NW, D, XIN>), dim3((unsigned)wgs), dim3(64 * NW), 0, s, a);
    return hipGetLastError();
}

template <typename OT>
static hipError_t launch_gemm_f8_t(const F8Args &a, hipStream_t s) {
    if (a.R <= 16) return launch_stream<OT, 1, 1, 8, 1, X_F8>(a, s);
    if (a.R <= 32) return launch_stream<OT, 1, 2, 8, 1, X_F8>(a, s);
    return launch_stream<OT, 2, 4, 8, 1, X_F8>(a, s);
}

hipError_t launch_gemm_f8(const F8Args &a, hipStream_t s) {
    return a.y_dtype == DT_F32 ? launch_gemm_f8_t<float>(a, s) : launch_gemm_f8_t<__bf16>(a, s);
}

}  // namespace sd
