// e4m3 product with block scales, and the quantiser of its rows.
//
//   y[r][n] = sum_b xs[b][r] ws[n / 128][b] sum_{k in block b} x[r][k] w[n][k],   blocks of 128 columns
//
// The matrix instructions sum one block from zero, 16 rows of w by 16 rows of x, and one fused multiply-add per element
// adds the result to the fp32 accumulators with the product of the two scales.  w is the first operand, so a lane's four
// results are four neighbouring columns of one row of y: they share one scale product, and they are stored together.  The
// k order inside a block is free as long as both operands use the same one: lane l holds row l % 16 and the 16-byte
// chunks l / 16 and l / 16 + 4 of the block's eight, so that each load of a wave covers whole halves of 128-byte lines of
// the row-major operands.
//
// How the products of a block are summed.  v_mfma_f32_16x16x128_f8f6f4 takes the whole block at once, at twice the rate
// of the 16-bit instructions, but inside each group of eight neighbouring products it drops what lies below 2^-13 of the
// power of two of the largest one (measured: 2^16 + 2^3 comes out whole, 2^16 + 2^2 as 2^16).  Its results are 3e-5 off in
// the 2-norm.  A bf16 result rounds by 2e-3, and the instruction serves it; an fp32 result is summed from the values as
// fp16 (which holds every e4m3 value, so the products are exact) by v_mfma_f32_16x16x32_f16, and is 1e-7 off.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>
#include <type_traits>

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

// a lane's 32 values of a fragment as fp16, and the two of its dwords `v` of them alone
__device__ __forceinline__ void widen(const u4_t &c0, const u4_t &c1, h8_t (&h)[4]) {
    h[0] = to_f16(c0[0], c0[1]); h[1] = to_f16(c0[2], c0[3]);
    h[2] = to_f16(c1[0], c1[1]); h[3] = to_f16(c1[2], c1[3]);
}
__device__ __forceinline__ void widen2(const u4_t &c0, const u4_t &c1, h8_t (&h)[4], int v) {
    const uint32_t d = v < 4 ? c0[v] : c1[v - 4];
    const h2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(d, 1.f, true);
    h[v >> 1][(v & 1) * 4] = a[0]; h[v >> 1][(v & 1) * 4 + 1] = a[1];
    h[v >> 1][(v & 1) * 4 + 2] = b[0]; h[v >> 1][(v & 1) * 4 + 3] = b[1];
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

template <int N> using num = std::integral_constant<int, N>;
// f(num<0>) .. f(num<N - 1>)
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(num<N - 1>());
    }
}

}  // namespace

// ---- quantiser -------------------------------------------------------------------------------------------------
// Sixteen lanes per block of 128 columns, eight columns each: x is read once, and the block's largest is four shuffles
// away.  VEC: the rows start on 16 bytes, so that the eight columns are one or two loads.  Bound by memory (4096 x 14336 bf16:
// 35 us, 5.0 TB/s read and written) or, for few rows, by the launch (9 x 5120 fp32: 2.5 us).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quant_f8_k(const T *__restrict__ x, int64_t ldx, int R, int K, int KB,
                                                  uint8_t *__restrict__ q, float *__restrict__ scale) {
    const uint32_t grp = workgroup() * 16 + (threadIdx.x >> 4);  // below 2^32: the host bounds R * KB
    const int sub = threadIdx.x & 15;
    const uint32_t r = grp / KB, b = grp % KB;
    if (r >= (uint32_t)R) return;
    const int k = b * F8_BLOCK + sub * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (k < K) {
        const T *p = x + (int64_t)r * ldx + k;
        if constexpr (VEC && sizeof(T) == 4) {
            const f4_t u0 = *reinterpret_cast<const f4_t *>(p), u1 = *reinterpret_cast<const f4_t *>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = u0[i]; v[4 + i] = u1[i]; }
        } else if constexpr (VEC) {
            const u4_t u = *reinterpret_cast<const u4_t *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i % 2 ? bf16_hi(u[i / 2]) : bf16_lo(u[i / 2]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)p[i];
        }
    }
    float a = F8_LEAST;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, fabsf(v[i]));
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) a = fmaxf(a, __shfl_xor(a, m, WAVE));
    const float f = F8_MAX / a;
    if (k < K) *reinterpret_cast<uint2 *>(q + (int64_t)r * K + k) = make_uint2(quant4(v, f), quant4(v + 4, f));
    if (sub == 0) scale[(int64_t)b * R + r] = a / F8_MAX;
}

template <typename T>
static void launch_quant_t(const void *x, int64_t ldx, int R, int K, int KB, void *q, float *scale, dim3 grid, hipStream_t s) {
    const T *p = reinterpret_cast<const T *>(x);
    uint8_t *o = reinterpret_cast<uint8_t *>(q);
    if (reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * sizeof(T) % 16 == 0)
        hipLaunchKernelGGL((quant_f8_k<T, true>), grid, dim3(256), 0, s, p, ldx, R, K, KB, o, scale);
    else
        hipLaunchKernelGGL((quant_f8_k<T, false>), grid, dim3(256), 0, s, p, ldx, R, K, KB, o, scale);
}

hipError_t launch_quant_f8(const void *x, int dtype, int64_t ldx, int R, int K, void *q, float *scale, hipStream_t s) {
    const int KB = (K + F8_BLOCK - 1) / F8_BLOCK;
    if ((int64_t)R * KB > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid = grid_of(((int64_t)R * KB + 15) / 16);
    if (dtype == DT_F32) launch_quant_t<float>(x, ldx, R, K, KB, q, scale, grid, s);
    else launch_quant_t<__bf16>(x, ldx, R, K, KB, q, scale, grid, s);
    return hipGetLastError();
}

// ---- product: the waves of a workgroup share K ------------------------------------------------------------------
// A workgroup computes 16 NG columns by 16 RB rows of y.  Its NW waves take the blocks of k in turn, each with fragments
// of its own straight from memory (no wave needs another's, so there is no LDS to fill), and their sums meet in LDS in a
// fixed order.  The e4m3 values enter v_mfma_f32_16x16x32_f16 as fp16, which holds every one of them.
// Bound by the stream of w from memory where w is large (1 x 28672 x 4096: 24.6 us, 4.8 TB/s; 9 x 5120 x 13824: 18 us, 3.9 TB/s;
// 9 x 4096 x 14336: 13.8 us, 4.3 TB/s), by the latency of each wave's few loads where it is small (1 x 2048 x 2048: 3.8 us).
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
    const uint32_t wg = workgroup();
    const int n0 = (wg % n_tiles) * 16 * NG, r0 = (wg / n_tiles) * 16 * RB;
    if (r0 >= a.R) return;
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
    // multiplies block b, which `s` holds; `more`: `s` is loaded anew, each register as soon as its values have been converted
    auto step = [&](Stage &s, int b, auto more) {
        const int nb = b + D * NW;
        h8_t hw[NG][4];
#pragma unroll
        for (int i = 0; i < NG; ++i) widen(s.w[i][0], s.w[i][1], hw[i]);
        const float sw = s.sw;
        if constexpr (more) load_w(s, nb);
        const bool part = (b + 1) * F8_BLOCK > K;
        const bool dead0 = part && b * F8_BLOCK + g * 16 >= K, dead1 = part && b * F8_BLOCK + 64 + g * 16 >= K;
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            h8_t hx[4];
            const float sc = sw * take_x<XIN>(s.x[j], s.sx[j], dead0, dead1, hx);
            if constexpr (more) load_x(s, nb, j);
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                f4_t t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int q = 0; q < 4; ++q) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(hw[i][q], hx[q], t, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[e], sc, acc[i][j][e]);
            }
        }
    };
    const std::true_type yes;
    const std::false_type no;
    // full rounds while every stage has a block to come (loads past the last block would cost as much as real ones)
    int b0 = wave;
    for (; b0 + (2 * D - 1) * NW < KB; b0 += D * NW) {
#pragma unroll
        for (int d = 0; d < D; ++d) step(st[d], b0 + d * NW, yes);
    }
#pragma unroll
    for (int d = 0; d < 2 * D - 1; ++d) {
        const int b = b0 + d * NW;
        if (b >= KB) break;
        if (d < D - 1 && b + D * NW < KB) step(st[d], b, yes);
        else step(st[d % D], b, no);
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
    hipLaunchKernelGGL((f8_stream_k<OT, NG, RB, NW, D, XIN>), grid_of(wgs), dim3(64 * NW), 0, s, a);
    return hipGetLastError();
}

// ---- product: tiles in LDS -------------------------------------------------------------------------------------
// The workgroup meets once every wave's reads of LDS are done and its copies into LDS, but for the last N, have landed.  (A
// barrier alone promises neither, and __syncthreads() would wait for the last N as well.)
template <int N>
__device__ __forceinline__ void meet_but() {
    static_assert(N < 64, "six bits");
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // no instruction: keeps memory operations on their side
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);  // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A workgroup computes TN columns by TR rows of y with PN x PR waves.  A stage of LDS holds one block of k of both
// operands; S stages go round, and while one multiplies, the others are on their way from memory straight into LDS (16 bytes
// a lane, no registers).  A step cannot be shorter than a copy takes divided by the S - 1 blocks in flight: with two stages
// and one workgroup a compute unit it took 0.8 us whatever the tile (64 x 4096 x 14336, tiles of 64 x 64: 94.5 us with two
// stages, 50.7 with three, 39.5 with four), so the small tiles have three stages.  The large ones have two, which fill LDS,
// and are long enough by themselves.  The stages are separate arrays, and the loop is unrolled over them: the compiler
// then sees that fragment reads do not touch the stages in flight and does not wait for them.  A row of a stage is 128
// bytes, eight chunks; position p of row i holds chunk p ^ (i / 2 % 8), which spreads the sixteen rows a fragment read
// touches over all banks.
// F16: the fragments are turned into fp16 (exact sums), otherwise multiplied as e4m3.
// What bounds it: 4096 x 28672 x 4096 in tiles of 256 x 256 takes 470 us, 2.0 PFLOP/s, with the matrix units busy 52 % of the
// cycles: 5.7 vector instructions for each matrix instruction (four of them additions, the others mostly addresses of the
// copies), and a clock that the power limit holds at 1.8 GHz (zeros instead of data took a tenth less); a library product of
// the same operands without block scales takes 331 us.  With fp32 results 918 us, 1.05 PFLOP/s: half the rate, and four
// vector instructions (conversions, additions) for each matrix instruction, which share the issue with it: without three
// quarters of the additions it would take a tenth less, and the small tiles gained 3 % from offsets kept in registers.
// Measured and not taken: four waves of 128 x 128 each (their accumulators do not fit the vector registers: 1020 us), copies
// through registers (606), 32 x 32 x 64 instructions (spills: 578), all copies of a step at once (485), wave priorities (475).
template <typename OT, bool F16, int TN, int TR, int PN, int PR, int S>
__global__ __launch_bounds__(64 * PN * PR, 2) void f8_tile_k(const F8Args a, const int n_tiles, const int r_tiles, const int shares) {
    constexpr int NT = 64 * PN * PR, WN = TN / PN / 16, WR = TR / PR / 16;
    constexpr int LW = TN * 8 / NT, LX = TR * 8 / NT;  // 16-byte chunks a thread moves per stage
    constexpr int LAG = 2;                             // matrix instructions between a tile's own and its additions
    static_assert(S == 2 || S == 3, "");
    constexpr int SCALES = (TN + TR) * F8_BLOCK, SIZE = SCALES + (S > 2 ? TR * 4 : 0);  // a stage's scales of x, its size
    __shared__ __attribute__((aligned(16))) uint8_t stage0[SIZE];
    __shared__ __attribute__((aligned(16))) uint8_t stage1[SIZE];
    __shared__ __attribute__((aligned(16))) uint8_t stage2[SIZE];  // takes LDS only where it is used
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sub = lane & 15, g = lane >> 4;
    const int wn = wave % PN, wr = wave / PN;
    // consecutive workgroups go round the eight XCDs: each takes one run of tiles, in bands of eight tiles of rows, so that
    // the tiles it works on together share rows of w and x in its L2
    // (a tile's shares of K stand side by side: they run together)
    const int total = n_tiles * r_tiles * shares, per = (total + 7) >> 3;
    const int wg = (int)workgroup(), id = (wg & 7) * per + (wg >> 3);
    if (id >= total || (wg >> 3) >= per) return;
    const int tile = id / shares, share = id % shares;
    const int band = tile / (8 * n_tiles), in_band = tile % (8 * n_tiles), rows_in_band = min(8, r_tiles - band * 8);
    const int n0 = in_band / rows_in_band * TN, r0 = (band * 8 + in_band % rows_in_band) * TR;
    // this share's blocks of K; from here on K and KB are those of the share
    const int b_share = (int)((int64_t)a.KB * share / shares);
    const int KB = (int)((int64_t)a.KB * (share + 1) / shares) - b_share, ld = a.K, K = min(ld - b_share * F8_BLOCK, KB * F8_BLOCK);
    const uint8_t *wb = a.w + (int64_t)n0 * ld + b_share * F8_BLOCK;
    const uint8_t *xb = reinterpret_cast<const uint8_t *>(a.x) + (int64_t)r0 * ld + b_share * F8_BLOCK;

    // copy i of a thread moves chunk `chunk` of row `row` + i NT / 8 of w, or of x for i >= LW; rows past the last repeat it
    const int row = tid >> 3, chunk = (tid & 7) ^ ((tid >> 4) & 7);
    const int last_n = a.N - 1 - n0, last_r = a.R - 1 - r0;
    // the rows of this tile as buffers (a tile's rows span less than 2^31 bytes: the host bounds K)
    const __amdgpu_buffer_rsrc_t wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(wb), 0, min(TN - 1, last_n) * ld + K, 0x27000);
    const __amdgpu_buffer_rsrc_t xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(xb), 0, min(TR - 1, last_r) * ld + K, 0x27000);
    uint32_t offset[LW + LX];  // of the rows of every copy; the large tiles have no registers for them and work them out anew
    if constexpr (S > 2) {
#pragma unroll
        for (int i = 0; i < LW + LX; ++i)
            offset[i] = __umul24(min(row + (i < LW ? i : i - LW) * (NT / 8), i < LW ? last_n : last_r), ld);
    }
    auto copy = [&](int b, int i, uint8_t *stage) {  // 16 bytes a lane, 1 KiB of LDS a wave
        // a chunk past the end of the rows reads the block's first one; it is zeroed before the block is multiplied
        const uint32_t c = b * F8_BLOCK + chunk * 16 < K ? chunk * 16 : 0;
        const int ii = i < LW ? i : i - LW;
        uint32_t o;
        if constexpr (S > 2) {
            o = offset[i] + c;
        } else {
            int own = row;
            asm volatile("" : "+v"(own));  // no instruction: keeps the compiler from holding the offset of every copy in a register
            o = __umul24(min(own + ii * (NT / 8), i < LW ? last_n : last_r), ld) + c;
        }
        uint8_t *to = stage + (i < LW ? 0 : TN * F8_BLOCK) + ii * NT * 16 + wave * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(i < LW ? wbuf : xbuf, (__attribute__((address_space(3))) void *)to, 16, o,
                                                 b * F8_BLOCK, 0, 0);
    };
    f4_t acc[WN][WR];
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int j = 0; j < WR; ++j) acc[i][j] = f4_t{0.f, 0.f, 0.f, 0.f};
    const float *wsp = a.ws + (int64_t)(min(n0 + wn * WN * 16, a.N - 1) / F8_BLOCK) * a.KB + b_share;
    // Scales of a block.  Two stages: loads into registers, a step ahead.  More: those of x go into the stage as well, one copy
    // a wave (64 rows; waves beyond the rows repeat them), so that the copies in flight can be counted, and that of w is a
    // scalar load.
    float xs[WR], ws = 0.f;
    auto load_scales = [&](int b, uint8_t *stage) {
        if constexpr (S == 2) {
            const char *p = reinterpret_cast<const char *>(a.xs + (int64_t)(b_share + b) * a.R + r0);
            int own = wr * WR * 16 + sub;
            asm volatile("" : "+v"(own));
#pragma unroll
            for (int j = 0; j < WR; ++j) xs[j] = *reinterpret_cast<const float *>(p + (uint32_t)min(own + j * 16, last_r) * 4);
            ws = wsp[b];
        } else {
            static_assert(TR % 64 == 0 && TR <= NT, "");
            const __amdgpu_buffer_rsrc_t buf = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<float *>(a.xs + (int64_t)(b_share + b) * a.R + r0), 0, (min(TR - 1, last_r) + 1) * 4, 0x27000);
            const int first = wave * 64 % TR;
            int own = first + lane;
            asm volatile("" : "+v"(own));
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)(stage + SCALES + first * 4), 4,
                                                     min(own, last_r) * 4, 0, 0, 0);
        }
    };
    auto take_scales = [&](int b, const uint8_t *stage) {
        if constexpr (S > 2) {
#pragma unroll
            for (int j = 0; j < WR; ++j) xs[j] = *reinterpret_cast<const float *>(stage + SCALES + (wr * WR * 16 + j * 16 + sub) * 4);
            ws = *(const __attribute__((address_space(4))) float *)(uintptr_t)(wsp + b);
        }
    };
    const int f0 = sub * F8_BLOCK + ((g ^ (sub >> 1)) * 16), f1 = f0 ^ 64;
    auto frag = [&](const uint8_t *p, u4_t &c0, u4_t &c1) {
        c0 = *reinterpret_cast<const u4_t *>(p + f0);
        c1 = *reinterpret_cast<const u4_t *>(p + f1);
    };
    auto add1 = [&](int i, int j, int e, const f4_t t, float sc) {
        acc[i][j][e] = fmaf(t[e], sc, acc[i][j][e]);
        asm volatile("" : "+v"(acc[i][j][e]));  // no instruction: keeps the addition in front of the step's end
    };
    auto add = [&](int i, int j, const f4_t t, float sc) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(t[e], sc, acc[i][j][e]);
        asm volatile("" : "+v"(acc[i][j]));  // no instruction: keeps the additions in front of the barrier at the step's end
    };
    // the last block may be short: its missing columns of x count as zeros
    auto trim = [&](int b, uint8_t *stage) {
        if ((b + 1) * F8_BLOCK > K) {
            if (b * F8_BLOCK + chunk * 16 >= K) {
#pragma unroll
                for (int i = 0; i < LX; ++i) *reinterpret_cast<u4_t *>(stage + TN * F8_BLOCK + (i * NT + tid) * 16) = u4_t{0, 0, 0, 0};
            }
            __syncthreads();
        }
    };
    const int lw = wn * WN * 16 * F8_BLOCK, lx = (TN + wr * WR * 16) * F8_BLOCK;
    u4_t x0[WR], x1[WR], w0[2], w1[2];
    h8_t hx[F16 ? WR : 1][4], hw[2][4];  // fp16 fragments
    // Step b multiplies the stage `cur` while block b + S - 1 is copied into `far` (the stage of step b - 1), CPR copies a row of
    // tiles (all at once they would hold up the matrix instructions behind them).  Fragments are read a row of tiles ahead;
    // in front of the last row, whose fragments are in registers by then, the workgroup meets: `nxt` is complete and nobody
    // reads `cur` any more, and the first fragments of `nxt` are read behind the last row's instructions.
    // `more`: there is a block b + 1; `load`: there is a block b + S - 1.
    // Matrix and vector instructions of a wave alternate (left alone, the scheduler groups them, and each unit waits for
    // the other): a tile's additions follow matrix instructions issued after its own.
    constexpr int CPR = (LW + LX + WN / 2 - 1) / (WN / 2);
    constexpr int FLIGHT = (S - 2) * (LW + LX + 1);  // copies younger than those of block b + 1 when step b meets
    float sc[WR];           // scales of this step
    f4_t t[4];              // the last results; those of a step's last tiles are added in the next one
#pragma unroll
    for (int u = 0; u < 4; ++u) t[u] = f4_t{0.f, 0.f, 0.f, 0.f};
    auto step = [&](int b, uint8_t *cur, uint8_t *nxt, uint8_t *far, auto more, auto load) __attribute__((always_inline)) {
        float old[LAG];
#pragma unroll
        for (int q = 0; q < LAG; ++q) old[q] = sc[WR - LAG + q];
#pragma unroll
        for (int j = 0; j < WR; ++j) sc[j] = xs[j] * ws;
        auto meet = [&] {
            meet_but<load ? FLIGHT : 0>();
            trim(b + 1, nxt);
            frag(nxt + lw, w0[0], w1[0]);
            take_scales(b + 1, nxt);
        };
        if constexpr (F16) {
#pragma unroll
            for (int j = 0; j < WR; ++j) widen(x0[j], x1[j], hx[j]);
            __builtin_amdgcn_sched_barrier(0);
            // two tiles at a time: four matrix instructions each, in turn
#pragma unroll
            for (int p = 0; p < WN * WR / 2; ++p) {
                const int i = p / (WR / 2), jp = p % (WR / 2);
                if (jp == 0 && i + 1 < WN) frag(cur + lw + (i + 1) * 16 * F8_BLOCK, w0[0], w1[0]);
                if constexpr (more) {
                    if (jp == 0 && i + 1 == WN) {
                        meet();
#pragma unroll
                        for (int j = 0; j < WR; ++j) frag(nxt + lx + j * 16 * F8_BLOCK, x0[j], x1[j]);
                    }
                }
                if constexpr (load) {
                    if (jp == 0 && i == WN / 2 - 1) load_scales(b + S - 1, far);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    const int q = v >> 1, u = 2 * p + (v & 1), j = u % WR;
                    const f4_t z = {0.f, 0.f, 0.f, 0.f};
                    t[u & 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hw[i & 1][q], hx[j][q], q == 0 ? z : t[u & 3], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (load) {
                        const int k = i * CPR + jp * 8 + v;
                        if (jp * 8 + v < CPR && i < WN / 2 && k < LW + LX) copy(b + S - 1, k, far);
                    }
                    const int d = u - 2;  // the pair before, one element of each tile at a time
                    if (d >= 0) add1(d / WR, d % WR, q, t[d & 3], sc[d % WR]);
                    else add1(WN - 1, WR + d, q, t[d & 3], old[LAG + d]);
                    if (jp == WR / 2 - 1 && (i + 1 < WN || more)) widen2(w0[0], w1[0], hw[(i + 1) & 1], v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < WN * WR; ++u) {
                const int i = u / WR, j = u % WR;
                if (j == 0 && i + 1 < WN) frag(cur + lw + (i + 1) * 16 * F8_BLOCK, w0[(i + 1) & 1], w1[(i + 1) & 1]);
                if constexpr (more) {
                    if (j == 0 && i + 1 == WN) meet();
                }
                if constexpr (load) {
                    if (j == 0 && i == WN / 2 - 1) load_scales(b + S - 1, far);
                }
                __builtin_amdgcn_sched_barrier(0);
                t[u & 3] = mfma_f8(w0[i & 1], w1[i & 1], x0[j], x1[j]);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (more) {
                    if (i + 1 == WN) frag(nxt + lx + j * 16 * F8_BLOCK, x0[j], x1[j]);
                }
                if constexpr (load) {
                    if (j % (WR / 2) == 0 && i < WN / 2) {
#pragma unroll
                        for (int q = 0; q < (CPR + 1) / 2; ++q) {
                            const int k = i * CPR + j / (WR / 2) * ((CPR + 1) / 2) + q;
                            if (k < (i + 1) * CPR && k < LW + LX) copy(b + S - 1, k, far);
                        }
                    }
                }
                if (u >= LAG) add((u - LAG) / WR, (u - LAG) % WR, t[(u - LAG) & 3], sc[(u - LAG) % WR]);
                else add(WN - 1, WR - LAG + u, t[(u - LAG) & 3], old[u]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    static_assert(WN % 2 == 0 && WR % 2 == 0 && WN * WR % 4 == 0 && WR >= LAG, "the fragments of w alternate over whole steps");
    auto stage = [&](auto n) -> uint8_t * {
        constexpr int i = n % S;
        if constexpr (i == 0) return stage0;
        else if constexpr (i == 1) return stage1;
        else return stage2;
    };
    // the first S - 1 blocks (a short product's last one over and over)
    each<S - 1>([&](auto n) {
        const int b = min((int)n, KB - 1);
#pragma unroll
        for (int i = 0; i < LW + LX; ++i) copy(b, i, stage(n));
        load_scales(b, stage(n));
    });
    meet_but<FLIGHT>();
    trim(0, stage0);
#pragma unroll
    for (int j = 0; j < WR; ++j) sc[j] = 0.f;
    frag(stage0 + lw, w0[0], w1[0]);
    take_scales(0, stage0);
#pragma unroll
    for (int j = 0; j < WR; ++j) frag(stage0 + lx + j * 16 * F8_BLOCK, x0[j], x1[j]);
    if constexpr (F16) widen(w0[0], w1[0], hw[0]);
    const std::true_type yes;
    const std::false_type no;
    int b = 0;
    // rounds over the stages while every step has a block to load, then up to 2 S - 2 steps that may have none
    for (; b + 2 * S - 2 < KB; b += S)
        each<S>([&](auto n) { step(b + n, stage(n), stage(num<n + 1>()), stage(num<n + S - 1>()), yes, yes); });
    if constexpr (S == 2) {
        // One or two blocks are left.  Both ways share the last step, with its stage known only at run time: with a last step
        // of its own for each, the accumulators met in different registers behind them, through scratch memory (4096 x 28672 x
        // 4224, an odd number of blocks: 483 us, 559 that way; 128 x 128 tiles with fp32 results 951 and 980).
        uint8_t *last = stage0;
        if (b + 1 < KB) {
            step(b++, stage0, stage1, stage1, yes, yes);
            last = stage1;
        }
        step(b, last, nullptr, nullptr, no, no);
    } else {
        auto rest = [&](auto self, auto n) __attribute__((always_inline)) {
            if constexpr (n + 1 < 2 * S - 2) {
                if (b + n + 1 < KB) {
                    uint8_t *const cur = stage(n), *const nxt = stage(num<n + 1>()), *const far = stage(num<n + S - 1>());
                    if constexpr (n < S - 1) {
                        if (b + n + S - 1 < KB) step(b + n, cur, nxt, far, yes, yes);
                        else step(b + n, cur, nxt, far, yes, no);
                    } else {
                        step(b + n, cur, nxt, far, yes, no);
                    }
                    self(self, num<n + 1>());
                    return;
                }
            }
            step(b + n, stage(n), nullptr, nullptr, no, no);
        };
        rest(rest, num<0>());
    }
#pragma unroll
    for (int q = 0; q < LAG; ++q) add(WN - 1, WR - LAG + q, t[(q - LAG) & 3], sc[WR - LAG + q]);
    OT *y = reinterpret_cast<OT *>(a.y) + (int64_t)share * a.R * a.ldy;  // several shares: slabs of partial sums
    const bool aligned = a.ldy % 4 == 0 && reinterpret_cast<uintptr_t>(a.y) % (4 * sizeof(OT)) == 0;
#pragma unroll
    for (int j = 0; j < WR; ++j) {
        const int r = r0 + (wr * WR + j) * 16 + sub;
        if (r >= a.R) continue;
#pragma unroll
        for (int i = 0; i < WN; ++i) store_y4(y + (int64_t)r * a.ldy, acc[i][j], n0 + (wn * WN + i) * 16 + 4 * g, a.N, aligned);
    }
}

// y = sum of the shares' slabs, in their order
template <typename OT>
__global__ __launch_bounds__(256) void f8_sum_k(const float *__restrict__ part, int shares, int R, int N, OT *__restrict__ y, int64_t ldy) {
    const int64_t slab = (int64_t)R * N;
    const int n4 = (N + 3) >> 2;
    const bool whole = N % 4 == 0, aligned = ldy % 4 == 0 && reinterpret_cast<uintptr_t>(y) % (4 * sizeof(OT)) == 0;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)R * n4) return;
    const int r = (int)(i / n4), n = (int)(i % n4) * 4;
    const float *p = part + (int64_t)r * N + n;
    f4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < shares; ++s, p += slab) {
        if (whole) {
            v += *reinterpret_cast<const f4_t *>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < N) v[e] += p[e];
        }
    }
    store_y4(y + (int64_t)r * ldy, v, n, N, aligned);
}

template <typename OT, bool F16, int TN, int TR, int PN, int PR, int S>
static hipError_t launch_tile(const F8Args &a, hipStream_t s, int shares = 1) {
    const int64_t n_tiles = (a.N + TN - 1) / TN, r_tiles = (a.R + TR - 1) / TR, total = n_tiles * r_tiles * shares;
    if (total > 1 << 30) return hipErrorInvalidValue;  // beyond any memory: N and R are at most 2^30 each
    hipLaunchKernelGGL((f8_tile_k<OT, F16, TN, TR, PN, PR, S>), grid_of((total + 7) / 8 * 8), dim3(64 * PN * PR), 0, s, a, (int)n_tiles,
                       (int)r_tiles, shares);
    return hipGetLastError();
}

template <typename OT, bool F16, int TN, int TR, int PN, int PR, int S>
static hipError_t launch_shared(const F8Args &a, int shares, hipStream_t s) {
    if (shares == 1) return launch_tile<OT, F16, TN, TR, PN, PR, S>(a, s);
    F8Args p = a;  // partial sums: [shares][R][N]
    p.y = a.part; p.ldy = a.N;
    const hipError_t e = launch_tile<float, F16, TN, TR, PN, PR, S>(p, s, shares);
    if (e != hipSuccess) return e;
    const int64_t items = (int64_t)a.R * ((a.N + 3) / 4);  // few tiles share: far below 2^32
    hipLaunchKernelGGL((f8_sum_k<OT>), dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, a.part, shares, a.R, a.N,
                       reinterpret_cast<OT *>(a.y), a.ldy);
    return hipGetLastError();
}

// ---- which kernel runs ---------------------------------------------------------------------------------------------
// Times below: fresh weights from HBM for every call, in microseconds, launches back to back.

// Tiles of rows the stream makes of more than 32: of 48 rows if they are no more than tiles of 64 would be.
static int64_t stream_row_tiles(const F8Args &a) { return (a.R + 63) / 64; }
static bool tiles_of_48(const F8Args &a) { return (a.R + 47) / 48 == stream_row_tiles(a); }

// Whether the product quantises fp32 / bf16 rows itself, in every workgroup anew, instead of by a launch of the quantiser
// in front: where that costs the GPU little, for it saves the host a launch (3 us).  Itself against both, in a graph, fp32
// rows: 1 x 2048 x 2048 4.8 / 5.9, 1 x 4096 x 4096 8.3 / 8.2, 16 x 2048 x 2048 7.4 / 6.7, but 12 x 4096 x 4096 11.1 / 9.3, 1 x 2048 x 8192
// 12.4 / 9.8; bf16: 16 x 4096 x 4096 9.2 / 9.5, 32 x 2048 x 2048 8.0 / 8.0, 200 x 512 x 1024 8.1 / 7.5, 4096 x 128 x 512 6.7 / 9.1, but 24 x 4096 x
// 4096 13.4 / 11.0, 48 x 2048 x 2048 10.3 / 9.2.  Many columns make it too many times: 8 x 28672 x 512 9.9 / 8.1.
bool gemm_f8_takes_wide(const F8Args &a) {
    const int64_t size = a.x_type == X_F32 ? 4 : 2;
    const int blocks = a.x_type == X_F32 ? (a.R <= 8 ? 32 : a.R <= 16 ? 16 : 0) : (a.R <= 16 ? 32 : a.R <= 32 ? 16 : 8);
    return a.KB <= blocks && (int64_t)a.N * a.K <= 4096 * 4096 &&
           (a.R <= 16 ? a.N <= 16384 : ((int64_t)a.N + 31) / 32 * stream_row_tiles(a) <= 256) &&
           reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * size % 16 == 0;
}

// Shares of K for a grid of `tiles` tiles: one workgroup a compute unit, and two where that leaves each more than sixteen
// blocks of k (137 x 4096 x 11008, 96 tiles: 44.6 / 28.7 / 24.7 / 28.7 with 1 / 2 / 5 / 8; 256 x 2048 x 8192, 64 tiles: 33.3 / 16.0 / 17.8
// with 1 / 4 / 8; 192 x 8192 x 2048, 192 tiles: 12.3 / 15.4 with 1 / 2).  At most eight, eight blocks each, and the partial sums
// have to fit the scratch.
static int64_t pick_shares(const F8Args &a, int64_t tiles) {
    const int64_t slab = (int64_t)a.R * a.N * 4;
    const int64_t fit = a.part == nullptr ? 1 : a.part_bytes / slab;
    const int64_t two = std::min<int64_t>(8, 512 / tiles), n = a.KB > 16 * two ? two : 256 / tiles;
    return std::max<int64_t>(1, std::min({n, (int64_t)8, (int64_t)a.KB / 8, fit}));
}

// The stream with 16 RB rows a workgroup: 16, 32 or 64 columns, the fewest that need no more than one workgroup a compute
// unit.  With more columns x is read less often, with fewer the chip fills sooner (16 / 32 / 64 columns: 9 x 4096 x 14336 13.8 /
// 20 / -, 9 x 6144 x 4096 9.3 / 8.2 / -, 1 x 28672 x 4096 26.5 / 25.9 / 25.9, 32 x 4096 x 4096 8.2 / 9.7 / -, 32 x 6144 x 4096
// 14.4 / 10.7 / -, 32 x 14336 x 4096 26.7 / 19.5 / 15.9).  Waves and stages: 9 x 4096 x 14336 13.8 with eight of two, 14.4 with
// eight of one, 14.8 with sixteen of one (rows quantised here, 1 x 2048 x 2048: 5.4 with two stages, 4.8 with one); 64 x 4096 x 4096 12.9 with four waves, 13.3 with eight.
template <typename OT, int RB, int XIN>
static hipError_t launch_columns(const F8Args &a, hipStream_t s) {
    const int64_t r_tiles = (a.R + 16 * RB - 1) / (16 * RB), groups = (a.N + 15) / 16;
    constexpr int NW = RB == 4 ? 4 : 8;
    if (groups * r_tiles <= 256) return launch_stream<OT, 1, RB, NW, RB == 1 && XIN == X_F8 ? 2 : 1, XIN>(a, s);
    if constexpr (XIN == X_F8 && RB <= 2) {  // the others come with columns that fit
        if ((groups + 1) / 2 * r_tiles > 256) return launch_stream<OT, 4, RB, 4, 1, XIN>(a, s);
    }
    return launch_stream<OT, 2, RB, NW, 1, XIN>(a, s);
}

template <typename OT, int XIN>
static hipError_t launch_rows(const F8Args &a, hipStream_t s) {
    if constexpr (XIN == X_F32) {
        return launch_columns<OT, 1, XIN>(a, s);  // comes with no more rows
    } else {
        if (a.R <= 16) return launch_columns<OT, 1, XIN>(a, s);
        if (a.R <= 32) return launch_columns<OT, 2, XIN>(a, s);
        return tiles_of_48(a) ? launch_columns<OT, 3, XIN>(a, s) : launch_columns<OT, 4, XIN>(a, s);
    }
}

// Whether the stream takes the product: up to 16 rows always; more where the tiles would need longer, 0.37 a block of k a
// share and 6 to start and to join the shares against 0.22 a block of k, as long as (more than 32 rows) workgroups of 32
// columns fit the compute units.  Stream against tiles, fp32 / bf16 results: 24 x 4096 x 14336 22.1 against 19.4 / 17.5, 32 x 14336 x
// 4096 15.9 against 19 / 17, 40 x 4096 x 4096 10.1 against 12.8 / 11.4, 40 x 2048 x 8192 16.2 against 14.1 / 12.8, 128 x 2048 x 2048 7.7 against
// 11.2 / 9.6, 64 x 4096 x 14336 35.2 against 20.1 / 19.0 with eight shares and 74.2 / 60.3 with one, 48 x 28672 x 4096 32.6 against 31.1 / 29.1.
static bool streams(const F8Args &a, int64_t shares) {
    if (a.R <= 16) return true;
    if (a.R > 32 && ((int64_t)a.N + 31) / 32 * stream_row_tiles(a) > 256) return false;
    return 37 * (int64_t)a.KB / shares + 600 > 22 * (int64_t)a.KB;
}

template <typename OT>
static hipError_t launch_gemm_f8_t(const F8Args &a, hipStream_t s) {
    if (a.x_type == X_F32) return launch_rows<OT, X_F32>(a, s);
    if (a.x_type == X_BF16) return launch_rows<OT, X_BF16>(a, s);
    auto tiles = [&](int64_t tn, int64_t tr) { return (a.N + tn - 1) / tn * ((a.R + tr - 1) / tr); };
    const int64_t shares = pick_shares(a, tiles(128, 64));
    if (streams(a, shares)) return launch_rows<OT, X_F8>(a, s);
    // Large tiles read each operand less often, but a round of them over the chip leaves more of it idle when it is not full:
    // they are taken from two rounds on, or for one that fills.
    auto fills = [](int64_t t, int64_t round, int64_t idle) { return t >= 2 * round || (round - t % round) % round <= idle; };
    if constexpr (sizeof(OT) == 4) {
        // tiles of 128 x 128 (two a compute unit) against 128 x 64: 4096 x 28672 x 4096 895 against 1047, 1300 x 14336 x 4096 164 against 184,
        // 4096 x 2048 x 8192 (512 tiles) 129 against 151, 1024 x 6144 x 4096 (384) 66 against 63
        if (fills(tiles(128, 128), 512, 64)) return launch_tile<OT, true, 128, 128, 2, 2, 2>(a, s);
        return launch_shared<OT, true, 128, 64, 2, 2, 3>(a, (int)shares, s);
    } else {
        // tiles of 256 x 256 (one) against 128 x 64: 4096 x 28672 x 4096 464 against 715, 4096 x 6144 x 4096 (384 tiles) 123 against 156,
        // 3000 x 6144 x 4096 (288) 114 against 105, 1500 x 6144 x 4096 (144) 61 against 65, 2048 x 4096 x 4096 (128) 58 against 56
        const int64_t t = tiles(256, 256);
        if (t > 128 && fills(t, 256, 128)) return launch_tile<OT, false, 256, 256, 2, 4, 2>(a, s);
        // tiles of 128 x 128 (one) against 128 x 64: 500 x 6144 x 4096 (192 tiles) 26 against 29, 900 x 4096 x 11008 (256) 61 against 67,
        // 1024 x 6144 x 4096 (384) 48 against 43; with shares of K neither wins by much (96 tiles: 27 / 31, 44 / 41)
        const int64_t m = tiles(128, 128);
        if (a.R > 64 && m > 128 && fills(m, 256, 64)) return launch_tile<OT, false, 128, 128, 4, 2, 3>(a, s);
        return launch_shared<OT, false, 128, 64, 2, 2, 3>(a, (int)shares, s);
    }
}

hipError_t launch_gemm_f8(const F8Args &a, hipStream_t s) {
    return a.y_dtype == DT_F32 ? launch_gemm_f8_t<float>(a, s) : launch_gemm_f8_t<__bf16>(a, s);
}

}  // namespace sd
