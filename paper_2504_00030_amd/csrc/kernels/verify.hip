// Verification of drafted tokens against given uniforms, a batch at once.
//
// Only one row a sequence needs summing: the accept test reads single elements.  verify_sum_k finds the row (every wave for
// itself: two dependent loads, cheaper than a launch in front) and sums its tiles of max(0, p - q) and p, a wave each;
// verify_pick_k, one wave a sequence, finds the tile the draw falls into and the element inside it.  Sums are in 64 bits:
// a draw in 2^17 elements moves by 1e-13 of the mass at most, and the tests u q < p are exact.  Bound by memory and two launches:
// 64 sequences of 128256 fp32 12.8 + 4.9 us (62 MB, 4.9 TB/s in the first), one of 32000 3.8 + 3.3.  Tiles of 512 elements: with 1024
// these take 17.8 and 8.0 us together, with 2048 20.3 and 10.2, with 512 18.3 and 7.0.
#include "common.hpp"
#include "params.hpp"

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

constexpr int PER = VERIFY_TILE / 64;  // elements of a tile a lane takes

// sequence b's first draft and their number; false where draft_start does not make sense
__device__ __forceinline__ bool drafts_of(const VerifyArgs &a, int b, int &first, int &k) {
    first = a.draft_start[b];
    const int end = a.draft_start[b + 1];
    k = end - first;
    return first >= 0 && end >= first && end <= a.n_drafts;
}

// leading drafts that pass the test, sixty-four at a time; every wave works them out for itself
template <typename T>
__device__ __forceinline__ int accepted_of(const VerifyArgs &a, int b, int first, int k) {
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < k; base += 64) {
        const int i = base + lane;
        bool kept = true;
        if (i < k) {
            const int d = first + i, x = a.drafted[d];
            kept = x >= 0 && x < a.vocab;
            if (kept) {
                const double px = (double)(float)reinterpret_cast<const T *>(a.p)[(int64_t)(d + b) * a.ldp + x];
                const double qx = a.q ? (double)(float)reinterpret_cast<const T *>(a.q)[(int64_t)d * a.ldq + x] : 1.0;
                kept = (double)a.u_accept[d] * qx < px;  // exact: products of two 24-bit numbers
            }
        }
        const uint64_t refused = __ballot(!kept);
        if (refused) return base + __ffsll((unsigned long long)refused) - 1;
    }
    return k;
}

// This lane's elements of a tile that begins with element j0, zeros past the row's end: PER neighbours, or every 64th
// vector (SPREAD: each load of the wave is then one run of memory; only sums can do with that order)
template <bool SPREAD, typename T>
__device__ __forceinline__ void load_tile(const T *row, int j0, int n, float (&v)[PER]) {
    constexpr int N = 16 / sizeof(T);  // elements of a vector
    const int lane = threadIdx.x & 63;
    const bool whole = j0 + VERIFY_TILE <= n && (reinterpret_cast<uintptr_t>(row + j0) & 15) == 0;
#pragma unroll
    for (int w = 0; w < PER / N; ++w) {
        const int j = j0 + (SPREAD ? (w * 64 + lane) * N : lane * PER + w * N);
        if (whole) {
            if constexpr (sizeof(T) == 4) {
                const f4_t x = *reinterpret_cast<const f4_t *>(row + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * w + e] = x[e];
            } else {
                const b8_t x = *reinterpret_cast<const b8_t *>(row + j);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * w + e] = (float)x[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[N * w + e] = j + e < n ? (float)row[j + e] : 0.f;
        }
    }
}
// element e of load_tile()
template <bool SPREAD, typename T>
__device__ __forceinline__ int place(int j0, int e) {
    constexpr int N = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    return j0 + (SPREAD ? (e / N * 64 + lane) * N + e % N : lane * PER + e);
}

// the two weights of an element: of the residual and of the target's row alone (comparisons with NaN are false)
__device__ __forceinline__ double weight_p(float p) { return p > 0.f ? (double)p : 0.0; }
__device__ __forceinline__ double weight_rest(float p, float q) {
    const double d = (double)p - (double)q;
    return d > 0.0 ? d : 0.0;
}

// Row of the draw: p, and q where one is subtracted (draw_q), or the token left out (out, else -1).
template <typename T>
struct Draw {
    const T *p, *q;
    int out;
};
template <typename T>
__device__ __forceinline__ Draw<T> draw_of(const VerifyArgs &a, int b, int first, int k, int A) {
    Draw<T> d;
    d.p = reinterpret_cast<const T *>(a.p) + (int64_t)(first + b + A) * a.ldp;
    d.q = A < k && a.q ? reinterpret_cast<const T *>(a.q) + (int64_t)(first + A) * a.ldq : nullptr;
    d.out = A < k && !a.q ? a.drafted[first + A] : -1;
    return d;
}

// sum over the lanes below this one and itself
__device__ __forceinline__ double wave_scan(double v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double o = __shfl_up(v, m, WAVE);
        if (lane >= m) v += o;
    }
    return v;
}
}  // namespace

template <typename T>
__global__ __launch_bounds__(256) void verify_sum_k(const VerifyArgs a) {
    const int b = blockIdx.y, tile = blockIdx.x * 4 + (threadIdx.x >> 6);
    int first, k;
    if (tile >= a.tiles || !drafts_of(a, b, first, k)) return;
    const int A = accepted_of<T>(a, b, first, k);
    const Draw<T> d = draw_of<T>(a, b, first, k, A);
    const int j0 = tile * VERIFY_TILE;
    float p[PER], q[PER];
    load_tile<true>(d.p, j0, a.vocab, p);
    double sp = 0.0, sr = 0.0;
    if (d.q) {
        load_tile<true>(d.q, j0, a.vocab, q);
#pragma unroll
        for (int e = 0; e < PER; ++e) { sp += weight_p(p[e]); sr += weight_rest(p[e], q[e]); }
    } else {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const double w = weight_p(p[e]);
            sp += w;
            sr += place<true, T>(j0, e) == d.out ? 0.0 : w;
        }
    }
    sp = wave_sum(sp);
    sr = wave_sum(sr);
    if ((threadIdx.x & 63) == 0) {
        double *to = a.sums + ((int64_t)b * a.tiles + tile) * 2;
        to[0] = sr;
        to[1] = sp;
        if (tile == 0) a.taken[b] = A;
    }
}

template <typename T>
__global__ __launch_bounds__(64) void verify_pick_k(const VerifyArgs a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    int first, k;
    if (!drafts_of(a, b, first, k)) {
        if (lane == 0) { a.n_accepted[b] = -1; a.next_token[b] = -1; }
        return;
    }
    const int A = a.taken[b];
    const double *sums = a.sums + (int64_t)b * a.tiles * 2;
    const int each = (a.tiles + 63) / 64, t0 = min(lane * each, a.tiles), t1 = min(t0 + each, a.tiles);
    double rest = 0.0, full = 0.0;
    for (int t = t0; t < t1; ++t) { rest += sums[2 * t]; full += sums[2 * t + 1]; }
    const double u = (double)a.u_next[b];
    Draw<T> d = draw_of<T>(a, b, first, k, A);
    // sums up to the end of this lane's tiles
    double upto = wave_scan(rest), total = __shfl(upto, 63, WAVE);
    int which = 0;
    if (A == k || !(total > 0.0)) {  // no draft was refused, or the residual is empty: the target's row
        which = 1;
        d.q = nullptr;
        d.out = -1;
        rest = full;
        upto = wave_scan(rest);
        total = __shfl(upto, 63, WAVE);
    }
    const double target = u * total;
    // the first tile whose end lies beyond the target, or the last one with any weight, and the mass in front of it
    int hit = -1, last = -1;
    double at = upto - rest, before = 0.0;
    for (int t = t0; t < t1; ++t) {
        const double w = sums[2 * t + which];
        if (w > 0.0 && hit < 0) {
            last = t;
            before = at;
            if (at + w > target) hit = t;
        }
        at += w;
    }
    const uint64_t hits = __ballot(hit >= 0), some = __ballot(last >= 0);
    if (!some) {  // no weight anywhere
        if (lane == 0) { a.n_accepted[b] = A; a.next_token[b] = 0; }
        return;
    }
    const int from = hits ? __ffsll((unsigned long long)hits) - 1 : 63 - __clzll((long long)some);
    const int j0 = __shfl(last, from, WAVE) * VERIFY_TILE;
    before = __shfl(before, from, WAVE);
    // inside the tile
    float p[PER], q[PER];
    double w[PER], sum = 0.0;
    load_tile<false>(d.p, j0, a.vocab, p);
    if (d.q) load_tile<false>(d.q, j0, a.vocab, q);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        w[e] = d.q ? weight_rest(p[e], q[e]) : (place<false, T>(j0, e) == d.out ? 0.0 : weight_p(p[e]));
        sum += w[e];
    }
    at = before + (wave_scan(sum) - sum);
    int found = -1, behind = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
            behind = place<false, T>(j0, e);
            if (found < 0 && at > target) found = behind;
        }
    }
    const uint64_t founds = __ballot(found >= 0), any = __ballot(behind >= 0);
    const int y = founds ? __shfl(found, __ffsll((unsigned long long)founds) - 1, WAVE) : __shfl(behind, any ? 63 - __clzll((long long)any) : 0, WAVE);
    if (lane == 0) {
        a.n_accepted[b] = A;
        a.next_token[b] = max(y, 0);
    }
}

template <typename T>
static hipError_t launch_verify_t(const VerifyArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((verify_sum_k<T>), dim3((a.tiles + 3) / 4, a.n_seq), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_pick_k<T>), dim3(a.n_seq), dim3(64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs &a, hipStream_t s) {
    return a.dtype == DT_F32 ? launch_verify_t<float>(a, s) : launch_verify_t<__bf16>(a, s);
}

}  // namespace sd
