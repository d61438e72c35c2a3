// Verification of drafted tokens against given uniforms, a batch at once.
//
// Only one row a sequence needs summing: the accept test reads single elements.  verify_sum_k finds the row (every
// workgroup for itself: two dependent loads, cheaper than a launch in front) and sums its tiles of max(0, p - q) and p;
// verify_pick_k, one workgroup a sequence, finds the tile the draw falls into and the element inside it.  Sums are in 64 bits:
// a draw in 2^17 elements moves by 1e-13 of the mass at most, and the tests u q < p are exact.
#include "common.hpp"
#include "params.hpp"

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));

constexpr int PER = VERIFY_TILE / 256;  // elements of a tile a thread takes: 16 neighbours

// sequence b's first draft and their number; false where draft_start does not make sense
__device__ __forceinline__ bool drafts_of(const VerifyArgs &a, int b, int &first, int &k) {
    first = a.draft_start[b];
    const int end = a.draft_start[b + 1];
    k = end - first;
    return first >= 0 && end >= first && end <= a.n_drafts;
}

// leading drafts that pass the test; the same for every wave, sixty-four drafts at a time
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

// PER neighbours of a row from element j on, zeros past its end
template <typename T>
__device__ __forceinline__ void load_row(const T *row, int j, int n, float (&v)[PER]) {
    if (j + PER <= n && (reinterpret_cast<uintptr_t>(row + j) & 15) == 0) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int w = 0; w < PER / 4; ++w) {
                const f4_t x = reinterpret_cast<const f4_t *>(row + j)[w];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * w + e] = x[e];
            }
        } else {
#pragma unroll
            for (int w = 0; w < PER / 8; ++w) {
                const b8_t x = reinterpret_cast<const b8_t *>(row + j)[w];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * w + e] = (float)x[e];
            }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) v[e] = j + e < n ? (float)row[j + e] : 0.f;
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
// inclusive sums over the 256 threads; `waves` is shared, four elements
__device__ __forceinline__ double block_scan(double v, double *waves, double &total) {
    const int wave = threadIdx.x >> 6;
    v = wave_scan(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) waves[wave] = v;
    __syncthreads();
    double before = 0.0;
    for (int w = 0; w < wave; ++w) before += waves[w];
    total = ((waves[0] + waves[1]) + waves[2]) + waves[3];
    return before + v;
}

}  // namespace

template <typename T>
__global__ __launch_bounds__(256) void verify_sum_k(const VerifyArgs a) {
    __shared__ double part[4][2];
    const int b = blockIdx.y, tile = blockIdx.x;
    int first, k;
    if (!drafts_of(a, b, first, k)) return;
    const int A = accepted_of<T>(a, b, first, k);
    if (tile == 0 && threadIdx.x == 0) a.taken[b] = A;
    const Draw<T> d = draw_of<T>(a, b, first, k, A);
    const int j = tile * VERIFY_TILE + (int)threadIdx.x * PER;
    float p[PER], q[PER];
    load_row(d.p, j, a.vocab, p);
    double sp = 0.0, sr = 0.0;
    if (d.q) {
        load_row(d.q, j, a.vocab, q);
#pragma unroll
        for (int e = 0; e < PER; ++e) { sp += weight_p(p[e]); sr += weight_rest(p[e], q[e]); }
    } else {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const double w = weight_p(p[e]);
            sp += w;
            sr += j + e == d.out ? 0.0 : w;
        }
    }
    sp = wave_sum(sp);
    sr = wave_sum(sr);
    if ((threadIdx.x & 63) == 0) { part[threadIdx.x >> 6][0] = sr; part[threadIdx.x >> 6][1] = sp; }
    __syncthreads();
    if (threadIdx.x < 2) {
        const int w = threadIdx.x;
        a.sums[((int64_t)b * a.tiles + tile) * 2 + w] = ((part[0][w] + part[1][w]) + part[2][w]) + part[3][w];
    }
}

template <typename T>
__global__ __launch_bounds__(256) void verify_pick_k(const VerifyArgs a) {
    __shared__ double waves[4];
    __shared__ double before;   // mass in front of the chosen tile
    __shared__ int hit, last;
    const int b = blockIdx.x, tid = threadIdx.x;
    int first, k;
    if (!drafts_of(a, b, first, k)) {
        if (tid == 0) { a.n_accepted[b] = -1; a.next_token[b] = -1; }
        return;
    }
    const int A = a.taken[b];
    Draw<T> d = draw_of<T>(a, b, first, k, A);
    const double *sums = a.sums + (int64_t)b * a.tiles * 2;
    const int each = (a.tiles + 255) / 256, t0 = min(tid * each, a.tiles), t1 = min(t0 + each, a.tiles);
    double mine[2] = {0.0, 0.0}, total;
    for (int t = t0; t < t1; ++t) { mine[0] += sums[2 * t]; mine[1] += sums[2 * t + 1]; }
    if (tid == 0) { hit = 0x7fffffff; last = -1; }
    double upto = block_scan(mine[0], waves, total);
    int which = 0;
    if (A == k || !(total > 0.0)) {  // no draft was refused, or the residual is empty: the target's row
        which = 1;
        d.q = nullptr;
        d.out = -1;
        upto = block_scan(mine[1], waves, total);
    }
    const double target = (double)a.u_next[b] * total;
    // the first tile whose end lies beyond the target, or the last one with any weight
    {
        double at = upto - mine[which];
        int full = -1;
        for (int t = t0; t < t1; ++t) {
            const double w = sums[2 * t + which];
            at += w;
            if (w > 0.0) full = t;
            if (at > target && w > 0.0) { atomicMin(&hit, t); break; }
        }
        if (full >= 0) atomicMax(&last, full);
    }
    __syncthreads();
    const int tile = hit != 0x7fffffff ? hit : last;
    if (tile < 0) {  // no weight anywhere
        if (tid == 0) { a.n_accepted[b] = A; a.next_token[b] = 0; }
        return;
    }
    if (tile >= t0 && tile < t1) {
        double at = upto - mine[which];
        for (int t = t0; t < tile; ++t) at += sums[2 * t + which];
        before = at;
    }
    __syncthreads();
    if (tid == 0) { hit = 0x7fffffff; last = -1; }
    const int j = tile * VERIFY_TILE + tid * PER;
    float p[PER], q[PER];
    double w[PER], sum = 0.0;
    load_row(d.p, j, a.vocab, p);
    if (d.q) load_row(d.q, j, a.vocab, q);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        w[e] = d.q ? weight_rest(p[e], q[e]) : (j + e == d.out ? 0.0 : weight_p(p[e]));
        sum += w[e];
    }
    double at = before + (block_scan(sum, waves, total) - sum);
    int found = 0x7fffffff, full = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        at += w[e];
        if (w[e] > 0.0) {
            full = j + e;
            if (found == 0x7fffffff && at > target) found = j + e;
        }
    }
    if (found != 0x7fffffff) atomicMin(&hit, found);
    if (full >= 0) atomicMax(&last, full);
    __syncthreads();
    if (tid == 0) {
        a.n_accepted[b] = A;
        a.next_token[b] = hit != 0x7fffffff ? hit : last;
    }
}

template <typename T>
static hipError_t launch_verify_t(const VerifyArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((verify_sum_k<T>), dim3(a.tiles, a.n_seq), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((verify_pick_k<T>), dim3(a.n_seq), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs &a, hipStream_t s) {
    return a.dtype == DT_F32 ? launch_verify_t<float>(a, s) : launch_verify_t<__bf16>(a, s);
}

}  // namespace sd
