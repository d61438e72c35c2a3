// Attention of a batch's rows over a prefix that all sequences share and over every sequence's own positions, from pages.
//
//   o = sum_j softmax_j(scale q . k_j) v_j,   one pass over the positions with a running maximum m and sum l
//
// Columns and lanes.  The query heads that read one cache head, of all rows of a piece, are the columns of one product:
// S^T = K Q^T (16 positions x 16 columns an instruction), then O^T += V^T P^T.  Transposed, column c of S, P and O is held by
// lanes c, c + 16, c + 32, c + 48, so m, l and the rescaling are one number a lane, and what a lane holds of S^T (positions
// 4 g .. 4 g + 3 of each 16, g = lane / 16) is, rounded, its share of the second product's operand: no exchange between lanes
// and no shared memory in the loop.  The positions' order inside a product is free, so a lane loads the rows of V for just
// those positions, 16 bytes of each, and turns 2 x 2 blocks in registers.  Which channels a lane holds is free too: lane
// l % 16 takes W neighbours, so loads and stores are whole vectors.
//
// Pieces.  The prefix is read once for all rows (columns: every row of the batch), the own positions once a sequence; either
// is split into parts along the positions, and a second kernel joins the parts of a row.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>
#include <math.h>

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef float f2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

constexpr int TILE = 32;      // positions a wave takes at a time
constexpr int MIN_PART = 128; // least positions of a part: a tile for each of a workgroup's four waves
constexpr int MAX_PARTS = 64;

template <int N> struct words { uint32_t w[N]; };
template <int BYTES, typename E> struct vec_of;
template <> struct vec_of<16, uint32_t> { typedef uint32_t type __attribute__((ext_vector_type(4))); };
template <> struct vec_of<8, uint32_t> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct vec_of<4, uint32_t> { typedef uint32_t type; };

// N words from N * 4-byte aligned memory
template <int N>
__device__ __forceinline__ void load_words(const void *p, uint32_t (&w)[N]) {
    const typename vec_of<N * 4, uint32_t>::type v = *reinterpret_cast<const typename vec_of<N * 4, uint32_t>::type *>(p);
    if constexpr (N == 1) w[0] = v;
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = v[i];
    }
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// What one lane keeps of QT x 16 columns in bf16.  HDP: head size rounded up to 32, 64, 128 or 256; channels from hd on are
// zeros.  W: neighbouring channels of V a lane holds, NB blocks of 16 W.
template <int HDP_, int QT_, bool EXACT>
struct CoreBf16 {
    typedef __bf16 T;
    static constexpr int HDP = HDP_, QT = QT_, W = HDP >= 128 ? 8 : HDP / 16, NB = HDP / (16 * W), KC = HDP / 32;
    b8_t q[QT][KC];
    u4_t k[2][KC];            // positions lane % 16 of the tile's two sixteens, channels 32 c + 8 g ..
    uint32_t v[8][NB][W / 2]; // positions 4 g + i of the first (i < 4) and second sixteen, channels W (lane % 16) ..

    __device__ __forceinline__ void load_q(int t, const T *row, bool whole, int hd, int g) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const int ch = 32 * c + 8 * g;
            b8_t x = {};
            if (EXACT || ch < hd) {
                if (whole) x = *reinterpret_cast<const b8_t *>(row + ch);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = row[ch + e];
                }
            }
            q[t][c] = x;
        }
    }
    __device__ __forceinline__ void load_k(int s, const T *row, int hd, int g) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const int ch = 32 * c + 8 * g;
            // (beyond hd the queries are zero: any finite value would do, and the row's memory need not hold one)
            k[s][c] = EXACT || ch < hd ? *reinterpret_cast<const u4_t *>(row + ch) : u4_t{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void load_v(int s, const T *rows, int hd, int c16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int ch = 16 * W * n + W * c16;
                if (EXACT || ch < hd) load_words<W / 2>(rows + (int64_t)i * hd + ch, v[4 * s + i][n]);
                else {
#pragma unroll
                    for (int w = 0; w < W / 2; ++w) v[4 * s + i][n][w] = 0;
                }
            }
    }
    __device__ __forceinline__ void scores(int t, f4_t (&s)[2]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, k[h][c]), q[t][c], s[h], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void forget(int i, bool keep) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W / 2; ++w) v[i][n][w] = keep ? v[i][n][w] : 0u;
    }
    // whether row i of this lane's values holds an infinity or a NaN
    __device__ __forceinline__ bool odd(int i) const {
        bool bad = false;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W / 2; ++w) bad |= (v[i][n][w] & 0x7f80u) == 0x7f80u || (v[i][n][w] & 0x7f800000u) == 0x7f800000u;
        return bad;
    }
    struct Weights { b8_t p; };
    __device__ __forceinline__ static Weights weights(const f4_t (&s)[2]) {
        Weights x;
#pragma unroll
        for (int i = 0; i < 4; ++i) { x.p[i] = (__bf16)s[0][i]; x.p[4 + i] = (__bf16)s[1][i]; }
        return x;
    }
    __device__ __forceinline__ static Weights none() { return Weights{b8_t{}}; }
    // channel pair w of block n, positions turned into rows: the first product operand of channels 2 w and 2 w + 1
    __device__ __forceinline__ void turned(int n, int w, b8_t &even, b8_t &odd_) const {
        u4_t lo, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = __builtin_amdgcn_perm(v[2 * i + 1][n][w], v[2 * i][n][w], 0x05040100u);
            hi[i] = __builtin_amdgcn_perm(v[2 * i + 1][n][w], v[2 * i][n][w], 0x07060302u);
        }
        even = __builtin_bit_cast(b8_t, lo);
        odd_ = __builtin_bit_cast(b8_t, hi);
    }
    __device__ __forceinline__ void values(const Weights (&p)[QT], f4_t (&o)[QT][NB * W]) const {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W / 2; ++w) {
                b8_t even, odd_;
                turned(n, w, even, odd_);
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    f4_t &x = o[t][n * W + 2 * w], &y = o[t][n * W + 2 * w + 1];
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, p[t].p, x, 0, 0, 0);
                    y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd_, p[t].p, y, 0, 0, 0);
                }
            }
    }
};

// The same in fp32: 16 x 16 x 4 instructions, their four channels (positions) those of the four groups of lanes.
template <int HDP_, bool EXACT>
struct CoreF32 {
    typedef float T;
    static constexpr int HDP = HDP_, QT = 1, W = HDP >= 64 ? 4 : HDP / 16, NB = HDP / (16 * W), KC = HDP / 16;
    f4_t q[1][KC];   // channels 16 c + 4 g ..
    f4_t k[2][KC];
    uint32_t v[8][NB][W];

    __device__ __forceinline__ void load_q(int t, const T *row, bool whole, int hd, int g) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const int ch = 16 * c + 4 * g;
            f4_t x = {0.f, 0.f, 0.f, 0.f};
            if (EXACT || ch < hd) {
                if (whole) x = *reinterpret_cast<const f4_t *>(row + ch);
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = row[ch + e];
                }
            }
            q[t][c] = x;
        }
    }
    __device__ __forceinline__ void load_k(int s, const T *row, int hd, int g) {
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            const int ch = 16 * c + 4 * g;
            k[s][c] = EXACT || ch < hd ? *reinterpret_cast<const f4_t *>(row + ch) : f4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void load_v(int s, const T *rows, int hd, int c16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int ch = 16 * W * n + W * c16;
                if (EXACT || ch < hd) load_words<W>(rows + (int64_t)i * hd + ch, v[4 * s + i][n]);
                else {
#pragma unroll
                    for (int w = 0; w < W; ++w) v[4 * s + i][n][w] = 0;
                }
            }
    }
    __device__ __forceinline__ void scores(int t, f4_t (&s)[2]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            s[h] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[h][c][e], q[t][c][e], s[h], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void forget(int i, bool keep) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W; ++w) v[i][n][w] = keep ? v[i][n][w] : 0u;
    }
    __device__ __forceinline__ bool odd(int i) const {
        bool bad = false;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W; ++w) bad |= (v[i][n][w] & 0x7f800000u) == 0x7f800000u;
        return bad;
    }
    struct Weights { f4_t p[2]; };
    __device__ __forceinline__ static Weights weights(const f4_t (&s)[2]) { return Weights{{s[0], s[1]}}; }
    __device__ __forceinline__ static Weights none() { return Weights{{f4_t{0.f, 0.f, 0.f, 0.f}, f4_t{0.f, 0.f, 0.f, 0.f}}}; }
    __device__ __forceinline__ void values(const Weights (&p)[1], f4_t (&o)[1][NB * W]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int w = 0; w < W; ++w)
                    o[0][n * W + w] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][n][w]), p[0].p[i / 4][i % 4], o[0][n * W + w], 0, 0, 0);
    }
};

// Parts of a sequence's own positions: `chunk` positions each, `used` of them (one, perhaps empty, at least).
struct OwnParts { int len, chunk, used; };
__device__ __forceinline__ OwnParts own_parts_of(const SharedAttnArgs &a, int b) {
    OwnParts p;
    p.len = max(0, min(a.own_len[b], a.table_pages << a.page_shift));
    p.chunk = max(MIN_PART, ((p.len + a.own_parts - 1) / a.own_parts + TILE - 1) & ~(TILE - 1));
    p.used = max(1, (p.len + p.chunk - 1) / p.chunk);
    return p;
}

// Sequence s's rows, within 0 .. R whatever row_start holds.
__device__ __forceinline__ void rows_of(const SharedAttnArgs &a, int s, int &first, int &n) {
    first = max(0, min(a.row_start[s], a.R));
    n = max(first, min(a.row_start[s + 1], a.R)) - first;
}

// One workgroup's share: columns of `tile` of the rows row0 .. row0 + n - 1, positions begin .. end - 1 of a table.
struct Piece {
    const int32_t *table;
    int pages;              // of the table, 1 at least
    int row0, n, tile, h;
    int len;                // positions of the prefix or the sequence
    bool own, direct;
    int part, begin, chunk;
};

// Which piece workgroup `id` has: prefix pieces first, tiles of `cols` columns.  false: none.  Same answer in every wave.
template <int COLS>
__device__ __forceinline__ bool piece_of(const SharedAttnArgs &a, uint32_t id, Piece &p) {
    if (id < a.prefix_groups) {
        // tiles outermost: the workgroups that read one head's part follow each other at a distance of heads x parts,
        // a multiple of eight where the heads are, so that they meet in one cache
        const uint32_t per_tile = (uint32_t)(a.nkv * a.prefix_parts), c = id % per_tile;
        p.tile = (int)(id / per_tile);
        p.h = (int)(c % a.nkv);
        p.part = (int)(c / a.nkv);
        p.table = a.prefix_table;
        p.pages = ((a.prefix_len - 1) >> a.page_shift) + 1;
        p.row0 = 0; p.n = a.R; p.len = a.prefix_len; p.own = false; p.direct = false;
        p.chunk = a.prefix_chunk;
        p.begin = p.part * p.chunk;
        return true;
    }
    id -= a.prefix_groups;
    p.h = (int)(id % a.nkv);
    id /= a.nkv;
    int64_t tile = id % a.own_tiles;
    const int part = (int)(id / a.own_tiles);
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
        int first = 0, n = 0;
        if (s0 + lane < a.n_seq) rows_of(a, s0 + lane, first, n);
        const int64_t tiles = ((int64_t)n * a.g + COLS - 1) / COLS;
        int64_t upto = tiles;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int64_t o = __shfl_up(upto, m, WAVE);
            if (lane >= m) upto += o;
        }
        const uint64_t beyond = __ballot(upto > tile);
        if (beyond) {
            const int src = uniform(__ffsll((unsigned long long)beyond) - 1), b = s0 + src;
            p.tile = uniform((int)(tile - __shfl(upto - tiles, src, WAVE)));
            p.row0 = uniform(__shfl(first, src, WAVE));
            p.n = uniform(__shfl(n, src, WAVE));
            const OwnParts parts = own_parts_of(a, b);
            if (part >= parts.used) return false;
            p.own = true;
            p.len = uniform(parts.len);
            p.chunk = uniform(parts.chunk);
            p.direct = a.prefix_parts == 0 && parts.used == 1;
            p.part = a.prefix_parts + part;
            p.begin = part * p.chunk;
            p.table = a.table + (int64_t)b * a.table_pages;
            p.pages = a.table_pages;
            return true;
        }
        tile -= __shfl(upto, 63, WAVE);
    }
    return false;
}

// Positions a lane loads of one tile, by page.
struct Places {
    int k[2], v[2];  // pages of the K row of each sixteen and of the V rows' quad
};
__device__ __forceinline__ Places places_of(const SharedAttnArgs &a, const Piece &p, int t0, int c16, int g) {
    Places x;
    const int last = p.pages - 1;
    if (a.page_shift >= 5) {
        const int page = p.table[min(t0 >> a.page_shift, last)];
        x.k[0] = x.k[1] = x.v[0] = x.v[1] = page;
    } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            x.k[s] = p.table[min((t0 + 16 * s + c16) >> a.page_shift, last)];
            x.v[s] = p.table[min((t0 + 16 * s + 4 * g) >> a.page_shift, last)];
        }
    }
    return x;
}
// element of position t of head h on `page` (page 0 stands in for one outside the pool)
__device__ __forceinline__ int64_t element(const SharedAttnArgs &a, int page, int h, int t) {
    const int pg = (uint32_t)page < (uint32_t)a.n_pages ? page : 0;
    return ((((int64_t)pg * a.nkv + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1))) * a.hd;
}

__device__ __forceinline__ float group_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, WAVE));
    return fmaxf(x, __shfl_xor(x, 32, WAVE));
}
__device__ __forceinline__ float group_sum(float x) {
    x += __shfl_xor(x, 16, WAVE);
    return x + __shfl_xor(x, 32, WAVE);
}

// One tile's softmax step of one column tile: scores -> weights, running maximum, sum and results brought up to date.
template <int NO>
__device__ __forceinline__ void soften(f4_t (&s)[2], float scale2, float &m, float &l, f4_t (&o)[NO]) {
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i / 4][i % 4]);
    top = fmaxf(m, group_max(top) * scale2);
    if (__ballot(top > m)) {
        const float by = exp2_(m - (top == -INFINITY ? 0.f : top));
        l *= by;
#pragma unroll
        for (int i = 0; i < NO; ++i) o[i] *= by;
        m = top;
    }
    const float base = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float e = exp2_(fmaf(s[i / 4][i % 4], scale2, -base));
        s[i / 4][i % 4] = e;
        sum += e;
    }
    l += sum;
}

}  // namespace

// Few columns: the four waves of a workgroup take the same QT x 16 columns and every fourth tile of the positions, and
// join their sums through shared memory at the end.
template <class C>
__global__ __launch_bounds__(256) void attn_split_k(const SharedAttnArgs a) {
    typedef typename C::T T;
    constexpr int QT = C::QT, NO = C::NB * C::W, LD = C::HDP + 4;
    __shared__ float so[4][16][LD];
    __shared__ float sm[4][QT * 16], sl[4][QT * 16];
    Piece p;
    if (!piece_of<QT * 16>(a, workgroup(), p)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
    const int cols = p.n * a.g, m0 = p.tile * QT * 16;
    const bool whole = a.q_whole;
    C core;
    int lim[QT];  // positions a column sees
    float m[QT], l[QT];
    f4_t o[QT][NO];
    auto sees = [&](int row) { return p.own ? max(0, p.len - p.n + row + 1) : p.len; };
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int col = min(m0 + 16 * t + c16, cols - 1), row = col / a.g;
        lim[t] = sees(row);
        core.load_q(t, reinterpret_cast<const T *>(a.q) + (int64_t)(p.row0 + row) * a.ldq + (int64_t)(p.h * a.g + col % a.g) * a.hd, whole, a.hd, g);
        m[t] = -INFINITY;
        l[t] = 0.f;
#pragma unroll
        for (int i = 0; i < NO; ++i) o[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int least = sees(m0 / a.g), most = sees(min(m0 + QT * 16, cols) - 1) , end = min(p.begin + p.chunk, sees((min(m0 + QT * 16, cols) - 1) / a.g));
    (void)most;
    const T *kp = reinterpret_cast<const T *>(a.k_pages), *vp = reinterpret_cast<const T *>(a.v_pages);
    auto load_k = [&](const Places &x, int t0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) core.load_k(s, kp + element(a, x.k[s], p.h, t0 + 16 * s + c16), a.hd, g);
    };
    auto load_v = [&](const Places &x, int t0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) core.load_v(s, vp + element(a, x.v[s], p.h, t0 + 16 * s + 4 * g), a.hd, c16);
    };
    int t0 = p.begin + TILE * wave;
    if (t0 < end) {
        Places now = places_of(a, p, t0, c16, g), next = places_of(a, p, t0 + 4 * TILE, c16, g);
        load_k(now, t0);
        load_v(now, t0);
        for (; t0 < end; t0 += 4 * TILE) {
            f4_t s[QT][2];
#pragma unroll
            for (int t = 0; t < QT; ++t) core.scores(t, s[t]);
            const int t1 = t0 + 4 * TILE;
            const bool more = t1 < end;
            if (more) load_k(next, t1);
            const bool there[2] = {(uint32_t)now.v[0] < (uint32_t)a.n_pages, (uint32_t)now.v[1] < (uint32_t)a.n_pages};
            bool apart = false;  // whether a column has to be kept from values that another one sees
            if (t0 + TILE > least || __ballot(!(there[0] && there[1]))) {
                bool bad = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int at = t0 + 16 * (i / 4) + 4 * g + i % 4;
                    const bool seen = there[i / 4] && at < end;
#pragma unroll
                    for (int t = 0; t < QT; ++t)
                        if (!seen || at >= lim[t]) s[t][i / 4][i % 4] = -INFINITY;
                    core.forget(i, seen);
                    bad |= at >= least && core.odd(i);
                }
                apart = __ballot(bad) != 0;
            }
            typename C::Weights w[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                soften<NO>(s[t], a.scale2, m[t], l[t], o[t]);
                w[t] = C::weights(s[t]);
            }
            if (!apart) {
                core.values(w, o);
            } else {
                // an infinity or a NaN that some columns see and others do not: 0 times it would reach those, so each
                // column is multiplied by itself, with the values it sees
                for (int c = 0; c < 16; ++c) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const int see = __builtin_amdgcn_readlane(lim[t], c);
                        C alone = core;
#pragma unroll
                        for (int i = 0; i < 8; ++i) alone.forget(i, t0 + 16 * (i / 4) + 4 * g + i % 4 < see);
                        typename C::Weights one[QT];
                        f4_t sum[QT][NO];
#pragma unroll
                        for (int u = 0; u < QT; ++u) {
                            one[u] = u == t && c16 == c ? w[u] : C::none();
#pragma unroll
                            for (int i = 0; i < NO; ++i) sum[u][i] = f4_t{0.f, 0.f, 0.f, 0.f};
                        }
                        alone.values(one, sum);
#pragma unroll
                        for (int i = 0; i < NO; ++i)
                            if (c16 == c) o[t][i] += sum[t][i];
                    }
                }
            }
            if (more) {
                load_v(next, t1);
                now = next;
                next = places_of(a, p, t1 + 4 * TILE, c16, g);
            }
        }
    }
    // the waves' sums meet: 16 columns at a time
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        l[t] = group_sum(l[t]);
        if (g == 0) { sm[wave][16 * t + c16] = m[t]; sl[wave][16 * t + c16] = l[t]; }
    }
    const int parts = a.prefix_parts + a.own_parts, my = threadIdx.x >> 4, sub = threadIdx.x & 15;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        __syncthreads();
#pragma unroll
        for (int n = 0; n < C::NB; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int w = 0; w < C::W; ++w) so[wave][c16][16 * C::W * n + C::W * (4 * g + r) + w] = o[t][n * C::W + w][r];
        __syncthreads();
        const int col = m0 + 16 * t + my;
        if (col >= cols) continue;
        float top = -INFINITY, f[4], sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][16 * t + my]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = exp2_(sm[w][16 * t + my] - (top == -INFINITY ? 0.f : top));
            sum += f[w] * sl[w][16 * t + my];
        }
        const int row = p.row0 + col / a.g, head = p.h * a.g + col % a.g;
        if (p.direct) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T *dst = reinterpret_cast<T *>(a.out) + (int64_t)row * a.ldo + (int64_t)head * a.hd;
            for (int ch = sub; ch < a.hd; ch += 16) {
                float x = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) x += f[w] * so[w][my][ch];
                dst[ch] = (T)(sum == 0.f ? 0.f : x * inv);
            }
        } else {
            const int64_t at = ((int64_t)row * a.nq + head) * parts + p.part;
            float *dst = a.part_o + at * a.hd;
            for (int ch = 4 * sub; ch < a.hd; ch += 64) {
                f4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) x += f[w] * *reinterpret_cast<const f4_t *>(&so[w][my][ch]);
                *reinterpret_cast<f4_t *>(dst + ch) = x;
            }
            if (sub == 0) *reinterpret_cast<f2_t *>(a.part_ml + 2 * at) = f2_t{top, sum};
        }
    }
}

// The parts of one row and head, a wave each.
template <typename T>
__global__ __launch_bounds__(256) void attn_join_k(const SharedAttnArgs a) {
    const uint32_t item = workgroup() * 4 + (threadIdx.x >> 6);  // below 2^31: the host bounds R * nq
    if (item >= (uint32_t)a.R * (uint32_t)a.nq) return;
    const int lane = threadIdx.x & 63, row = (int)(item / a.nq), head = (int)(item % a.nq);
    int b = -1;
    for (int s0 = 0; s0 < a.n_seq && b < 0; s0 += 64) {
        int first = 0, n = 0;
        if (s0 + lane < a.n_seq) rows_of(a, s0 + lane, first, n);
        const uint64_t mine = __ballot(row >= first && row < first + n);
        if (mine) b = s0 + __ffsll((unsigned long long)mine) - 1;
    }
    if (b < 0) return;  // a row of no sequence
    int used = 0;
    if (a.own_parts) used = own_parts_of(a, b).used;
    const int n = a.prefix_parts + used, parts = a.prefix_parts + a.own_parts;
    if (a.prefix_parts == 0 && used == 1) return;  // written by its only part
    const float *ml = a.part_ml + (int64_t)item * parts * 2, *po = a.part_o + (int64_t)item * parts * a.hd;
    float m = -INFINITY, l = 0.f;
    if (lane < n) { m = ml[2 * lane]; l = ml[2 * lane + 1]; }
    float m2 = -INFINITY, l2 = 0.f;
    if (lane + 64 < n) { m2 = ml[2 * lane + 128]; l2 = ml[2 * lane + 129]; }
    const float top = wave_max(fmaxf(m, m2)), base = top == -INFINITY ? 0.f : top;
    const float f = exp2_(m - base), f2 = exp2_(m2 - base);
    const float sum = wave_sum(f * l + f2 * l2);
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; ++i) {
        const float w = __shfl(i < 64 ? f : f2, i & 63, WAVE);
        // (a part without positions seen holds zeros)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < a.hd) acc[c] += w * po[(int64_t)i * a.hd + lane + 64 * c];
    }
    const float inv = 1.f / sum;
    T *dst = reinterpret_cast<T *>(a.out) + (int64_t)row * a.ldo + (int64_t)head * a.hd;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < a.hd) dst[lane + 64 * c] = (T)(sum == 0.f ? 0.f : acc[c] * inv);
}

// Parts and tiles of a call; a function of the sizes alone, so that the workspace is known beforehand.
void plan_shared_attention(SharedAttnArgs &a, int64_t own_capacity) {
    const int64_t columns = (int64_t)a.R * a.g;
    a.qt = a.dtype == DT_BF16 && columns > (int64_t)16 * a.n_seq ? 2 : 1;
    const int64_t cols = 16 * a.qt;
    const int64_t tiles = (columns + cols - 1) / cols;
    auto parts = [&](int64_t positions, int64_t groups) {
        groups = std::max<int64_t>(groups, 1);
        const int64_t want = (1024 + groups - 1) / groups, most = (positions + MIN_PART - 1) / MIN_PART;
        return std::max<int64_t>(1, std::min<int64_t>({want, most, MAX_PARTS}));
    };
    a.prefix_parts = 0;
    a.prefix_chunk = 0;
    if (a.prefix_len > 0) {
        const int64_t n = parts(a.prefix_len, tiles * a.nkv);
        a.prefix_chunk = (int)(((a.prefix_len + n - 1) / n + TILE - 1) / TILE * TILE);
        a.prefix_parts = (a.prefix_len + a.prefix_chunk - 1) / a.prefix_chunk;
    }
    a.own_tiles = (uint32_t)(a.n_seq + columns / cols);
    a.own_parts = own_capacity > 0 ? (int)parts(own_capacity, std::max<int64_t>(tiles, a.n_seq) * a.nkv) : 0;
    // (prefix_groups, own_groups beyond 2^31 are refused by the launcher)
    a.prefix_groups64 = a.prefix_len > 0 ? tiles * a.nkv * a.prefix_parts : 0;
    a.own_groups64 = (int64_t)a.own_tiles * a.nkv * a.own_parts;
    a.prefix_groups = (uint32_t)a.prefix_groups64;
}

int64_t shared_attention_parts(const SharedAttnArgs &a) {
    const int n = a.prefix_parts + a.own_parts;
    return a.prefix_parts == 0 && a.own_parts <= 1 ? 0 : n;
}

template <class C>
static hipError_t launch_split(const SharedAttnArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((attn_split_k<C>), grid_of(a.prefix_groups64 + a.own_groups64), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int HDP, bool EXACT>
static hipError_t launch_core(const SharedAttnArgs &a, hipStream_t s) {
    if (a.dtype == DT_F32) return launch_split<CoreF32<HDP, EXACT>>(a, s);
    if (a.qt == 1) return launch_split<CoreBf16<HDP, 1, EXACT>>(a, s);
    return launch_split<CoreBf16<HDP, 2, EXACT>>(a, s);
}

template <int HDP>
static hipError_t launch_exact(const SharedAttnArgs &a, hipStream_t s) {
    return a.hd == HDP ? launch_core<HDP, true>(a, s) : launch_core<HDP, false>(a, s);
}

hipError_t launch_shared_attention(const SharedAttnArgs &a, hipStream_t s) {
    if (a.prefix_groups64 + a.own_groups64 > 0x7fffffff) return hipErrorInvalidValue;
    if (a.prefix_groups64 + a.own_groups64 > 0) {
        const hipError_t e = a.hd <= 32 ? launch_exact<32>(a, s) : a.hd <= 64 ? launch_exact<64>(a, s) : a.hd <= 128 ? launch_exact<128>(a, s) : launch_exact<256>(a, s);
        if (e != hipSuccess) return e;
    }
    if (a.prefix_parts == 0 && a.own_parts == 1) return hipSuccess;  // every row is written by its only part
    const dim3 grid = grid_of(((int64_t)a.R * a.nq + 3) / 4);
    if (a.dtype == DT_F32) hipLaunchKernelGGL((attn_join_k<float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_join_k<__bf16>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sd
