// Attention of a batch's rows over a prefix that all sequences share and over every sequence's own positions, from pages.
//
//   o = sum_j softmax_j(scale q . k_j) v_j,   one pass over the positions with a running maximum m and sum l
//
// Columns and lanes.  The query heads that read one cache head, of all rows of a piece, are the columns of one product:
// S^T = K Q^T (16 positions x 16 columns an instruction), then O^T += V^T P^T.  Transposed, column c of S, P and O is held by
// lanes c, c + 16, c + 32, c + 48, so m, l and the rescaling are one number a lane, and what a lane holds of S^T (positions
// 4 g .. 4 g + 3 of each 16, g = lane / 16) is, rounded, its share of the second product's operand: no exchange between lanes
// and no shared memory needed in between.  The positions' order inside a product is free, so a lane loads the rows of V for just
// those positions, 16 bytes of each, and turns 2 x 2 blocks in registers.  Which channels a lane holds is free too: lane
// l % 16 takes W neighbours, so loads and stores are whole vectors.
//
// Pieces.  The prefix is read once for all rows (columns: every row of the batch), the own positions once a sequence; either
// is split into parts along the positions, and a second kernel joins the parts of a row.  Two kernels, by columns: up to 32 a
// workgroup's waves split the positions (bound by memory), from 33 on they share them (bound by the issue of instructions beside
// the matrix units).  4 sequences of 48 columns, 8000 positions: 55 us split, 41 shared; 64 of 36 columns, 1000: 90 and 76.
#include "common.hpp"
#include "params.hpp"

#include <algorithm>
#include <math.h>
#include <type_traits>

namespace sd {

namespace {

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef float f2_t __attribute__((ext_vector_type(2)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

constexpr int TILE = 32;      // positions a wave takes at a time
constexpr int MIN_PART = 128; // least positions of a part: a tile for each of a workgroup's four waves
constexpr int MAX_PARTS = 64;
constexpr int STAGE = 64;     // positions of a stage in shared memory

// What a lane loads at once stays one vector: words that are loop variables of their own share a register tuple whose elements
// the compiler may take for undefined (see isa_guard.py).
template <int N> using words = uint32_t __attribute__((ext_vector_type(N)));

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// over the four lanes of a column
__device__ __forceinline__ float group_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, WAVE));
    return fmaxf(x, __shfl_xor(x, 32, WAVE));
}
__device__ __forceinline__ float group_sum(float x) {
    x += __shfl_xor(x, 16, WAVE);
    return x + __shfl_xor(x, 32, WAVE);
}

// What one lane keeps of QT x 16 columns in bf16.  HDP: head size rounded up to 32, 64, 128 or 256; channels from hd on are
// zeros.  W: neighbouring channels of V a lane holds, NB blocks of 16 W.
template <int HDP_, int QT_, bool EXACT>
struct CoreBf16 {
    typedef __bf16 T;
    static constexpr int HDP = HDP_, QT = QT_, W = HDP >= 128 ? 8 : HDP / 16, NB = HDP / (16 * W), KC = HDP / 32;
    static constexpr int ROOM = HDP <= 128 || EXACT ? 2 : 1;  // waves a SIMD that leave it registers enough
    static constexpr bool LATE = HDP == 256;  // walk() loads V when K's registers are free: both do not fit
    // channel of row r of a lane's i-th block of results
    __device__ __forceinline__ static int channel(int i, int r, int g) { return 16 * W * (i / W) + W * (4 * g + r) + i % W; }
    b8_t q[QT][KC];
    u4_t k[2][KC];            // positions lane % 16 of the tile's two sixteens, channels 32 c + 8 g ..
    words<W / 2> v[8][NB];    // positions 4 g + i of the first (i < 4) and second sixteen, channels W (lane % 16) ..

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
                v[4 * s + i][n] = EXACT || ch < hd ? *reinterpret_cast<const words<W / 2> *>(rows + i * (EXACT ? HDP : hd) + ch) : words<W / 2>(0);
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
        for (int n = 0; n < NB; ++n) v[i][n] = keep ? v[i][n] : words<W / 2>(0);
    }
    // infinities and NaN of row i of this lane's values become zeros (where `on`); whether there were any
    __device__ __forceinline__ bool clean(int i, bool on) {
        bool bad = false;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W / 2; ++w) {
                const uint32_t x = v[i][n][w];
                const bool lo = on && (x & 0x7f80u) == 0x7f80u, hi = on && (x & 0x7f800000u) == 0x7f800000u;
                v[i][n][w] = x & (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
                bad |= lo || hi;
            }
        return bad;
    }
    // Weights in two bf16 terms, 16 significant bits: these pieces wait for memory, and the second instruction comes free.
    struct Weights { b8_t p, rest; };
    __device__ __forceinline__ static Weights weights(const f4_t (&s)[2]) {
        Weights x;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x.p[i] = (__bf16)s[i / 4][i % 4];
            x.rest[i] = (__bf16)(s[i / 4][i % 4] - (float)x.p[i]);
        }
        return x;
    }
    // sums of the weights as they were rounded: products with ones, which leave a column's whole sum with all its lanes
    __device__ __forceinline__ static void add_up(const Weights &w, f4_t &l) {
        const __bf16 one = (__bf16)1.f;
        const b8_t ones = {one, one, one, one, one, one, one, one};
        l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w.p, l, 0, 0, 0);
        l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w.rest, l, 0, 0, 0);
    }
    __device__ __forceinline__ static float total(const f4_t &l) { return l[0]; }
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
                    x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, p[t].rest, x, 0, 0, 0);
                    y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd_, p[t].rest, y, 0, 0, 0);
                }
            }
    }
};

// The same with positions that lie in shared memory, rows of HDP elements.  Values are read turned (a lane's address names four
// channels of a row, and it gets one channel of four rows), so channels stay in their order.  Chunk u (16 bytes) of row r is at
// place u ^ turn(r), which spreads over all banks both the eight rows of one chunk that an eighth of a key load reads and the
// four rows of two chunks that a quarter of a value load does.
template <int HDP_, int QT_, bool EXACT>
struct CoreLds : CoreBf16<HDP_, QT_, EXACT> {
    typedef CoreBf16<HDP_, QT_, EXACT> Base;
    static constexpr int HDP = HDP_, QT = QT_, KC = Base::KC, W = 1, NB = HDP / 16, UNITS = HDP / 8;
    uint32_t v[NB][4];  // channel 16 n + lane % 16, positions 4 g .. + 3 of the first and the second sixteen
    __device__ __forceinline__ static int channel(int i, int r, int g) { return 16 * i + 4 * g + r; }
    __device__ __forceinline__ static int turn(int row) {
        return UNITS == 4 ? (row & 2) | (row >> 2 & 1) : ((row & 3) << 1 | (row >> 2 & 1) | (row & 8)) & (UNITS - 1);
    }
    __device__ __forceinline__ void read_k(int s, const uint8_t *stage, int row, int g) {
#pragma unroll
        for (int c = 0; c < KC; ++c) this->k[s][c] = *reinterpret_cast<const u4_t *>(stage + row * HDP * 2 + (((4 * c + g) ^ turn(row)) << 4));
    }
    __device__ __forceinline__ void read_v(const uint8_t *stage, int row0, int g, int c16) {
        typedef short s4_t __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int row = row0 + 16 * s + 4 * g + (c16 >> 2);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const uint8_t *from = stage + row * HDP * 2 + (((2 * n + (c16 >> 1 & 1)) ^ turn(row)) << 4) + 8 * (c16 & 1);
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t *)from));
                v[n][2 * s] = x.x;
                v[n][2 * s + 1] = x.y;
            }
        }
    }
    // positions i of this lane's (bit i of `keep` off) become zeros
    __device__ __forceinline__ void forget(uint32_t keep) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t both = (keep >> 2 * w & 1 ? 0x0000ffffu : 0u) | (keep >> (2 * w + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
            for (int n = 0; n < NB; ++n) v[n][w] &= both;
        }
    }
    // infinities and NaN at positions whose bit is on become zeros; whether there were any
    __device__ __forceinline__ bool clean(uint32_t on) {
        bool bad = false;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                uint32_t &x = v[n][w];
                const bool lo = (on >> 2 * w & 1) && (x & 0x7f80u) == 0x7f80u, hi = (on >> (2 * w + 1) & 1) && (x & 0x7f800000u) == 0x7f800000u;
                x &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
                bad |= lo || hi;
            }
        return bad;
    }
    // Weights rounded once, as the values are: results are off by 0.0023 of their norm then, with two terms by 0.0017, their own
    // rounding.  Here the second instructions would not come free: 8 x 256 rows behind 8192 positions 280 -> 381 us, heads of 64
    // 166 -> 253, 64 sequences of 36 columns behind 8192 106 -> 123.
    struct Weights { b8_t p; };
    __device__ __forceinline__ static Weights weights(const f4_t (&s)[2]) {
        Weights x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x.p[i] = (__bf16)s[i / 4][i % 4];
        return x;
    }
    __device__ __forceinline__ static void add_up(const Weights &w, f4_t &l) {
        const __bf16 one = (__bf16)1.f;
        const b8_t ones = {one, one, one, one, one, one, one, one};
        l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, w.p, l, 0, 0, 0);
    }
    __device__ __forceinline__ void values(const Weights (&p)[QT], f4_t (&o)[QT][NB]) const {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int t = 0; t < QT; ++t)
                o[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8_t, u4_t{v[n][0], v[n][1], v[n][2], v[n][3]}), p[t].p, o[t][n], 0, 0, 0);
    }
};

// The same in fp32: 16 x 16 x 4 instructions, their four channels (positions) those of the four groups of lanes.
template <int HDP_, bool EXACT>
struct CoreF32 {
    typedef float T;
    static constexpr int HDP = HDP_, QT = 1, W = HDP >= 64 ? 4 : HDP / 16, NB = HDP / (16 * W), KC = HDP / 16;
    static constexpr int ROOM = HDP < 128 ? 2 : 1;
    static constexpr bool LATE = HDP == 256;
    __device__ __forceinline__ static int channel(int i, int r, int g) { return 16 * W * (i / W) + W * (4 * g + r) + i % W; }
    f4_t q[1][KC];   // channels 16 c + 4 g ..
    f4_t k[2][KC];
    words<W> v[8][NB];

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
                v[4 * s + i][n] = EXACT || ch < hd ? *reinterpret_cast<const words<W> *>(rows + i * (EXACT ? HDP : hd) + ch) : words<W>(0);
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
        for (int n = 0; n < NB; ++n) v[i][n] = keep ? v[i][n] : words<W>(0);
    }
    __device__ __forceinline__ bool clean(int i, bool on) {
        bool bad = false;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const bool odd = on && (v[i][n][w] & 0x7f800000u) == 0x7f800000u;
                v[i][n][w] = odd ? 0u : v[i][n][w];
                bad |= odd;
            }
        return bad;
    }
    struct Weights { f4_t p[2]; };
    __device__ __forceinline__ static Weights weights(const f4_t (&s)[2]) { return Weights{{s[0], s[1]}}; }
    __device__ __forceinline__ static void add_up(const Weights &w, f4_t &l) { l += w.p[0] + w.p[1]; }
    __device__ __forceinline__ static float total(const f4_t &l) { return group_sum((l[0] + l[1]) + (l[2] + l[3])); }
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
__device__ __forceinline__ OwnParts own_parts_of(const SharedAttnArgs &a, int own_len) {
    OwnParts p;
    p.len = max(0, min(own_len, a.table_pages << a.page_shift));
    p.chunk = max(MIN_PART, ((p.len + a.own_parts - 1) / a.own_parts + STAGE - 1) & ~(STAGE - 1));  // stages begin with their pages
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
    __device__ __forceinline__ int sees(int row) const { return own ? max(0, len - n + row + 1) : len; }  // positions
};

// Which piece workgroup `id` has: prefix pieces first, tiles of COLS columns.  false: none.  Same answer in every wave.  Sequences
// are looked through sixty-four at a time, a load and seven exchanges each.
template <int COLS>
__device__ __forceinline__ bool piece_of(const SharedAttnArgs &a, uint32_t id, Piece &p) {
    if (id >= a.groups) return false;  // a long grid ends in whole rows
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
    uint32_t tile = id % a.own_tiles;
    const int part = (int)(id / a.own_tiles);
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
        int first = 0, n = 0, len = 0;
        if (s0 + lane < a.n_seq) {
            len = a.own_len[s0 + lane];
            rows_of(a, s0 + lane, first, n);
        }
        // tiles of this sequence, and of it and those in front (row numbers that make no sense may run past 2^32: then the
        // tile found is not one of its sequence, and nobody works on it)
        const uint32_t tiles = (uint32_t)(((int64_t)n * a.g + COLS - 1) / COLS);
        uint32_t upto = tiles;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t o = __shfl_up(upto, m, WAVE);
            if (lane >= m) upto += o;
        }
        const uint64_t beyond = __ballot(upto > tile);
        if (beyond) {
            const int src = uniform(__ffsll((unsigned long long)beyond) - 1), b = s0 + src;
            auto from = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
            p.tile = from((int)(tile - (upto - tiles)));
            if ((uint32_t)p.tile >= (uint32_t)from((int)tiles)) return false;
            p.row0 = from(first);
            p.n = from(n);
            const OwnParts parts = own_parts_of(a, from(len));
            if (part >= parts.used) return false;
            p.own = true;
            p.len = parts.len;
            p.chunk = parts.chunk;
            p.direct = a.prefix_parts == 0 && parts.used == 1;
            p.part = a.prefix_parts + part;
            p.begin = part * p.chunk;
            p.table = a.table + (int64_t)b * a.table_pages;
            p.pages = a.table_pages;
            return true;
        }
        tile -= (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    return false;
}

// The prefix in front of a piece of own positions, for the same rows.
__device__ __forceinline__ Piece prefix_of(const SharedAttnArgs &a, const Piece &own) {
    Piece p = own;
    p.table = a.prefix_table;
    p.pages = ((a.prefix_len - 1) >> a.page_shift) + 1;
    p.len = p.chunk = a.prefix_len;
    p.begin = 0;
    p.own = false;
    return p;
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
    const uint32_t pg = (uint32_t)page < (uint32_t)a.n_pages ? page : 0;
    // (slots are below 2^31, and so are slots of all heads below 2^51)
    return (int64_t)(((uint64_t)(pg * (uint64_t)(uint32_t)a.nkv + (uint32_t)h) << a.page_shift) + (uint32_t)(t & ((1 << a.page_shift) - 1))) * a.hd;
}

// Reference, sum and results of a wave's columns.  Weights are powers of two over a reference, which follows the maximum
// at a distance: it moves when a score (in powers of two) lies more than 8 above it.  Weights stay below 2^8, which costs no
// precision, and most tiles need neither the exchange between lanes nor the rescaling.
// An exponent is one multiply-add, s * scale2 - m * scale2: rounding the second product moves a reference below FAR by 2^-14
// at most, in the range of what rounding the scores themselves does, but beyond it would grow past the range of the weights.
// There every tile looks at its maximum, and the reference is taken off before the scaling.
template <class C>
struct Running {
    static constexpr int QT = C::QT, NO = C::NB * C::W;
    static constexpr float FAR = 1024.f;
    float m[QT];      // the reference, a score not yet scaled: -infinity before there is one
    float base[QT];   // scaled; 0 before there is one and beyond FAR
    float bound[QT];  // scores, not yet scaled, that move it
    f4_t l[QT], o[QT][NO];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            m[t] = bound[t] = -INFINITY;
            base[t] = 0.f;
            l[t] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NO; ++i) o[t][i] = l[t];
        }
    }
    __device__ __forceinline__ void follow(f4_t (&s)[QT][2], float scale2, float lift) {
        float top[QT];
        bool above = false;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            top[t] = s[t][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top[t] = fmaxf(top[t], s[t][i / 4][i % 4]);
            above |= top[t] > bound[t];
        }
        if (__ballot(above)) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const float to = fmaxf(m[t], group_max(top[t]));
                const float ref = to == -INFINITY ? 0.f : to, by = exp2_((m[t] - ref) * scale2), scaled = ref * scale2;
                const bool far = fabsf(scaled) >= FAR;
                m[t] = to;
                base[t] = far ? 0.f : scaled;
                bound[t] = far ? -INFINITY : to + lift;
                l[t] *= by;
#pragma unroll
                for (int i = 0; i < 8; ++i) s[t][i / 4][i % 4] -= far ? ref : 0.f;
#pragma unroll
                for (int i = 0; i < NO; ++i) o[t][i] *= by;
            }
        }
    }
    __device__ __forceinline__ void weigh(f4_t (&s)[QT][2], float scale2, typename C::Weights (&w)[QT]) const {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s[t][i / 4][i % 4] = exp2_(fmaf(s[t][i / 4][i % 4], scale2, -base[t]));
            w[t] = C::weights(s[t]);
        }
    }
    __device__ __forceinline__ void add(const C &core, const typename C::Weights (&w)[QT]) {
#pragma unroll
        for (int t = 0; t < QT; ++t) C::add_up(w[t], l[t]);
        core.values(w, o);
    }
};

// Values that are infinite or NaN at positions that some columns of a tile see and others do not: 0 times them would reach the
// others, so the products have zeros in their place, and at the end every column adds those it sees (times any weight they
// are what they are).  Positions from .. end - 1, of every `of` tiles those of number `nth`.
template <class C, int QT = C::QT>
__device__ __forceinline__ void add_odd(const SharedAttnArgs &a, const Piece &p, int from, int end, int nth, int of, const int (&lim)[QT],
                                        Running<C> &run) {
    typedef typename C::T T;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    for (int x = max(from, p.begin); x < end; ++x) {
        if ((x - p.begin) / TILE % of != nth) continue;
        const int page = p.table[min(x >> a.page_shift, p.pages - 1)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
        const T *row = reinterpret_cast<const T *>(a.v_pages) + element(a, page, p.h, x);
#pragma unroll
        for (int i = 0; i < C::NB * C::W; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int ch = C::channel(i, r, g);
                float v = ch < a.hd ? (float)row[ch] : 0.f;
                if ((__float_as_uint(v) & 0x7f800000u) != 0x7f800000u) v = 0.f;
#pragma unroll
                for (int t = 0; t < QT; ++t) run.o[t][i][r] += x < lim[t] ? v : 0.f;
            }
    }
}

// Tiles t0, t0 + step, .. up to `end`, straight from the pages; columns see at least `least` positions.  odd: whether values
// were left for add_odd().  The loads of a tile are on their way while the one before is worked on: K's from its scores on, V's
// from its values' product on.
template <class C>
__device__ __forceinline__ void walk(const SharedAttnArgs &a, const Piece &p, C &core, const int (&lim)[C::QT], Running<C> &run, int t0, const int step,
                                     const int end, const int least, int &odd) {
    typedef typename C::T T;
    constexpr int QT = C::QT;
    const int lane = threadIdx.x & 63, g = lane >> 4, c16 = lane & 15;
    const T *kp = reinterpret_cast<const T *>(a.k_pages), *vp = reinterpret_cast<const T *>(a.v_pages);
    auto load_k = [&](const Places &x, int t0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) core.load_k(s, kp + element(a, x.k[s], p.h, t0 + 16 * s + c16), a.hd, g);
    };
    auto load_v = [&](const Places &x, int t0) {
#pragma unroll
        for (int s = 0; s < 2; ++s) core.load_v(s, vp + element(a, x.v[s], p.h, t0 + 16 * s + 4 * g), a.hd, c16);
    };
    if (t0 >= end) return;
    Places now = places_of(a, p, t0, c16, g), next = places_of(a, p, t0 + step, c16, g);
    load_k(now, t0);
    if constexpr (!C::LATE) load_v(now, t0);
    for (; t0 < end; t0 += step) {
        f4_t s[QT][2];
#pragma unroll
        for (int t = 0; t < QT; ++t) core.scores(t, s[t]);
        const int t1 = t0 + step;
        const bool more = t1 < end;
        if constexpr (C::LATE) load_v(now, t0);
        else if (more) load_k(next, t1);
        const bool there[2] = {(uint32_t)now.v[0] < (uint32_t)a.n_pages, (uint32_t)now.v[1] < (uint32_t)a.n_pages};
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
                if (core.clean(i, at >= least)) bad = true;
            }
            if (__ballot(bad)) odd = 1;
        }
        run.follow(s, a.scale2, a.lift);
        typename C::Weights w[QT];
        run.weigh(s, a.scale2, w);
        run.add(core, w);
        if (more) {
            if constexpr (C::LATE) load_k(next, t1);
            else load_v(next, t1);
            now = next;
            next = places_of(a, p, t1 + step, c16, g);
        }
    }
}

// Queries of a wave's columns from m0 on; columns past the last one repeat it.
template <class C>
__device__ __forceinline__ void take_columns(const SharedAttnArgs &a, const Piece &p, int m0, C &core) {
    const int lane = threadIdx.x & 63, cols = p.n * a.g;
#pragma unroll
    for (int t = 0; t < C::QT; ++t) {
        const int col = min(m0 + 16 * t + (lane & 15), cols - 1), row = col / a.g;
        core.load_q(t, reinterpret_cast<const typename C::T *>(a.q) + (int64_t)(p.row0 + row) * a.ldq + (int64_t)(p.h * a.g + col % a.g) * a.hd,
                    a.q_whole, a.hd, lane >> 4);
    }
}
// Positions each of them sees.
template <int QT>
__device__ __forceinline__ void limits(const SharedAttnArgs &a, const Piece &p, int m0, int (&lim)[QT]) {
    const int lane = threadIdx.x & 63, cols = p.n * a.g;
#pragma unroll
    for (int t = 0; t < QT; ++t) lim[t] = p.sees(min(m0 + 16 * t + (lane & 15), cols - 1) / a.g);
}

}  // namespace

// Few columns: the four waves of a workgroup take the same QT x 16 columns and every fourth tile of the positions, and
// join their sums through shared memory at the end.  8 sequences of 40 heads of 128, 2001 + up to 4096 positions: 84 us for
// 398 MB, 4.7 TB/s (read only; a copy reaches 6.1 both ways).  One token behind 356 positions: 7.7, a chain of dependent loads
// (row numbers, pages, keys).
template <class C, bool THROUGH>
__device__ __forceinline__ void split(const SharedAttnArgs &a, float (*so)[16][C::HDP + 4], float (*sm)[32], float (*sl)[32]) {
    typedef typename C::T T;
    constexpr int QT = C::QT;
    Piece whole;
    if (!piece_of<QT * 16>(a, workgroup(), whole)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
    const int cols = whole.n * a.g, m0 = whole.tile * QT * 16;
    C core;
    Running<C> run;
    take_columns(a, whole, m0, core);
    run.clear();
#pragma unroll 1
    for (int segment = THROUGH ? 0 : 1; segment < 2; ++segment) {
        const Piece p = THROUGH && segment == 0 ? prefix_of(a, whole) : whole;
        int lim[QT], odd = 0;
        limits(a, p, m0, lim);
        // positions that the first column sees, and those that the last one does within this part
        const int least = p.sees(m0 / a.g), end = min(p.begin + p.chunk, p.sees((min(m0 + QT * 16, cols) - 1) / a.g));
        walk(a, p, core, lim, run, p.begin + TILE * wave, 4 * TILE, end, least, odd);
        if (uniform(odd)) add_odd(a, p, least, end, wave, 4, lim, run);
    }
    // the waves' sums meet: 16 columns at a time
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const float sum = C::total(run.l[t]);
        if (g == 0) { sm[wave][16 * t + c16] = run.m[t]; sl[wave][16 * t + c16] = sum; }
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
                for (int w = 0; w < C::W; ++w) so[wave][c16][16 * C::W * n + C::W * (4 * g + r) + w] = run.o[t][n * C::W + w][r];
        __syncthreads();
        const int col = m0 + 16 * t + my;
        if (col >= cols) continue;
        float top = -INFINITY, f[4], sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w][16 * t + my]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = exp2_((sm[w][16 * t + my] - (top == -INFINITY ? 0.f : top)) * a.scale2);
            sum += f[w] * sl[w][16 * t + my];
        }
        const int row = whole.row0 + col / a.g, head = whole.h * a.g + col % a.g;
        if (whole.direct) {
            const float inv = 1.f / sum;
            T *dst = reinterpret_cast<T *>(a.out) + (int64_t)row * a.ldo + (int64_t)head * a.hd;
            for (int ch = sub; ch < a.hd; ch += 16) {
                float x = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) x += f[w] * so[w][my][ch];
                dst[ch] = (T)(sum == 0.f ? 0.f : x * inv);
            }
        } else {
            const int64_t at = ((int64_t)row * a.nq + head) * parts + whole.part;
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

// Pieces of the prefix as CP, of own positions as CO: the rows of all sequences are more columns than those of one.  THROUGH:
// pieces of own positions alone, and each goes through the prefix first.
template <class CP, class CO, bool THROUGH>
__global__ __launch_bounds__(256, CP::ROOM) void attn_split_k(const SharedAttnArgs a) {
    __shared__ float so[4][16][CP::HDP + 4], sm[4][32], sl[4][32];
    if (std::is_same<CP, CO>::value || workgroup() < a.prefix_groups) split<CP, THROUGH>(a, so, sm, sl);
    else split<CO, THROUGH>(a, so, sm, sl);
}

// f(num<0>) .. f(num<N - 1>)
template <int N> using num = std::integral_constant<int, N>;
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(num<N - 1>());
    }
}

// The copies of this wave have arrived, and with the barrier those of all waves.
__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // no instruction: keeps memory operations on their side
    __builtin_amdgcn_s_waitcnt(0x0070);                     // vmcnt(0), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 bytes a lane from memory to a wave's KiB of shared memory, without passing through registers
__device__ __forceinline__ void copy16(const void *from, uint8_t *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// Many columns: every wave has QT x 16 of its own, and those of a workgroup share the positions, which pass through shared
// memory in stages of 64, three in turn.  The loop is for whole stages that all columns see; the positions behind them, and
// pieces with pages outside the pool, follow stage by stage.
// 8 x 256 rows of 32 heads of 128 on 8 behind 8192 positions (256 columns, eight waves of 32): 272 - 288 us, 1.0 PFLOP/s, about 2 us
// a stage: the matrix units are busy 42 % of the cycles, shared memory 40 %; a SIMD's two waves leave each meeting together, and
// each issues 16 exponentials, 16 multiply-adds, 8 conversions and 24 LDS reads for its 34 matrix instructions.  Four waves of 64
// columns read LDS half as often, but what ends in the second half of the register file has to be moved: 352.  Turning values
// by permutes costs 32 instructions more: 307.
// Heads up to 64 are compiled for two waves a SIMD, also four waves a workgroup: with one, the compiler spreads what fits over both
// halves of the file and moves it (8 x 256 rows behind 8192 positions, heads of 32: 182 us for 155; 4 sequences of 80 columns,
// 8000 positions, heads of 64: 35.3 for 32.5).  Larger heads' stages leave room for one workgroup anyway.
template <int HDP, int QT, int WAVES, bool EXACT>
__global__ __launch_bounds__(64 * WAVES, HDP <= 64 ? 2 : WAVES / 4) void attn_share_k(const SharedAttnArgs a) {
    typedef CoreLds<HDP, QT, EXACT> C;
    typedef __bf16 T;
    constexpr int UNITS = C::UNITS, BYTES = STAGE * HDP * 2, SHARE = WAVES * 1024, COPIES = BYTES / SHARE, COLS = 16 * QT * WAVES;
    static_assert(COPIES >= 1 && BYTES % SHARE == 0, "every thread copies");
    __shared__ __attribute__((aligned(16))) uint8_t k0[BYTES], k1[BYTES], k2[BYTES], v0[BYTES], v1[BYTES], v2[BYTES];
    Piece whole;
    if (!piece_of<COLS>(a, workgroup(), whole)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, c16 = lane & 15;
    const int cols = whole.n * a.g, first = whole.tile * COLS, m0 = first + wave * 16 * QT;
    C core;
    Running<C> run;
    int lim[QT], odd = 0;
    take_columns(a, whole, m0, core);
    run.clear();
    if constexpr (!EXACT) {  // chunks beyond hd are never copied: the products need numbers there
        uint8_t *every[6] = {k0, k1, k2, v0, v1, v2};
#pragma unroll
        for (int i = 0; i < 6; ++i)
            for (int b = threadIdx.x * 16; b < BYTES; b += SHARE) *reinterpret_cast<u4_t *>(every[i] + b) = u4_t{0, 0, 0, 0};
    }
    const T *kp = reinterpret_cast<const T *>(a.k_pages), *vp = reinterpret_cast<const T *>(a.v_pages);
    // what this thread copies of a stage: one chunk each of rows i * STEP + mine
    constexpr int STEP = SHARE / 16 / UNITS;
    static_assert(STEP % 16 == 0, "the chunk is the same in each of them");
    const int mine = (wave * 64 + lane) / UNITS, chunk = lane % UNITS ^ C::turn(mine), step = STEP * (EXACT ? HDP : a.hd);
    const uint32_t at = mine * (EXACT ? HDP : a.hd) + chunk * 8;
#pragma unroll 1
    for (int segment = a.through ? 0 : 1; segment < 2; ++segment) {
        const Piece p = segment == 0 ? prefix_of(a, whole) : whole;
        auto page_at = [&](int st) { return p.table[min((p.begin + st * STAGE + lane) >> a.page_shift, p.pages - 1)]; };
        auto copy = [&](int st, int page, uint8_t *ks, uint8_t *vs) {
            const int t0 = p.begin + st * STAGE;
            const bool there = EXACT || chunk * 8 < a.hd;
            if (a.page_shift >= 6) {  // one page
                const int64_t base = element(a, uniform(page), p.h, t0);
                if (there) {
#pragma unroll
                    for (int i = 0; i < COPIES; ++i) {
                        copy16(kp + base + i * step + at, ks + i * SHARE + wave * 1024);
                        copy16(vp + base + i * step + at, vs + i * SHARE + wave * 1024);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < COPIES; ++i) {  // (every lane takes part in the exchange)
                    const int64_t from = element(a, __shfl(page, i * STEP + mine, WAVE), p.h, t0 + i * STEP + mine) + chunk * 8;
                    if (there) {
                        copy16(kp + from, ks + i * SHARE + wave * 1024);
                        copy16(vp + from, vs + i * SHARE + wave * 1024);
                    }
                }
            }
        };
        limits(a, p, m0, lim);
        // positions: of the part that some column sees, and stages that all columns see
        const int end = min(p.begin + p.chunk, p.sees((min(first + COLS, cols) - 1) / a.g));
        const int all = (max(0, end - p.begin) + STAGE - 1) / STAGE;
        int stages = max(0, min(end, p.sees(first / a.g)) - p.begin) / STAGE, page = 0;
        if (stages > 0) {
            // the first copies set out, and meanwhile every wave looks at the pages and comes to the same answer
            __syncthreads();
            const int page0 = page_at(0), page1 = page_at(1);
            bool gone = false;
            const int last = (p.begin + stages * STAGE - 1) >> a.page_shift;
            for (int i = (p.begin >> a.page_shift) + lane; i <= last; i += 64) gone |= (uint32_t)p.table[min(i, p.pages - 1)] >= (uint32_t)a.n_pages;
            copy(0, page0, k0, v0);
            if (stages > 1) copy(1, page1, k1, v1);
            page = page_at(2);  // of the stage after the last copy's
            if (__ballot(gone)) stages = 0;
        }
        f4_t s[2][QT][2];
        auto scores = [&](const uint8_t *ks, int half, f4_t (&to)[QT][2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) core.read_k(h, ks, 32 * half + 16 * h + c16, g);
#pragma unroll
            for (int t = 0; t < QT; ++t) core.scores(t, to[t]);
        };
        if (stages > 0) {
            auto kst = [&](auto n) -> uint8_t * { return n % 3 == 0 ? k0 : n % 3 == 1 ? k1 : k2; };
            auto vst = [&](auto n) -> uint8_t * { return n % 3 == 0 ? v0 : n % 3 == 1 ? v1 : v2; };
            // one half of a stage, whose scores are there; `next` computes those of the half behind it meanwhile
            auto half_step = [&](const uint8_t *vs, int half, f4_t (&x)[QT][2], auto next) {
                run.follow(x, a.scale2, a.lift);
                next();
                typename C::Weights w[QT];
                run.weigh(x, a.scale2, w);
                core.read_v(vs, 32 * half, g, c16);
                run.add(core, w);
            };
            meet();
            scores(k0, 0, s[0]);
            for (int st0 = 0; st0 < stages; st0 += 3) {
                each<3>([&](auto n) {
                    const int st = st0 + n;
                    if (st >= stages) return;
                    half_step(vst(n), 0, s[0], [&]() { scores(kst(n), 1, s[1]); });
                    // the next stage has arrived; the one before this has been read by all
                    meet();
                    if (st + 2 < stages) {
                        copy(st + 2, page, kst(num<n + 2>()), vst(num<n + 2>()));
                        page = page_at(st + 3);
                    }
                    // (behind the last stage: scores of an old one, which nobody reads)
                    half_step(vst(n), 1, s[1], [&]() { scores(kst(num<n + 1>()), 0, s[0]); });
                });
            }
        }
        const int least = p.sees(min(m0, cols - 1) / a.g);  // positions that all of this wave's columns see
        for (int st = stages; st < all; ++st) {
            const int page = page_at(st);
            const uint64_t there = __ballot((uint32_t)page < (uint32_t)a.n_pages);
            __syncthreads();
            copy(st, page, k0, v0);
            meet();
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                const int t0 = p.begin + st * STAGE + 32 * half;
                scores(k0, half, s[0]);
                core.read_v(v0, 32 * half, g, c16);
                uint32_t keep = 0, apart = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int pos = 16 * (i / 4) + 4 * g + i % 4;
                    const bool seen = (there >> (32 * half + pos) & 1) && t0 + pos < end;
#pragma unroll
                    for (int t = 0; t < QT; ++t)
                        if (!seen || t0 + pos >= lim[t]) s[0][t][i / 4][i % 4] = -INFINITY;
                    keep |= (uint32_t)seen << i;
                    apart |= (uint32_t)(t0 + pos >= least) << i;
                }
                core.forget(keep);
                if (__ballot(core.clean(apart))) odd = 1;
                run.follow(s[0], a.scale2, a.lift);
                typename C::Weights w[QT];
                run.weigh(s[0], a.scale2, w);
                run.add(core, w);
            }
        }
        if (uniform(odd)) add_odd(a, p, max(least, p.begin + stages * STAGE), end, 0, 1, lim, run);
        odd = 0;
    }
    const int parts = a.prefix_parts + a.own_parts;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int col = m0 + 16 * t + c16;
        if (col >= cols) continue;
        const int row = whole.row0 + col / a.g, head = whole.h * a.g + col % a.g;
        const float sum = C::total(run.l[t]), inv = 1.f / sum;
        const int64_t at = ((int64_t)row * a.nq + head) * parts + whole.part;
        float *po = a.part_o + at * a.hd;
        T *out = reinterpret_cast<T *>(a.out) + (int64_t)row * a.ldo + (int64_t)head * a.hd;
        if (!whole.direct && g == 0) *reinterpret_cast<f2_t *>(a.part_ml + 2 * at) = f2_t{run.m[t], sum};
#pragma unroll
        for (int n = 0; n < C::NB; ++n) {
            const int ch = 16 * n + 4 * g;
            if (!EXACT && ch >= a.hd) continue;
            if (whole.direct) {
#pragma unroll
                for (int r = 0; r < 4; ++r) out[ch + r] = (T)(sum == 0.f ? 0.f : run.o[t][n][r] * inv);
            } else {
                *reinterpret_cast<f4_t *>(po + ch) = run.o[t][n];
            }
        }
    }
}

// The parts of one row and head, a wave each: LPP lanes hold four neighbouring channels each, 64 / LPP parts at a time, four of
// these on their way (319 rows of 32 heads, eight parts: 10 us, 42 MB; 24 rows of 40 heads, one part at a time: 21, so 5).
template <typename T, int LPP>
__global__ __launch_bounds__(256) void attn_join_k(const SharedAttnArgs a) {
    const uint32_t item = workgroup() * 4 + (threadIdx.x >> 6);  // below 2^31: the host bounds R * nq
    if (item >= (uint32_t)a.R * (uint32_t)a.nq) return;
    const int lane = threadIdx.x & 63, row = (int)(item / a.nq), head = (int)(item % a.nq);
    int used = -1;
    for (int s0 = 0; s0 < a.n_seq && used < 0; s0 += 64) {
        int first = 0, n = 0, len = 0;
        if (s0 + lane < a.n_seq) {
            if (a.own_parts) len = a.own_len[s0 + lane];
            rows_of(a, s0 + lane, first, n);
        }
        const uint64_t mine = __ballot(row >= first && row < first + n);
        if (mine) used = a.own_parts ? own_parts_of(a, uniform(__shfl(len, __ffsll((unsigned long long)mine) - 1, WAVE))).used : 0;
    }
    if (used < 0) return;  // a row of no sequence
    const int n = a.prefix_parts + used, parts = a.prefix_parts + a.own_parts;
    if (a.prefix_parts == 0 && used == 1) return;  // written by its only part
    const float *ml = a.part_ml + (int64_t)item * parts * 2, *po = a.part_o + (int64_t)item * parts * a.hd;
    f2_t x = {-INFINITY, 0.f}, y = {-INFINITY, 0.f};
    if (lane < n) x = *reinterpret_cast<const f2_t *>(ml + 2 * lane);
    if (lane + 64 < n) y = *reinterpret_cast<const f2_t *>(ml + 2 * lane + 128);
    const float top = wave_max(fmaxf(x[0], y[0])), base = top == -INFINITY ? 0.f : top;
    // (a part without positions seen has weight 0 and holds zeros)
    const float f = exp2_((x[0] - base) * a.scale2), f2 = exp2_((y[0] - base) * a.scale2), sum = wave_sum(f * x[1] + f2 * y[1]);
    const int ch = 4 * (lane % LPP), which = lane / LPP;
    f4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < n; i0 += 4 * (64 / LPP)) {
        f4_t v[4];
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * (64 / LPP) + which;
            const float fi = __shfl(f, i & 63, WAVE), fj = __shfl(f2, i & 63, WAVE);
            w[j] = i < 64 ? fi : fj;
            v[j] = f4_t{0.f, 0.f, 0.f, 0.f};
            if (i < n && ch < a.hd) v[j] = *reinterpret_cast<const f4_t *>(po + (int64_t)i * a.hd + ch);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + j * (64 / LPP) + which < n) acc += w[j] * v[j];
    }
#pragma unroll
    for (int m = LPP; m < 64; m <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], m, WAVE);
    if (which != 0 || ch >= a.hd) return;
    const float inv = 1.f / sum;
    T *dst = reinterpret_cast<T *>(a.out) + (int64_t)row * a.ldo + (int64_t)head * a.hd + ch;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = (T)(sum == 0.f ? 0.f : acc[e] * inv);
}

// Parts and tiles of a call; a function of the sizes alone, so that the workspace is known beforehand.
void plan_shared_attention(SharedAttnArgs &a, int64_t own_capacity) {
    const int64_t columns = (int64_t)a.R * a.g, each_seq = columns / a.n_seq;  // of a cache head; of one sequence, on average
    // Columns a workgroup takes: 16 or 32 where its waves split the positions, 64, 128 or 256 where they share them.
    auto kind = [&](int64_t n) {
        if (a.dtype != DT_BF16) return 16;
        if (n > 32 && a.hd <= 128) return n > 128 ? 256 : n > 64 ? 128 : 64;
        return n > 16 && a.hd <= 128 ? 32 : 16;
    };
    a.prefix_cols = kind(columns);
    a.own_cols = kind(each_seq);
    const int64_t prefix_tiles = a.prefix_len > 0 ? (columns + a.prefix_cols - 1) / a.prefix_cols : 0;
    const int64_t own_tiles = own_capacity > 0 ? std::max<int64_t>((columns + a.own_cols - 1) / a.own_cols, a.n_seq) : 0;
    // Pieces whose waves split the positions, of prefix and own together: a thousand workgroups, parts of the same length; no
    // shorter ones than 512 where the pieces are enough by themselves (16 sequences of 40 fp32 heads, 500 positions behind
    // 500: 88 us in two parts, 76 in one)
    const int64_t pieces = a.nkv * ((a.prefix_cols < 64 ? prefix_tiles : 0) + (a.own_cols < 64 ? own_tiles : 0));
    const int64_t work = a.nkv * ((a.prefix_cols < 64 ? prefix_tiles * a.prefix_len : 0) + (a.own_cols < 64 ? own_tiles * own_capacity : 0));
    const int64_t length = std::max<int64_t>(pieces >= 512 ? 512 : MIN_PART, (work + 1023) / 1024);
    auto parts = [&](int64_t positions, int64_t groups, int cols) -> int64_t {
        groups = std::max<int64_t>(groups, 1);
        const int64_t most = std::min<int64_t>((positions + MIN_PART - 1) / MIN_PART, MAX_PARTS);
        if (cols < 64) return std::max<int64_t>(1, std::min((positions + length - 1) / length, most));
        // one workgroup a compute unit, in rounds of 256.  Measured: 2 us a stage, 6 a start, and what the parts' sums take to
        // be written and read (5 TB/s)
        int64_t best = 1;
        double least = 1e300;
        const double stages = (double)((positions + STAGE - 1) / STAGE), join = 8e-6 / 5.0 * (double)a.R * a.nq * a.hd;
        for (int64_t n = 1; n <= most; ++n) {
            const double cost = (double)((groups * n + 255) / 256) * (2.0 * std::ceil(stages / n) + 6.0) + join * n;
            if (cost < least) { least = cost; best = n; }
        }
        return best;
    };
    a.prefix_parts = a.own_parts = a.prefix_chunk = 0;
    a.prefix_groups64 = a.own_groups64 = 0;
    if (a.prefix_len > 0) {
        const int64_t n = parts(a.prefix_len, prefix_tiles * a.nkv, a.prefix_cols);
        a.prefix_chunk = (int)(((a.prefix_len + n - 1) / n + STAGE - 1) / STAGE * STAGE);
        a.prefix_parts = (a.prefix_len + a.prefix_chunk - 1) / a.prefix_chunk;
        a.prefix_groups64 = prefix_tiles * a.nkv * a.prefix_parts;
    }
    a.own_tiles = (uint32_t)(a.n_seq + columns / a.own_cols);
    if (own_capacity > 0) {
        a.own_parts = (int)parts(own_capacity, own_tiles * a.nkv, a.own_cols);
        a.own_groups64 = (int64_t)a.own_tiles * a.nkv * a.own_parts;
    }
    // A workgroup goes through prefix and own positions by itself, and nothing is left to join, where there are enough of them
    // without sharing out the prefix (8 x 256 rows behind 8192 positions: 285 us, 316 in parts; few columns, whose prefix would take
    // a launch of its own: 32 tokens behind 512 + 512 positions 21 and 32, behind 1000 + 1000 42 and 53), or so little to go
    // through that the second launch would take longer.  One token of 32 heads on 8, through and in parts, by positions of
    // both: heads of 32 (64 bytes) 512 6.6 and 7.6; of 64 448 7.6 and 7.8, 512 8.0 and 7.8; of 128 320 8.6 and 8.8, 384 9.4 and
    // 8.8; of 256 192 9.9 and 10.2, 256 10.9 and 10.3; fp32 like the bf16 heads of as many bytes.
    const int64_t groups = (a.own_cols >= 64 ? (columns + a.own_cols - 1) / a.own_cols : own_tiles) * a.nkv;
    const bool most = groups >= 192 && (a.own_cols >= 64 || (a.prefix_cols >= 64 && a.prefix_len <= 1024 && own_capacity <= 1024));
    const int64_t bytes = (int64_t)a.hd * (a.dtype == DT_F32 ? 4 : 2);
    const bool little = a.own_cols < 64 && (a.prefix_len + own_capacity) * (128 + bytes) <= 125000;
    a.through = a.prefix_len > 0 && own_capacity > 0 && (most || little);
    if (a.through) {
        a.prefix_parts = 0;
        a.prefix_groups64 = 0;
        a.own_parts = 1;
        a.own_groups64 = (int64_t)a.own_tiles * a.nkv;
    }
    a.prefix_groups = (uint32_t)a.prefix_groups64;
}

int64_t shared_attention_parts(const SharedAttnArgs &a) {
    const int n = a.prefix_parts + a.own_parts;
    return a.prefix_parts == 0 && a.own_parts <= 1 ? 0 : n;
}

// Pieces of the prefix and of own positions, of either kind or (parts that split the positions) both.
template <int HDP, bool EXACT>
static hipError_t launch_cols(const SharedAttnArgs &a, int prefix_cols, int own_cols, int64_t groups, hipStream_t s) {
    const dim3 grid = grid_of(groups), block(256);
    typedef CoreBf16<HDP, 1, EXACT> One;
    if (a.dtype == DT_F32) {
        typedef CoreF32<HDP, EXACT> C;
        if (a.through) hipLaunchKernelGGL((attn_split_k<C, C, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((attn_split_k<C, C, false>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    if constexpr (HDP <= 128) {
        typedef CoreBf16<HDP, 2, EXACT> Two;
        constexpr int WIDE = HDP == 32 ? 4 : 8;  // waves of 256 columns (heads of 32: a stage is too small to be copied by eight)
        switch (prefix_cols) {
            case 256: hipLaunchKernelGGL((attn_share_k<HDP, 16 / WIDE, WIDE, EXACT>), grid, dim3(64 * WIDE), 0, s, a); return hipGetLastError();
            case 128: hipLaunchKernelGGL((attn_share_k<HDP, 2, 4, EXACT>), grid, block, 0, s, a); return hipGetLastError();
            case 64: hipLaunchKernelGGL((attn_share_k<HDP, 1, 4, EXACT>), grid, block, 0, s, a); return hipGetLastError();
            case 32:
                if (a.through) hipLaunchKernelGGL((attn_split_k<Two, Two, true>), grid, block, 0, s, a);
                else if (own_cols == 32) hipLaunchKernelGGL((attn_split_k<Two, Two, false>), grid, block, 0, s, a);
                else hipLaunchKernelGGL((attn_split_k<Two, One, false>), grid, block, 0, s, a);
                return hipGetLastError();
            default: break;
        }
    }
    if (a.through) hipLaunchKernelGGL((attn_split_k<One, One, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attn_split_k<One, One, false>), grid, block, 0, s, a);
    return hipGetLastError();
}

static hipError_t launch_head(const SharedAttnArgs &a, int prefix_cols, int own_cols, int64_t groups, hipStream_t s) {
    if (groups == 0) return hipSuccess;
    if (a.hd <= 32) return a.hd == 32 ? launch_cols<32, true>(a, prefix_cols, own_cols, groups, s) : launch_cols<32, false>(a, prefix_cols, own_cols, groups, s);
    if (a.hd <= 64) return a.hd == 64 ? launch_cols<64, true>(a, prefix_cols, own_cols, groups, s) : launch_cols<64, false>(a, prefix_cols, own_cols, groups, s);
    if (a.hd <= 128) return a.hd == 128 ? launch_cols<128, true>(a, prefix_cols, own_cols, groups, s) : launch_cols<128, false>(a, prefix_cols, own_cols, groups, s);
    return a.hd == 256 ? launch_cols<256, true>(a, prefix_cols, own_cols, groups, s) : launch_cols<256, false>(a, prefix_cols, own_cols, groups, s);
}

template <typename T>
static hipError_t launch_join(const SharedAttnArgs &a, hipStream_t s) {
    const dim3 grid = grid_of(((int64_t)a.R * a.nq + 3) / 4), block(256);
    if (a.hd <= 32) hipLaunchKernelGGL((attn_join_k<T, 8>), grid, block, 0, s, a);
    else if (a.hd <= 64) hipLaunchKernelGGL((attn_join_k<T, 16>), grid, block, 0, s, a);
    else if (a.hd <= 128) hipLaunchKernelGGL((attn_join_k<T, 32>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((attn_join_k<T, 64>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_shared_attention(const SharedAttnArgs &args, hipStream_t s) {
    SharedAttnArgs a = args;
    auto launch = [&](int prefix_cols, int64_t groups) {
        a.groups = (uint32_t)groups;
        return launch_head(a, prefix_cols, a.own_cols, groups, s);
    };
    if (a.prefix_groups64 + a.own_groups64 > 0x7fffffff) return hipErrorInvalidValue;
    hipError_t e;
    if (a.through) {
        e = launch(a.own_cols, a.own_groups64);
    } else if (a.prefix_cols == a.own_cols || (a.prefix_cols == 32 && a.own_cols == 16)) {  // in one launch
        e = launch(a.prefix_cols, a.prefix_groups64 + a.own_groups64);
    } else {
        e = launch(a.prefix_cols, a.prefix_groups64);
        a.prefix_groups = 0;
        if (e == hipSuccess) e = launch(a.own_cols, a.own_groups64);
    }
    if (e != hipSuccess) return e;
    if (a.prefix_parts == 0 && a.own_parts == 1) return hipSuccess;  // every row is written by its only part
    return a.dtype == DT_F32 ? launch_join<float>(a, s) : launch_join<__bf16>(a, s);
}

}  // namespace sd
