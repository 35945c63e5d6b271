// What the kernels of attention share: tiles of rows in LDS, fragments of them, and the mapping of work-groups to work.
//
// The queries that share a key head are taken together: row u of a sequence and key head is position u / group, head u % group of the group, so a tile of 32
// of them holds several heads of one position as well as several positions of one head, and every tile of keys and values is read once for all of them.
//
// Products go through v_mfma_f32_32x32: out[m][n] += sum_k A[m][k] B[k][n], with lane l = 32 h + i holding A[i][...] and B[...][i], and of the result
// column i, rows 8 (r / 4) + 4 h + r % 4 in register r.  A kernel's own rows are columns of its results: sums along the other side (softmax) stay in a lane
// and its partner 32 lanes away, and a result's registers are, as they are, the right operand of the next product, whose sum runs over its rows:
// registers 8 s ... 8 s + 7 (bf16; floats: 4 s ... 4 s + 3) of half h are rows {16 s + 4 h + j, 16 s + 8 + 4 h + j} (8 s + 4 h + j), j < 4, and the left
// operand is read in that order.
#pragma once
#include "pg_rows.h"

namespace pg {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Rows of a tile in LDS: one block of a product.  64 need more registers than two wavefronts a SIMD have, and those two count for more (forward, 2 x 4096 x 8192, 16 heads of
// 128, bf16: tiles of 64 661 us, of 32 561 us; with one wavefront a SIMD 772 and more).
constexpr int KT = 32;
constexpr uint32_t kAllRows = ~0u;

// Floats are multiplied as three bf16 pieces that add up to them, six products: 8/3 times the rate of the float
// instructions, which heads wider than 128 take, whose pieces do not fit LDS and registers.  Pieces are cut, not rounded, so that none overflows; second and third ones are up to 2^-7 and
// 2^-15 of the float, so each of the two larger products left out is up to 2^-22 of the whole (mantissas near 1; 2^-24 as a rule) and of its sign.  Results are off by 3e-7 to 6e-7 in norm where
// float products leave 1.6e-7 to 5.7e-7.  Floats below 2^-110 lose what lies below 2^-133, where bf16 ends.  Infinities and NaN are
// first pieces with nothing behind them: a product of tiles that hold one (`ODD`) leaves them out where they would meet the other's lower pieces, 0 or of any sign.
constexpr int kPieces = 2;
template <> struct Elem<kPieces> {
    static constexpr int bytes = 4;
};

// bf16 whose weights and their gradients keep 16 bits instead of 8 on the way into their products: a part that is cut off and what it leaves, two products for one.  Calls of
// few weights take it.  Rounded weights put results 1.4 times as far off as their own rounding does where many average out (forward 1.35), but up to 1.7 times where a few large
// ones decide (16 rows of 200 states); with two parts 1.0 to 1.1.  The price is one product in four to one in two: for many weights, which average, half a forward pass; below 2^17 of them a
// call is launch and latency (gradients of 16 rows of 43 states, heads of 192: 22.5 us with rounded weights, 23.5 with two parts).
constexpr int kFine = 3;
template <> struct Elem<kFine> {
    static constexpr int bytes = 2;
};
inline bool few_weights(const AttentionArgs &a, int type) { return type == kBf16 && (double)a.n * a.sequences * a.heads * a.rows * a.memory <= 1 << 17; }
constexpr int stored_as(int et) { return et == kPieces ? kF32 : (et == kFine ? kBf16 : et); }  // in memory

template <int ET> struct FragOf {
    typedef bf16x8 type;
};
template <> struct FragOf<kF32> {
    typedef f32x4 type;
};
struct Pieces {
    bf16x8 p[3];
};
template <> struct FragOf<kPieces> {
    typedef Pieces type;
};
template <int ET> using Frag = typename FragOf<ET>::type;
// Registers of a result as a right operand.
struct TwoParts {
    bf16x8 high, low;
};
template <int ET> struct RightOf {
    typedef Frag<ET> type;
};
template <> struct RightOf<kFine> {
    typedef TwoParts type;
};
template <int ET> using Right = typename RightOf<ET>::type;

__device__ __forceinline__ uint32_t high_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float first_piece(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
// of a float that is not below 0; 0 stays 0
__device__ __forceinline__ float next_smaller(float v) { return __uint_as_float(__builtin_elementwise_sub_sat(__float_as_uint(v), 1u)); }
// Eight floats in three pieces, word by word; `odd` becomes other than 0 where one is not finite.
struct Split {
    u32x4 w[3];
};
__device__ __forceinline__ Split split8(const float (&v)[8], float &odd) {
    Split s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = v[2 * j], b = v[2 * j + 1], ra = a - first_piece(a), rb = b - first_piece(b);
        s.w[0][j] = high_halves(a, b);
        s.w[1][j] = high_halves(ra, rb);
        s.w[2][j] = high_halves(ra - first_piece(ra), rb - first_piece(rb));
        odd += a * 0.f + b * 0.f;
    }
    return s;
}
// ... where some are not
__device__ __forceinline__ void mend_odd(const float (&v)[8], Split &s) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (__builtin_fabsf(v[j]) < __builtin_inff()) continue;
        const uint32_t keep = j % 2 ? 0x0000ffffu : 0xffff0000u, top = (__float_as_uint(v[j]) >> 16 | (v[j] != v[j] ? 0x40u : 0u)) << (j % 2 * 16);
        s.w[0][j / 2] = (s.w[0][j / 2] & keep) | top;
        s.w[1][j / 2] &= keep;
        s.w[2][j / 2] &= keep;
    }
}
// first pieces, those that are not finite as 0
__device__ __forceinline__ bf16x8 finite(const bf16x8 &v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if ((w[j] & 0x7f80u) == 0x7f80u) w[j] &= 0xffff0000u;
        if ((w[j] & 0x7f800000u) == 0x7f800000u) w[j] &= 0x0000ffffu;
    }
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ f32x16 mul_bf16(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

template <int ET, bool ODD = false> __device__ __forceinline__ f32x16 mul(const Frag<ET> &a, const Frag<ET> &b, f32x16 c) {
    if constexpr (ET == kBf16 || ET == kFine) {
        return mul_bf16(a, b, c);
    } else if constexpr (ET == kPieces) {
        const bf16x8 a0 = ODD ? finite(a.p[0]) : a.p[0], b0 = ODD ? finite(b.p[0]) : b.p[0];
        c = mul_bf16(a.p[2], b0, c);
        c = mul_bf16(a0, b.p[2], c);
        c = mul_bf16(a.p[1], b.p[1], c);
        c = mul_bf16(a.p[1], b0, c);
        c = mul_bf16(a0, b.p[1], c);
        return mul_bf16(a.p[0], b.p[0], c);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}
template <int ET, bool ODD = false> __device__ __forceinline__ f32x16 mul_right(const Frag<ET> &a, const Right<ET> &b, f32x16 c) {
    if constexpr (ET == kFine) return mul_bf16(a, b.high, mul_bf16(a, b.low, c));
    else return mul<ET, ODD>(a, b, c);
}
__device__ __forceinline__ f32x16 zero16() { return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// Rows of DP elements (the head's width, filled up with zeros) in LDS, and how a lane reads them.
//
// The 16-byte units of a row lie in another order in every row: unit u of row r is at u ^ swap(r).  LDS serves 16 lanes of a reading along rows at a time, one unit
// of 16 rows, and 32 lanes of a transposing one, four units of 4 rows: both lie on all 64 banks then.  (Counted, forward, width 128: rows padded by 16 bytes spent half of
// LDS's cycles on conflicts, this order none.)
template <int ET, int DP> struct Tile {
    static constexpr int EB = Elem<ET>::bytes;                                       // bytes of an element in memory
    static constexpr int LB = ET == kF32 ? 4 : 2, PLANES = ET == kPieces ? 3 : 1;    // in LDS: its bytes, and the tiles of pieces, one behind the other
    static constexpr int NK = DP * LB / 32, NB = DP / 32;                            // fragments along a row, blocks of 32 columns
    static constexpr int STEP = LB == 2 ? 16 : 8, STEPS = 32 / STEP;                 // rows that a fragment of a result spans
    static constexpr int PITCH = DP * LB, PLANE = KT * PITCH, SIZE = PLANES * PLANE;
    static constexpr int PER = 16 / LB, CHUNKS = DP / PER;                           // elements of a unit, units of a row
    static constexpr int APART = CHUNKS % 16 == 0 ? 1 : (CHUNKS % 8 == 0 ? 2 : 4);   // rows until one starts on the first's bank again
    static __device__ __forceinline__ constexpr int swap(int row) {
        const int j = row / APART;
        return APART == 1 ? j % 4 * 4 + j / 4 % 4 : (APART == 2 ? j % 2 * 4 + j / 2 % 4 : j % 4);
    }
    // unit `unit` of row `row`
    static __device__ __forceinline__ int at(int row, int unit) { return row * PITCH + (unit ^ swap(row)) * 16; }

    // Places of this lane's fragments in a tile: units keep their place among GROUP others, so few registers and constants give all of them.
    static constexpr int GROUP = 16 / APART, ROWS = NK < GROUP / 2 ? NK : GROUP / 2, COLUMNS = LB == 4 ? 4 : (NB < GROUP / 4 ? NB : GROUP / 4);
    int rows[ROWS], columns[COLUMNS];
    __device__ __forceinline__ explicit Tile(int lane) {
        const int i = lane % 32, h = lane / 32;
#pragma unroll
        for (int kk = 0; kk < ROWS; ++kk) rows[kk] = at(i, 2 * kk + h);
#pragma unroll
        for (int c = 0; c < COLUMNS; ++c) {
            // bf16, a transposing read: of 16 lanes, four to a row of 16 columns, lane i receives column i of the four rows
            if (LB == 2) columns[c] = at(4 * h + lane % 16 / 4, c * 4 + i / 16 * 2 + lane % 4 / 2) + lane % 2 * 8;
            // floats, column i of row 4 h: swap(8 step + 4 h + j) = 4 j + 2 (step % 2) + h, of which 4 (j % 2) + 2 (step % 2) is left to c
            else columns[c] = 4 * h * PITCH + (i / 4 ^ h ^ 2 * c) * 16;
        }
    }
    __device__ __forceinline__ int row_place(int kk) const { return rows[kk % ROWS] + kk / ROWS * ROWS * 32; }
    // fragment kk of row lane % 32
    __device__ __forceinline__ Frag<ET> along(const char *tile, int kk) const {
        const char *const from = tile + row_place(kk);
        if constexpr (ET == kPieces) return Pieces{{*(const bf16x8 *)from, *(const bf16x8 *)(from + PLANE), *(const bf16x8 *)(from + 2 * PLANE)}};
        else return *(const Frag<ET> *)from;
    }
    __device__ __forceinline__ void put_along(char *tile, int kk, const Frag<ET> &f) const {
        char *const to = tile + row_place(kk);
        if constexpr (ET == kPieces) {
#pragma unroll
            for (int k = 0; k < 3; ++k) *(bf16x8 *)(to + k * PLANE) = f.p[k];
        } else {
            *(Frag<ET> *)to = f;
        }
    }
    __device__ __forceinline__ bf16x8 turned(const char *from, int nb) const {
        typedef __attribute__((address_space(3))) s16x4 *lds4;
        // eight rows on, units lie two further apart: swap(row + 8) = swap(row) ^ 2
        const int place = columns[nb % COLUMNS], behind = nb / COLUMNS * COLUMNS * 64;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(from + place + behind)),
                    b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(from + (place ^ 32) + behind + 8 * PITCH));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // column block nb of rows STEP * step ... + STEP - 1, transposed: this lane's column in the order of a result's registers
    __device__ __forceinline__ Frag<ET> across(const char *tile, int step, int nb, int lane) const {
        const char *const from = tile + step * STEP * PITCH;
        if constexpr (ET == kBf16 || ET == kFine) {
            return turned(from, nb);
        } else if constexpr (ET == kPieces) {
            return Pieces{{turned(from, nb), turned(from + PLANE, nb), turned(from + 2 * PLANE, nb)}};
        } else {
            static_assert(APART == 1, "rows swap units among 16");
            f32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const float *)(from + columns[2 * (j % 2) + step % 2] + j * PITCH + (nb * 8 ^ j / 2 * 8) * 16 + lane % 4 * 4);
            return v;
        }
    }
    // step s of a result as a right operand.  bf16: rounded to nearest, off by 2^-9 of itself on average; the sums they enter hold floats.
    // WEIGHTS: no value is below 0.  The first of two parts is then that of the next smaller float, which leaves something to the second one of every weight: an infinity times
    // a weight stays one (times a second part of 0 it is NaN, as times weights below 2^-110, whose second part may be less than any bf16).
    template <bool ODD = false, bool WEIGHTS = false> static __device__ __forceinline__ Right<ET> of(const f32x16 &c, int s) {
        if constexpr (ET == kBf16) {
            const u32x4 w = {bf16_pack(c[8 * s], c[8 * s + 1]), bf16_pack(c[8 * s + 2], c[8 * s + 3]), bf16_pack(c[8 * s + 4], c[8 * s + 5]),
                             bf16_pack(c[8 * s + 6], c[8 * s + 7])};
            return __builtin_bit_cast(bf16x8, w);
        } else if constexpr (ET == kFine) {
            u32x4 high, low;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = c[8 * s + 2 * j], b = c[8 * s + 2 * j + 1];
                if constexpr (WEIGHTS) {
                    const float below_a = next_smaller(a), below_b = next_smaller(b);
                    high[j] = high_halves(below_a, below_b);
                    low[j] = bf16_pack(a - first_piece(below_a), b - first_piece(below_b));
                } else {
                    high[j] = high_halves(a, b);
                    low[j] = bf16_pack(__builtin_fabsf(a) == __builtin_inff() ? 0.f : a - first_piece(a), __builtin_fabsf(b) == __builtin_inff() ? 0.f : b - first_piece(b));
                }
            }
            return TwoParts{__builtin_bit_cast(bf16x8, high), __builtin_bit_cast(bf16x8, low)};
        } else if constexpr (ET == kPieces) {
            const float v[8] = {c[8 * s], c[8 * s + 1], c[8 * s + 2], c[8 * s + 3], c[8 * s + 4], c[8 * s + 5], c[8 * s + 6], c[8 * s + 7]};
            float odd = 0.f;
            Split w = split8(v, odd);
            if (ODD && odd != 0.f) mend_odd(v, w);
            return Pieces{{__builtin_bit_cast(bf16x8, w.w[0]), __builtin_bit_cast(bf16x8, w.w[1]), __builtin_bit_cast(bf16x8, w.w[2])}};
        } else {
            return f32x4{c[4 * s], c[4 * s + 1], c[4 * s + 2], c[4 * s + 3]};
        }
    }
};

// A unit's elements as they are in memory, at any address of their own; `have` of them exist, the rest is zero.
template <int ET> struct Unit {
    static constexpr int EB = Elem<ET>::bytes, WORDS = ET == kPieces ? 2 : 1, PER = 16 * WORDS / EB;
    u32x4 w[WORDS];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (auto &v : w) v = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void load(gin p) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = at_global<u32x4_any>(p + 16 * j);
    }
    __device__ __forceinline__ void load(gin p, int have) {
        if (have >= PER) return load(p);
        zero();
#pragma unroll
        for (int i = 0; i < PER - 1; ++i) {
            if (i >= have) continue;
            if constexpr (EB == 4) w[i / 4][i % 4] = at_global<uint32_t>(p + 4 * i);
            else w[0][i / 2] |= (uint32_t)at_global<uint16_t>(p + 2 * i) << (i % 2 * 16);
        }
    }
    // pieces; `odd` as for split8
    __device__ __forceinline__ Split split(bool &odd) const {
        const float v[8] = {__uint_as_float(w[0][0]), __uint_as_float(w[0][1]), __uint_as_float(w[0][2]), __uint_as_float(w[0][3]),
                            __uint_as_float(w[WORDS - 1][0]), __uint_as_float(w[WORDS - 1][1]), __uint_as_float(w[WORDS - 1][2]), __uint_as_float(w[WORDS - 1][3])};
        float some = 0.f;
        Split s = split8(v, some);
        if (some != 0.f) {  // NaN
            mend_odd(v, s);
            odd = true;
        }
        return s;
    }
    __device__ __forceinline__ Frag<ET> frag(bool &odd) const {
        if constexpr (ET == kPieces) {
            const Split s = split(odd);
            return Pieces{{__builtin_bit_cast(bf16x8, s.w[0]), __builtin_bit_cast(bf16x8, s.w[1]), __builtin_bit_cast(bf16x8, s.w[2])}};
        } else {
            return __builtin_bit_cast(Frag<ET>, w[0]);
        }
    }
};

// A tile's rows on their way from memory to LDS: thread `id` of THREADS holds its share.  WHOLE: the width is a multiple of 16 bytes, so that every load is one
// instruction behind no branch: what does not exist is read from where something does (the tile's last row, the row's first unit).  Units that no row has are zero in
// LDS from the start (clear()) and stay so.
template <int ET, int DP, int THREADS, bool WHOLE> struct Staged {
    typedef Tile<ET, DP> T;
    static constexpr int COUNT = (KT * T::CHUNKS + THREADS - 1) / THREADS;
    static constexpr bool EVEN = KT * T::CHUNKS % THREADS == 0;
    Unit<ET> w[COUNT];
    // row and unit of share j; no thread reads behind the tile
    static __device__ __forceinline__ int share(int id, int j) {
        constexpr int last = KT * T::CHUNKS - 1;
        return EVEN || id + j * THREADS < last ? id + j * THREADS : last;
    }
    static __device__ __forceinline__ int row_of(int id, int j) { return share(id, j) / T::CHUNKS; }
    static __device__ __forceinline__ int unit_of(int id, int j) { return share(id, j) % T::CHUNKS; }
    static __device__ __forceinline__ bool has(int id, int j, int width) { return (EVEN || id + j * THREADS < KT * T::CHUNKS) && unit_of(id, j) * T::PER < width; }

    // Of a tile that exists as a whole: bytes from its start, once, if its rows lie at(row) in every tile; the rest is one load each.
    struct Places {
        uint32_t from[COUNT];
    };
    template <typename At> static __device__ __forceinline__ Places places(int id, int width, At at) {
        Places p;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) p.from[j] = at(row_of(id, j)) + (unit_of(id, j) * T::PER < width ? unit_of(id, j) : 0) * (T::PER * T::EB);
        return p;
    }
    __device__ __forceinline__ void load_whole(gin from, const Places &p) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) w[j].load(from + p.from[j]);
    }
    __device__ __forceinline__ void put(char *tile, int id, int j, bool keep, bool &odd) const {
        char *const to = tile + T::at(row_of(id, j), unit_of(id, j));
        if constexpr (ET == kPieces) {
            const Split s = w[j].split(odd);
#pragma unroll
            for (int k = 0; k < 3; ++k) *(u32x4 *)(to + k * T::PLANE) = keep ? s.w[k] : u32x4{0u, 0u, 0u, 0u};
        } else {
            *(u32x4 *)to = keep ? w[j].w[0] : u32x4{0u, 0u, 0u, 0u};
        }
    }
    // Both return whether something was not finite, where a product has to know.
    __device__ __forceinline__ bool store_whole(char *tile, int id, int width) const {
        bool odd = false;
        if (EVEN && width == DP) {  // one branch for all of them
#pragma unroll
            for (int j = 0; j < COUNT; ++j) put(tile, id, j, true, odd);
            return odd;
        }
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (has(id, j, width)) put(tile, id, j, true, odd);
        return odd;
    }
    // Of any tile, of which `have` > 0 rows exist (others are not read); at(row): bytes from `from`.
    template <typename At> __device__ __forceinline__ void load(gin from, int id, int have, int width, At at) {
#pragma unroll
        for (int j = 0; j < COUNT; ++j) {
            const int row = row_of(id, j), col = unit_of(id, j) * T::PER;
            if constexpr (WHOLE) {
                w[j].load(from + at(row < have ? row : have - 1) + (col < width ? col : 0) * T::EB);
            } else {
                w[j].zero();
                if (row < have && col < width) w[j].load(from + at(row) + col * T::EB, width - col);
            }
        }
    }
    // rows whose bit is clear become zero
    __device__ __forceinline__ bool store(char *tile, int id, int width, uint32_t keep) const {
        if (keep == kAllRows) return store_whole(tile, id, width);
        bool odd = false;
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
            if (has(id, j, width)) put(tile, id, j, keep >> row_of(id, j) & 1, odd);
        return odd;
    }
    // the units that no row has
    static __device__ __forceinline__ void clear(char *tile, int id, int width) {
        if (width == DP) return;
#pragma unroll
        for (int j = 0; j < COUNT; ++j)
#pragma unroll
            for (int k = 0; k < T::PLANES; ++k)
                if (!has(id, j, width)) *(u32x4 *)(tile + k * T::PLANE + T::at(row_of(id, j), unit_of(id, j))) = u32x4{0u, 0u, 0u, 0u};
    }
};

// with the lane 32 away
__device__ __forceinline__ float across_halves_max(float v) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ __forceinline__ float across_halves_sum(float v) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}

// Whether sequences and key heads are dealt out to the dies one by one: no die stands idle for more than an eighth of the time.
__host__ __device__ constexpr bool dealt_out(uint32_t problems) { return problems % 8 == 0 || problems >= 64; }

// Work-groups of a sequence and key head, and the parts that their steps along the other side are split into.
struct Cut {
    int tiles, splits;
};
constexpr int kMostParts = 64;
// By the least estimated time: rounds of work-groups, `per_cu` of them on each of 256 compute units, of so many steps of `us` and as much as three for their start and
// end; parts are joined by a launch that reads `part_bytes` each, at 4 TB/s written and read.
inline Cut cut_of(int64_t problems, int64_t tiles, int64_t steps, int per_cu, double us, double part_bytes, int forced) {
    const int64_t least_steps = us >= 4.0 ? 1 : (us >= 2.0 ? 2 : 4), parts = steps / least_steps;  // a part takes 4 us and more
    const int most = (int)(parts < 1 ? 1 : (parts > kMostParts ? kMostParts : parts));
    Cut best = {(int)tiles, 1};
    if (forced > 0) {   // no more work-groups than a launch takes, which the estimate stays far below: it splits what is at most 8 rounds
        const int64_t room = (kMostAttentionGroups - 1) / (problems * tiles > 0 ? problems * tiles : 1);
        best.splits = forced < most ? forced : most;
        if (best.splits > room) best.splits = room > 0 ? (int)room : 1;
        return best;
    }
    double least = 1e30;
    for (int s = 1; s <= most; ++s) {
        const int64_t groups = problems * tiles * s, room = 256 * per_cu, rounds = (groups + room - 1) / room;
        const double time = (double)rounds * (double)((steps + s - 1) / s + 3) * us + (s > 1 ? 6.0 + 2.0 * s * part_bytes / 4e6 : 0.0);
        if (time < least) {
            least = time;
            best.splits = s;
        }
        if (rounds > 8) break;
    }
    return best;
}

// Which of a ring's tiles hold something that is not finite: a tag for each place, the number of its tile and 1 where it does.
template <int ET> struct Odd {
    int *tags;
    __device__ __forceinline__ void clear(int places) const {
        if constexpr (ET == kPieces) {
            if ((int)threadIdx.x < places) tags[threadIdx.x] = 0;
            __syncthreads();
        }
    }
    __device__ __forceinline__ void note(int place, int tile, bool odd) const {
        if constexpr (ET == kPieces)
            if (odd) tags[place] = tile + 1;
    }
    __device__ __forceinline__ bool at(int place, int tile) const {
        if constexpr (ET == kPieces) return __builtin_amdgcn_readfirstlane(tags[place]) == tile + 1;
        return false;
    }
};

// Which part of the work a work-group does.  Consecutive work-groups go to the eight dies in turn: all work-groups of a sequence and key head, which read the same rows,
// are on one die, whose L2 serves them.  Where there are many, each die takes every eighth, so that long and short sequences spread; else a contiguous eighth of all
// work-groups.  (32 sequences of up to 512 x 1024, 16 heads of 64, dk and dv: 164 us; with contiguous eighths, which hold
// whole sequences, 188.)
struct Work {
    int worker, sequence, head, tile, split;   // head: of the keys
    int64_t where;                             // worker * sequences + sequence
    bool any;
};
__device__ __forceinline__ Work work_of(const AttentionArgs &a) {
    const uint32_t problems = (uint32_t)a.n * a.sequences * a.kv_heads, each = (uint32_t)a.tiles * a.splits;  // fewer than kMostAttentionGroups in all
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, die = id % 8, turn = id / 8;
    const uint32_t in_order = die * (gridDim.x * gridDim.y / 8) + turn;
    const bool dealt = dealt_out(problems);
    uint32_t problem = dealt ? turn / each * 8 + die : in_order / each;
    const uint32_t inside = dealt ? turn % each : in_order % each;
    Work k;
    k.any = problem < problems;
    if (!k.any) problem = 0;
    k.split = inside % (uint32_t)a.splits;
    k.tile = inside / (uint32_t)a.splits;
    k.head = problem % (uint32_t)a.kv_heads, problem /= (uint32_t)a.kv_heads;
    k.where = problem;
    k.sequence = problem % (uint32_t)a.sequences;
    k.worker = problem / (uint32_t)a.sequences;
    return k;
}
__device__ __forceinline__ int length_of(const int32_t *counts, int64_t where, int most) {
    if (!counts) return most;
    const int c = counts[where];
    return c < 0 ? 0 : (c > most ? most : c);
}
// row 0 of a sequence
__device__ __forceinline__ gin sequence_of(const RowsArg &r, const Work &k, int rows, int eb) {
    return (gin)r.data + (k.worker * r.worker + (int64_t)k.sequence * rows * r.row) * eb;
}
// Tiles of `size` rows of `length`, the split's share: [first, last)
__device__ __forceinline__ void share_of(int length, int size, int split, int splits, int &first, int &last) {
    const int tiles = (length + size - 1) / size, per = (tiles + splits - 1) / splits;
    first = split * per;
    last = first + per < tiles ? first + per : tiles;
}
// Bits of the states of a tile that are seen.  The mask's bytes are fetched with a tile's rows and taken when these go into LDS.
struct Seen {
    const uint8_t *mask;  // of the sequence; null: none
    int count;
    int next;
    __device__ __forceinline__ uint32_t there(int tile) const {
        const int left = count - tile * KT;
        return left >= KT ? kAllRows : (1u << left) - 1;
    }
    __device__ __forceinline__ void fetch(int tile) {
        if (!mask) return;
        const int lane = threadIdx.x % 64, at = tile * KT + lane;
        next = lane < KT && at < count ? mask[at] : 0;
    }
    __device__ __forceinline__ uint32_t take(int tile) const { return mask ? there(tile) & (uint32_t)__ballot(next != 0) : there(tile); }
};
// Scores of rows that are not become -inf.
__device__ __forceinline__ void hide(f32x16 &s, uint32_t seen, int h) {
    if (seen == kAllRows) return;
    const uint32_t bits = seen >> (4 * h);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = bits >> (8 * (r / 4) + r % 4) & 1 ? s[r] : -__builtin_inff();
}

// A wavefront's own 32 rows as right operands: row i in lanes i and i + 32.  WHOLE: `row` is one that exists also where the lane's own does not, and every load is behind
// no branch, so that all of them are on their way together (behind branches they came one after the other: 12 us at the head of a work-group).  What does not exist is zero.
// Returns whether something of the wavefront's rows was not finite, where a product has to know.
template <int ET, int DP, bool WHOLE> __device__ __forceinline__ bool own_rows(Frag<ET> *f, gin row, bool there, int width, int h) {
    typedef Tile<ET, DP> T;
    Unit<ET> w[T::NK];
#pragma unroll
    for (int kk = 0; kk < T::NK; ++kk) {
        const int col = (2 * kk + h) * T::PER;
        w[kk].zero();
        if constexpr (WHOLE) w[kk].load(row + (col < width ? col : 0) * T::EB);
        else if (there && col < width) w[kk].load(row + col * T::EB, width - col);
    }
    bool odd = false;
#pragma unroll
    for (int kk = 0; kk < T::NK; ++kk) {
        if (WHOLE && (!there || (2 * kk + h) * T::PER >= width)) w[kk].zero();
        f[kk] = w[kk].frag(odd);
    }
    return ET == kPieces && __any(odd);
}
// A result, transposed: register r of block nb is column 32 nb + 8 (r / 4) + 4 h + r % 4 of the lane's own row.
template <int ET, int NB> __device__ __forceinline__ void put_rows(gout row, const f32x16 (&c)[NB], float times, int width, int h) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int col = nb * 32 + 8 * b + 4 * h;
            if (col >= width) continue;
            store4<stored_as(ET)>(row + col * Elem<ET>::bytes, f32x4{c[nb][4 * b] * times, c[nb][4 * b + 1] * times, c[nb][4 * b + 2] * times, c[nb][4 * b + 3] * times}, width - col);
        }
}

}  // namespace pg
