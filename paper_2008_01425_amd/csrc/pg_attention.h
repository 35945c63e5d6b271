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

// Widest head, and the work-groups of a launch.
constexpr int kMostWidth = 256;
constexpr int64_t kMostAttentionGroups = 1 << 30;

struct AttentionArgs {
    int n, sequences, rows, memory, heads, kv_heads, group, width;
    float scale;
    const int32_t *counts, *memory_counts;  // per sequence (null: all)
    const uint8_t *mask;                    // per sequence and state, 0: hidden (null: none)
    RowsArg q, k, v, y, dy, dq, dk, dv;
    float *lse;                             // per position and head
    float *delta;                           // backward: the same of dy . y
    int tiles, splits;                      // of a sequence and key head: tiles of its own rows, parts of the other side
    float *part, *part_stats;               // partial results [split][row][head][width], and [split][row][head] largest score and sum
};

#ifdef __HIP__
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

template <int ET> struct FragOf {
    typedef bf16x8 type;
};
template <> struct FragOf<kF32> {
    typedef f32x4 type;
};
template <int ET> using Frag = typename FragOf<ET>::type;

template <int ET> __device__ __forceinline__ f32x16 mul(const Frag<ET> &a, const Frag<ET> &b, f32x16 c) {
    if constexpr (ET == kBf16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
}
__device__ __forceinline__ f32x16 zero16() { return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// Rows of DP elements (the head's width, filled up with zeros) in LDS.
template <int ET, int DP> struct Tile {
    static constexpr int EB = Elem<ET>::bytes, NK = DP * EB / 32, NB = DP / 32;   // fragments along a row, blocks of 32 columns
    static constexpr int STEP = ET == kBf16 ? 16 : 8, STEPS = 32 / STEP;          // rows that a fragment of a result spans
    static constexpr int PITCH = DP * EB + (ET == kBf16 ? 16 : 32);
    static constexpr int PER = 16 / EB, CHUNKS = DP / PER;                        // elements of 16 bytes, those of a row

    // fragment kk of row `row`
    static __device__ __forceinline__ Frag<ET> along(const char *tile, int row, int kk, int h) { return *(const Frag<ET> *)(tile + row * PITCH + kk * 32 + h * 16); }
    // column block nb of rows first ... first + STEP - 1, transposed: this lane's column in the order of a result's registers
    static __device__ __forceinline__ Frag<ET> across(const char *tile, int first, int nb, int lane) {
        if constexpr (ET == kBf16) {
            // a transposing read: of 16 lanes, four to a row of 16 columns, lane i receives column i of the four rows
            const int at = (first + 4 * (lane / 32) + (lane % 16) / 4) * PITCH + (nb * 32 + (lane % 32) / 16 * 16 + lane % 4 * 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 *lds4;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tile + at)), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(tile + at + 8 * PITCH));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const char *const at = tile + (first + 4 * (lane / 32)) * PITCH + (nb * 32 + lane % 32) * 4;
            return f32x4{*(const float *)at, *(const float *)(at + PITCH), *(const float *)(at + 2 * PITCH), *(const float *)(at + 3 * PITCH)};
        }
    }
    // step s of a result as a right operand.  bf16: rounded to nearest, off by 2^-9 of itself on average; the sums they enter hold floats.
    static __device__ __forceinline__ Frag<ET> of(const f32x16 &c, int s) {
        if constexpr (ET == kBf16) {
            const u32x4 w = {bf16_pack(c[8 * s], c[8 * s + 1]), bf16_pack(c[8 * s + 2], c[8 * s + 3]), bf16_pack(c[8 * s + 4], c[8 * s + 5]),
                             bf16_pack(c[8 * s + 6], c[8 * s + 7])};
            return __builtin_bit_cast(bf16x8, w);
        } else {
            return f32x4{c[4 * s], c[4 * s + 1], c[4 * s + 2], c[4 * s + 3]};
        }
    }
};

// 16 bytes at any address of their elements, of which `have` elements exist; the rest zero.
template <int ET> __device__ __forceinline__ u32x4 load16(gin p, int have) {
    constexpr int EB = Elem<ET>::bytes, PER = 16 / EB;
    if (have >= PER) return at_global<u32x4_any>(p);
    u32x4 w = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < PER - 1; ++i) {
        if (i >= have) continue;
        if constexpr (ET == kF32) w[i] = at_global<uint32_t>(p + 4 * i);
        else w[i / 2] |= (uint32_t)at_global<uint16_t>(p + 2 * i) << (i % 2 * 16);
    }
    return w;
}

// A tile's rows on their way from memory to LDS: thread `id` of THREADS holds its share.
template <int ET, int DP, int ROWS, int THREADS> struct Staged {
    typedef Tile<ET, DP> T;
    static constexpr int COUNT = (ROWS * T::CHUNKS + THREADS - 1) / THREADS;
    static constexpr bool EVEN = ROWS * T::CHUNKS % THREADS == 0;
    u32x4 w[COUNT];
    // at(row) is the address of row `row` of the tile, for rows below `have` only; the others become zero
    template <typename At> __device__ __forceinline__ void load(int id, int have, int width, At at) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + i * THREADS, row = c / T::CHUNKS, col = c % T::CHUNKS * T::PER;
            w[i] = u32x4{0u, 0u, 0u, 0u};
            if (row < have && row < ROWS && col < width) w[i] = load16<ET>(at(row) + col * T::EB, width - col);
        }
    }
    // rows whose bit is clear become zero
    __device__ __forceinline__ void store(char *tile, int id, uint64_t keep) const {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int c = id + i * THREADS, row = c / T::CHUNKS;
            if (!EVEN && row >= ROWS) continue;
            *(u32x4 *)(tile + row * T::PITCH + c % T::CHUNKS * 16) = keep >> row & 1 ? w[i] : u32x4{0u, 0u, 0u, 0u};
        }
    }
};

__device__ __forceinline__ float across_halves_max(float v) { return __builtin_fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float across_halves_sum(float v) { return v + __shfl_xor(v, 32); }

// Which part of the work a work-group does.  Consecutive work-groups go to the eight dies in turn: each die takes a contiguous eighth of the list, so that the tiles
// of a sequence and key head, which read the same keys and values, meet in one L2.
struct Work {
    int worker, sequence, head, tile, split;   // head: of the keys
    int64_t where;                             // worker * sequences + sequence
    bool any;
};
__device__ __forceinline__ Work work_of(const AttentionArgs &a) {
    const uint32_t total = (uint32_t)a.n * a.sequences * a.kv_heads * a.tiles * a.splits;  // fewer than kMostAttentionGroups
    const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x;
    uint32_t at = id % 8 * (gridDim.x * gridDim.y / 8) + id / 8;
    Work k;
    k.any = at < total;
    if (!k.any) at = 0;
    k.split = at % (uint32_t)a.splits, at /= (uint32_t)a.splits;
    k.tile = at % (uint32_t)a.tiles, at /= (uint32_t)a.tiles;
    k.head = at % (uint32_t)a.kv_heads, at /= (uint32_t)a.kv_heads;
    k.where = at;
    k.sequence = at % (uint32_t)a.sequences;
    k.worker = at / (uint32_t)a.sequences;
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
// Bits of the rows of a tile that are seen.
template <int ROWS> __device__ __forceinline__ uint64_t seen_of(const AttentionArgs &a, int64_t where, int first, int count) {
    const int left = count - first;
    uint64_t seen = left >= 64 ? ~0ull : (1ull << left) - 1;
    if (ROWS < 64) seen &= (1ull << (ROWS % 64)) - 1;
    if (a.mask) {
        const int lane = threadIdx.x % 64;
        bool on = lane < ROWS && lane < left;
        if (on) on = a.mask[where * a.memory + first + lane] != 0;
        seen &= __ballot(on);
    }
    return seen;
}
template <int ROWS> __device__ __forceinline__ constexpr uint64_t all_rows() { return ROWS >= 64 ? ~0ull : (1ull << (ROWS % 64)) - 1; }

// A wavefront's own 32 rows as right operands: row i in lanes i and i + 32, zero where it does not exist.
template <int ET, int DP> __device__ __forceinline__ void own_rows(Frag<ET> *f, gin row, bool there, int width, int h) {
    typedef Tile<ET, DP> T;
#pragma unroll
    for (int kk = 0; kk < T::NK; ++kk) {
        const int col = (2 * kk + h) * T::PER;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (there && col < width) w = load16<ET>(row + col * T::EB, width - col);
        f[kk] = __builtin_bit_cast(Frag<ET>, w);
    }
}
// A result, transposed: register r of block nb is column 32 nb + 8 (r / 4) + 4 h + r % 4 of the lane's own row.
template <int ET, int NB> __device__ __forceinline__ void put_rows(gout row, const f32x16 (&c)[NB], float times, int width, int h) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int col = nb * 32 + 8 * b + 4 * h;
            if (col >= width) continue;
            store4<ET>(row + col * Elem<ET>::bytes, f32x4{c[nb][4 * b] * times, c[nb][4 * b + 1] * times, c[nb][4 * b + 2] * times, c[nb][4 * b + 3] * times}, width - col);
        }
}

// rows of a tile in LDS: 16 KB of them, 32 or 64
template <int ET, int DP> constexpr int tile_rows() { return DP * Elem<ET>::bytes * 64 <= 16384 ? 64 : 32; }
#endif

dim3 attention_grid(const AttentionArgs &a);
size_t attention_forward_workspace(const AttentionArgs &a, int type);
size_t attention_backward_workspace(const AttentionArgs &a, int type);  // delta, from a multiple of 256 bytes on the parts
void launch_attention(AttentionArgs a, int type, hipStream_t st);
void launch_attention_dq(AttentionArgs a, int type, hipStream_t st);
void launch_attention_delta(const AttentionArgs &a, int type, hipStream_t st);
void launch_attention_dkv(AttentionArgs a, int type, hipStream_t st);

}  // namespace pg
