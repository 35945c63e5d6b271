// The products of a linear layer, all workers in one launch, straight on their parameter and gradient buffers:
//
//   forward    Y[t][j]  = act(sum_c X[t][c] W[j][c] + b[j]) + R[t][j]            (kForward)
//   input      dX[t][c] = (sum_j dZ[t][j] W[j][c]) act'(z[t][c]) + R[t][c]       (kInput)
//   weights    dW[j][c] = sum_t dZ[t][j] X[t][c],  db[j] = sum_t dZ[t][j]        (kWeights)
//
// Each is out[m][n] = sum_k M[m][k] N[n][k]; the operands differ in whether k runs along their rows in memory
// (X, dZ and W of the forward product, dZ of the second one) or across them (W of the second, both of the third).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "pg_rows.h"

namespace pg {

constexpr int kForward = 0, kInput = 1, kWeights = 2;
constexpr int kComputeUnits = 256;
constexpr int kMostSplit = 1024;   // work-groups of a split product: 256 MB of partial sums at most
constexpr int64_t kMostTiles = 1 << 22;  // of a launch: its lanes are counted in 32 bits
constexpr int kSrcF32 = 0, kSrcBf16 = 1, kSrcKept = 2;

// Matrix instructions take bf16.  An activation type of bf16 enters as it is, a kept one exactly (e4m3 times a power of two), and float
// weights beside them are rounded to bf16, the precision of what they are multiplied with.  Where activations are float, every float operand enters as three
// bf16 pieces, x = x1 + x2 + x3 with x1 = bf16(x), x2 = bf16(x - x1), x3 = x - x1 - x2: 24 bits, the whole significand
// (of floats below 2^-110 the part above 2^-133, where bf16 ends; the matrix cores take its subnormal values as they are).  Of
// the nine products of pieces the three smallest (2^-26 of the product and less) are left out.  A product that is kept in 8 bits beside bf16
// takes the weights in two pieces, 16 bits: what rounded weights move a sum by, 2^-9 of it, sends one value in fifty to the next e4m3 one, a sixteenth away, and the
// kept values would be off by 1e-2 in norm that way (two pieces: 4e-4; 8 x 2048 x 8192 x 2048: 811 us with rounded weights, 1190 with two pieces, 1480
// with three, for 2e-4, where 8 bits themselves are 2.65e-2 off).
// Elsewhere the type alone decides, also where few rows leave the matrix cores time: the precision of a row's result does not depend on how many come with it, and a second piece is not free there
// either (16 x 10 x 33278 x 650: 266 -> 302 us).
template <int MODE, int ET, bool X8, bool KEEP, int BK> struct Product {
    static constexpr int whole = ET == kF32 ? 3 : 1;     // pieces of a float operand
    static constexpr int xsrc = X8 ? kSrcKept : (ET == kF32 ? kSrcF32 : kSrcBf16);
    static constexpr int dsrc = ET == kF32 ? kSrcF32 : kSrcBf16;
    static constexpr int msrc = MODE == kForward ? xsrc : dsrc;
    static constexpr int nsrc = MODE == kWeights ? xsrc : kSrcF32;
    static constexpr bool macross = MODE == kWeights;    // k runs across the rows of M
    static constexpr bool nacross = MODE != kForward;
    static constexpr int pm = msrc == kSrcF32 ? whole : 1, pn = nsrc == kSrcF32 ? (KEEP && ET == kBf16 ? 2 : whole) : 1;
    static constexpr bool split = pm * pn > 1;
    static constexpr int bk = BK;                        // k of a step
};

struct Source {
    gin data;                  // element (first row of the tile, k = 0) or (k = 0, first row of the tile)
    const PG_GLOBAL uint8_t *scales;  // kept: of the same element
    int ld, scale_ld;          // elements (kept: bytes) between rows in memory
    int limit;                 // rows of the operand from the tile's first one on
};

// LDS holds a tile as [piece][row][BK] bf16, rows of 16-byte chunks along k.  Chunks of a 128-byte line are permuted by a
// function of the line that is one to one on any eight lines in a row (the lanes that read a matrix operand) and on every fourth of
// 32 (the lanes that write a transposed tile), so both touch all banks.
template <int BK> __device__ __forceinline__ int chunk_at(int row, int chunk) {
    const int line = BK == 64 ? row : row >> 1;
    const int c = BK == 64 ? chunk : ((row & 1) * 4 + chunk);
    return line * 8 + (c ^ ((line ^ (line >> 3 & 3)) & 7));
}

// A float in bf16 pieces.  `odd`: not finite, or too large to be rounded to bf16 (then pieces are cut instead of rounded, so that no
// sum of them exceeds it).
__device__ __forceinline__ void pieces_of(float x, float p[3]) {
    p[0] = (float)(__bf16)x;
    const float r = x - p[0];
    p[1] = (float)(__bf16)r;
    p[2] = r - p[1];
}
__device__ __forceinline__ void odd_pieces_of(float x, float p[3]) {
    if (!(__builtin_fabsf(x) < __builtin_inff())) {
        p[0] = x;
        p[1] = p[2] = 0.f;
        return;
    }
    p[0] = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    const float r = x - p[0];
    p[1] = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    p[2] = r - p[1];
}
constexpr float kLargestRounded = 0x1.fep127f;  // at most this, a float rounds to a finite bf16

// One operand's way from memory through registers into LDS.  ROWS of the tile, BK of k; ACROSS as above.
// CHECK: bf16 that is multiplied with more than one piece is looked through for what is not finite, codes for the scale that alone can make them infinite (NaN
// needs no care: its sums are NaN whatever the other pieces add).
template <int SRC, bool ACROSS, int ROWS, int BK, int PIECES, int THREADS, bool CHECK> struct Stage {
    static constexpr int kPlane = ROWS * BK;   // bf16 of one piece
    // along: 16 bytes of a row, so that the lanes of an access read whole lines;  across: units of KU k x 4 rows
    static constexpr int kLen = SRC == kSrcF32 ? 4 : (SRC == kSrcBf16 ? 8 : 16);
    static constexpr int kAcross = BK / kLen;                   // lanes side by side on a row
    static constexpr int kChunks = ROWS * kAcross / THREADS > 0 ? ROWS * kAcross / THREADS : 1;
    static constexpr bool kSome = ROWS * kAcross < THREADS;     // not every thread has one
    // the permutation of LDS repeats after 32 lines: units this many apart differ by a constant
    static constexpr int kApart = THREADS / kAcross * BK / 64;  // lines from one unit to the next
    static constexpr int kPeriod = ACROSS || kApart >= 32 ? 1 : 32 / kApart;
    static constexpr int KU = ROWS * BK / 4 / THREADS >= 8 ? 8 : (ROWS * BK / 4 / THREADS >= 4 ? 4 : 2);
    static constexpr int kUnits = ACROSS ? ROWS * BK / (4 * KU) / THREADS : kChunks;
    static constexpr int kWords = SRC == kSrcKept ? (ACROSS ? KU : 4) : (ACROSS ? (SRC == kSrcF32 ? 4 * KU : 2 * KU) : 4);
    static constexpr int kScales = SRC == kSrcKept ? (ACROSS ? KU : 1) : 0;
    static constexpr int kBytes = SRC == kSrcF32 ? 4 : (SRC == kSrcBf16 ? 2 : 1);
    static_assert(ACROSS || 32 % kApart == 0 || kApart % 32 == 0, "units along k repeat the permutation");
    static_assert(!ACROSS || kUnits * THREADS * 4 * KU == ROWS * BK, "units cover the tile");

    uint32_t w[kUnits][kWords];
    uint8_t sc[kUnits][kScales > 0 ? kScales : 1];

    // Rows of the tile past the operand's last one are read as another of its rows or not written: their results are not stored.  What lies past the last k is zero.
    // Addresses are one base for the work-group and 32 bits a lane (strides are at most 2^21 elements).  The whole step, without a branch, is
    // one body and the ragged one another: the compiler waits for every load before a branch that another load depends on.
    __device__ __forceinline__ void load(const Source &s, int k0, int K, int tid) {
        if (k0 + BK <= K && plain(s)) load_whole(s, k0, tid);
        else load_ragged(s, k0, K, tid);
    }
    __device__ __forceinline__ static bool plain(const Source &s) { return !ACROSS || SRC == kSrcKept || s.limit >= 4; }
    // across: the first of a thread's four rows.  Threads past the operand's last row double its last four (codes: its last word, rows of codes are filled
    // up): they load and store the same as another thread, and no access is a partial one.
    __device__ __forceinline__ static int row_at(int id, int limit) {
        return min(id % (ROWS / 4) * 4, SRC == kSrcKept ? (limit - 1) / 4 * 4 : max(limit - 4, 0));
    }
    __device__ __forceinline__ void load_whole(const Source &s, int k0, int tid) {
        const gin base = s.data + (int64_t)k0 * (ACROSS ? s.ld : 1) * kBytes;
        const PG_GLOBAL uint8_t *const scale = s.scales + (ACROSS ? (int64_t)k0 * s.scale_ld : k0 / kScaled);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int id = u * THREADS + tid;
            if constexpr (!ACROSS) {
                if (kSome && id >= ROWS * kAcross) break;
                const int row = min(id / kAcross, s.limit - 1), k = id % kAcross * kLen;
                const gin at = base + ((uint32_t)(row * s.ld + k) * kBytes);
                if constexpr (SRC == kSrcF32) {
                    *(f32x4 *)&w[u][0] = at_global<f32x4_any>(at);
                } else if constexpr (SRC == kSrcBf16) {
                    *(u32x4 *)&w[u][0] = at_global<u32x4_any>(at);
                } else {
                    *(u32x4 *)&w[u][0] = at_global<u32x4>(at);
                    sc[u][0] = scale[(uint32_t)(row * s.scale_ld + k / kScaled)];
                }
            } else {
                const int row = row_at(id, s.limit), k = id / (ROWS / 4) * KU;
                const uint32_t at = (uint32_t)(k * s.ld + row) * kBytes, scale_at = (uint32_t)(k * s.scale_ld + row / kScaled);
                constexpr int W = kWords / KU;
#pragma unroll
                for (int i = 0; i < KU; ++i) {
                    const gin p = base + (int64_t)i * s.ld * kBytes + at;
                    if constexpr (SRC == kSrcKept) {
                        w[u][i] = at_global<uint32_t>(p);
                        sc[u][i] = (scale + (int64_t)i * s.scale_ld)[scale_at];
                    } else if constexpr (SRC == kSrcF32) {
                        *(f32x4 *)&w[u][i * W] = at_global<f32x4_any>(p);
                    } else {
                        *(u32x2 *)&w[u][i * W] = at_global<u32x2_any>(p);
                    }
                }
            }
        }
    }
    // A step that ends past the last k, or a tile of fewer than four rows across.  Where the operand is long enough the accesses are whole ones that
    // end with its last element, moved into place, and what lies behind is made zero: no branch here either.
    __device__ __forceinline__ void load_ragged(const Source &s, int k0, int K, int tid) {
        const gin base = s.data + (int64_t)k0 * (ACROSS ? s.ld : 1) * kBytes;
        const PG_GLOBAL uint8_t *const scale = s.scales + (ACROSS ? (int64_t)k0 * s.scale_ld : k0 / kScaled);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int id = u * THREADS + tid;
            if constexpr (!ACROSS) {
                if (kSome && id >= ROWS * kAcross) break;
                const int row = min(id / kAcross, s.limit - 1), k = id % kAcross * kLen, have = K - k0 - k;
                u32x4 v = {0u, 0u, 0u, 0u};
                if constexpr (SRC == kSrcKept) {  // rows of codes are filled up with zeros to whole blocks
                    const gin at = base + ((uint32_t)(row * s.ld + k));
                    if (have > 0) v = at_global<u32x4>(at);
                    sc[u][0] = have > 0 ? scale[(uint32_t)(row * s.scale_ld + k / kScaled)] : 127;
                } else if (K >= kLen) {
                    const int by = max(0, kLen - have);          // elements the access is moved back
                    const gin at = base + (int64_t)row * s.ld * kBytes + (k - by) * kBytes;
                    v = at_global<u32x4_any>(at);
                    if constexpr (SRC == kSrcF32) {
                        if (by & 1) v = u32x4{v[1], v[2], v[3], 0u};
                        if (by & 2) v = u32x4{v[2], v[3], 0u, 0u};
                    } else {
                        if (by & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
                        if (by & 2) v = u32x4{v[1], v[2], v[3], 0u};
                        if (by & 4) v = u32x4{v[2], v[3], 0u, 0u};
                    }
                    if (by >= kLen) v = u32x4{0u, 0u, 0u, 0u};
                } else {
                    const gin at = base + (int64_t)row * s.ld * kBytes + k * kBytes;
#pragma unroll
                    for (int i = 0; i < kLen - 1; ++i)
                        if (i < have) {
                            if constexpr (SRC == kSrcF32) v[i] = at_global<uint32_t>(at + 4 * i);
                            else v[i / 2] |= (uint32_t)at_global<uint16_t>(at + 2 * i) << (i % 2 * 16);
                        }
                }
                *(u32x4 *)&w[u][0] = v;
            } else {
                const int row = row_at(id, s.limit), k = id / (ROWS / 4) * KU, have = s.limit - row;
                constexpr int W = kWords / KU;
#pragma unroll
                for (int i = 0; i < KU; ++i) {
                    const bool in = k0 + k + i < K;
                    const int64_t at = in ? k + i : K - 1 - k0;
                    const gin p = base + (at * s.ld + row) * kBytes;
                    if constexpr (SRC == kSrcKept) {
                        const uint32_t v = at_global<uint32_t>(p);
                        w[u][i] = in ? v : 0u;
                        sc[u][i] = scale[at * s.scale_ld + row / kScaled];
                    } else if constexpr (SRC == kSrcF32) {
                        const f32x4 v = load4<kF32>(p, have);
                        *(f32x4 *)&w[u][i * W] = in ? v : f32x4{0.f, 0.f, 0.f, 0.f};
                    } else {
                        u32x2 v = {0u, 0u};
                        if (have >= 4) {
                            v = at_global<u32x2_any>(p);
                        } else {
#pragma unroll
                            for (int j = 0; j < 3; ++j)
                                if (j < have) v[j / 2] |= (uint32_t)at_global<uint16_t>(p + 2 * j) << (j % 2 * 16);
                        }
                        *(u32x2 *)&w[u][i * W] = in ? v : u32x2{0u, 0u};
                    }
                }
            }
        }
    }

    // Sums over k of the four rows a thread holds (across, floats or bf16).
    __device__ __forceinline__ void add_to(f32x4 &sum) const {
        static_assert(ACROSS && SRC != kSrcKept && kUnits == 1, "a unit of the tile per thread");
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            if constexpr (SRC == kSrcF32) sum += *(const f32x4 *)&w[0][i * 4];
            else sum += f32x4{bf16_low(w[0][2 * i]), bf16_high(w[0][2 * i]), bf16_low(w[0][2 * i + 1]), bf16_high(w[0][2 * i + 1])};
        }
    }

    // Returns whether a value was odd (see pieces_of).
    __device__ __forceinline__ bool store(uint16_t *lds, int limit, int tid) const {
        bool odd = false;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int id = u * THREADS + tid;
            if constexpr (!ACROSS) {
                if (kSome && id >= ROWS * kAcross) break;
                const int one = u % kPeriod * THREADS + tid, k = one % kAcross * kLen;
                uint16_t *const at = lds + chunk_at<BK>(one / kAcross, k / 8) * 8 + k % 8 + u / kPeriod * kPeriod * THREADS * kLen;
                if constexpr (SRC == kSrcBf16) {
                    *(u32x4 *)at = *(const u32x4 *)&w[u][0];
                    if constexpr (CHECK) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) odd |= (w[u][i] & 0x7fffu) >= 0x7f80u || (w[u][i] & 0x7fffffffu) >= 0x7f800000u;
                    }
                } else if constexpr (SRC == kSrcKept) {
                    if constexpr (CHECK) odd |= sc[u][0] >= kLargestScale;
                    const float f = scale_of(sc[u][0]);
                    uint16_t *const second = lds + chunk_at<BK>(one / kAcross, k / 8 + 1) * 8 + u / kPeriod * kPeriod * THREADS * kLen;
                    u32x4 out[2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        out[i / 2][i % 2 * 2] = decode_bf16<false>(w[u][i], f);
                        out[i / 2][i % 2 * 2 + 1] = decode_bf16<true>(w[u][i], f);
                    }
                    *(u32x4 *)at = out[0];
                    *(u32x4 *)second = out[1];
                } else {
                    uint32_t out[PIECES][2];
                    float x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[u][i]);
                    odd |= cut<4>(x, out);
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) *(u32x2 *)(at + p * kPlane) = u32x2{out[p][0], out[p][1]};
                }
            } else {
                const int row = row_at(id, limit), k = id / (ROWS / 4) * KU;
                constexpr int W = kWords / KU;
                if constexpr (SRC == kSrcKept && CHECK) {
#pragma unroll
                    for (int i = 0; i < KU; ++i) odd |= sc[u][i] >= kLargestScale;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t out[PIECES][KU / 2];
                    if constexpr (SRC == kSrcBf16) {
#pragma unroll
                        for (int i = 0; i < KU / 2; ++i)
                            out[0][i] = __builtin_amdgcn_perm(w[u][(2 * i + 1) * W + j / 2], w[u][2 * i * W + j / 2],
                                                              j & 1 ? 0x07060302u : 0x05040100u);
                    } else if constexpr (SRC == kSrcKept) {
#pragma unroll
                        for (int i = 0; i < KU / 2; ++i) {
                            const float f = scale_of(sc[u][2 * i]), g = scale_of(sc[u][2 * i + 1]);
                            const uint32_t a = j < 2 ? decode_bf16<false>(w[u][2 * i], f) : decode_bf16<true>(w[u][2 * i], f);
                            const uint32_t b = j < 2 ? decode_bf16<false>(w[u][2 * i + 1], g) : decode_bf16<true>(w[u][2 * i + 1], g);
                            out[0][i] = __builtin_amdgcn_perm(b, a, j & 1 ? 0x07060302u : 0x05040100u);
                        }
                    } else {
                        float x[KU];
#pragma unroll
                        for (int i = 0; i < KU; ++i) x[i] = __uint_as_float(w[u][i * W + j]);
                        odd |= cut<KU>(x, out);
                    }
                    uint16_t *at = lds + chunk_at<BK>(row + j, k / 8) * 8 + k % 8;
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) {
                        if constexpr (KU == 8) *(u32x4 *)(at + p * kPlane) = u32x4{out[p][0], out[p][1], out[p][2], out[p][3]};
                        else if constexpr (KU == 4) *(u32x2 *)(at + p * kPlane) = u32x2{out[p][0], out[p][1]};
                        else *(uint32_t *)(at + p * kPlane) = out[p][0];
                    }
                }
            }
        }
        return odd;
    }

    template <int E, int WORDS> __device__ __forceinline__ static bool cut(const float (&x)[E], uint32_t (*out)[WORDS]) {
        static_assert(WORDS * 2 == E, "two to a word");
        static_assert(PIECES <= 3, "three pieces are all of a float");
        if constexpr (PIECES == 1) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) out[0][i] = bf16_pack(x[2 * i], x[2 * i + 1]);
            return false;
        } else {
            bool odd = false;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float a[3], b[3];
                pieces_of(x[2 * i], a);
                pieces_of(x[2 * i + 1], b);
                odd |= !(__builtin_fabsf(x[2 * i]) <= kLargestRounded) || !(__builtin_fabsf(x[2 * i + 1]) <= kLargestRounded);
#pragma unroll
                for (int p = 0; p < PIECES; ++p) out[p][i] = bf16_pack(a[p], b[p]);
            }
            if (odd) {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    float a[3], b[3];
                    if (__builtin_fabsf(x[2 * i]) <= kLargestRounded) pieces_of(x[2 * i], a);
                    else odd_pieces_of(x[2 * i], a);
                    if (__builtin_fabsf(x[2 * i + 1]) <= kLargestRounded) pieces_of(x[2 * i + 1], b);
                    else odd_pieces_of(x[2 * i + 1], b);
#pragma unroll
                    for (int p = 0; p < PIECES; ++p) out[p][i] = bf16_pack(a[p], b[p]);
                }
            }
            return odd;
        }
    }
};

// bf16 pairs with what is not finite replaced by zero
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0x0000ffffu;
    }
    return v;
}

// Where a wavefront reads its operands of a tile: 16 rows at a time from row `first` on.  The permutation repeats after 32 lines, so
// a few addresses and constants do.
template <int BK> struct Reader {
    static constexpr int kPeriod = BK == 64 ? 2 : 4;
    int at[BK / 32][kPeriod];
    __device__ __forceinline__ Reader(int first, int lane) {
#pragma unroll
        for (int ks = 0; ks < BK / 32; ++ks)
#pragma unroll
            for (int i = 0; i < kPeriod; ++i) at[ks][i] = chunk_at<BK>(first + 16 * i + lane % 16, ks * 4 + lane / 16) * 8;
    }
    __device__ __forceinline__ u32x4 read(const uint16_t *plane, int ks, int i) const {
        return *(const u32x4 *)(plane + at[ks][i % kPeriod] + i / kPeriod * kPeriod * 16 * BK);
    }
};

// Work-groups go to the eight dies in turn; each die gets a contiguous part of the tiles, so that the operands its work-groups
// share stay in its own L2.
__device__ __forceinline__ int die_order(int id, int total) {
    const int die = id & 7, k = id >> 3, each = total >> 3, rest = total & 7;
    return die * each + min(die, rest) + k;
}

// One tile of one worker's product.
struct Job {
    Source sm, sn;
    int w, m0, n0, M, N, K;   // K < 0: no such rows
};

template <int MODE, int ET, bool X8, int BM, int BN> __device__ __forceinline__ Job job_of(const LinearArgs &a, int tile) {
    constexpr int EB = Elem<ET>::bytes;
    const int tiles = a.tiles_m * a.tiles_n;
    int id = tile;
    Job j{};
    const int w = id / tiles;
    id -= w * tiles;
    // eight tiles of m under each other, then the next n: what runs at the same time is a square of tiles
    const int band = id / (8 * a.tiles_n), high = min(8, a.tiles_m - band * 8);
    id -= band * 8 * a.tiles_n;
    const int m0 = (band * 8 + id % high) * BM, n0 = id / high * BN;
    const int count = rows_of(a.counts, w, a.rows);
    j.w = w;
    j.m0 = m0;
    j.n0 = n0;
    j.M = MODE == kWeights ? a.p : count;
    j.N = MODE == kForward ? a.p : a.q;
    j.K = MODE == kForward ? a.q : (MODE == kInput ? a.p : count);
    if (m0 >= j.M) {
        j.K = -1;
        return j;
    }
    const float *const params = MODE == kWeights ? nullptr : a.params[w];
    Source &sm = j.sm, &sn = j.sn;
    sm.limit = j.M - m0;
    sn.limit = j.N - n0;
    const int64_t kept_row = (int64_t)w * a.rows;  // a worker's first row in a checkpoint
    if constexpr (MODE == kForward) {
        if constexpr (X8) {
            sm.data = (gin)a.x8.codes + (kept_row + m0) * a.x8.pitch;
            sm.scales = (const PG_GLOBAL uint8_t *)a.x8.scales + (kept_row + m0) * (a.x8.pitch / kScaled);
            sm.ld = a.x8.pitch;
            sm.scale_ld = a.x8.pitch / kScaled;
        } else {
            sm.data = (gin)a.x.data + (w * a.x.worker + m0 * a.x.row) * EB;
            sm.ld = (int)a.x.row;
        }
        sn.data = (gin)(params + a.w_off + (int64_t)n0 * a.w_ld);
        sn.ld = a.w_ld;
    } else if constexpr (MODE == kInput) {
        sm.data = (gin)a.dz.data + (w * a.dz.worker + m0 * a.dz.row) * EB;
        sm.ld = (int)a.dz.row;
        sn.data = (gin)(params + a.w_off + n0);
        sn.ld = a.w_ld;
    } else {
        sm.data = (gin)a.dz.data + (w * a.dz.worker + m0) * EB;
        sm.ld = (int)a.dz.row;
        if constexpr (X8) {
            sn.data = (gin)a.x8.codes + kept_row * a.x8.pitch + n0;
            sn.scales = (const PG_GLOBAL uint8_t *)a.x8.scales + kept_row * (a.x8.pitch / kScaled) + n0 / kScaled;
            sn.ld = a.x8.pitch;
            sn.scale_ld = a.x8.pitch / kScaled;
        } else {
            sn.data = (gin)a.x.data + (w * a.x.worker + n0) * EB;
            sn.ld = (int)a.x.row;
        }
    }
    return j;
}

template <int MF, int NF> __device__ __forceinline__ void multiply(const u32x4 (&m)[MF], const u32x4 (&n)[NF], f32x4 (&acc)[MF][NF]) {
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, n[j]), __builtin_bit_cast(bf16x8, m[i]), acc[i][j], 0, 0, 0);
}

// What a tile's sums become.  Everything an element needs from memory is asked for before any of it is used, a few rows of results at
// a time; INNER tiles have all their columns, so that no access there is a partial one.
template <int MODE, int ET, bool INNER, int BM, int BN, int WM, int WN, int MF, int NF>
__device__ __forceinline__ void put_rows(const LinearArgs &a, const Job &job, const f32x4 (&acc)[MF][NF]) {
    constexpr int EB = Elem<ET>::bytes;
    constexpr int IR = MF * NF >= 32 ? 2 : (MF < 4 ? MF : 4);  // times 16 rows at once
    const int w = job.w, M = job.M, N = job.N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nfirst = job.n0 + wave / WM * (BN / WN);         // of the wavefront: a multiple of 32
    const int mw = job.m0 + wave % WM * (BM / WM) + lane % 16, nw = nfirst + lane / 16 * 4;
    auto have = [&](int j) { return INNER ? 4 : N - nw - 16 * j; };
    if constexpr (MODE == kWeights) {
        PG_GLOBAL float *const g = (PG_GLOBAL float *)(a.grads[w] + a.w_off + nw);
#pragma unroll
        for (int i0 = 0; i0 < MF; i0 += IR) {
            f32x4 old[IR][NF];
            if (a.accumulate)
#pragma unroll
                for (int i = 0; i < IR; ++i)
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        if (have(j) > 0) old[i][j] = load4<kF32>((gin)(g + (int64_t)min(mw + 16 * (i0 + i), M - 1) * a.w_ld + 16 * j), have(j));
#pragma unroll
            for (int i = 0; i < IR; ++i) {
                const int m = mw + 16 * (i0 + i);
                if (m >= M) continue;
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    if (have(j) > 0) store4<kF32>((gout)(g + (int64_t)m * a.w_ld + 16 * j), a.accumulate ? acc[i0 + i][j] + old[i][j] : acc[i0 + i][j], have(j));
            }
        }
    } else {
        const PG_GLOBAL float *const params = (const PG_GLOBAL float *)a.params[w];
        const int64_t kept_row = (int64_t)w * a.rows;
        const bool back = MODE == kInput && a.act != kActNone;
        f32x4 bias[NF] = {};
        if (MODE == kForward && a.b_off >= 0)
#pragma unroll
            for (int j = 0; j < NF; ++j)
                if (have(j) > 0) bias[j] = load4<kF32>((gin)(params + a.b_off + nw + 16 * j), have(j));
#pragma unroll
        for (int i0 = 0; i0 < MF; i0 += IR) {
            f32x4 res[IR][NF];
            uint32_t codes[IR][NF];
            uint8_t scales[IR][(NF + 1) / 2];
            if (a.res.data)
#pragma unroll
                for (int i = 0; i < IR; ++i) {
                    const gin row = (gin)a.res.data + (w * a.res.worker + min(mw + 16 * (i0 + i), M - 1) * a.res.row + nw) * EB;
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        if (have(j) > 0) res[i][j] = load4<ET>(row + 16 * j * EB, have(j));
                }
            if (back)
#pragma unroll
                for (int i = 0; i < IR; ++i) {
                    const int64_t row = (kept_row + min(mw + 16 * (i0 + i), M - 1)) * a.z8.pitch;
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        if (have(j) > 0) {
                            codes[i][j] = *(const uint32_t *)(a.z8.codes + row + nw + 16 * j);
                            if (j % 2 == 0) scales[i][j / 2] = a.z8.scales[row / kScaled + nfirst / kScaled + j / 2];
                        }
                }
            if (MODE == kForward && a.z8.codes)
#pragma unroll
                for (int i = 0; i < IR; ++i) {
                    const int m = mw + 16 * (i0 + i);
                    const int64_t row = (kept_row + m) * a.z8.pitch;
#pragma unroll
                    for (int j = 0; j < NF; j += 2) {
                        if (!INNER && nfirst + 16 * j >= N) continue;  // the whole wavefront
                        f32x4 z[2] = {acc[i0 + i][j] + bias[j], acc[i0 + i][j + 1] + bias[j + 1]};
                        if (!INNER)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (e % 4 >= have(j + e / 4)) z[e / 4][e % 4] = 0.f;
                        // lanes of rows that do not exist take part as well
                        auto most = [&] {
                            float top = larger(larger(0.f, z[0]), z[1]);
                            top = __builtin_fmaxf(top, __shfl_xor(top, 16));
                            return __builtin_fmaxf(top, __shfl_xor(top, 32));
                        };
                        float top = most();
                        if (__any(top == __builtin_inff())) {
                            z[0] = infinite_to_nan(z[0]);
                            z[1] = infinite_to_nan(z[1]);
                            top = most();
                        }
                        const int e = scale_exp(top);
                        const float inv = exp2_of(-e);
                        if (m < M) {
                            uint8_t *const to = a.z8.codes + row + nw + 16 * j;
                            *(uint32_t *)to = encode4(z[0], inv);
                            *(uint32_t *)(to + 16) = encode4(z[1], inv);
                            if (lane < 16) a.z8.scales[row / kScaled + nfirst / kScaled + j / 2] = (uint8_t)(e + 127);
                        }
                    }
                }
#pragma unroll
            for (int i = 0; i < IR; ++i) {
                const int m = mw + 16 * (i0 + i);
                if (m >= M) continue;
                const gout row = (gout)a.out.data + (w * a.out.worker + m * a.out.row + nw) * EB;
#pragma unroll
                for (int j = 0; j < NF; ++j) {
                    if (have(j) <= 0) continue;
                    f32x4 v = acc[i0 + i][j] + bias[j];
                    if (MODE == kForward && a.act != kActNone)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = act_of(a.act, v[e]);
                    if (back) {
                        const f32x4 z = decode4(codes[i][j], scale_of(scales[i][j / 2]));
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] *= slope_of(a.act, z[e]);
                    }
                    if (a.res.data) v += res[i][j];
                    store4<ET>(row + 16 * j * EB, v, have(j));
                }
            }
        }
    }
}
template <int MODE, int ET, int BM, int BN, int WM, int WN, int MF, int NF>
__device__ __forceinline__ void put_out(const LinearArgs &a, const Job &job, const f32x4 (&acc)[MF][NF]) {
    if (job.n0 + BN <= job.N) put_rows<MODE, ET, true, BM, BN, WM, WN>(a, job, acc);
    else put_rows<MODE, ET, false, BM, BN, WM, WN>(a, job, acc);
}

// A tile of BM x BN by WM x WN wavefronts.  acc[i][j]: lane l holds out rows m = 16 i + l % 16 of its wavefront's part and columns
// n = 16 j + 4 (l / 16) + 0..3, so that a lane's four results lie side by side in memory.  LDS holds two steps: while one is multiplied, the next
// is written from registers and the one after it is on its way from memory.
//
// Bound by the matrix cores and what feeds them: 8 x 2048 x 2048 x 8192 bf16, weight gradient 669 us (822 TFLOP/s; the library's one large product reaches 1325),
// input gradient 620 (886), forward 670 (820; 720 on another card); floats, six products each, 8 x 2048 x 2048 x 2048 750 us (183, 1100 on the matrix cores; the
// library's float product 154).  Of the forward pass 480 us remain without its loads from memory and writes to LDS, 520 without the loads, 660 without its stores.
// Few rows are bound by reading the weights: 16 x 10 x 33278 x 650 in 266 us, 5.3 TB/s.
//
// Where a product has too few tiles for the chip, `splits` work-groups share a tile's steps and leave their sums, in the order of their registers, for
// linear_join_kernel.
template <int MODE, int ET, bool X8, bool KEEP, int BM, int BN, int BK, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, ET == kBf16 || WM * WN == 8 ? 2 : 1) linear_kernel(const LinearArgs a) {
    using P = Product<MODE, ET, X8, KEEP, BK>;
    constexpr int THREADS = 64 * WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
    constexpr bool SUMS = MODE == kWeights;
    using StageM = Stage<P::msrc, P::macross, BM, BK, P::pm, THREADS, (P::pn > 1)>;
    using StageN = Stage<P::nsrc, P::nacross, BN, BK, P::pn, THREADS, (P::pm > 1)>;
    constexpr int kStep = P::pm * BM * BK + P::pn * BN * BK;
    __shared__ __attribute__((aligned(128))) uint16_t lds[2 * kStep];
    __shared__ int odd_step[2];
    const int slot = die_order(blockIdx.x, gridDim.x), tile = slot / a.splits, split = slot - tile * a.splits;
    const Job job = job_of<MODE, ET, X8, BM, BN>(a, tile);
    if (job.K < 0) return;
    const int each = a.split_steps * BK, first = split * each, end = min(job.K, first + each);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Reader<BK> rm(wave % WM * (BM / WM), lane), rn(wave / WM * (BN / WN), lane);
    StageM stm;
    StageN stn;
    f32x4 acc[MF][NF] = {}, sum = {0.f, 0.f, 0.f, 0.f};
    const bool want_sums = SUMS && job.n0 == 0 && a.b_off >= 0;

    auto store = [&](int at, int step) {
        if constexpr (SUMS)
            if (want_sums) stm.add_to(sum);
        uint16_t *const to = lds + at * kStep;
        const bool odd_m = stm.store(to, job.sm.limit, tid), odd_n = stn.store(to + P::pm * StageM::kPlane, job.sn.limit, tid);
        if (P::split && (odd_m || odd_n)) odd_step[at] = step;
    };
    auto part = [&](int at, bool odd, int ks) {
        const uint16_t *const lm = lds + at * kStep, *const ln = lm + P::pm * StageM::kPlane;
        u32x4 fm[P::pm][MF], fn[P::pn][NF];
#pragma unroll
        for (int p = 0; p < P::pn; ++p)
#pragma unroll
            for (int j = 0; j < NF; ++j) fn[p][j] = rn.read(ln + p * StageN::kPlane, ks, j);
#pragma unroll
        for (int p = 0; p < P::pm; ++p)
#pragma unroll
            for (int i = 0; i < MF; ++i) fm[p][i] = rm.read(lm + p * StageM::kPlane, ks, i);
        multiply(fm[0], fn[0], acc);
        if constexpr (P::split) {
            // The first pieces alone give what infinities and NaN give; the other products go without them.
            if (odd) {
#pragma unroll
                for (int j = 0; j < NF; ++j) fn[0][j] = finite_only(fn[0][j]);
#pragma unroll
                for (int i = 0; i < MF; ++i) fm[0][i] = finite_only(fm[0][i]);
            }
#pragma unroll
            for (int s = 1; s < 3; ++s)
#pragma unroll
                for (int p = 0; p <= s; ++p)
                    if (p < P::pm && s - p < P::pn) multiply(fm[p < P::pm ? p : 0], fn[s - p < P::pn ? s - p : 0], acc);
        }
    };

    const int steps = max(0, end - first + BK - 1) / BK;
    const bool whole = stm.plain(job.sm) && stn.plain(job.sn);
    if (P::split && tid < 2) odd_step[tid] = -1;
    if (steps > 0) {
        stm.load(job.sm, first, end, tid);
        stn.load(job.sn, first, end, tid);
        if (P::split) __syncthreads();
        store(0, 0);
        if (steps > 1) {
            stm.load(job.sm, first + BK, end, tid);
            stn.load(job.sn, first + BK, end, tid);
        }
        __syncthreads();
    }
    int step = 0;
    // the steps whose next but one is a whole one: no branch in their body, so that the compiler moves its parts into one another
    for (const int last = whole ? (end - first) / BK - 2 : 0; step < last; ++step) {
        const int at = step & 1;
        const bool odd = P::split && odd_step[at] == step;
        part(at, odd, 0);
        store(at ^ 1, step + 1);
        stm.load_whole(job.sm, first + (step + 2) * BK, tid);
        stn.load_whole(job.sn, first + (step + 2) * BK, tid);
#pragma unroll
        for (int ks = 1; ks < BK / 32; ++ks) part(at, odd, ks);
        __syncthreads();
    }
    for (; step < steps; ++step) {
        const int at = step & 1;
        const bool odd = P::split && odd_step[at] == step;
        part(at, odd, 0);
        if (step + 1 < steps) store(at ^ 1, step + 1);
        if (step + 2 < steps) {
            stm.load(job.sm, first + (step + 2) * BK, end, tid);
            stn.load(job.sn, first + (step + 2) * BK, end, tid);
        }
#pragma unroll
        for (int ks = 1; ks < BK / 32; ++ks) part(at, odd, ks);
        __syncthreads();
    }
    if constexpr (SUMS) {
        if (want_sums) {
            float *const all = (float *)lds;
            f32x4_any *const at = (f32x4_any *)(all + tid / (BM / 4) * BM + StageM::row_at(tid, job.sm.limit));
            *at = sum;
            __syncthreads();
            if (tid < min(job.M - job.m0, BM)) {
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < THREADS * 4 / BM; ++g) v += all[g * BM + tid];
                if (a.splits > 1) {
                    a.part_sums[((int64_t)split * a.n + job.w) * a.p + job.m0 + tid] = v;
                } else {
                    float *const out = a.grads[job.w] + a.b_off + job.m0 + tid;
                    *out = a.accumulate ? *out + v : v;
                }
            }
        }
    }
    if (a.splits > 1) {
        f32x4 *const part = (f32x4 *)a.part + (int64_t)slot * MF * NF * THREADS + tid;
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) part[(i * NF + j) * THREADS] = acc[i][j];
        return;
    }
    put_out<MODE, ET, BM, BN, WM, WN, MF, NF>(a, job, acc);
}

// Adds up what the work-groups of a tile left, always in the same order: 16 rows of every wavefront's part per work-group.
template <int MODE, int ET, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN) linear_join_kernel(const LinearArgs a) {
    constexpr int THREADS = 64 * WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
    const int tile = blockIdx.x / MF, i = blockIdx.x - tile * MF, tid = threadIdx.x;
    Job job = job_of<MODE, ET, false, BM, BN>(a, tile);
    if (job.K < 0) return;
    f32x4 acc[1][NF] = {};
    const f32x4 *part = (const f32x4 *)a.part + ((int64_t)tile * a.splits * MF + i) * NF * THREADS + tid;
    for (int s = 0; s < a.splits; ++s, part += MF * NF * THREADS)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[0][j] += part[j * THREADS];
    if (MODE == kWeights && i == 0 && job.n0 == 0 && a.b_off >= 0 && tid < min(job.M - job.m0, BM)) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v += a.part_sums[((int64_t)s * a.n + job.w) * a.p + job.m0 + tid];
        float *const out = a.grads[job.w] + a.b_off + job.m0 + tid;
        *out = a.accumulate ? *out + v : v;
    }
    job.m0 += 16 * i;
    put_out<MODE, ET, BM, BN, WM, WN, 1, NF>(a, job, acc);
}

namespace {

// Steps of 32 for the largest bf16 tiles where those of 64 do not fit the registers (scratch memory: input gradients 859 against 639 us, 8 x 2048 x 2048 x 8192;
// forward 672 against 687); codes, which take fewer, are faster in steps of 64 (704 against 759 us).
constexpr bool short_steps(int mode, bool x8) { return mode == kInput || (mode == kForward && !x8); }

// How a product is cut into tiles, and each tile's k among work-groups.
struct Cut {
    int bm, bn, bk, tiles_m, tiles_n, splits, split_steps;
};
// What a tile takes: work-groups that share a compute unit, microseconds for 64 of k where a compute unit has one of them and where it has as many as
// fit, and microseconds for its start and end.  Measured with every tile forced (8 x 2048 x 2048 x 2048 for full units, 1 x 512 x 2048 x 2048 for
// single ones).  bf16, full: 171, 248, 299, 442 us from the largest tile to the smallest; single: 69, 37, 26, 26 us.  float: 814, 880, 970, 1355 and 167, 100, 93 us.
struct TileCost {
    int bm, bn, fit;
    float one, full, ends;
};
constexpr TileCost kTilesBf16[] = {{256, 256, 1, 2.1f, 2.1f, 15.f}, {128, 128, 2, 1.f, 1.75f, 5.f}, {64, 128, 3, 0.65f, 1.6f, 4.f}, {32, 128, 3, 0.6f, 1.2f, 4.f}};
constexpr TileCost kTilesF32[] = {{256, 128, 1, 5.f, 6.f, 8.f}, {128, 128, 1, 3.f, 3.2f, 5.f}, {64, 128, 2, 2.6f, 3.6f, 5.f}, {32, 128, 2, 1.8f, 2.6f, 4.f}};

// The cut with the least estimated time: rounds of work-groups, no less than the operands take from memory, and the joining of split sums.  Split or not, measured
// (bf16, us): 1 x 512 x 2048 x 2048 37 -> 23 in four, 1 x 16 x 4096 x 4096 43 -> 20 in eight; 8 x 1 x 2048 x 2048, whose weights
// take as long to read, 27 -> 29 in four.
Cut cut_of(int mode, int type, bool x8, bool keep, int n, int rows, int p, int q, CutForced forced) {
    const int M = mode == kWeights ? p : rows, N = mode == kForward ? p : q, K = mode == kForward ? q : (mode == kInput ? p : rows);
    const float element = type == kF32 ? 4.f : 2.f;
    const float memory = ((float)p * q * 4.f + ((float)p + q) * rows * element) * n / 5e6f;  // us
    Cut best{};
    float least = 0.f;
    for (const TileCost &t : type == kF32 ? kTilesF32 : kTilesBf16) {
        if (mode == kWeights && t.bm == 32) continue;
        if (forced.tile && t.bm != (mode == kWeights ? std::max(64, forced.tile) : forced.tile)) continue;
        Cut c{};
        c.bm = t.bm;
        c.bn = t.bn;
        c.bk = type == kF32 || keep || (t.bm == 256 && short_steps(mode, x8)) ? 32 : 64;
        c.tiles_m = (M + t.bm - 1) / t.bm;
        c.tiles_n = (N + t.bn - 1) / t.bn;
        const int64_t tiles = (int64_t)c.tiles_m * c.tiles_n * n;
        if (tiles > kMostTiles && t.bm != 256) continue;
        const int steps = std::max(1, (K + c.bk - 1) / c.bk);
        for (int wanted : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (wanted > 1 && (wanted * 2 > steps || tiles * wanted > kMostSplit)) break;
            if (forced.splits && wanted < forced.splits && wanted * 4 <= steps && tiles * wanted * 2 <= kMostSplit) continue;
            c.split_steps = (steps + wanted - 1) / wanted;
            c.splits = (steps + c.split_steps - 1) / c.split_steps;
            const float groups = (float)(tiles * c.splits), per_unit = groups / kComputeUnits;
            const float along = c.split_steps * c.bk / 64.f;
            float time;
            if (per_unit <= t.fit) {
                const float shared = t.fit > 1 ? (std::max(1.f, std::ceil(per_unit)) - 1.f) / (t.fit - 1) : 0.f;
                time = along * (t.one + (t.full - t.one) * shared) + t.ends;
            } else {
                const float rounds = per_unit / t.fit;
                time = 0.5f * (rounds + std::ceil(rounds)) * (along * t.full + t.ends);  // work-groups drift apart: half of a last round's gap is filled
            }
            time = std::max(time, memory) + 0.1f * time;
            if (c.splits > 1) time += 5.f + groups * t.bm * t.bn * 8.f / 8e6f;
            if (best.bm == 0 || time < least) {
                best = c;
                least = time;
            }
        }
    }
    return best;
}
int64_t part_floats(const Cut &c, int n) { return c.splits > 1 ? (int64_t)c.splits * c.tiles_m * c.tiles_n * n * c.bm * c.bn : 0; }

template <int MODE, int ET, bool X8, bool KEEP, int BM, int BN, int BK, int WM, int WN> void launch(const LinearArgs &a, hipStream_t st) {
    const unsigned tiles = (unsigned)a.tiles_m * a.tiles_n * a.n;
    if (!tiles) return;
    linear_kernel<MODE, ET, X8, KEEP, BM, BN, BK, WM, WN><<<dim3(tiles * a.splits), dim3(64 * WM * WN), 0, st>>>(a);
    if (a.splits > 1) linear_join_kernel<MODE, ET, BM, BN, WM, WN><<<dim3(tiles * (BM / WM / 16)), dim3(64 * WM * WN), 0, st>>>(a);
}
template <int MODE, int ET, bool X8, bool KEEP = false> void launch_cut(LinearArgs a, hipStream_t st) {
    const Cut c = cut_of(MODE, ET, X8, KEEP, a.n, a.rows, a.p, a.q, a.forced);
    a.tiles_m = c.tiles_m;
    a.tiles_n = c.tiles_n;
    a.splits = c.splits;
    a.split_steps = c.split_steps;
    a.part_sums = a.part + part_floats(c, a.n);
    constexpr int BK = ET == kF32 || KEEP ? 32 : 64;
    if (c.bm == 256) {
        if constexpr (ET == kF32) launch<MODE, ET, X8, KEEP, 256, 128, 32, 4, 2>(a, st);
        else launch<MODE, ET, X8, KEEP, 256, 256, short_steps(MODE, X8) ? 32 : BK, 2, 4>(a, st);
    } else if (c.bm == 128) {
        if constexpr (ET == kF32) launch<MODE, ET, X8, KEEP, 128, 128, BK, 2, 4>(a, st);
        else launch<MODE, ET, X8, KEEP, 128, 128, BK, 2, 2>(a, st);
    } else if (c.bm == 64) {
        launch<MODE, ET, X8, KEEP, 64, 128, BK, 2, 2>(a, st);
    } else {
        if constexpr (MODE != kWeights) launch<MODE, ET, X8, KEEP, 32, 128, BK, 1, 4>(a, st);
    }
}

}  // namespace

void launch_linear(const LinearArgs &a, int type, hipStream_t st) {
    if (type == kF32) a.x8.codes ? launch_cut<kForward, kF32, true>(a, st) : launch_cut<kForward, kF32, false>(a, st);
    else if (a.z8.codes) a.x8.codes ? launch_cut<kForward, kBf16, true, true>(a, st) : launch_cut<kForward, kBf16, false, true>(a, st);
    else a.x8.codes ? launch_cut<kForward, kBf16, true>(a, st) : launch_cut<kForward, kBf16, false>(a, st);
}
void launch_linear_dx(const LinearArgs &a, int type, hipStream_t st) {
    type == kF32 ? launch_cut<kInput, kF32, false>(a, st) : launch_cut<kInput, kBf16, false>(a, st);
}
void launch_linear_dw(const LinearArgs &a, int type, hipStream_t st) {
    if (type == kF32) a.x8.codes ? launch_cut<kWeights, kF32, true>(a, st) : launch_cut<kWeights, kF32, false>(a, st);
    else a.x8.codes ? launch_cut<kWeights, kBf16, true>(a, st) : launch_cut<kWeights, kBf16, false>(a, st);
}

namespace {
// Every cut that a call on these sizes may take: fn(mode, cut).
template <typename F> void each_cut(int n, int rows, int p, int q, int type, CutForced forced, F fn) {
    for (int mode : {kForward, kInput, kWeights})
        for (int x8 = 0; x8 < 2; ++x8)
            for (int keep = 0; keep < 2; ++keep)
                if ((mode == kForward || !keep) && (mode != kInput || !x8) && (type != kF32 || !keep)) 
                    fn(mode, cut_of(mode, type, x8, keep, n, rows, p, q, forced));
}
}  // namespace

// The two gradients of a call run one after the other and share the workspace.
size_t linear_workspace(int n, int rows, int p, int q, int type, CutForced forced) {
    int64_t most = 0;
    each_cut(n, rows, p, q, type, forced, [&](int mode, const Cut &c) {
        if (c.splits > 1) most = std::max(most, part_floats(c, n) + (mode == kWeights ? (int64_t)c.splits * n * p : 0));
    });
    return sizeof(float) * (size_t)most;
}
bool linear_fits(int n, int rows, int p, int q, int type, CutForced forced) {
    bool fits = true;
    each_cut(n, rows, p, q, type, forced, [&](int, const Cut &c) { fits &= c.bm > 0 && (int64_t)c.tiles_m * c.tiles_n * n <= kMostTiles; });  // bm 0: no tile of the forced size does
    return fits;
}

}  // namespace pg
