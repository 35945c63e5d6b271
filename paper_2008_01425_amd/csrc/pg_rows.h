// Rows of activations: what the kernels that turn parameters into gradients take, and the number formats they share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pg {

// Element types of activations (PG_F32, PG_BF16) and activation functions (PG_ACT_*), as in the C header.
constexpr int kF32 = 0, kBf16 = 1;
constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3;

// Longest rows a norm takes: what 16 wavefronts hold in registers.
constexpr int kMostCols = 16384;

// Elements a checkpoint scales together, and the smallest exponent of their scale: 2^-117 times the smallest
// e4m3 value, 2^-9, is the smallest normal float, so no decoded value is a subnormal one.
constexpr int kScaled = 32;
constexpr int kLeastExp = -117;
// The scale byte of the largest exponent, 120: the only one under which a value, 256 * 2^120 and more, is no finite float and is read as an infinity.
constexpr int kLargestScale = 120 + 127;

struct RowsArg {
    char *data;
    int64_t row, worker;  // elements between rows, between workers
};
struct KeptArg {
    uint8_t *codes, *scales;  // null: none
    int pitch;                // bytes of a row of codes (a multiple of 32); a row of scales has pitch / 32
};

// Tuning experiments and tests: the rows of every tile (32, 64, 128, 256) and the parts its steps are split into; 0: by the estimate.
struct CutForced {
    int tile = 0, splits = 0;
};

struct LinearArgs {
    float *const *params;
    float *const *grads;
    int64_t w_off, b_off;     // floats inside a worker's buffer; b_off < 0: no bias
    int w_ld;
    int n, rows, p, q;
    const int32_t *counts;    // rows of each worker (null: all)
    RowsArg x, dz, res, out;  // null data: absent
    KeptArg x8, z8;
    int act, accumulate;
    CutForced forced;
    int tiles_m, tiles_n, splits, split_steps;
    float *part, *part_sums;  // partial sums of a split product, and of its bias gradient
};

struct NormArgs {
    float *const *params;
    float *const *grads;
    int64_t g_off, b_off;      // b_off < 0: no bias
    int n, rows, cols;
    const int32_t *counts;
    RowsArg x, res, sum, out;  // forward: input, its addend, their sum, result; backward: dy, gradient that passes by, sum, result
    KeptArg y8;
    float *mean, *rstd;        // mean: layer norms
    float eps;
    int accumulate, blocks;    // backward: work-groups per worker
    float *part;               // ... and their column sums
};

// Most entries of a teacher's a row has.
constexpr int kMostTop = 1024;

struct DistillArgs {
    int n, rows, cols;
    const int32_t *counts;
    RowsArg z, dz;
    const int32_t *labels;     // null: no cross entropy
    int top;                   // 0: no teacher
    const int32_t *top_index;
    const float *top_logits, *weights;
    float *loss;
    float temperature, hard, soft;
};

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
    int forced;                             // tests: parts; 0: by the estimate
    int tiles, splits;                      // of a sequence and key head: tiles of its own rows, parts of the other side
    float *part, *part_stats;               // partial results [split][row][head][width], and [split][row][head] largest score and sum
};

struct KeptArgs {  // storing, reading back, and going back through an activation
    int n, rows, cols;
    const int32_t *counts;
    RowsArg x, out;
    KeptArg kept;
    int act;
};

// type: kF32 or kBf16
void launch_linear(const LinearArgs &a, int type, hipStream_t st);
void launch_linear_dx(const LinearArgs &a, int type, hipStream_t st);
void launch_linear_dw(const LinearArgs &a, int type, hipStream_t st);
size_t linear_workspace(int n, int rows, int p, int q, int type, CutForced forced);
bool linear_fits(int n, int rows, int p, int q, int type, CutForced forced);   // few enough tiles for a launch
void launch_norm(const NormArgs &a, int type, hipStream_t st);
void launch_norm_backward(const NormArgs &a, int type, hipStream_t st);
void launch_layer_norm(const NormArgs &a, int type, hipStream_t st);
void launch_layer_norm_backward(const NormArgs &a, int type, hipStream_t st);
int norm_backward_blocks(int n, int rows, int cols, bool center);
void launch_store(const KeptArgs &a, int type, hipStream_t st);
void launch_load(const KeptArgs &a, int type, hipStream_t st);
void launch_distill(const DistillArgs &a, int type, hipStream_t st);
dim3 attention_grid(const AttentionArgs &a);
size_t attention_forward_workspace(const AttentionArgs &a, int type);
size_t attention_backward_workspace(const AttentionArgs &a, int type);  // delta, from a multiple of 256 bytes on the parts
void launch_attention(AttentionArgs a, int type, hipStream_t st);
void launch_attention_dq(AttentionArgs a, int type, hipStream_t st);
void launch_attention_delta(const AttentionArgs &a, int type, hipStream_t st);
void launch_attention_dkv(AttentionArgs a, int type, hipStream_t st);
void launch_activation_backward(const KeptArgs &a, int type, hipStream_t st);

#ifdef __HIP__
// Pointers that come out of the workers' pointer tables are generic to the compiler, and a generic (flat) load also waits for LDS: what a kernel
// reads or writes through them is cast to global memory.
#define PG_GLOBAL __attribute__((address_space(1)))
typedef const PG_GLOBAL char *gin;
typedef PG_GLOBAL char *gout;
template <typename T> __device__ __forceinline__ T at_global(gin p) { return *(const PG_GLOBAL T *)p; }
template <typename T> __device__ __forceinline__ void to_global(gout p, const T &v) { *(PG_GLOBAL T *)p = v; }

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));  // four bf16 at any address of their own
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // eight
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int ET> struct Elem;
template <> struct Elem<kF32> {
    static constexpr int bytes = 4;
};
template <> struct Elem<kBf16> {
    static constexpr int bytes = 2;
};

__device__ __forceinline__ float bf16_low(uint32_t two) { return __uint_as_float(two << 16); }
__device__ __forceinline__ float bf16_high(uint32_t two) { return __uint_as_float(two & 0xffff0000u); }
// to nearest even, two in one instruction
__device__ __forceinline__ uint32_t bf16_pack(float a, float b) {
    bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint16_t bf16_bits(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

// `have` (1..4) elements at any address of their own type, the rest zero
template <int ET> __device__ __forceinline__ f32x4 load4(gin p, int have) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if constexpr (ET == kF32) {
        if (have >= 4) return at_global<f32x4_any>(p);
        for (int i = 0; i < 3; ++i)
            if (i < have) v[i] = at_global<float>(p + 4 * i);
    } else {
        if (have >= 4) {
            const u32x2 w = at_global<u32x2_any>(p);
            return f32x4{bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])};
        }
        for (int i = 0; i < 3; ++i)
            if (i < have) v[i] = bf16_low(at_global<uint16_t>(p + 2 * i));
    }
    return v;
}
template <int ET> __device__ __forceinline__ void store4(gout p, const f32x4 &v, int have) {
    if constexpr (ET == kF32) {
        if (have >= 4) {
            to_global<f32x4_any>(p, v);
            return;
        }
        for (int i = 0; i < 3; ++i)
            if (i < have) to_global<float>(p + 4 * i, v[i]);
    } else {
        if (have >= 4) {
            to_global<u32x2_any>(p, u32x2{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])});
            return;
        }
        for (int i = 0; i < 3; ++i)
            if (i < have) to_global<uint16_t>(p + 2 * i, bf16_bits(v[i]));
    }
}

// ---- 8-bit checkpoints ---------------------------------------------------------------------
//
// 32 elements of a row share a scale 2^e, e the least integer >= kLeastExp with max |x| <= 448 * 2^e (448 is the
// largest e4m3 value, so nothing saturates and every rounding is by half a step at most); each is held as the nearest e4m3 value of x * 2^-e, ties
// to even.  What is not finite is held as e4m3's NaN and does not enter the maximum.

// 448 = 0.875 * 2^9, so the exponent is that of the maximum less 8, one more where its mantissa exceeds 1.75.
__device__ __forceinline__ int scale_exp(float top) {
    const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8;
    return e < kLeastExp ? kLeastExp : e;
}
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// max |x|, NaN left out
__device__ __forceinline__ float larger(float top, const f32x4 &v) {
    top = __builtin_fmaxf(__builtin_fmaxf(top, __builtin_fabsf(v[0])), __builtin_fabsf(v[1]));
    return __builtin_fmaxf(__builtin_fmaxf(top, __builtin_fabsf(v[2])), __builtin_fabsf(v[3]));
}
__device__ __forceinline__ f32x4 infinite_to_nan(f32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (__builtin_fabsf(v[i]) == __builtin_inff()) v[i] = __builtin_nanf("");
    return v;
}
// four codes in a word, the first in the low byte; inv = 2^-e
__device__ __forceinline__ uint32_t encode4(const f32x4 &v, float inv) {
    const uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, (int)w, true);
}
__device__ __forceinline__ f32x4 decode4(uint32_t w, float scale) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}
// two of a word's codes as bf16, exactly
template <bool HIGH> __device__ __forceinline__ uint32_t decode_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}
__device__ __forceinline__ float scale_of(uint8_t byte) { return __uint_as_float((uint32_t)byte << 23); }

// ---- activation functions, in float ----------------------------------------------------------
// NaN in, NaN out, in functions and slopes: a checkpoint holds what is not finite as NaN.
//   relu z > 0 ? z : 0;  gelu z Phi(z), Phi the normal distribution function;  silu z / (1 + exp(-z))
// The hardware's 2^x and 1 / x, an ulp each.  Phi by Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26, off by 0.75e-7 at most, which
// shares its exponential with the density: with the library's erf and exp the tiles' last part alone took longer (8 x 2048 x 8192 x 2048 bf16 with gelu
// forward 1023 -> 955 us, input gradient through gelu 1599 -> 1458 us).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + exp_of(-z)); }
// Phi(-|z|), and exp(-z^2 / 2)
__device__ __forceinline__ float lower_tail(float z, float &density) {
    const float x = __builtin_fabsf(z) * 0.70710678f, t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * x);
    density = exp_of(-x * x);
    return t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f)))) * density;
}
__device__ __forceinline__ float act_of(int act, float z) {
    if (act == kActRelu) return z > 0.f ? z : (z != z ? z : 0.f);
    if (act == kActGelu) {
        float density;
        const float low = lower_tail(z, density);
        return z * (z > 0.f ? 1.f - low : low);
    }
    if (act == kActSilu) return z * sigmoid(z);
    return z;
}
__device__ __forceinline__ float slope_of(int act, float z) {
    if (act == kActRelu) return z > 0.f ? 1.f : (z != z ? z : 0.f);
    if (act == kActGelu) {
        float density;
        const float low = lower_tail(z, density);
        return (z > 0.f ? 1.f - low : low) + 0.39894228f * z * density;
    }
    if (act == kActSilu) {
        const float g = sigmoid(z);
        return g * (1.f + z * (1.f - g));
    }
    return 1.f;
}

// rows of worker w that count
__device__ __forceinline__ int rows_of(const int32_t *counts, int w, int rows) {
    if (!counts) return rows;
    const int c = counts[w];
    return c < 0 ? 0 : (c > rows ? rows : c);
}
#endif

}  // namespace pg
