// Norms of rows of activations, by their root mean square or by mean and variance (layer norms), and their gradients, rows kept in 8 bits, and the way back through an activation
// whose input was kept: everything beside the products that one pass over the rows does, so all of it is bound by memory.  Measured, bf16, bytes read and
// written once (a copy of 2 GiB: 4.9 TB/s): norm of 8 x 8192 x 2048 with residual, sum and 8-bit result 186 us, 5.1 TB/s; its backward 223 us, 4.8 TB/s; layer norm without the
// 8 bits 215 us, 5.0 TB/s, and back 205 us, 5.2 TB/s; 16 x 700 ragged rows of 1301 floats back 38 us;
// 8 x 2048 x 8192 back through an activation 134 us, 5.0 TB/s, read back from 8 bits 69 us, 5.9 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pg_rows.h"

namespace pg {

namespace {

constexpr int kWave = 64;

struct Eight {
    f32x4 a, b;
};
template <int ET> __device__ __forceinline__ Eight load8(gin p, int have) {
    if constexpr (ET == kBf16) {
        if (have >= 8) {
            const u32x4 w = at_global<u32x4_any>(p);
            return {{bf16_low(w[0]), bf16_high(w[0]), bf16_low(w[1]), bf16_high(w[1])},
                    {bf16_low(w[2]), bf16_high(w[2]), bf16_low(w[3]), bf16_high(w[3])}};
        }
    }
    Eight v = {load4<ET>(p, have), {0.f, 0.f, 0.f, 0.f}};
    if (have > 4) v.b = load4<ET>(p + 4 * Elem<ET>::bytes, have - 4);
    return v;
}
template <int ET> __device__ __forceinline__ void store8(gout p, const Eight &v, int have) {
    if constexpr (ET == kBf16) {
        if (have >= 8) {
            to_global<u32x4_any>(p, u32x4{bf16_pack(v.a[0], v.a[1]), bf16_pack(v.a[2], v.a[3]), bf16_pack(v.b[0], v.b[1]), bf16_pack(v.b[2], v.b[3])});
            return;
        }
    }
    store4<ET>(p, v.a, have);
    if (have > 4) store4<ET>(p + 4 * Elem<ET>::bytes, v.b, have - 4);
}
// Eight elements as they are in memory: half the registers of their floats where they are bf16, for rows that wait for their sums.
template <int ET> struct Raw {
    u32x4 w[ET == kF32 ? 2 : 1];
    __device__ __forceinline__ void load(gin p, int have) {
        if (have >= 8) {
            w[0] = at_global<u32x4_any>(p);
            if constexpr (ET == kF32) w[1] = at_global<u32x4_any>(p + 16);
            return;
        }
        const Eight v = load8<ET>(p, have);
        if constexpr (ET == kF32) {
            w[0] = __builtin_bit_cast(u32x4, v.a);
            w[1] = __builtin_bit_cast(u32x4, v.b);
        } else {
            w[0] = u32x4{bf16_pack(v.a[0], v.a[1]), bf16_pack(v.a[2], v.a[3]), bf16_pack(v.b[0], v.b[1]), bf16_pack(v.b[2], v.b[3])};
        }
    }
    __device__ __forceinline__ Eight get() const {
        if constexpr (ET == kF32) return {__builtin_bit_cast(f32x4, w[0]), __builtin_bit_cast(f32x4, w[1])};
        else return {{bf16_low(w[0][0]), bf16_high(w[0][0]), bf16_low(w[0][1]), bf16_high(w[0][1])},
                     {bf16_low(w[0][2]), bf16_high(w[0][2]), bf16_low(w[0][3]), bf16_high(w[0][3])}};
    }
};
template <int ET> __device__ __forceinline__ f32x4 rounded(const f32x4 &v) {
    if constexpr (ET == kF32) return v;
    return f32x4{(float)(__bf16)v[0], (float)(__bf16)v[1], (float)(__bf16)v[2], (float)(__bf16)v[3]};
}

// Eight consecutive elements of a row per lane, four lanes to a scale; all four take part.
__device__ __forceinline__ void keep8(Eight v, uint8_t *codes, uint8_t *scale, bool first) {
    auto most = [&] {
        float top = larger(larger(0.f, v.a), v.b);
        top = __builtin_fmaxf(top, __shfl_xor(top, 1));
        return __builtin_fmaxf(top, __shfl_xor(top, 2));
    };
    float top = most();
    if (__any(top == __builtin_inff())) {
        v = {infinite_to_nan(v.a), infinite_to_nan(v.b)};
        top = most();
    }
    const int e = scale_exp(top);
    const float inv = exp2_of(-e);
    *(u32x2 *)codes = u32x2{encode4(v.a, inv), encode4(v.b, inv)};
    if (first) *scale = (uint8_t)(e + 127);
}

// Sum over the LANES that share a row, the same value in every lane.  One barrier: sums in a row use the two halves of `lds` in turn.
template <int LANES> __device__ __forceinline__ float row_sum(float v, float *lds) {
    constexpr int WAVES = LANES / kWave;
#pragma unroll
    for (int d = 1; d < (LANES < kWave ? LANES : kWave); d *= 2) v += __shfl_xor(v, d);
    if constexpr (WAVES > 1) {
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += lds[i];
    }
    return v;
}

// The same of two values with one barrier.
template <int LANES> __device__ __forceinline__ f32x2 row_sum2(f32x2 v, f32x2 *lds) {
    constexpr int WAVES = LANES / kWave;
#pragma unroll
    for (int d = 1; d < (LANES < kWave ? LANES : kWave); d *= 2) v += f32x2{__shfl_xor(v[0], d), __shfl_xor(v[1], d)};
    if constexpr (WAVES > 1) {
        if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = v;
        __syncthreads();
        v = f32x2{0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += lds[i];
    }
    return v;
}

}  // namespace

// Lanes of a launch are counted in 32 bits along each side of its grid: work-groups beyond kMostGroups go to the next y.
constexpr int64_t kMostGroups = 1 << 20;
__device__ __forceinline__ int64_t group_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// A row per LANES, NV times eight elements of it in each lane's registers: read once, written once.  A lane's eights lie LANES * 8
// apart, so that every access of a wavefront is one piece of a row (or of several short ones).
//
// CENTER: the layer norm, whose rows lose their mean and gain a bias.  The mean is that of the row as it is in registers, and the squares are those of
// what is left of it, never a difference of two large sums; what rounding left in the mean comes out of the same second sum.
template <int ET, int LANES, int NV, bool CENTER>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) norm_kernel(const NormArgs a) {
    constexpr int EB = Elem<ET>::bytes, ROWS = LANES < 256 ? 256 / LANES : 1;
    __shared__ float lds[LANES / kWave + 1];
    __shared__ f32x2 lds2[CENTER ? LANES / kWave + 1 : 1];
    const int r = (int)group_of() * ROWS + threadIdx.x / LANES;
    if (r >= a.n * a.rows) return;
    const int w = r / a.rows, t = r - w * a.rows, lane = threadIdx.x % LANES;
    if (t >= rows_of(a.counts, w, a.rows)) return;
    const gin x = (gin)a.x.data + (w * a.x.worker + t * a.x.row) * EB;
    const gin res = a.res.data ? (gin)a.res.data + (w * a.res.worker + t * a.res.row) * EB : nullptr;
    Eight v[NV];
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * 8, have = a.cols - c;
        v[k] = {};
        if (have <= 0) continue;
        v[k] = load8<ET>(x + c * EB, have);
        if (res) {
            const Eight y = load8<ET>(res + c * EB, have);
            // the norm is that of the sum as it is stored
            v[k].a = rounded<ET>(v[k].a + y.a);
            v[k].b = rounded<ET>(v[k].b + y.b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sq += CENTER ? v[k].a[i] + v[k].b[i] : v[k].a[i] * v[k].a[i] + v[k].b[i] * v[k].b[i];
    }
    sq = row_sum<LANES>(sq, lds);
    float mean = 0.f;
    if constexpr (CENTER) {
        const float near = sq / (float)a.cols;
        f32x2 left = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int have = a.cols - (k * LANES + lane) * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = i < have ? v[k].a[i] - near : 0.f, e = i + 4 < have ? v[k].b[i] - near : 0.f;
                left += f32x2{d + e, d * d + e * e};
            }
        }
        left = row_sum2<LANES>(left, lds2);
        const float off = left[0] / (float)a.cols;
        mean = near + off;
        sq = __builtin_fmaxf(left[1] - left[0] * off, 0.f);
        if (left[1] != left[1]) sq = left[1];  // the maximum drops a NaN
    }
    const float rstd = 1.f / sqrtf(sq / (float)a.cols + a.eps);
    if (lane == 0 && a.rstd) a.rstd[(int64_t)w * a.rows + t] = rstd;
    if (CENTER && lane == 0 && a.mean) a.mean[(int64_t)w * a.rows + t] = mean;
    const PG_GLOBAL float *const gain = (const PG_GLOBAL float *)(a.params[w] + a.g_off);
    const PG_GLOBAL float *const bias = CENTER && a.b_off >= 0 ? (const PG_GLOBAL float *)(a.params[w] + a.b_off) : nullptr;
    const int64_t at = (int64_t)w * a.rows + t;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * 8, have = a.cols - c;
        if (c >= (a.cols + kScaled - 1) / kScaled * kScaled) continue;
        Eight g = {};
        if (have > 0) {
            if (a.sum.data) store8<ET>((gout)a.sum.data + (w * a.sum.worker + t * a.sum.row + c) * EB, v[k], have);
            g = load8<kF32>((gin)(gain + c), have);
        }
        Eight y;
        if constexpr (CENTER) {
            Eight b = {};
            if (bias && have > 0) b = load8<kF32>((gin)(bias + c), have);
            y = {(v[k].a - mean) * rstd * g.a + b.a, (v[k].b - mean) * rstd * g.b + b.b};
        } else {
            y = {v[k].a * rstd * g.a, v[k].b * rstd * g.b};
        }
        if (have > 0 && a.out.data) store8<ET>((gout)a.out.data + (w * a.out.worker + t * a.out.row + c) * EB, y, have);
        if (have < 8) {  // what fills a row of codes up is zero, also where rstd is not a number
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= have) y.a[i] = 0.f;
                if (i + 4 >= have) y.b[i] = 0.f;
            }
        }
        if (a.y8.codes) keep8(y, a.y8.codes + at * a.y8.pitch + c, a.y8.scales + (at * a.y8.pitch + c) / kScaled, lane % 4 == 0);
    }
}

// ds = dr + rstd (g dy - xhat mean(g dy xhat)), xhat = s rstd;  dg = sum over rows of dy xhat.  A work-group walks along the rows of
// one worker, its columns' part of dg in registers; the parts are added up by norm_join_kernel, always in the same order.
//
// CENTER: ds = dr + rstd (g dy - mean(g dy) - xhat mean(g dy xhat)), xhat = (s - mean) rstd;  db = sum over rows of dy, behind dg among the parts.
template <int ET, int LANES, int NV, bool CENTER>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES, (CENTER && LANES < 256 ? 4 : 1)) norm_backward_kernel(const NormArgs a) {
    constexpr int EB = Elem<ET>::bytes, GROUPS = LANES < 256 ? 256 / LANES : 1, WAVES = LANES / kWave;
    __shared__ float lds[2 * WAVES + 1];
    __shared__ f32x2 lds2[CENTER ? 2 * WAVES + 1 : 1];
    __shared__ __attribute__((aligned(16))) float sums[GROUPS > 1 ? GROUPS * NV * LANES * 8 : 4];
    const int w = blockIdx.x / a.blocks, b = blockIdx.x - w * a.blocks;
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int count = rows_of(a.counts, w, a.rows);
    const PG_GLOBAL float *const gain = (const PG_GLOBAL float *)(a.params[w] + a.g_off);
    Eight g[NV], dg[NV], db[CENTER ? NV : 1];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (k * LANES + lane) * 8;
        g[k] = dg[k] = {};
        if constexpr (CENTER) db[k] = {};
        if (c < a.cols) g[k] = load8<kF32>((gin)(gain + c), a.cols - c);
    }
    struct Row {
        Raw<ET> dy[NV], sum[NV], res[NV];
        float rstd, center;
    };
    auto fetch = [&](Row &r, int t) __attribute__((always_inline)) {
        const gin dy_row = (gin)a.x.data + (w * a.x.worker + t * a.x.row) * EB, sum_row = (gin)a.sum.data + (w * a.sum.worker + t * a.sum.row) * EB;
        const gin res_row = a.res.data ? (gin)a.res.data + (w * a.res.worker + t * a.res.row) * EB : nullptr;
        r.rstd = a.rstd[(int64_t)w * a.rows + t];
        r.center = CENTER ? a.mean[(int64_t)w * a.rows + t] : 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * 8, have = a.cols - c;
            r.dy[k] = r.sum[k] = r.res[k] = {};
            if (have <= 0) continue;
            r.dy[k].load(dy_row + c * EB, have);
            r.sum[k].load(sum_row + c * EB, have);
            if (res_row) r.res[k].load(res_row + c * EB, have);
        }
    };
    // The next row sets out before the barrier of this one: layer norms, 16 x 700 ragged rows of 1301 floats 41.6 us for 44.5; the other norms, which have fewer sums and run more
    // work-groups at a time, are slower (16 x 700 x 1301 bf16 37 us for 28).
    constexpr bool AHEAD = CENTER && NV == 1;
    const int apart = a.blocks * GROUPS;
    int half = 0;
    Row now, next;
    if (AHEAD && b * GROUPS + group < count) fetch(next, b * GROUPS + group);
    for (int t = b * GROUPS + group; t < count; t += apart, half ^= WAVES) {
        if (AHEAD) {
            now = next;
            if (t + apart < count) fetch(next, t + apart);
        } else {
            fetch(now, t);
        }
        const float rstd = now.rstd, center = now.center;
        // What lies behind the row is multiplied by zeros of dy and g, so -center rstd has to be finite.  Where it is not, the row's elements are one value, its mean (two neighbouring floats
        // among them would leave an rstd below 2^32 / |center|): they are 0 with any rstd.
        const float rstd_h = CENTER && __builtin_fabsf(center) * rstd > 0x1p127f ? 0.f : rstd;
        const auto &dy = now.dy, &sum = now.sum, &res = now.res;
        float dot = 0.f, total = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const Eight y = dy[k].get();
            Eight h = sum[k].get();
            if constexpr (CENTER) {
                h.a = (h.a - center) * rstd_h;
                h.b = (h.b - center) * rstd_h;
                db[k].a += y.a;
                db[k].b += y.b;
            } else {
                h.a *= rstd;
                h.b *= rstd;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = y.a[i] * h.a[i], q = y.b[i] * h.b[i];
                dot += p * g[k].a[i] + q * g[k].b[i];
                if constexpr (CENTER) total += y.a[i] * g[k].a[i] + y.b[i] * g[k].b[i];
                dg[k].a[i] += p;
                dg[k].b[i] += q;
            }
        }
        float mean;
        f32x2 means = {0.f, 0.f};
        if constexpr (CENTER) {
            means = row_sum2<LANES>(f32x2{total, dot}, lds2 + half) / (float)a.cols;
            mean = means[1];
        } else {
            mean = row_sum<LANES>(dot, lds + half) / (float)a.cols;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * 8, have = a.cols - c;
            if (have <= 0) continue;
            const Eight y = dy[k].get(), v = sum[k].get(), r = res[k].get();
            Eight ds;
            if constexpr (CENTER)
                ds = {(g[k].a * y.a - means[0] - (v.a - center) * rstd_h * mean) * rstd + r.a, (g[k].b * y.b - means[0] - (v.b - center) * rstd_h * mean) * rstd + r.b};
            else
                ds = {(g[k].a * y.a - v.a * rstd * mean) * rstd + r.a, (g[k].b * y.b - v.b * rstd * mean) * rstd + r.b};
            store8<ET>((gout)a.out.data + (w * a.out.worker + t * a.out.row + c) * EB, ds, have);
        }
    }
    if (!a.part) return;
    float *const part = a.part + ((int64_t)w * a.blocks + b) * a.cols * (CENTER ? 2 : 1);
    if constexpr (CENTER) {
        if constexpr (GROUPS > 1) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                f32x4 *const at = (f32x4 *)(sums + group * NV * LANES * 8 + (k * LANES + lane) * 8);
                at[0] = db[k].a;
                at[1] = db[k].b;
            }
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += 256) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < GROUPS; ++i) s += sums[i * NV * LANES * 8 + c];
                part[a.cols + c] = s;
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (k * LANES + lane) * 8, have = a.cols - c;
                if (have > 0) store8<kF32>((gout)(part + a.cols + c), db[k], have);
            }
        }
    }
    if constexpr (GROUPS > 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            f32x4 *const at = (f32x4 *)(sums + group * NV * LANES * 8 + (k * LANES + lane) * 8);
            at[0] = dg[k].a;
            at[1] = dg[k].b;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += 256) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) s += sums[i * NV * LANES * 8 + c];
            part[c] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c = (k * LANES + lane) * 8, have = a.cols - c;
            if (have > 0) store8<kF32>((gout)(part + c), dg[k], have);
        }
    }
}

// 32 columns per work-group, eight lanes to each: the parts of 8 x 2048 columns from 224 work-groups in 7 us, one lane to a column 18 us.
// `length` columns to a part: those of the gain's gradient and, where there are more, those of the bias's behind them.
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs a, int length) {
    __shared__ float sums[8][32];
    const int cols = a.b_off >= 0 ? length : a.cols, parts = (cols + 31) / 32;
    const int64_t id = group_of();
    const int w = (int)(id / parts), c = (int)(id - (int64_t)w * parts) * 32 + threadIdx.x % 32, group = threadIdx.x / 32;
    if (w >= a.n) return;
    float s = 0.f;
    if (c < cols) {
        const float *const part = a.part + (int64_t)w * a.blocks * length + c;
#pragma unroll 4
        for (int b = group; b < a.blocks; b += 8) s += part[(int64_t)b * length];
    }
    sums[group][threadIdx.x % 32] = s;
    __syncthreads();
    if (group > 0 || c >= cols) return;
    s = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) s += sums[g][threadIdx.x];
    PG_GLOBAL float *const at = (PG_GLOBAL float *)(a.grads[w] + (c < a.cols ? a.g_off + c : a.b_off + (c - a.cols)));
    *at = a.accumulate ? *at + s : s;
}

// Rows side by side: 4 to 64 lanes (1 << shift) walk along a row, eight elements each.
constexpr int kStore = 0, kLoad = 1, kBack = 2;
template <int ET, int WHAT> __global__ void __launch_bounds__(256) kept_kernel(const KeptArgs a, int shift) {
    constexpr int EB = Elem<ET>::bytes;
    const int64_t id = group_of() * 256 + threadIdx.x, r = id >> shift;
    if (r >= (int64_t)a.n * a.rows) return;
    const int w = (int)(r / a.rows), t = (int)(r - (int64_t)w * a.rows), lanes = 1 << shift;
    if (t >= rows_of(a.counts, w, a.rows)) return;
    const gin x = WHAT == kLoad ? nullptr : (gin)a.x.data + (w * a.x.worker + t * a.x.row) * EB;
    const gout out = WHAT == kStore ? nullptr : (gout)a.out.data + (w * a.out.worker + t * a.out.row) * EB;
    uint8_t *const codes = a.kept.codes + r * a.kept.pitch, *const scales = a.kept.scales + r * (a.kept.pitch / kScaled);
    for (int c = (int)(id & (lanes - 1)) * 8; c < a.kept.pitch; c += lanes * 8) {
        const int have = a.cols - c;
        if constexpr (WHAT == kStore) {
            Eight v = {};
            if (have > 0) v = load8<ET>(x + c * EB, have);
            keep8(v, codes + c, scales + c / kScaled, c % kScaled == 0);
        } else if (have > 0) {
            const u32x2 code = *(const u32x2 *)(codes + c);
            const float scale = scale_of(scales[c / kScaled]);
            Eight v = {decode4(code[0], scale), decode4(code[1], scale)};
            if constexpr (WHAT == kBack) {
                const Eight dy = load8<ET>(x + c * EB, have);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v.a[i] = dy.a[i] * slope_of(a.act, v.a[i]);
                    v.b[i] = dy.b[i] * slope_of(a.act, v.b[i]);
                }
            }
            store8<ET>(out + c * EB, v, have);
        }
    }
}

namespace {

dim3 grid_of(int64_t groups) {
    const int64_t y = (groups + kMostGroups - 1) / kMostGroups;
    return dim3((unsigned)((groups + y - 1) / y), (unsigned)y);
}

// Lanes to a row and their eights, by columns (kMostCols at most): few registers, so that many rows are on their way at once.  Backward, 2048
// columns of bf16: 4 wavefronts with one eight a lane 235 us, one wavefront with four 342 us (8 x 8192 rows).
#define PG_BY_COLS(LAUNCH)                     \
    if (a.cols <= 128) LAUNCH(16, 1);          \
    else if (a.cols <= 256) LAUNCH(32, 1);     \
    else if (a.cols <= 512) LAUNCH(32, 2);     \
    else if (a.cols <= 1024) LAUNCH(64, 2);    \
    else if (a.cols <= 2048) LAUNCH(256, 1);   \
    else if (a.cols <= 4096) LAUNCH(256, 2);   \
    else if (a.cols <= 8192) LAUNCH(1024, 1);  \
    else LAUNCH(1024, 2)
// ... and the rows a work-group takes side by side
int rows_at_once(int cols) { return cols <= 128 ? 16 : (cols <= 512 ? 8 : (cols <= 1024 ? 4 : 1)); }

template <int ET, bool CENTER> void norm_launch(const NormArgs &a, hipStream_t st) {
    const dim3 grid = grid_of(((int64_t)a.n * a.rows + rows_at_once(a.cols) - 1) / rows_at_once(a.cols));
#define PG_NORM(LANES, NV) norm_kernel<ET, LANES, NV, CENTER><<<grid, dim3(LANES < 256 ? 256 : LANES), 0, st>>>(a)
    PG_BY_COLS(PG_NORM);
#undef PG_NORM
}
template <int ET, bool CENTER> void norm_backward_launch(const NormArgs &a, hipStream_t st) {
#define PG_NORM(LANES, NV) norm_backward_kernel<ET, LANES, NV, CENTER><<<dim3((unsigned)a.n * a.blocks), dim3(LANES < 256 ? 256 : LANES), 0, st>>>(a)
    PG_BY_COLS(PG_NORM);
#undef PG_NORM
}
template <int WHAT> void kept_launch(const KeptArgs &a, int type, hipStream_t st) {
    int shift = 2;
    while (shift < 6 && (8 << shift) < a.kept.pitch) ++shift;
    const dim3 grid = grid_of((((int64_t)a.n * a.rows << shift) + 255) / 256);
    if (type == kF32) kept_kernel<kF32, WHAT><<<grid, dim3(256), 0, st>>>(a, shift);
    else kept_kernel<kBf16, WHAT><<<grid, dim3(256), 0, st>>>(a, shift);
}

}  // namespace

// Layer norms: sums for the bias and the next row's loads take registers, so fewer run at the same time.  Of 8 x 4096 x 2048 bf16 768 work-groups 115 us, 1792 122; 4 x 8192 x 650
// floats 1024 82 us, 1792 91, 768 89; 8 x 500 x 16384 floats 256 228 us, 512 241.
int norm_backward_blocks(int n, int rows, int cols, bool center) {
    const int at_once = rows_at_once(cols);
    int most = cols <= 256 || (cols > 1024 && cols <= 2048) ? 1792 : (cols <= 4096 ? 1024 : 512);  // work-groups that run at the same time
    if (center) most = cols <= 1024 ? 1024 : (cols <= 4096 ? 768 : 256);
    return std::max(1, std::min((rows + at_once - 1) / at_once, most / n));
}
void launch_norm(const NormArgs &a, int type, hipStream_t st) { type == kF32 ? norm_launch<kF32, false>(a, st) : norm_launch<kBf16, false>(a, st); }
void launch_layer_norm(const NormArgs &a, int type, hipStream_t st) { type == kF32 ? norm_launch<kF32, true>(a, st) : norm_launch<kBf16, true>(a, st); }
static void join(const NormArgs &a, int length, hipStream_t st) {
    if (!a.part) return;
    const int cols = a.b_off >= 0 ? length : a.cols;
    norm_join_kernel<<<grid_of((int64_t)a.n * ((cols + 31) / 32)), dim3(256), 0, st>>>(a, length);  // a grid's y ends at 65536: fewer than workers may be
}
void launch_norm_backward(const NormArgs &a, int type, hipStream_t st) {
    type == kF32 ? norm_backward_launch<kF32, false>(a, st) : norm_backward_launch<kBf16, false>(a, st);
    join(a, a.cols, st);
}
void launch_layer_norm_backward(const NormArgs &a, int type, hipStream_t st) {
    type == kF32 ? norm_backward_launch<kF32, true>(a, st) : norm_backward_launch<kBf16, true>(a, st);
    join(a, 2 * a.cols, st);
}
void launch_store(const KeptArgs &a, int type, hipStream_t st) { kept_launch<kStore>(a, type, st); }
void launch_load(const KeptArgs &a, int type, hipStream_t st) { kept_launch<kLoad>(a, type, st); }
void launch_activation_backward(const KeptArgs &a, int type, hipStream_t st) { kept_launch<kBack>(a, type, st); }

}  // namespace pg
