// The loss behind the last layer and the gradient of its logits, in one pass: cross entropy against a label, and the divergence from a teacher of which
// the largest logits are known.  Per row, with z the logits, c the label, t_j the teacher's logit of entry i_j, u the temperature:
//     p = softmax_j(t / u),  q = softmax(z / u),  s = softmax(z)
//     loss = w (hard (log sum exp z - z_c) + soft u^2 sum_j p_j (log p_j - log q_i_j))
//     dz_v = w (hard (s_v - [v = c]) + soft u (q_v - sum over j with i_j = v of p_j))
// Bound by memory: a row is read once and its gradient written once, the row waits for its sums in registers (11200 rows of 33278 in bf16, 32 entries: 335 us,
// 4.5 TB/s); rows of more than 65536 are read twice (2048 of 128256: 264 us, 4.0 TB/s of one reading).  Entries cost their square, as each looks for itself among the others: 2048 rows of 33278
// take 58 us without a teacher, 100 with 128 entries, 160 with 256, 996 with 1024, of which bytes are no more than 60 us.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pg_rows.h"

namespace pg {

namespace {

constexpr int kWave = 64;
constexpr float kLog2e = 1.44269504f;

constexpr int64_t kMostGroups = 1 << 20;
__device__ __forceinline__ int64_t group_of() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }
dim3 grid_of(int64_t groups) {
    const int64_t y = (groups + kMostGroups - 1) / kMostGroups;
    return dim3((unsigned)((groups + y - 1) / y), (unsigned)y);
}

struct Entry {
    int at;         // -1: none
    float t, p, z;  // the teacher's logit and its weight, the student's logit
};

template <int LANES> __device__ __forceinline__ float largest(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v = __builtin_fmaxf(v, __shfl_xor(v, d));
    return v;
}
template <int LANES> __device__ __forceinline__ float sum(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// Eight elements at any address of their own type; those behind the row's end are -inf, whose exponential is 0.
template <int ET> struct Raw8 {
    u32x4 w[ET == kF32 ? 2 : 1];
    __device__ __forceinline__ void load(gin p, int have) {
        if (have >= 8) {
            w[0] = at_global<u32x4_any>(p);
            if constexpr (ET == kF32) w[1] = at_global<u32x4_any>(p + 16);
            return;
        }
        constexpr uint32_t none = ET == kF32 ? 0xff800000u : 0xff80ff80u;
        for (auto &v : w) v = u32x4{none, none, none, none};
#pragma unroll
        for (int i = 0; i < 7; ++i) {
            if (i >= have) continue;
            if constexpr (ET == kF32) {
                w[i / 4][i % 4] = at_global<uint32_t>(p + 4 * i);
            } else {
                const uint32_t one = at_global<uint16_t>(p + 2 * i);
                w[0][i / 2] = i % 2 ? (w[0][i / 2] & 0xffffu) | one << 16 : (w[0][i / 2] & 0xffff0000u) | one;
            }
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (ET == kF32) return __uint_as_float(w[i / 4][i % 4]);
        else return i % 2 ? bf16_high(w[0][i / 2]) : bf16_low(w[0][i / 2]);
    }
};
template <int ET> __device__ __forceinline__ void put8(gout p, const float (&v)[8], int have) {
    store4<ET>(p, f32x4{v[0], v[1], v[2], v[3]}, have);
    if (have > 4) store4<ET>(p + 4 * Elem<ET>::bytes, f32x4{v[4], v[5], v[6], v[7]}, have - 4);
}
template <> __device__ __forceinline__ void put8<kBf16>(gout p, const float (&v)[8], int have) {
    if (have >= 8) {
        to_global<u32x4_any>(p, u32x4{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3]), bf16_pack(v[4], v[5]), bf16_pack(v[6], v[7])});
        return;
    }
    store4<kBf16>(p, f32x4{v[0], v[1], v[2], v[3]}, have);
    if (have > 4) store4<kBf16>(p + 8, f32x4{v[4], v[5], v[6], v[7]}, have - 4);
}

// e^x - 1 - x: below 1/2, where that difference loses digits, its series, off by less than x^9 / 9! or 2^-26 of it.
__device__ __forceinline__ float above_tangent(float x) {
    if (__builtin_fabsf(x) >= 0.5f) return expm1f(x) - x;
    return x * x * (1.f / 2 + x * (1.f / 6 + x * (1.f / 24 + x * (1.f / 120 + x * (1.f / 720 + x * (1.f / 5040 + x * (1.f / 40320)))))));
}

// Largest value and, relative to it, the sums of both exponentials.
struct Stats {
    float top, one, two;
};

}  // namespace

// A row per LANES lanes.  NV > 0: NV times eight of its elements in each lane's registers, read once; NV = 0: rows of any length, read twice, with running
// maximum and sums the first time.  BOTH: two temperatures, 1 for the label and that of the teacher; else the one that is asked for.
template <int ET, int LANES, int NV, bool BOTH>
__global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) distill_kernel(const DistillArgs a) {
    constexpr int EB = Elem<ET>::bytes, ROWS = LANES < 256 ? 256 / LANES : 1, WAVES = LANES / kWave, GROUP = LANES < kWave ? LANES : kWave;
    extern __shared__ Entry entries[];
    __shared__ Stats stats[WAVES > 1 ? WAVES : 1];
    __shared__ float shares[1];
    const int64_t r = group_of() * ROWS + threadIdx.x / LANES;
    const int lane = threadIdx.x % LANES;
    const bool in = r < (int64_t)a.n * a.rows;
    const int w = in ? (int)(r / a.rows) : 0, t = in ? (int)(r - (int64_t)w * a.rows) : 0;
    const bool there = in && t < rows_of(a.counts, w, a.rows);
    const float kt = kLog2e / a.temperature;
    const float weight = there ? (a.weights ? a.weights[r] : 1.f) : 0.f;
    int label = there && a.labels ? a.labels[r] : -1;
    if ((unsigned)label >= (unsigned)a.cols) label = -1;
    const float hard = label >= 0 ? weight * a.hard : 0.f;
    bool live = weight != 0.f && (label >= 0 || a.top > 0);
    const gin z = (gin)a.z.data + (w * a.z.worker + t * a.z.row) * EB;
    const gout dz = a.dz.data ? (gout)a.dz.data + (w * a.dz.worker + t * a.dz.row) * EB : nullptr;
    // x -> 2^x of the distance to the largest logit; with one temperature it is that of whichever part there is
    const float k1 = BOTH || a.top == 0 ? kLog2e : kt, k2 = kt;
    Entry *const mine = entries + (threadIdx.x / LANES) * (a.top + 1);  // the last one is the label

    Raw8<ET> x[NV > 0 ? NV : 1];
    if constexpr (NV > 0) {
        if (live)
#pragma unroll
            for (int k = 0; k < NV; ++k) x[k].load(z + (k * LANES + lane) * 8 * EB, a.cols - (k * LANES + lane) * 8);
    }
    // The entries, by the group's first wavefront.
    float top_t = -__builtin_inff(), sum_p = 0.f;
    if (live && lane < GROUP) {
        for (int j = lane; j <= a.top; j += GROUP) {
            const int64_t e = r * a.top + j;
            int at = j < a.top ? a.top_index[e] : label;
            if ((unsigned)at >= (unsigned)a.cols) at = -1;
            float logit = -__builtin_inff();
            if (at >= 0 && j < a.top) {
                logit = a.top_logits[e];
                if (logit == -__builtin_inff()) at = -1;
            }
            float student = 0.f;
            if (at >= 0) {
                if constexpr (ET == kF32) student = at_global<float>(z + at * 4);
                else student = bf16_low(at_global<uint16_t>(z + at * 2));
            }
            mine[j] = Entry{at, logit, 0.f, student};
            top_t = __builtin_fmaxf(top_t, logit);  // drops a NaN, which comes back with the sum
        }
        top_t = largest<GROUP>(top_t);
    }
    // Whether the row's entries are all classes, each once: every entry marks its class, in a place of its own.
    constexpr bool ALL = NV > 0 && (LANES * NV <= kMostTop / 8 || LANES * NV == 256);   // lanes of rows that short
    bool all = false;
    if (ALL && a.top == a.cols && a.temperature > 1.f) {
        __syncthreads();
        if (live && lane < GROUP)
            for (int j = lane; j < a.top; j += GROUP)
                if (mine[j].at >= 0) mine[mine[j].at].p = __int_as_float(j);
        __syncthreads();
        if (live && lane < GROUP) {
            float missed = 0.f;
            for (int j = lane; j < a.top; j += GROUP)
                if (mine[j].at < 0 || __float_as_int(mine[mine[j].at].p) != j) missed = 1.f;
            all = sum<GROUP>(missed) == 0.f;
        }
        __syncthreads();
    }
    bool taught = false;
    if (live && lane < GROUP) {
        for (int j = lane; j < a.top; j += GROUP) {
            if (mine[j].at < 0) continue;
            taught = true;
            mine[j].p = __builtin_amdgcn_exp2f((mine[j].t - top_t) * kt);
            sum_p += mine[j].p;
        }
        sum_p = sum<GROUP>(sum_p);
        taught = sum<GROUP>(taught ? 1.f : 0.f) > 0.f;
        if (WAVES > 1 && lane == 0) shares[0] = taught ? 1.f : 0.f;
    }

    // largest logit and sums
    Stats s = {-__builtin_inff(), 0.f, 0.f};
    if (live) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((k * LANES + lane) * 8 < a.cols) s.top = __builtin_fmaxf(s.top, x[k].get(i));
        } else {
            constexpr int AHEAD = 4;  // eights on their way at once
            for (int c = lane * 8; c < a.cols; c += AHEAD * LANES * 8) {
                Raw8<ET> y[AHEAD];
                float top = s.top;
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) y[k].load(z + (int64_t)(c + k * LANES * 8) * EB, a.cols - c - k * LANES * 8);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = __builtin_fmaxf(top, y[k].get(i));
                if (top > s.top) {
                    s.one *= __builtin_amdgcn_exp2f((s.top - top) * k1);
                    if constexpr (BOTH) s.two *= __builtin_amdgcn_exp2f((s.top - top) * k2);
                    s.top = top;
                }
                const float from = s.top == -__builtin_inff() ? 0.f : s.top;
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float d = y[k].get(i) - from;
                        s.one += __builtin_amdgcn_exp2f(d * k1);
                        if constexpr (BOTH) s.two += __builtin_amdgcn_exp2f(d * k2);
                    }
            }
        }
    }
    float top = largest<GROUP>(s.top);
    if constexpr (WAVES > 1) {
        if (lane % kWave == 0) stats[lane / kWave].top = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = __builtin_fmaxf(top, stats[i].top);
        taught = live && shares[0] != 0.f;
    } else {
        __syncthreads();  // the entries
    }
    if (live) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if ((k * LANES + lane) * 8 >= a.cols) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = x[k].get(i) - top;
                    s.one += __builtin_amdgcn_exp2f(d * k1);
                    if constexpr (BOTH) s.two += __builtin_amdgcn_exp2f(d * k2);
                }
            }
        } else {
            const float k = s.top == -__builtin_inff() ? 0.f : 1.f;
            s.one *= k * __builtin_amdgcn_exp2f(k != 0.f ? (s.top - top) * k1 : 0.f);
            if constexpr (BOTH) s.two *= k * __builtin_amdgcn_exp2f(k != 0.f ? (s.top - top) * k2 : 0.f);
        }
    }
    s.one = sum<GROUP>(s.one);
    if constexpr (BOTH) s.two = sum<GROUP>(s.two);
    if constexpr (WAVES > 1) {
        __syncthreads();
        if (lane % kWave == 0) stats[lane / kWave] = s;
        __syncthreads();
        s.one = s.two = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            s.one += stats[i].one;
            s.two += stats[i].two;
        }
    }
    const float sum2 = BOTH ? s.two : s.one;
    live = live && (label >= 0 || taught);
    // What an exponential counts in the gradient.
    const float soft = taught ? weight * a.soft * a.temperature : 0.f;
    float c1 = 0.f, c2 = 0.f;
    if (label >= 0 && hard != 0.f) c1 = hard / s.one;
    if (taught && soft != 0.f) c2 = soft / sum2;
    if (!BOTH) c1 += c2;
    // The logarithms of p and q at a high temperature u are alike, and the loss is what u^2 makes of their difference.  Where entries are all classes, it needs no difference: with d_j the distance
    // of the student's logits from the teacher's, over u, and m = sum p d, sum q = 1 makes the divergence log sum p e^(d - m) = log(1 + sum p (e^x - 1 - x)), x = d - m, of terms that are all positive, and q_j - p_j =
    // p_j (e^(x_j - divergence) - 1).  (Ten classes, u = 2^20: the loss was off by 9 x 10^4 times itself, at u = 30 by 1 part in 10^4.)  Weights p that round to 0 have no d; their q counts as it is.
    float apart_mean = 0.f, divergence = 0.f;
    const auto apart = [&](const Entry &e) { return ((e.z - top) - (e.t - top_t)) / a.temperature; };
    if (ALL && all) {
        for (int j = lane; j < a.top; j += GROUP)
            if (mine[j].p != 0.f) apart_mean += mine[j].p * apart(mine[j]);
        apart_mean = sum<GROUP>(apart_mean) / sum_p;
        float far = 0.f, more = 0.f, rest = 0.f;
        for (int j = lane; j < a.top; j += GROUP) {
            const Entry e = mine[j];
            if (e.p == 0.f) {
                rest += __builtin_amdgcn_exp2f((e.z - top) * k2);
                continue;
            }
            const float x = apart(e) - apart_mean;
            far = __builtin_fmaxf(far, __builtin_fabsf(x));
            more += e.p * above_tangent(x);
        }
        all = largest<GROUP>(far) <= 64.f && __builtin_fabsf(apart_mean) <= 64.f;   // else, and where something is not finite, the difference is none of near values
        divergence = log1pf((sum<GROUP>(more) + sum<GROUP>(rest) * __builtin_amdgcn_exp2f(-apart_mean * kLog2e)) / sum_p);
    }
    auto slope = [&](float logit) {
        const float d = logit - top;
        float g = c1 * __builtin_amdgcn_exp2f(d * k1);
        if constexpr (BOTH) g += c2 * __builtin_amdgcn_exp2f(d * k2);
        return g;
    };
    if (there && lane < GROUP && a.loss) {
        float loss = 0.f;
        if (live) {
            const float log_p = logf(sum_p), log_q = logf(sum2);
            float kl = 0.f;
            if (taught) {
                for (int j = lane; j < a.top; j += GROUP) {
                    const Entry e = mine[j];
                    // a weight that rounds to 0 counts as 0, whatever its logarithm
                    if (e.at >= 0 && e.p != 0.f) kl += e.p / sum_p * ((e.t - top_t) / a.temperature - log_p - ((e.z - top) / a.temperature - log_q));
                }
                kl = ALL && all ? divergence : sum<GROUP>(kl);
                loss += weight * a.soft * a.temperature * a.temperature * kl;
            }
            if (label >= 0) loss += hard * (logf(s.one) - (mine[a.top].z - top));
        }
        if (lane == 0) a.loss[r] = loss;
    }
    if (!a.dz.data) return;
    if (there) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int c = (k * LANES + lane) * 8;
                if (c >= a.cols) continue;
                float g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) g[i] = live ? slope(x[k].get(i)) : 0.f;
                put8<ET>(dz + c * EB, g, a.cols - c);
            }
        } else {
            for (int c = lane * 8; c < a.cols; c += LANES * 8) {
                float g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (live) {
                    x[0].load(z + (int64_t)c * EB, a.cols - c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = slope(x[0].get(i));
                }
                put8<ET>(dz + (int64_t)c * EB, g, a.cols - c);
            }
        }
    }
    // The label and the entries once more, each element from all that is known of it: an index that comes twice is written twice, with the same value.
    __syncthreads();
    if (!live || lane >= GROUP) return;
    for (int j = lane; j <= a.top; j += GROUP) {
        const Entry e = mine[j];
        if (e.at < 0) continue;
        if (ALL && all && j == a.top) continue;   // one of the entries
        if (ALL && all && e.p != 0.f) {
            float g = soft * (e.p / sum_p) * expm1f(apart(e) - apart_mean - divergence);
            if constexpr (BOTH) g += c1 * __builtin_amdgcn_exp2f((e.z - top) * k1);
            if (e.at == label) g -= hard;
            if constexpr (ET == kF32) to_global<float>(dz + e.at * 4, g);
            else to_global<uint16_t>(dz + e.at * 2, bf16_bits(g));
            continue;
        }
        float p = 0.f;
        if (soft != 0.f)
            for (int i = 0; i < a.top; ++i)
                if (mine[i].at == e.at) p += mine[i].p;
        float g = slope(e.z);
        if (soft != 0.f) g -= soft * (p / sum_p);
        if (e.at == label) g -= hard;
        if constexpr (ET == kF32) to_global<float>(dz + e.at * 4, g);
        else to_global<uint16_t>(dz + e.at * 2, bf16_bits(g));
    }
}

namespace {

template <int ET, bool BOTH> void distill_launch(const DistillArgs &a, hipStream_t st) {
    const int64_t rows = (int64_t)a.n * a.rows;
    const size_t lds = sizeof(Entry) * (a.top + 1);
#define PG_DISTILL(LANES, NV)                                                                                                   \
    distill_kernel<ET, LANES, NV, BOTH><<<grid_of((rows + (LANES < 256 ? 256 / LANES : 1) - 1) / (LANES < 256 ? 256 / LANES : 1)), \
                                          dim3(LANES < 256 ? 256 : LANES), lds * (LANES < 256 ? 256 / LANES : 1), st>>>(a)
    // Few lanes to a row, so that several work-groups of a compute unit are at different places of theirs: 11200 rows of 33278 in bf16 take 459 us with 1024 lanes
    // a row, 370 with 512, 353 with 256; 65536 of 2048 259 with 256, 158 with 64.  Rows that are few are a matter of latency (4 of 33278: 14 us with 1024 lanes, 18
    // with 256), and so go those of a teacher whose entries would fill LDS.
    const bool few = rows <= 512 || (a.top > 256 && a.cols <= 4096);
    if (a.cols <= 128) PG_DISTILL(16, 1);
    else if (a.cols <= 512) PG_DISTILL(64, 1);
    else if (few && a.cols <= 2048) PG_DISTILL(256, 1);
    else if (few && a.cols <= 8192) PG_DISTILL(1024, 1);
    else if (few && a.cols <= 16384) PG_DISTILL(1024, 2);
    else if (few && a.cols <= 40960) PG_DISTILL(1024, 5);
    else if (a.cols <= 1024) PG_DISTILL(64, 2);
    else if (a.cols <= 2048) PG_DISTILL(64, 4);
    else if (a.cols <= 4096) PG_DISTILL(64, 8);
    else if (a.cols <= 8192) PG_DISTILL(256, 4);
    else if (a.cols <= 16384) PG_DISTILL(256, 8);
    else if (a.cols <= 24576) PG_DISTILL(256, 12);
    else if (a.cols <= 40960) {
        if constexpr (ET == kF32) {
            PG_DISTILL(512, 10);
        } else {
            if (a.cols <= 32768) PG_DISTILL(256, 16);
            else if (a.cols <= 36864) PG_DISTILL(256, 18);
            else PG_DISTILL(256, 20);
        }
    } else if (a.cols <= 65536) PG_DISTILL(1024, 8);
    else PG_DISTILL(1024, 0);
#undef PG_DISTILL
}

}  // namespace

void launch_distill(const DistillArgs &a, int type, hipStream_t st) {
    const bool both = a.labels && a.top > 0 && a.temperature != 1.f;
    if (type == kF32) both ? distill_launch<kF32, true>(a, st) : distill_launch<kF32, false>(a, st);
    else both ? distill_launch<kBf16, true>(a, st) : distill_launch<kBf16, false>(a, st);
}

}  // namespace pg
