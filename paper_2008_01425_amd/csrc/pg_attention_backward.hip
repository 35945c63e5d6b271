// Gradients of attention, without the scores of the way there: they are formed again from queries and keys, and their weights from the sums that were kept.
//     P = exp(scale q k^T - lse),  dS = P (dy v^T - dy . y),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dy
// Two kernels, one that owns queries and one that owns states: each writes its own rows once and in a fixed order of sums, at the price of forming S and dy v^T twice (7
// products for the 5 that one kernel with atomic additions would take).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pg_attention.h"

namespace pg {

namespace {

template <int ET> __device__ __forceinline__ float dot(const Frag<ET> &a, const Frag<ET> &b, float sum) {
    if constexpr (ET == kF32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += a[j] * b[j];
    } else {
        const u32x4 x = __builtin_bit_cast(u32x4, a), y = __builtin_bit_cast(u32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += bf16_low(x[j]) * bf16_low(y[j]) + bf16_high(x[j]) * bf16_high(y[j]);
    }
    return sum;
}

}  // namespace

// dy . y of every position and head, a wavefront each; attention_dq_kernel leaves the same where it runs.
template <int ET> __global__ void __launch_bounds__(256) attention_delta_kernel(const AttentionArgs a) {
    constexpr int EB = Elem<ET>::bytes;
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64;
    if (at >= (int64_t)a.n * a.sequences * a.rows * a.heads) return;
    const int lane = threadIdx.x % 64, head = (int)(at % a.heads);
    const int64_t row = at / a.heads, where = row / a.rows;
    const int t = (int)(row - where * a.rows);
    if (t >= length_of(a.counts, where, a.rows)) return;
    const int64_t place = (where % a.sequences) * a.rows + t;
    const gin dy = (gin)a.dy.data + ((where / a.sequences) * a.dy.worker + place * a.dy.row + head * a.width) * EB;
    const gin y = (gin)a.y.data + ((where / a.sequences) * a.y.worker + place * a.y.row + head * a.width) * EB;
    float sum = 0.f;
    for (int c = lane; c < a.width; c += 64) {
        if constexpr (ET == kF32) sum += at_global<float>(dy + c * 4) * at_global<float>(y + c * 4);
        else sum += bf16_low(at_global<uint16_t>(dy + c * 2)) * bf16_low(at_global<uint16_t>(y + c * 2));
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) a.delta[at] = sum;
}

template <int ET, int DP, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) attention_dq_kernel(const AttentionArgs a) {
    typedef Tile<ET, DP> T;
    constexpr int KT = WAVES == 1 ? 32 : tile_rows<ET, DP>(), THREADS = 64 * WAVES, SIZE = KT * T::PITCH;
    __shared__ __attribute__((aligned(16))) char lds[4 * SIZE];
    const Work k = work_of(a);
    if (!k.any) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 32, h = lane / 32;
    const int asked = length_of(a.counts, k.where, a.rows) * a.group, count = length_of(a.memory_counts, k.where, a.memory);
    if (k.tile * (32 * WAVES) >= asked) return;
    const int u = k.tile * (32 * WAVES) + wave * 32 + i, t = u / a.group, head = k.head * a.group + u % a.group;
    const bool there = u < asked;
    const int64_t at = (k.where * a.rows + t) * a.heads + head;
    Frag<ET> q[T::NK], dy[T::NK];
    float delta = 0.f, from = 0.f;
    {
        Frag<ET> y[T::NK];
        own_rows<ET, DP>(dy, sequence_of(a.dy, k, a.rows, T::EB) + ((int64_t)t * a.dy.row + head * a.width) * T::EB, there, a.width, h);
        own_rows<ET, DP>(y, sequence_of(a.y, k, a.rows, T::EB) + ((int64_t)t * a.y.row + head * a.width) * T::EB, there, a.width, h);
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) delta = dot<ET>(dy[kk], y[kk], delta);
        delta = across_halves_sum(delta);
    }
    if (there) {
        from = a.lse[at] * kLog2e;
        if (from == -__builtin_inff()) from = 0.f;   // nothing seen: every weight below is 2^-inf
        if (a.delta && k.split == 0 && h == 0) a.delta[at] = delta;
    }
    own_rows<ET, DP>(q, sequence_of(a.q, k, a.rows, T::EB) + ((int64_t)t * a.q.row + head * a.width) * T::EB, there, a.width, h);
    const gin keys = sequence_of(a.k, k, a.memory, T::EB) + k.head * a.width * T::EB, values = sequence_of(a.v, k, a.memory, T::EB) + k.head * a.width * T::EB;
    const float c = a.scale * kLog2e;
    f32x16 out[T::NB];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) out[nb] = zero16();

    int tile, last;
    share_of(count, KT, k.split, a.splits, tile, last);
    Staged<ET, DP, KT, THREADS> next_k, next_v;
    auto fetch = [&](int at) {
        const gin kb = keys + (int64_t)at * KT * a.k.row * T::EB, vb = values + (int64_t)at * KT * a.v.row * T::EB;
        const int have = count - at * KT;
        next_k.load(threadIdx.x, have, a.width, [&](int row) { return kb + (int64_t)row * a.k.row * T::EB; });
        next_v.load(threadIdx.x, have, a.width, [&](int row) { return vb + (int64_t)row * a.v.row * T::EB; });
    };
    if (tile < last) fetch(tile);
    for (int buffer = 0; tile < last; ++tile, buffer ^= 1) {
        char *const tk = lds + buffer * 2 * SIZE, *const tv = tk + SIZE;
        const uint64_t seen = seen_of<KT>(a, k.where, tile * KT, count);
        next_k.store(tk, threadIdx.x, seen);
        next_v.store(tv, threadIdx.x, seen);
        __syncthreads();
        if (tile + 1 < last) fetch(tile + 1);
#pragma unroll
        for (int b = 0; b < KT / 32; ++b) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int kk = 0; kk < T::NK; ++kk) {
                s = mul<ET>(T::along(tk, b * 32 + i, kk, h), q[kk], s);
                dp = mul<ET>(T::along(tv, b * 32 + i, kk, h), dy[kk], dp);
            }
            if (seen != all_rows<KT>()) {
                const uint32_t bits = (uint32_t)(seen >> (b * 32)) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(bits >> (8 * (r / 4) + r % 4) & 1)) s[r] = -__builtin_inff();
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -from)) * (dp[r] - delta);
#pragma unroll
            for (int step = 0; step < T::STEPS; ++step) {
                const Frag<ET> ds = T::of(s, step);
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) out[nb] = mul<ET>(T::across(tk, b * 32 + step * T::STEP, nb, lane), ds, out[nb]);
            }
        }
    }
    if (!there) return;
    if (a.splits > 1) {
        const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads;
        put_rows<kF32>((gout)(a.part + (k.split * rows + at) * a.width), out, a.scale, a.width, h);
    } else {
        put_rows<ET>((gout)sequence_of(a.dq, k, a.rows, T::EB) + ((int64_t)t * a.dq.row + head * a.width) * T::EB, out, a.scale, a.width, h);
    }
}

// A wavefront owns 32 states and walks along the rows of all queries that share the key head, whose gradients add up in its registers in that order.
// Queries that do not exist have a weight of 2^-inf.  WHAT: 1 dv, 2 dk, 3 both in one.
template <int ET, int DP, int WHAT>
__global__ void __launch_bounds__(256) attention_dkv_kernel(const AttentionArgs a) {
    typedef Tile<ET, DP> T;
    constexpr int KT = tile_rows<ET, DP>(), SIZE = KT * T::PITCH;
    constexpr bool DK = WHAT & 2, DV = WHAT & 1;
    __shared__ __attribute__((aligned(16))) char lds[4 * SIZE];
    __shared__ __attribute__((aligned(16))) float stats[2][2][KT];
    const Work k = work_of(a);
    if (!k.any) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 32, h = lane / 32;
    const int asked = length_of(a.counts, k.where, a.rows) * a.group, count = length_of(a.memory_counts, k.where, a.memory);
    if (k.tile * 128 >= count) return;
    const int own = k.tile * 128 + wave * 32 + i;
    const bool there = own < count, seen = there && (!a.mask || a.mask[k.where * a.memory + own] != 0);
    Frag<ET> key[T::NK], value[DK ? T::NK : 1];
    own_rows<ET, DP>(key, sequence_of(a.k, k, a.memory, T::EB) + ((int64_t)own * a.k.row + k.head * a.width) * T::EB, seen, a.width, h);
    if constexpr (DK) own_rows<ET, DP>(value, sequence_of(a.v, k, a.memory, T::EB) + ((int64_t)own * a.v.row + k.head * a.width) * T::EB, seen, a.width, h);
    const float c = a.scale * kLog2e;
    f32x16 dk[DK ? T::NB : 1], dv[DV ? T::NB : 1];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) {
        if constexpr (DK) dk[nb] = zero16();
        if constexpr (DV) dv[nb] = zero16();
    }

    int tile, last;
    share_of(asked, KT, k.split, a.splits, tile, last);
    Staged<ET, DP, KT, 256> next_q, next_dy;
    float next_from = 0.f, next_delta = 0.f;
    const gin queries = sequence_of(a.q, k, a.rows, T::EB) + (int64_t)k.head * a.group * a.width * T::EB,
              dys = sequence_of(a.dy, k, a.rows, T::EB) + (int64_t)k.head * a.group * a.width * T::EB;
    auto fetch = [&](int at) {
        const int first = at * KT, have = asked - first;
        next_q.load(threadIdx.x, have, a.width, [&](int row) {
            const int u = first + row, t = u / a.group;
            return queries + ((int64_t)t * a.q.row + (u - t * a.group) * a.width) * T::EB;
        });
        next_dy.load(threadIdx.x, have, a.width, [&](int row) {
            const int u = first + row, t = u / a.group;
            return dys + ((int64_t)t * a.dy.row + (u - t * a.group) * a.width) * T::EB;
        });
        if (threadIdx.x < KT) {
            next_from = __builtin_inff();
            next_delta = 0.f;
            if ((int)threadIdx.x < have) {
                const int u = first + threadIdx.x, t = u / a.group;
                const int64_t at = (k.where * a.rows + t) * a.heads + k.head * a.group + (u - t * a.group);
                next_from = a.lse[at] * kLog2e;
                if (next_from == -__builtin_inff()) next_from = __builtin_inff();   // saw nothing
                next_delta = a.delta[at];
            }
        }
    };
    if (tile < last) fetch(tile);
    for (int buffer = 0; tile < last; ++tile, buffer ^= 1) {
        char *const tq = lds + buffer * 2 * SIZE, *const td = tq + SIZE;
        next_q.store(tq, threadIdx.x, ~0ull);
        next_dy.store(td, threadIdx.x, ~0ull);
        if (threadIdx.x < KT) {
            stats[buffer][0][threadIdx.x] = next_from;
            stats[buffer][1][threadIdx.x] = next_delta;
        }
        __syncthreads();
        if (tile + 1 < last) fetch(tile + 1);
#pragma unroll
        for (int b = 0; b < KT / 32; ++b) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int kk = 0; kk < T::NK; ++kk) {
                s = mul<ET>(T::along(tq, b * 32 + i, kk, h), key[kk], s);
                if constexpr (DK) dp = mul<ET>(T::along(td, b * 32 + i, kk, h), value[kk], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const f32x4 from = *(const f32x4 *)&stats[buffer][0][b * 32 + 2 * r + 4 * h], delta = *(const f32x4 *)&stats[buffer][1][b * 32 + 2 * r + 4 * h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[r + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + j], c, -from[j]));
                    if constexpr (DK) dp[r + j] = s[r + j] * (dp[r + j] - delta[j]);
                }
            }
#pragma unroll
            for (int step = 0; step < T::STEPS; ++step) {
                if constexpr (DV) {
                    const Frag<ET> p = T::of(s, step);
#pragma unroll
                    for (int nb = 0; nb < T::NB; ++nb) dv[nb] = mul<ET>(T::across(td, b * 32 + step * T::STEP, nb, lane), p, dv[nb]);
                }
                if constexpr (DK) {
                    const Frag<ET> ds = T::of(dp, step);
#pragma unroll
                    for (int nb = 0; nb < T::NB; ++nb) dk[nb] = mul<ET>(T::across(tq, b * 32 + step * T::STEP, nb, lane), ds, dk[nb]);
                }
            }
        }
    }
    if (!there) return;
    if (!seen) {  // nothing reads it, whatever it holds
#pragma unroll
        for (int nb = 0; nb < T::NB; ++nb) {
            if constexpr (DK) dk[nb] = zero16();
            if constexpr (DV) dv[nb] = zero16();
        }
    }
    if (a.splits > 1) {
        const int64_t rows = (int64_t)a.n * a.sequences * a.memory * a.kv_heads, at = (k.where * a.memory + own) * a.kv_heads + k.head;
        if constexpr (DK) put_rows<kF32>((gout)(a.part + (k.split * rows + at) * a.width), dk, a.scale, a.width, h);
        if constexpr (DV) put_rows<kF32>((gout)(a.part + ((a.splits + k.split) * rows + at) * a.width), dv, 1.f, a.width, h);
    } else {
        if constexpr (DK) put_rows<ET>((gout)sequence_of(a.dk, k, a.memory, T::EB) + ((int64_t)own * a.dk.row + k.head * a.width) * T::EB, dk, a.scale, a.width, h);
        if constexpr (DV) put_rows<ET>((gout)sequence_of(a.dv, k, a.memory, T::EB) + ((int64_t)own * a.dv.row + k.head * a.width) * T::EB, dv, 1.f, a.width, h);
    }
}

// Sums of parts, a wavefront to a row and head, always in the same order; z: dk and dv.
template <int ET> __global__ void __launch_bounds__(256) attention_sum_kernel(const AttentionArgs a, RowsArg first, RowsArg second, int length, int heads, const int32_t *counts) {
    const int64_t rows = (int64_t)a.n * a.sequences * length * heads, at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64;
    if (at >= rows) return;
    const int lane = threadIdx.x % 64, head = (int)(at % heads);
    const int64_t row = at / heads, where = row / length;
    const int t = (int)(row - where * length);
    if (t >= length_of(counts, where, length)) return;
    const RowsArg r = blockIdx.z ? second : first;
    const float *const part = a.part + (blockIdx.z * a.splits * rows + at) * a.width;
    const gout out = (gout)r.data + ((where / a.sequences) * r.worker + ((where % a.sequences) * length + t) * r.row + head * a.width) * Elem<ET>::bytes;
    for (int col = lane; col < a.width; col += 64) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v += part[s * rows * a.width + col];
        if constexpr (ET == kF32) to_global<float>(out + col * 4, v);
        else to_global<uint16_t>(out + col * 2, bf16_bits(v));
    }
}

namespace {

struct Cut {
    int waves, tiles, splits;
};
Cut cut_of(const AttentionArgs &a, int64_t own, int64_t other, bool one_wave) {
    const int64_t problems = (int64_t)a.n * a.sequences * a.kv_heads;
    const int waves = one_wave ? 1 : 4;
    const int64_t tiles = (own + 32 * waves - 1) / (32 * waves), groups = problems * tiles, wanted = waves == 1 ? 2048 : 512;
    const int64_t splits = std::max<int64_t>(1, std::min({wanted / std::max<int64_t>(groups, 1), (other + 63) / 64 / 2, (int64_t)64}));
    return Cut{waves, (int)tiles, (int)splits};
}
Cut dq_cut(const AttentionArgs &a, int type) {
    const int64_t asked = (int64_t)a.rows * a.group;
    return cut_of(a, asked, a.memory, asked <= 32 && a.width <= 128 && type == kBf16);
}
Cut dkv_cut(const AttentionArgs &a) { return cut_of(a, a.memory, (int64_t)a.rows * a.group, false); }

template <int ET, int DP, int WAVES> void launch_dq(const AttentionArgs &a, hipStream_t st) {
    attention_dq_kernel<ET, DP, WAVES><<<attention_grid(a), dim3(64 * WAVES), 0, st>>>(a);
}
template <int ET, int DP> void launch_dkv(const AttentionArgs &a, hipStream_t st) {
    if constexpr (DP * Elem<ET>::bytes > 768) {  // both gradients and the own rows of the widest heads in float are more than the registers
        attention_dkv_kernel<ET, DP, 1><<<attention_grid(a), dim3(256), 0, st>>>(a);
        attention_dkv_kernel<ET, DP, 2><<<attention_grid(a), dim3(256), 0, st>>>(a);
    } else {
        attention_dkv_kernel<ET, DP, 3><<<attention_grid(a), dim3(256), 0, st>>>(a);
    }
}
#define PG_BY_WIDTH(LAUNCH)             \
    if (a.width <= 32) LAUNCH(32);      \
    else if (a.width <= 64) LAUNCH(64); \
    else if (a.width <= 96) LAUNCH(96); \
    else if (a.width <= 128) LAUNCH(128); \
    else if (a.width <= 192) LAUNCH(192); \
    else LAUNCH(256)
template <int ET> void dq_by_width(const AttentionArgs &a, int waves, hipStream_t st) {
    if constexpr (ET == kBf16) {
        if (waves == 1) {
            if (a.width <= 64) launch_dq<ET, 64, 1>(a, st);
            else launch_dq<ET, 128, 1>(a, st);
            return;
        }
    }
#define PG_DQ(DP) launch_dq<ET, DP, 4>(a, st)
    PG_BY_WIDTH(PG_DQ);
#undef PG_DQ
}
template <int ET> void dkv_by_width(const AttentionArgs &a, hipStream_t st) {
#define PG_DKV(DP) launch_dkv<ET, DP>(a, st)
    PG_BY_WIDTH(PG_DKV);
#undef PG_DKV
}
dim3 wavefronts(int64_t rows, int z = 1) {
    const int64_t groups = (rows + 3) / 4, y = (groups + (1 << 20) - 1) >> 20;
    return dim3((unsigned)((groups + y - 1) / y), (unsigned)y, (unsigned)z);
}

}  // namespace

size_t attention_backward_workspace(const AttentionArgs &a, int type) {
    const size_t asked = (size_t)a.n * a.sequences * a.rows * a.heads, states = (size_t)a.n * a.sequences * a.memory * a.kv_heads;
    const Cut q = dq_cut(a, type), kv = dkv_cut(a);
    const size_t parts = std::max(q.splits > 1 ? q.splits * asked * a.width : 0, kv.splits > 1 ? 2 * kv.splits * states * a.width : 0);
    return sizeof(float) * ((asked + 63) / 64 * 64 + parts);
}
void launch_attention_delta(const AttentionArgs &a, int type, hipStream_t st) {
    const dim3 grid = wavefronts((int64_t)a.n * a.sequences * a.rows * a.heads);
    if (type == kF32) attention_delta_kernel<kF32><<<grid, dim3(256), 0, st>>>(a);
    else attention_delta_kernel<kBf16><<<grid, dim3(256), 0, st>>>(a);
}
void launch_attention_dq(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = dq_cut(a, type);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    type == kF32 ? dq_by_width<kF32>(a, cut.waves, st) : dq_by_width<kBf16>(a, cut.waves, st);
    if (cut.splits == 1) return;
    const dim3 grid = wavefronts((int64_t)a.n * a.sequences * a.rows * a.heads);
    if (type == kF32) attention_sum_kernel<kF32><<<grid, dim3(256), 0, st>>>(a, a.dq, a.dq, a.rows, a.heads, a.counts);
    else attention_sum_kernel<kBf16><<<grid, dim3(256), 0, st>>>(a, a.dq, a.dq, a.rows, a.heads, a.counts);
}
void launch_attention_dkv(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = dkv_cut(a);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    type == kF32 ? dkv_by_width<kF32>(a, st) : dkv_by_width<kBf16>(a, st);
    if (cut.splits == 1) return;
    const dim3 grid = wavefronts((int64_t)a.n * a.sequences * a.memory * a.kv_heads, 2);
    if (type == kF32) attention_sum_kernel<kF32><<<grid, dim3(256), 0, st>>>(a, a.dk, a.dv, a.memory, a.kv_heads, a.memory_counts);
    else attention_sum_kernel<kBf16><<<grid, dim3(256), 0, st>>>(a, a.dk, a.dv, a.memory, a.kv_heads, a.memory_counts);
}

}  // namespace pg
