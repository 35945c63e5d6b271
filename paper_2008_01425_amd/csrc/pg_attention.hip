// Attention of positions to an encoder's states: y = softmax(scale q k^T) v, one pass over the states with running maximum and sum; the scores never leave the registers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "pg_attention.h"

namespace pg {

// 32 rows of queries per wavefront, WAVES of them over the same tiles of states.  Scores are held transposed, a query to a lane and its partner.
// Without states to see: y = 0, lse = -inf.
template <int ET, int DP, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) attention_kernel(const AttentionArgs a) {
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
    Frag<ET> q[T::NK];
    own_rows<ET, DP>(q, sequence_of(a.q, k, a.rows, T::EB) + ((int64_t)t * a.q.row + head * a.width) * T::EB, there, a.width, h);
    const gin keys = sequence_of(a.k, k, a.memory, T::EB) + k.head * a.width * T::EB, values = sequence_of(a.v, k, a.memory, T::EB) + k.head * a.width * T::EB;
    const float c = a.scale * kLog2e;
    float top = -__builtin_inff(), sum = 0.f;
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
        f32x16 s[KT / 32];
        float most = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < KT / 32; ++b) {
            s[b] = zero16();
#pragma unroll
            for (int kk = 0; kk < T::NK; ++kk) s[b] = mul<ET>(T::along(tk, b * 32 + i, kk, h), q[kk], s[b]);
            if (seen != all_rows<KT>()) {
                const uint32_t bits = (uint32_t)(seen >> (b * 32)) >> (4 * h);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(bits >> (8 * (r / 4) + r % 4) & 1)) s[b][r] = -__builtin_inff();
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, s[b][r]);
        }
        most = across_halves_max(most) * c;
        // The maximum that the exponentials go by follows the true one once it is 2^8 behind: sums stay far from the ends of float's range, and most tiles leave
        // the results as they are.
        if (__any(most > top + 8.f)) {
            const float to = most > top + 8.f ? most : top, by = to == top ? 1.f : __builtin_amdgcn_exp2f(top - to);
            top = to;
            sum *= by;
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) out[nb] *= by;
        }
        const float from = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
        for (int b = 0; b < KT / 32; ++b) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], c, -from));
                sum += s[b][r];
            }
#pragma unroll
            for (int step = 0; step < T::STEPS; ++step) {
                const Frag<ET> p = T::of(s[b], step);
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) out[nb] = mul<ET>(T::across(tv, b * 32 + step * T::STEP, nb, lane), p, out[nb]);
            }
        }
    }
    sum = across_halves_sum(sum);
    if (!there) return;
    const int64_t at = (k.where * a.rows + t) * a.heads + head;
    if (a.splits > 1) {
        const int64_t mine = (int64_t)k.split * a.n * a.sequences * a.rows * a.heads + at;
        if (h == 0) {
            a.part_stats[2 * mine] = top;
            a.part_stats[2 * mine + 1] = sum;
        }
        if (sum != 0.f) put_rows<kF32>((gout)(a.part + mine * a.width), out, 1.f, a.width, h);
        return;
    }
    if (h == 0 && a.lse) a.lse[at] = sum == 0.f ? -__builtin_inff() : top * kLn2 + logf(sum);
    put_rows<ET>((gout)sequence_of(a.y, k, a.rows, T::EB) + ((int64_t)t * a.y.row + head * a.width) * T::EB, out, sum == 0.f ? 0.f : 1.f / sum, a.width, h);
}

// Parts of a position and head, one wavefront each, always in the same order.
template <int ET> __global__ void __launch_bounds__(256) attention_join_kernel(const AttentionArgs a) {
    const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads, at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64;
    if (at >= rows) return;
    const int lane = threadIdx.x % 64, head = (int)(at % a.heads);
    const int64_t row = at / a.heads, where = row / a.rows;
    const int t = (int)(row - where * a.rows);
    if (t >= length_of(a.counts, where, a.rows)) return;
    float top = -__builtin_inff(), sum = 0.f;
    for (int s = 0; s < a.splits; ++s) top = __builtin_fmaxf(top, a.part_stats[2 * (s * rows + at)]);
    const float from = top == -__builtin_inff() ? 0.f : top;
    float v[kMostWidth / 64] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float mine = a.part_stats[2 * (s * rows + at) + 1];
        if (mine == 0.f) continue;
        const float by = __builtin_amdgcn_exp2f(a.part_stats[2 * (s * rows + at)] - from);
        sum += mine * by;
#pragma unroll
        for (int j = 0; j < kMostWidth / 64; ++j)
            if (j * 64 + lane < a.width) v[j] += a.part[(s * rows + at) * a.width + j * 64 + lane] * by;
    }
    if (lane == 0 && a.lse) a.lse[at] = sum == 0.f ? -__builtin_inff() : top * kLn2 + logf(sum);
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    const gout y = (gout)a.y.data + ((where / a.sequences) * a.y.worker + ((where % a.sequences) * a.rows + t) * a.y.row + head * a.width) * Elem<ET>::bytes;
#pragma unroll
    for (int j = 0; j < kMostWidth / 64; ++j) {
        const int col = j * 64 + lane;
        if (col >= a.width) continue;
        if constexpr (ET == kF32) to_global<float>(y + col * 4, v[j] * by);
        else to_global<uint16_t>(y + col * 2, bf16_bits(v[j] * by));
    }
}

dim3 attention_grid(const AttentionArgs &a) {
    const int64_t groups = ((int64_t)a.n * a.sequences * a.kv_heads * a.tiles * a.splits + 7) / 8 * 8, most = 1 << 20;
    const int64_t y = (groups + most - 1) / most;
    return dim3((unsigned)(((groups + y - 1) / y + 7) / 8 * 8), (unsigned)y);
}

namespace {

// Splits: enough work-groups for the chip, of two tiles each at least.
struct Cut {
    int waves, tiles, splits;
};
Cut cut_of(const AttentionArgs &a, int type) {
    const int64_t asked = (int64_t)a.rows * a.group, problems = (int64_t)a.n * a.sequences * a.kv_heads;
    const int waves = asked <= 32 && (type == kBf16 || a.width <= 128) ? 1 : 4;
    const int64_t tiles = (asked + 32 * waves - 1) / (32 * waves), groups = problems * tiles, wanted = waves == 1 ? 2048 : 512;
    const int64_t steps = (a.memory + 63) / 64;
    const int64_t splits = std::max<int64_t>(1, std::min({wanted / std::max<int64_t>(groups, 1), steps / 2, (int64_t)64}));
    return Cut{waves, (int)tiles, (int)splits};
}

template <int ET, int DP, int WAVES> void launch_one(const AttentionArgs &a, hipStream_t st) {
    attention_kernel<ET, DP, WAVES><<<attention_grid(a), dim3(64 * WAVES), 0, st>>>(a);
}
template <int ET> void launch_by_width(const AttentionArgs &a, int waves, hipStream_t st) {
    if (waves == 1) {
        if (a.width <= 64) launch_one<ET, 64, 1>(a, st);
        else if (a.width <= 128) launch_one<ET, 128, 1>(a, st);
        else if constexpr (ET == kBf16) launch_one<ET, 256, 1>(a, st);
    } else {
        if (a.width <= 32) launch_one<ET, 32, 4>(a, st);
        else if (a.width <= 64) launch_one<ET, 64, 4>(a, st);
        else if (a.width <= 96) launch_one<ET, 96, 4>(a, st);
        else if (a.width <= 128) launch_one<ET, 128, 4>(a, st);
        else if (a.width <= 192) launch_one<ET, 192, 4>(a, st);
        else launch_one<ET, 256, 4>(a, st);
    }
}

}  // namespace

size_t attention_forward_workspace(const AttentionArgs &a, int type) {
    const Cut cut = cut_of(a, type);
    return cut.splits > 1 ? sizeof(float) * cut.splits * ((size_t)a.n * a.sequences * a.rows * a.heads) * (a.width + 2) : 0;
}

void launch_attention(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = cut_of(a, type);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads;
    a.part_stats = a.part + cut.splits * rows * a.width;
    if (type == kF32) launch_by_width<kF32>(a, cut.waves, st);
    else launch_by_width<kBf16>(a, cut.waves, st);
    if (cut.splits > 1) {
        const int64_t groups = (rows + 3) / 4, y = (groups + (1 << 20) - 1) >> 20;
        const dim3 grid((unsigned)((groups + y - 1) / y), (unsigned)y);
        if (type == kF32) attention_join_kernel<kF32><<<grid, dim3(256), 0, st>>>(a);
        else attention_join_kernel<kBf16><<<grid, dim3(256), 0, st>>>(a);
    }
}

}  // namespace pg
