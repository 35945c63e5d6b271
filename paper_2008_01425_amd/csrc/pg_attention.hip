// Attention of positions to an encoder's states: y = softmax(scale q k^T) v, one pass over the states with running maximum and sum; the scores never leave the registers.
// Bound by the matrix cores where positions are many (bf16, 2 x 4096 x 8192, 16 heads of 128 over 4: 552 to 573 us from card to card, 959 to 996 TFLOP/s of the 1244 that a large product reaches; the
// softmax's vector instructions are the rest), by reading the states where they are few (8 x 4 sequences, one position of up to 4096 states: 206 MB in 26 us, 4 more to join parts).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "pg_attention.h"

namespace pg {

// Wavefronts a SIMD has registers for.  (Float, 8 x 4 sequences of 512 x 1024, 16 heads of 64: 535 us with two, 628 with one; 4 x 2 of 1024 x 2048, 8 heads of 96: 350, 412.)
template <int ET, int DP> constexpr int forward_waves() { return DP <= (ET == kBf16 ? 128 : (ET == kPieces ? 96 : 0)) ? 2 : 1; }

// 32 queries per wavefront, four wavefronts over the same tiles of states; one without queries only helps to bring the tiles.  Scores are held transposed, a query to a lane and its partner.
// Without states to see: y = 0, lse = -inf.
//
// bf16: three tiles are on their way at once: while tile t's scores become weights, the scores of t + 1 are formed and the weights of t - 1 meet their values, so that
// matrix and vector instructions of one wavefront have something to do beside each other.  In LDS two tiles of keys and two of values: at step t, behind the
// barrier, the tiles that wait in registers (keys t + 2, values t) take the places of keys t and values t - 2, which no wavefront reads any more.  Floats, whose products take six times as long, have the registers for two
// wavefronts a SIMD instead, one tile after the other.
template <int ET, int DP, bool WHOLE>
__global__ void __launch_bounds__(256, (forward_waves<ET, DP>())) attention_kernel(const AttentionArgs a) {
    typedef Tile<ET, DP> T;
    constexpr bool PIPE = ET == kBf16;
    constexpr int SIZE = T::SIZE, OWN = 128, AHEAD = PIPE ? 3 : 2;
    __shared__ __attribute__((aligned(16))) char lds[4 * SIZE];
    __shared__ int tags[4];
    const Work k = work_of(a);
    if (!k.any) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 32, h = lane / 32;
    const T places(lane);
    const int asked = length_of(a.counts, k.where, a.rows) * a.group, count = length_of(a.memory_counts, k.where, a.memory);
    if (k.tile * OWN >= asked) return;
    const int u = k.tile * OWN + wave * 32 + i;
    const bool there = u < asked, busy = __builtin_amdgcn_readfirstlane(k.tile * OWN + wave * 32) < asked;
    const int mine = there ? u : asked - 1, t = mine / a.group, head = k.head * a.group + mine % a.group;
    Frag<ET> q[T::NK];
    const bool odd_q = own_rows<ET, DP, WHOLE>(q, sequence_of(a.q, k, a.rows, T::EB) + ((int64_t)t * a.q.row + head * a.width) * T::EB, there, a.width, h);
    const gin keys = sequence_of(a.k, k, a.memory, T::EB) + k.head * a.width * T::EB, values = sequence_of(a.v, k, a.memory, T::EB) + k.head * a.width * T::EB;
    const float c = a.scale * kLog2e;
    float top = -__builtin_inff(), sum = 0.f;
    f32x16 out[T::NB], s;
    Right<ET> p[T::STEPS];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) out[nb] = zero16();

    int first, last;
    share_of(count, KT, k.split, a.splits, first, last);
    // Tiles behind the last are the last once more: loads without a branch, of what nothing uses.
    const uint32_t key_row = (uint32_t)a.k.row * T::EB, value_row = (uint32_t)a.v.row * T::EB;
    Staged<ET, DP, 256, WHOLE> next_k, next_v;
    Seen seen{a.mask ? a.mask + k.where * a.memory : nullptr, count, 0};
    uint32_t seen_now = 0, seen_after = 0;  // masks only: of the tile of a step and the one behind it
    auto fetch_k = [&](int at) __attribute__((always_inline)) {
        at = at < last ? at : last - 1;
        seen.fetch(at);
        next_k.load(keys + (int64_t)at * KT * key_row, threadIdx.x, count - at * KT, a.width, [&](int row) { return __umul24(row, key_row); });
    };
    auto fetch_v = [&](int at) __attribute__((always_inline)) {
        at = at < last ? at : last - 1;
        next_v.load(values + (int64_t)at * KT * value_row, threadIdx.x, count - at * KT, a.width, [&](int row) { return __umul24(row, value_row); });
    };
    auto k_tile = [&](int parity) __attribute__((always_inline)) { return lds + parity * SIZE; };
    auto v_tile = [&](int parity) __attribute__((always_inline)) { return lds + (2 + parity) * SIZE; };
    const std::true_type yes{};
    const std::false_type no{};
    const Odd<ET> odd{tags};
    auto keep_k = [&](int at, int place) __attribute__((always_inline)) {
        const uint32_t on = seen.take(at < last ? at : last - 1);
        odd.note(place, at, next_k.store(k_tile(place), threadIdx.x, a.width, on));
        return on;
    };
    auto keep_v = [&](int at, int place, uint32_t keep) __attribute__((always_inline)) { odd.note(2 + place, at, next_v.store(v_tile(place), threadIdx.x, a.width, keep)); };
    auto score_as = [&](const char *tile, auto is_odd) __attribute__((always_inline)) {
        f32x16 to = zero16();
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) to = mul<ET, decltype(is_odd)::value>(places.along(tile, kk), q[kk], to);
        return to;
    };
    auto weigh_as = [&](const char *tile, auto is_odd) __attribute__((always_inline)) {  // values of a tile by the weights in p
#pragma unroll
        for (int step = 0; step < T::STEPS; ++step)
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) out[nb] = mul_right<ET, decltype(is_odd)::value>(places.across(tile, step, nb, lane), p[step], out[nb]);
    };
    auto score = [&](int at, int place) __attribute__((always_inline)) {
        if constexpr (ET == kPieces)
            if (odd_q || odd.at(place, at)) return score_as(k_tile(place), yes);
        return score_as(k_tile(place), no);
    };
    auto weigh = [&](int at, int place) __attribute__((always_inline)) {
        if constexpr (ET == kPieces)
            if (odd.at(2 + place, at)) return weigh_as(v_tile(place), yes);
        weigh_as(v_tile(place), no);
    };
    // Tiles of the split that exist as a whole, with nothing hidden, are plain: no bits, no ends.  A step takes in the tile AHEAD behind its own; where the last
    // tile is plain, tiles behind it are that one once more.
    const int whole = WHOLE && !a.mask ? (last < count / KT ? last : count / KT) : 0, plain_steps = whole == last ? last : whole - AHEAD;
    const auto key_places = next_k.places(threadIdx.x, a.width, [&](int row) { return __umul24(row, key_row); });
    const auto value_places = next_v.places(threadIdx.x, a.width, [&](int row) { return __umul24(row, value_row); });
    auto plain_k = [&](int at) __attribute__((always_inline)) { next_k.load_whole(keys + (int64_t)(at < whole ? at : whole - 1) * KT * key_row, key_places); };
    auto plain_v = [&](int at) __attribute__((always_inline)) { next_v.load_whole(values + (int64_t)(at < whole ? at : whole - 1) * KT * value_row, value_places); };
    // The maximum that the exponentials go by follows the true one once it is 2^8 behind: sums stay far from the ends of float's range, and most tiles leave the
    // results as they are.
    auto follow = [&]() __attribute__((always_inline)) {
        float most = -__builtin_inff();
#pragma unroll
        for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, s[r]);
        most *= c;
        if (__any(most > top + 8.f)) {
            most = across_halves_max(most);
            const float to = most > top + 8.f ? most : top, by = to == top ? 1.f : __builtin_amdgcn_exp2f(top - to);
            top = to;
            sum *= by;
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) out[nb] *= by;
        }
    };
    auto soften = [&]() __attribute__((always_inline)) {  // scores to weights
        const float from = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -from));
            sum += s[r];
        }
#pragma unroll
        for (int step = 0; step < T::STEPS; ++step) p[step] = T::template of<false, true>(s, step);
    };
    // before, behind: whether there is a tile; parity: of the tile, from the first on
    auto step = [&](int tile, int parity, auto before, auto behind, auto plain) __attribute__((always_inline)) {
        __syncthreads();
        if constexpr (decltype(plain)::value) {
            odd.note(parity, tile + 2, next_k.store_whole(k_tile(parity), threadIdx.x, a.width));
            odd.note(2 + parity, tile, next_v.store_whole(v_tile(parity), threadIdx.x, a.width));
            plain_k(tile + 3);
            plain_v(tile + 1);
        } else {
            const uint32_t on = a.mask ? seen_now : seen.there(tile);
            seen_now = seen_after;
            seen_after = keep_k(tile + 2, parity);
            keep_v(tile, parity, on);
            hide(s, on, h);
            fetch_k(tile + 3);
            fetch_v(tile + 1);
        }
        if (!busy) return;
        if constexpr (decltype(before)::value) weigh(tile - 1, parity ^ 1);
        follow();
        f32x16 after;
        if constexpr (decltype(behind)::value) after = score(tile + 1, parity ^ 1);
        soften();
        if constexpr (decltype(behind)::value) s = after;
    };
    // One after the other, in less registers.
    auto simple_step = [&](int tile, int parity, auto plain) __attribute__((always_inline)) {
        __syncthreads();
        uint32_t on = kAllRows;
        if constexpr (decltype(plain)::value) {
            odd.note(parity ^ 1, tile + 1, next_k.store_whole(k_tile(parity ^ 1), threadIdx.x, a.width));
            odd.note(2 + (parity ^ 1), tile + 1, next_v.store_whole(v_tile(parity ^ 1), threadIdx.x, a.width));
            plain_k(tile + 2);
            plain_v(tile + 2);
        } else {
            on = a.mask ? seen_now : seen.there(tile);
            seen_now = keep_k(tile + 1, parity ^ 1);
            keep_v(tile + 1, parity ^ 1, seen_now);
            fetch_k(tile + 2);
            fetch_v(tile + 2);
        }
        if (!busy) return;
        s = score(tile, parity);
        hide(s, on, h);
        follow();
        soften();
        weigh(tile, parity);
    };
    if (first < last) {
        odd.clear(4);
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) next_k.clear(lds + tile * SIZE, threadIdx.x, a.width);
        if constexpr (PIPE) {
            if (first < plain_steps) {
                Staged<ET, DP, 256, WHOLE> second;
                plain_k(first);
                second.load_whole(keys + (int64_t)(first + 1 < whole ? first + 1 : whole - 1) * KT * key_row, key_places);
                plain_v(first);
                odd.note(0, first, next_k.store_whole(k_tile(0), threadIdx.x, a.width));
                odd.note(1, first + 1, second.store_whole(k_tile(1), threadIdx.x, a.width));
                plain_k(first + 2);
            } else {
                fetch_k(first);
                fetch_v(first);
                seen_now = keep_k(first, 0);
                fetch_k(first + 1);
                seen_after = keep_k(first + 1, 1);
                fetch_k(first + 2);
            }
            __syncthreads();
            if (busy) s = score(first, 0);
            int tile = first;
            if (first + 1 == last) {
                step(first, 0, no, no, no);
            } else {
                if (tile < plain_steps) step(tile++, 0, no, yes, yes);
                else step(tile++, 0, no, yes, no);
                const int stop = plain_steps < last - 1 ? plain_steps : last - 1;
                for (; tile + 1 < stop; tile += 2) {
                    step(tile, 1, yes, yes, yes);
                    step(tile + 1, 0, yes, yes, yes);
                }
                for (; tile < last - 1; ++tile) step(tile, (tile - first) & 1, yes, yes, no);
                step(tile, (tile - first) & 1, yes, no, no);
            }
            __syncthreads();
            if (busy) weigh(last - 1, (last - 1 - first) & 1);
        } else {
            int tile = first;
            if (first < plain_steps) {
                plain_k(first);
                plain_v(first);
                odd.note(0, first, next_k.store_whole(k_tile(0), threadIdx.x, a.width));
                odd.note(2, first, next_v.store_whole(v_tile(0), threadIdx.x, a.width));
                plain_k(first + 1);
                plain_v(first + 1);
                for (; tile + 1 < plain_steps; tile += 2) {
                    simple_step(tile, 0, yes);
                    simple_step(tile + 1, 1, yes);
                }
            } else {
                fetch_k(first);
                fetch_v(first);
                seen_now = keep_k(first, 0);
                keep_v(first, 0, seen_now);
                fetch_k(first + 1);
                fetch_v(first + 1);
            }
            for (; tile < last; ++tile) simple_step(tile, (tile - first) & 1, no);
        }
    }
    sum = across_halves_sum(sum);
    if (!there) return;
    const int64_t at = (k.where * a.rows + t) * a.heads + head;
    if (a.splits > 1) {
        const int64_t part = (int64_t)k.split * a.n * a.sequences * a.rows * a.heads + at;
        if (h == 0) {
            a.part_stats[2 * part] = top;
            a.part_stats[2 * part + 1] = sum;
        }
        if (sum != 0.f) put_rows<kF32>((gout)(a.part + part * a.width), out, 1.f, a.width, h);
        return;
    }
    if (h == 0 && a.lse) a.lse[at] = sum == 0.f ? -__builtin_inff() : top * kLn2 + logf(sum);
    put_rows<ET>((gout)sequence_of(a.y, k, a.rows, T::EB) + ((int64_t)t * a.y.row + head * a.width) * T::EB, out, sum == 0.f ? 0.f : 1.f / sum, a.width, h);
}

// Parts of a position and head, one wavefront each, always in the same order: a lane to a part for the statistics, then eight parts' rows on their way at once (one after
// the other a part took 1.3 us).  NC: blocks of 64 columns.
template <int ET, int NC> __global__ void __launch_bounds__(256) attention_join_kernel(const AttentionArgs a) {
    constexpr int AHEAD = 8;
    const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads, at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64;
    if (at >= rows) return;
    const int lane = threadIdx.x % 64, head = (int)(at % a.heads);
    const int64_t row = at / a.heads, where = row / a.rows;
    const int t = (int)(row - where * a.rows);
    if (t >= length_of(a.counts, where, a.rows)) return;
    static_assert(kMostParts <= 64, "a lane to a part");
    float mine = -__builtin_inff(), sum = 0.f;
    if (lane < a.splits) {
        mine = a.part_stats[2 * (lane * rows + at)];
        sum = a.part_stats[2 * (lane * rows + at) + 1];
    }
    const uint64_t there = __ballot(sum != 0.f);  // others hold nothing, and their rows were not written
    float top = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = __builtin_fmaxf(top, __shfl_xor(top, d));
    const float by = sum != 0.f ? __builtin_amdgcn_exp2f(mine - (top == -__builtin_inff() ? 0.f : top)) : 0.f;
    sum *= by;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    float v[NC] = {};
    for (int s = 0; s < a.splits; s += AHEAD) {
        float part[AHEAD][NC];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int j = 0; j < NC; ++j)
                part[i][j] = (there >> (s + i) & 1) && j * 64 + lane < a.width ? a.part[((s + i) * rows + at) * a.width + j * 64 + lane] : 0.f;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float w = __shfl(by, s + i);
#pragma unroll
            for (int j = 0; j < NC; ++j) v[j] += part[i][j] * w;
        }
    }
    if (lane == 0 && a.lse) a.lse[at] = sum == 0.f ? -__builtin_inff() : top * kLn2 + logf(sum);
    const float times = sum == 0.f ? 0.f : 1.f / sum;
    const gout y = (gout)a.y.data + ((where / a.sequences) * a.y.worker + ((where % a.sequences) * a.rows + t) * a.y.row + head * a.width) * Elem<ET>::bytes;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int col = j * 64 + lane;
        if (col >= a.width) continue;
        if constexpr (ET == kF32) to_global<float>(y + col * 4, v[j] * times);
        else to_global<uint16_t>(y + col * 2, bf16_bits(v[j] * times));
    }
}

dim3 attention_grid(const AttentionArgs &a) {
    const int64_t problems = (int64_t)a.n * a.sequences * a.kv_heads, each = (int64_t)a.tiles * a.splits, most = 1 << 20;
    const int64_t groups = dealt_out((uint32_t)problems) ? (problems + 7) / 8 * 8 * each : (problems * each + 7) / 8 * 8;
    const int64_t y = (groups + most - 1) / most;
    return dim3((unsigned)(((groups + y - 1) / y + 7) / 8 * 8), (unsigned)y);
}

namespace {

// us of a step as measured with heads of 128 and 64, floats a multiple of that
Cut forward_cut(const AttentionArgs &a, int type) {
    const double us = (0.45 + 0.55 * a.width / 128) * 1.1 * (type == kBf16 ? 1 : (a.width <= 128 ? 2.5 : 6));
    return cut_of((int64_t)a.n * a.sequences * a.kv_heads, ((int64_t)a.rows * a.group + 127) / 128, (a.memory + KT - 1) / KT,
                  a.width <= (type == kBf16 ? 128 : 96) ? 2 : 1, us, 4.0 * a.n * a.sequences * a.rows * a.heads * a.width, a.forced);
}

template <int ET, int DP, bool WHOLE> void launch_one(const AttentionArgs &a, hipStream_t st) {
    attention_kernel<ET, DP, WHOLE><<<attention_grid(a), dim3(256), 0, st>>>(a);
}
// Heads that are no whole units wide are read element by element where they end: fewer widths of them are built.
template <int ET> void launch_by_width(const AttentionArgs &a, hipStream_t st) {
    const bool whole = a.width % Tile<ET, 32>::PER == 0;
#define PG_ATTENTION(DP) (whole ? launch_one<ET, DP, true>(a, st) : launch_one<ET, DP, false>(a, st))
    if constexpr (ET != kF32) {
        if (whole && a.width <= 32) return launch_one<ET, 32, true>(a, st);
        if (a.width <= 64) return PG_ATTENTION(64);
        if (whole && a.width <= 96) return launch_one<ET, 96, true>(a, st);
        if (a.width <= 128) return PG_ATTENTION(128);
    }
    if constexpr (ET != kPieces) {
        if (whole && a.width <= 192) return launch_one<ET, 192, true>(a, st);
        PG_ATTENTION(256);
    }
#undef PG_ATTENTION
}

}  // namespace

size_t attention_forward_workspace(const AttentionArgs &a, int type) {
    const Cut cut = forward_cut(a, type);
    return cut.splits > 1 ? sizeof(float) * cut.splits * ((size_t)a.n * a.sequences * a.rows * a.heads) * (a.width + 2) : 0;
}

void launch_attention(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = forward_cut(a, type);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads;
    a.part_stats = a.part + cut.splits * rows * a.width;
    if (few_weights(a, type)) launch_by_width<kFine>(a, st);
    else if (type == kBf16) launch_by_width<kBf16>(a, st);
    else if (a.width <= 128) launch_by_width<kPieces>(a, st);
    else launch_by_width<kF32>(a, st);
    if (cut.splits > 1) {
        const int64_t groups = (rows + 3) / 4, y = (groups + (1 << 20) - 1) >> 20;
        const dim3 grid((unsigned)((groups + y - 1) / y), (unsigned)y);
#define PG_JOIN(ET)                                                                       \
    a.width <= 64    ? attention_join_kernel<ET, 1><<<grid, dim3(256), 0, st>>>(a)        \
    : a.width <= 128 ? attention_join_kernel<ET, 2><<<grid, dim3(256), 0, st>>>(a)        \
                     : attention_join_kernel<ET, kMostWidth / 64><<<grid, dim3(256), 0, st>>>(a)
        type == kF32 ? PG_JOIN(kF32) : PG_JOIN(kBf16);
#undef PG_JOIN
    }
}

}  // namespace pg
