// Gradients of attention, without the scores of the way there: they are formed again from queries and keys, and their weights from the sums that were kept.
//     P = exp(scale q k^T - lse),  dS = P (dy v^T - dy . y),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dy
// Two kernels, one that owns queries and one that owns states: each writes its own rows once and in a fixed order of sums, at the price of forming S and dy v^T twice (7
// products for the 5 that one kernel with atomic additions would take).  bf16, 2 x 2048 x 4096, 16 heads of 128 over 4: dq 195 us, dk and dv 287 and 13 to join two parts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "pg_attention.h"

namespace pg {

namespace {

template <int ET> __device__ __forceinline__ float dot(const Frag<ET> &a, const Frag<ET> &b, float sum) {
    if constexpr (ET == kF32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += a[j] * b[j];
    } else if constexpr (ET == kPieces) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sum += ((float)a.p[0][j] + (float)a.p[1][j] + (float)a.p[2][j]) * ((float)b.p[0][j] + (float)b.p[1][j] + (float)b.p[2][j]);
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

// Wavefronts a SIMD has registers for; two hide each other's waits.  bf16, 8 x 4 sequences of 512 x 1024, 16 heads of 64: dq 128 us, dk and dv 256 us with two, 271 with one; width
// 128, 2 x 8192 x 8192, 16 heads over 4, dk and dv: 2160 us with two, which have registers for all but the own values, 3030 with one.
template <int ET, int DP> constexpr int dq_waves() { return DP <= (ET == kBf16 ? 128 : (ET == kPieces ? 64 : 0)) ? 2 : 1; }
// Where own values wait in LDS instead of registers.
template <int ET, int DP> constexpr bool stashes() { return (ET == kBf16 && DP == 128) || (ET == kPieces && DP == 96); }
template <int ET, int DP> constexpr int dkv_waves() { return DP <= (ET == kBf16 ? 128 : (ET == kPieces ? 32 : 0)) ? 2 : 1; }

// 32 queries per wavefront, four wavefronts; the next tile of keys and values waits in registers and goes, behind the barrier, where the last one was.
template <int ET, int DP, bool WHOLE>
__global__ void __launch_bounds__(256, (dq_waves<ET, DP>())) attention_dq_kernel(const AttentionArgs a) {
    typedef Tile<ET, DP> T;
    constexpr int SIZE = T::SIZE;
    __shared__ __attribute__((aligned(16))) char lds[4 * SIZE];
    __shared__ int tags[4];
    const Work k = work_of(a);
    if (!k.any) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 32, h = lane / 32;
    const T places(lane);
    const int asked = length_of(a.counts, k.where, a.rows) * a.group, count = length_of(a.memory_counts, k.where, a.memory);
    if (k.tile * 128 >= asked) return;
    const int u = k.tile * 128 + wave * 32 + i;
    const bool there = u < asked, busy = __builtin_amdgcn_readfirstlane(k.tile * 128 + wave * 32) < asked;
    const int mine = there ? u : asked - 1, t = mine / a.group, head = k.head * a.group + mine % a.group;
    const int64_t at = (k.where * a.rows + t) * a.heads + head;
    Frag<ET> q[T::NK], dy[T::NK];
    float delta = 0.f, from = a.lse[at] * kLog2e;
    bool odd_own;
    {
        Frag<ET> y[T::NK];
        // where nothing is seen, what comes back counts as 0: 0 times an infinity is NaN
        odd_own = own_rows<ET, DP, WHOLE>(dy, sequence_of(a.dy, k, a.rows, T::EB) + ((int64_t)t * a.dy.row + head * a.width) * T::EB, there && from != -__builtin_inff(), a.width, h);
        odd_own |= own_rows<ET, DP, WHOLE>(y, sequence_of(a.y, k, a.rows, T::EB) + ((int64_t)t * a.y.row + head * a.width) * T::EB, there, a.width, h);
        odd_own |= own_rows<ET, DP, WHOLE>(q, sequence_of(a.q, k, a.rows, T::EB) + ((int64_t)t * a.q.row + head * a.width) * T::EB, there, a.width, h);
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) delta = dot<ET>(dy[kk], y[kk], delta);
        delta = across_halves_sum(delta);
    }
    if (from == -__builtin_inff()) from = 0.f;   // nothing seen: every weight below is 2^-inf
    const gin keys = sequence_of(a.k, k, a.memory, T::EB) + k.head * a.width * T::EB, values = sequence_of(a.v, k, a.memory, T::EB) + k.head * a.width * T::EB;
    const float c = a.scale * kLog2e;
    f32x16 out[T::NB];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) out[nb] = zero16();

    int first, last;
    share_of(count, KT, k.split, a.splits, first, last);
    // A tile that holds all states gives dy . y as the sum of its weighted products, without the rounding of y, which few states do not average out (bf16, two states:
    // gradients off by 2.8e-3 in norm with y, 2.4e-3 so; their own rounding is 1.7e-3).
    const bool alone = count <= KT;  // then the first part has it
    const uint32_t key_row = (uint32_t)a.k.row * T::EB, value_row = (uint32_t)a.v.row * T::EB;
    Staged<ET, DP, 256, WHOLE> next_k, next_v;
    const auto key_places = next_k.places(threadIdx.x, a.width, [&](int row) { return __umul24(row, key_row); });
    const auto value_places = next_v.places(threadIdx.x, a.width, [&](int row) { return __umul24(row, value_row); });
    // Tiles of the split that exist as a whole, with nothing hidden, are plain: no bits, no ends.  A step takes in the tile two behind its own; where the last tile
    // is plain, tiles behind it are that one once more.
    const int whole = WHOLE && !a.mask ? (last < count / KT ? last : count / KT) : 0, plain_steps = whole == last ? last : whole - 2;
    auto fetch_whole = [&](int at) __attribute__((always_inline)) {
        at = at < whole ? at : whole - 1;
        next_k.load_whole(keys + (int64_t)at * KT * key_row, key_places);
        next_v.load_whole(values + (int64_t)at * KT * value_row, value_places);
    };
    Seen seen{a.mask ? a.mask + k.where * a.memory : nullptr, count, 0};
    uint32_t seen_after = 0;  // masks only: of the tile behind that of a step
    auto fetch = [&](int at) __attribute__((always_inline)) {  // tiles behind the last are the last once more, which nothing uses
        at = at < last ? at : last - 1;
        seen.fetch(at);
        next_k.load(keys + (int64_t)at * KT * key_row, threadIdx.x, count - at * KT, a.width, [&](int row) { return __umul24(row, key_row); });
        next_v.load(values + (int64_t)at * KT * value_row, threadIdx.x, count - at * KT, a.width, [&](int row) { return __umul24(row, value_row); });
    };
    auto k_tile = [&](int slot) __attribute__((always_inline)) { return lds + slot * 2 * SIZE; };
    auto v_tile = [&](int slot) __attribute__((always_inline)) { return lds + (slot * 2 + 1) * SIZE; };
    const std::true_type yes{};
    const std::false_type no{};
    const Odd<ET> odd{tags};
    auto keep = [&](int at, int slot) __attribute__((always_inline)) {
        const uint32_t on = seen_after = seen.take(at < last ? at : last - 1);
        const bool odd_k = next_k.store(k_tile(slot), threadIdx.x, a.width, on), odd_v = next_v.store(v_tile(slot), threadIdx.x, a.width, on);
        odd.note(slot, at, odd_k || odd_v);
    };
    auto keep_whole = [&](int at, int slot) __attribute__((always_inline)) {
        const bool odd_k = next_k.store_whole(k_tile(slot), threadIdx.x, a.width), odd_v = next_v.store_whole(v_tile(slot), threadIdx.x, a.width);
        odd.note(slot, at, odd_k || odd_v);
    };
    // The next tile, which waits in registers, goes into its slot, and the one behind it sets out.
    auto forward = [&](int at, int slot, auto plain) __attribute__((always_inline)) {
        if constexpr (decltype(plain)::value) {
            keep_whole(at, slot);
            fetch_whole(at + 1);
        } else {
            keep(at, slot);
            fetch(at + 1);
        }
    };
    auto work = [&](int slot, uint32_t on, auto is_odd) __attribute__((always_inline)) {
        constexpr bool ODD = decltype(is_odd)::value;
        const char *const tk = k_tile(slot), *const tv = v_tile(slot);
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) {
            s = mul<ET, ODD>(places.along(tk, kk), q[kk], s);
            dp = mul<ET, ODD>(places.along(tv, kk), dy[kk], dp);
        }
        hide(s, on, h);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -from));
        if (alone) {
            delta = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) delta += s[r] * dp[r];
            delta = across_halves_sum(delta);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
#pragma unroll
        for (int step = 0; step < T::STEPS; ++step) {
            const Right<ET> ds = T::template of<ODD>(s, step);
#pragma unroll
            for (int nb = 0; nb < T::NB; ++nb) out[nb] = mul_right<ET, ODD>(places.across(tk, step, nb, lane), ds, out[nb]);
        }
    };
    auto step = [&](int tile, int slot, auto plain) __attribute__((always_inline)) {
        __syncthreads();
        const uint32_t on = decltype(plain)::value ? kAllRows : (a.mask ? seen_after : seen.there(tile));
        forward(tile + 1, slot ^ 1, plain);
        if (!busy) return;
        if constexpr (ET == kPieces)
            if (odd_own || odd.at(slot, tile)) return work(slot, on, yes);
        work(slot, on, no);
    };
    if (first < last) {
        odd.clear(2);
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) next_k.clear(lds + tile * SIZE, threadIdx.x, a.width);
        int tile = first;
        if (first < plain_steps) {
            fetch_whole(first);
            keep_whole(first, 0);
            fetch_whole(first + 1);
            for (; tile + 1 < plain_steps; tile += 2) {
                step(tile, 0, yes);
                step(tile + 1, 1, yes);
            }
        } else {
            fetch(first);
            keep(first, 0);
            fetch(first + 1);
        }
        for (; tile < last; ++tile) step(tile, (tile - first) & 1, no);
    }
    if (!there) return;
    if (k.split == 0 && h == 0) a.delta[at] = delta;
    if (!a.dq.data) return;
    if (a.splits > 1) {
        const int64_t rows = (int64_t)a.n * a.sequences * a.rows * a.heads;
        put_rows<kF32>((gout)(a.part + (k.split * rows + at) * a.width), out, a.scale, a.width, h);
    } else {
        put_rows<ET>((gout)sequence_of(a.dq, k, a.rows, T::EB) + ((int64_t)t * a.dq.row + head * a.width) * T::EB, out, a.scale, a.width, h);
    }
}

// A wavefront owns 32 states and walks along the rows of all queries that share the key head, whose gradients add up in its registers in that order.
// Queries that do not exist have a weight of 2^-inf and zeros for dy.  Their q must not be zeros, whose product with an infinite key is NaN: WHOLE tiles hold the last query that exists in its place,
// whose score is not finite only where that one's own says the same; other tiles, whose loads are slower for it (floats, 4 x 2 x 333 x 777, heads of 203: 650 us for 597), have the score set to -inf.
// (So with all tiles: two registers more, which attention of 2 x 2048 x 4096, 16 heads of 128 over 4, pays with 600 us for 507.)  WHAT: 1 dv, 2 dk, 3 both in one.
template <int ET, int DP, int WHAT, bool WHOLE>
__global__ void __launch_bounds__(256, (dkv_waves<ET, DP>())) attention_dkv_kernel(const AttentionArgs a) {
    typedef Tile<ET, DP> T;
    constexpr int SIZE = T::SIZE;
    constexpr bool DK = WHAT & 2, DV = WHAT & 1, STASH = stashes<ET, DP>();
    __shared__ __attribute__((aligned(16))) char lds[4 * SIZE];
    __shared__ int tags[4];
    __shared__ __attribute__((aligned(16))) char own_values[STASH ? 4 * T::SIZE : 16];
    __shared__ __attribute__((aligned(16))) float stats[2][2][KT];
    const Work k = work_of(a);
    if (!k.any) return;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = lane % 32, h = lane / 32;
    const T places(lane);
    const int asked = length_of(a.counts, k.where, a.rows) * a.group, count = length_of(a.memory_counts, k.where, a.memory);
    if (k.tile * 128 >= count) return;
    const int own = k.tile * 128 + wave * 32 + i;
    const bool there = own < count, busy = __builtin_amdgcn_readfirstlane(k.tile * 128 + wave * 32) < count, seen = there && (!a.mask || a.mask[k.where * a.memory + own] != 0);
    Frag<ET> key[T::NK], value[DK ? T::NK : 1];
    char *const mine_in_lds = own_values + (STASH ? wave * T::SIZE : 0);
    const int mine = there ? own : count - 1;
    bool odd_own = own_rows<ET, DP, WHOLE>(key, sequence_of(a.k, k, a.memory, T::EB) + ((int64_t)mine * a.k.row + k.head * a.width) * T::EB, seen, a.width, h);
    if constexpr (DK) odd_own |= own_rows<ET, DP, WHOLE>(value, sequence_of(a.v, k, a.memory, T::EB) + ((int64_t)mine * a.v.row + k.head * a.width) * T::EB, seen, a.width, h);
    if constexpr (STASH && DK) {
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) places.put_along(mine_in_lds, kk, value[kk]);  // read by the lanes that write it
    }
    const float c = a.scale * kLog2e;
    f32x16 dk[DK ? T::NB : 1], dv[DV ? T::NB : 1];
#pragma unroll
    for (int nb = 0; nb < T::NB; ++nb) {
        if constexpr (DK) dk[nb] = zero16();
        if constexpr (DV) dv[nb] = zero16();
    }

    int first, last;
    share_of(asked, KT, k.split, a.splits, first, last);
    Staged<ET, DP, 256, WHOLE> next_q, next_dy;
    float next_from = 0.f, next_delta = 0.f;
    const gin queries = sequence_of(a.q, k, a.rows, T::EB) + (int64_t)k.head * a.group * a.width * T::EB,
              dys = sequence_of(a.dy, k, a.rows, T::EB) + (int64_t)k.head * a.group * a.width * T::EB;
    const float *const sums = a.lse + k.where * a.rows * a.heads + k.head * a.group, *const deltas = a.delta + k.where * a.rows * a.heads + k.head * a.group;
    // Positions of a tile begin with one as a whole where the group divides the tile; its rows then lie alike in every tile.
    const int group = a.group, per_tile = KT / group;
    const bool regular = per_tile * group == KT;
    const uint32_t query_row = (uint32_t)a.q.row * T::EB, dy_row = (uint32_t)a.dy.row * T::EB, head_bytes = a.width * T::EB;
    const auto query_places = next_q.places(threadIdx.x, a.width, [&](int row) { return __umul24(row / group, query_row) + row % group * head_bytes; });
    const auto dy_places = next_dy.places(threadIdx.x, a.width, [&](int row) { return __umul24(row / group, dy_row) + row % group * head_bytes; });
    const int stat_place = threadIdx.x % KT / group * a.heads + threadIdx.x % KT % group;
    // Tiles that exist as a whole are plain.  A step takes in the tile two behind its own; where the last tile is plain, tiles behind it are that one once more.  Float instructions take
    // all tiles as others: 4 x 2 x 333 x 777, 8 heads of 256 over 2, 1100 us, 1148 with plain ones.  (The body for plain tiles is theirs too, though no call enters it: where it is left out, the
    // compiler finds 244 bytes of scratch more, 1565 us.)
    const int whole = ET != kF32 && WHOLE && regular ? (last < asked / KT ? last : asked / KT) : 0, plain_steps = whole == last ? last : whole - 2;
    auto fetch_whole = [&](int at) __attribute__((always_inline)) {
        const int position = (at < whole ? at : whole - 1) * per_tile;
        next_q.load_whole(queries + (int64_t)position * query_row, query_places);
        next_dy.load_whole(dys + (int64_t)position * dy_row, dy_places);
        if (threadIdx.x < KT) {
            const int64_t at = (int64_t)position * a.heads + stat_place;
            next_from = sums[at] * kLog2e;
            if (next_from == -__builtin_inff()) next_from = __builtin_inff();   // saw nothing
            next_delta = deltas[at];
        }
    };
    auto fetch = [&](int at) __attribute__((always_inline)) {  // tiles behind the last are the last once more, which nothing uses
        at = at < last ? at : last - 1;
        const int begin = at * KT, have = asked - begin, position = begin / group, head = begin - position * group;
        const gin qb = queries + (int64_t)position * query_row, db = dys + (int64_t)position * dy_row;
        next_q.load(qb, threadIdx.x, have, a.width, [&](int row) {
            const int t = (head + row) / group;
            return __umul24(t, query_row) + (head + row - t * group) * head_bytes;
        });
        next_dy.load(db, threadIdx.x, have, a.width, [&](int row) {
            const int t = (head + row) / group;
            return __umul24(t, dy_row) + (head + row - t * group) * head_bytes;
        });
        if (threadIdx.x < KT) {
            next_from = __builtin_inff();
            next_delta = 0.f;
            if ((int)threadIdx.x < have) {
                const int t = (begin + (int)threadIdx.x) / group;
                const int64_t at = (int64_t)t * a.heads + (begin + (int)threadIdx.x - t * group);
                next_from = sums[at] * kLog2e;
                if (next_from == -__builtin_inff()) next_from = __builtin_inff();   // saw nothing
                next_delta = deltas[at];
            }
        }
    };
    auto q_tile = [&](int slot) __attribute__((always_inline)) { return lds + slot * 2 * SIZE; };
    auto d_tile = [&](int slot) __attribute__((always_inline)) { return lds + (slot * 2 + 1) * SIZE; };
    const std::true_type yes{};
    const std::false_type no{};
    const Odd<ET> odd{tags};
    auto keep_stats = [&](int slot) __attribute__((always_inline)) {
        if (threadIdx.x < KT) {
            stats[slot][0][threadIdx.x] = next_from;
            stats[slot][1][threadIdx.x] = next_delta;
        }
        return ET == kPieces && !(__builtin_fabsf(next_delta) < __builtin_inff());
    };
    auto keep = [&](int at, int slot) __attribute__((always_inline)) {
        const int left = asked - (at < last ? at : last - 1) * KT;
        const uint32_t on = left >= KT ? kAllRows : (1u << left) - 1;
        const bool odd_q = WHOLE ? next_q.store_whole(q_tile(slot), threadIdx.x, a.width) : next_q.store(q_tile(slot), threadIdx.x, a.width, on),
                   odd_d = next_dy.store(d_tile(slot), threadIdx.x, a.width, on);
        const bool odd_s = keep_stats(slot);
        odd.note(slot, at, odd_q || odd_d || odd_s);
    };
    auto keep_whole = [&](int at, int slot) __attribute__((always_inline)) {
        const bool odd_q = next_q.store_whole(q_tile(slot), threadIdx.x, a.width), odd_d = next_dy.store_whole(d_tile(slot), threadIdx.x, a.width);
        const bool odd_s = keep_stats(slot);
        odd.note(slot, at, odd_q || odd_d || odd_s);
    };
    // The next tile, which waits in registers, goes into its slot, and the one behind it sets out.
    auto forward = [&](int at, int slot, auto plain) __attribute__((always_inline)) {
        if constexpr (decltype(plain)::value) {
            keep_whole(at, slot);
            fetch_whole(at + 1);
        } else {
            keep(at, slot);
            fetch(at + 1);
        }
    };
    auto work = [&](int tile, int slot, auto is_odd, auto plain) __attribute__((always_inline)) {
        constexpr bool ODD = decltype(is_odd)::value;
        const char *const tq = q_tile(slot), *const td = d_tile(slot);
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < T::NK; ++kk) {
            s = mul<ET, ODD>(places.along(tq, kk), key[kk], s);
            if constexpr (DK) dp = mul<ET, ODD>(places.along(td, kk), STASH ? places.along(mine_in_lds, kk) : value[kk], dp);
        }
        if constexpr (!WHOLE && !decltype(plain)::value) {
            const int left = asked - tile * KT;
            if (left < KT) hide(s, (1u << left) - 1, h);
        }
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 from = *(const f32x4 *)&stats[slot][0][2 * r + 4 * h], delta = *(const f32x4 *)&stats[slot][1][2 * r + 4 * h];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + j], c, -from[j]));
                if constexpr (DK) dp[r + j] = s[r + j] * (dp[r + j] - delta[j]);
            }
        }
#pragma unroll
        for (int step = 0; step < T::STEPS; ++step) {
            if constexpr (DV) {
                const Right<ET> p = T::template of<ODD, true>(s, step);
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) dv[nb] = mul_right<ET, ODD>(places.across(td, step, nb, lane), p, dv[nb]);
            }
            if constexpr (DK) {
                const Right<ET> ds = T::template of<ODD>(dp, step);
#pragma unroll
                for (int nb = 0; nb < T::NB; ++nb) dk[nb] = mul_right<ET, ODD>(places.across(tq, step, nb, lane), ds, dk[nb]);
            }
        }
    };
    auto step = [&](int tile, int slot, auto plain) __attribute__((always_inline)) {
        __syncthreads();
        forward(tile + 1, slot ^ 1, plain);
        if (!busy) return;
        if constexpr (ET == kPieces)
            if (odd_own || odd.at(slot, tile)) return work(tile, slot, yes, plain);
        work(tile, slot, no, plain);
    };
    if (first < last) {
        odd.clear(2);
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) next_q.clear(lds + tile * SIZE, threadIdx.x, a.width);
        int tile = first;
        if (first < plain_steps) {
            fetch_whole(first);
            keep_whole(first, 0);
            fetch_whole(first + 1);
            for (; tile + 1 < plain_steps; tile += 2) {
                step(tile, 0, yes);
                step(tile + 1, 1, yes);
            }
        } else {
            fetch(first);
            keep(first, 0);
            fetch(first + 1);
        }
        for (; tile < last; ++tile) step(tile, (tile - first) & 1, no);
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

// Sums of parts, always in the same order, a thread to U elements of a row and head; z: dk and dv.
template <int ET, int U> __global__ void __launch_bounds__(256) attention_sum_kernel(const AttentionArgs a, RowsArg first, RowsArg second, int length, int heads, const int32_t *counts) {
    constexpr int AHEAD = 4;
    const int units = a.width / U;
    const int64_t rows = (int64_t)a.n * a.sequences * length * heads, id = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, at = id / units;
    if (at >= rows) return;
    const int col = (int)(id - at * units) * U, head = (int)(at % heads);
    const int64_t row = at / heads, where = row / length;
    const int t = (int)(row - where * length);
    if (t >= length_of(counts, where, length)) return;
    const RowsArg r = blockIdx.z ? second : first;
    const gin part = (gin)(a.part + (blockIdx.z * a.splits * rows + at) * a.width + col);
    const gout out = (gout)r.data + ((where / a.sequences) * r.worker + ((where % a.sequences) * length + t) * r.row + head * a.width + col) * Elem<ET>::bytes;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.splits; s += AHEAD) {
        f32x4 w[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            w[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (s + i < a.splits) w[i] = load4<kF32>(part + (s + i) * rows * a.width * 4, U);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) v += w[i];
    }
    store4<ET>(out, v, U);
}

namespace {

// us of a step as measured with heads of 128 and 64, floats a multiple of that
Cut dq_cut(const AttentionArgs &a, int type) {
    const double us = (0.45 + 0.55 * a.width / 128) * 1.5 * (type == kBf16 ? 1 : (a.width <= 128 ? 2.5 : 6));
    return cut_of((int64_t)a.n * a.sequences * a.kv_heads, ((int64_t)a.rows * a.group + 127) / 128, (a.memory + KT - 1) / KT,
                  a.width <= (type == kBf16 ? 128 : 64) ? 2 : 1, us, 4.0 * a.n * a.sequences * a.rows * a.heads * a.width, a.forced);
}
Cut dkv_cut(const AttentionArgs &a, int type) {
    const double us = (0.45 + 0.55 * a.width / 128) * 1.7 * (type == kBf16 ? 1 : (a.width <= 128 ? 2.5 : 6));
    return cut_of((int64_t)a.n * a.sequences * a.kv_heads, (a.memory + 127) / 128, ((int64_t)a.rows * a.group + KT - 1) / KT,
                  a.width <= (type == kBf16 ? 128 : 32) ? 2 : 1, us, 8.0 * a.n * a.sequences * a.memory * a.kv_heads * a.width, a.forced);
}

template <int ET, int DP, bool WHOLE> void launch_dq(const AttentionArgs &a, hipStream_t st) {
    attention_dq_kernel<ET, DP, WHOLE><<<attention_grid(a), dim3(256), 0, st>>>(a);
}
template <int ET, int DP, bool WHOLE> void launch_dkv(const AttentionArgs &a, hipStream_t st) {
    if constexpr (DP * Elem<ET>::bytes > (ET == kF32 ? 512 : 384)) {  // both gradients and the own rows of the widest heads are more than the registers
        attention_dkv_kernel<ET, DP, 1, WHOLE><<<attention_grid(a), dim3(256), 0, st>>>(a);
        attention_dkv_kernel<ET, DP, 2, WHOLE><<<attention_grid(a), dim3(256), 0, st>>>(a);
    } else {
        attention_dkv_kernel<ET, DP, 3, WHOLE><<<attention_grid(a), dim3(256), 0, st>>>(a);
    }
}
// Heads that are no whole units wide are read element by element where they end: fewer widths of them are built.
#define PG_BY_WIDTH(LAUNCH)                                             \
    const bool whole = a.width % Tile<ET, 32>::PER == 0;                \
    if constexpr (ET != kF32) {                                         \
        if (whole && a.width <= 32) return LAUNCH(32, true);        \
        if (a.width <= 64) return whole ? LAUNCH(64, true) : LAUNCH(64, false);     \
        if (whole && a.width <= 96) return LAUNCH(96, true);        \
        if (a.width <= 128) return whole ? LAUNCH(128, true) : LAUNCH(128, false);  \
    }                                                                   \
    if constexpr (ET != kPieces) {                                      \
        if (whole && a.width <= 192) return LAUNCH(192, true);      \
        whole ? LAUNCH(256, true) : LAUNCH(256, false);                 \
    }
template <int ET> void dq_by_width(const AttentionArgs &a, hipStream_t st) {
#define PG_DQ(DP, WHOLE) launch_dq<ET, DP, WHOLE>(a, st)
    PG_BY_WIDTH(PG_DQ)
#undef PG_DQ
}
template <int ET> void dkv_by_width(const AttentionArgs &a, hipStream_t st) {
#define PG_DKV(DP, WHOLE) launch_dkv<ET, DP, WHOLE>(a, st)
    PG_BY_WIDTH(PG_DKV)
#undef PG_DKV
}
dim3 groups_of(int64_t groups, int z = 1) {
    const int64_t y = (groups + (1 << 20) - 1) >> 20;
    return dim3((unsigned)((groups + y - 1) / y), (unsigned)y, (unsigned)z);
}

void sum_parts(const AttentionArgs &a, int type, const RowsArg &first, const RowsArg &second, int results, int length, int heads, const int32_t *counts, hipStream_t st) {
    const int unit = a.width % 4 ? 1 : 4;
    const dim3 grid = groups_of(((int64_t)a.n * a.sequences * length * heads * (a.width / unit) + 255) / 256, results);
    if (type == kF32) unit == 4 ? attention_sum_kernel<kF32, 4><<<grid, dim3(256), 0, st>>>(a, first, second, length, heads, counts)
                                : attention_sum_kernel<kF32, 1><<<grid, dim3(256), 0, st>>>(a, first, second, length, heads, counts);
    else unit == 4 ? attention_sum_kernel<kBf16, 4><<<grid, dim3(256), 0, st>>>(a, first, second, length, heads, counts)
                   : attention_sum_kernel<kBf16, 1><<<grid, dim3(256), 0, st>>>(a, first, second, length, heads, counts);
}

}  // namespace

size_t attention_backward_workspace(const AttentionArgs &a, int type) {
    const size_t asked = (size_t)a.n * a.sequences * a.rows * a.heads, states = (size_t)a.n * a.sequences * a.memory * a.kv_heads;
    const Cut q = dq_cut(a, type), kv = dkv_cut(a, type);
    const size_t parts = std::max(q.splits > 1 ? q.splits * asked * a.width : 0, kv.splits > 1 ? 2 * kv.splits * states * a.width : 0);
    return sizeof(float) * ((asked + 63) / 64 * 64 + parts);
}
void launch_attention_delta(const AttentionArgs &a, int type, hipStream_t st) {
    if (a.memory <= KT) return launch_attention_dq(a, type, st);  // which forms it from the weights
    const dim3 grid = groups_of(((int64_t)a.n * a.sequences * a.rows * a.heads + 3) / 4);
    if (type == kF32) attention_delta_kernel<kF32><<<grid, dim3(256), 0, st>>>(a);
    else attention_delta_kernel<kBf16><<<grid, dim3(256), 0, st>>>(a);
}
void launch_attention_dq(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = dq_cut(a, type);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    if (few_weights(a, type)) dq_by_width<kFine>(a, st);
    else if (type == kBf16) dq_by_width<kBf16>(a, st);
    else if (a.width <= 128) dq_by_width<kPieces>(a, st);
    else dq_by_width<kF32>(a, st);
    if (cut.splits == 1) return;
    sum_parts(a, type, a.dq, a.dq, 1, a.rows, a.heads, a.counts, st);
}
void launch_attention_dkv(AttentionArgs a, int type, hipStream_t st) {
    const Cut cut = dkv_cut(a, type);
    a.tiles = cut.tiles;
    a.splits = cut.splits;
    if (few_weights(a, type)) dkv_by_width<kFine>(a, st);
    else if (type == kBf16) dkv_by_width<kBf16>(a, st);
    else if (a.width <= 128) dkv_by_width<kPieces>(a, st);
    else dkv_by_width<kF32>(a, st);
    if (cut.splits == 1) return;
    sum_parts(a, type, a.dk, a.dv, 2, a.memory, a.kv_heads, a.memory_counts, st);
}

}  // namespace pg
