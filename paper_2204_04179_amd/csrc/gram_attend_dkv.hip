// Attention over item histories, backward pass over the keys (notation of gram_attend_fwd.hip and gram_attend_dq.hip):
//
//   dk_j = scale sum_i dz_ij q_i       dv_j = sum_i p_ij do_i       over the queries of every head that shares the key
//
// 1024 x 200 positions, 8 heads of 128, causal, bf16: 1.17 ms.  A block's own keys and values and its stores alone take 0.36 of
// it, as long as the memory needs; with two waves per SIMD (the accumulators of dk and dv are 64 registers, 253 in all) little of
// the staging and of the products hides behind the other.
#include "gram_attend.h"

namespace gram {

namespace {

template <typename T, int DP> struct DkvShared {
    __attribute__((aligned(1024))) unsigned char q[Shape<T, DP>::TILE], d[Shape<T, DP>::TILE];
    __attribute__((aligned(16))) int seg[kTile];
    __attribute__((aligned(16))) float less[kTile], delta[kTile], low[kTile];       // weights are 2^(s - less - low)
    uint32_t bad[2][2];                            // rows of a tile (by parity) that are marked
    float bias[2 * kTile];
    int border[kMaxBorders];
    TileMarks marks;
};

// NaN in the scores of marked rows.
__device__ __forceinline__ void spoil_rows(f32x4 (&s)[4], const uint32_t* bad, int g)
{
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if ((bad[n >> 1] >> (16 * (n & 1) + 4 * g + r)) & 1) s[n][r] = NAN;
}

// One block: 64 keys of one key head, 16 to a wave, against the queries of all heads of its group, one head after the
// other.
template <typename T, int DP, int UNIT, bool CAP, int WAVES, int SPLIT>
__global__ __launch_bounds__(kBlock * SPLIT, WAVES) void k_attend_dkv(const AttArgs a)
{
    using S = Shape<T, DP>;
    constexpr bool AHEAD = S::RB < 256;          // the next tile's loads under way; at 256 bytes it took 2 % longer
    __shared__ DkvShared<T, DP> sets[SPLIT];
    const int set = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kBlock) : 0;
    DkvShared<T, DP>& sh = sets[set];
    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int tid = threadIdx.x % kBlock, lane = lane_id();
    const int ntiles = (a.length + kTile - 1) / kTile;
    const int rows_item = (int)a.by_tiles.quotient((uint32_t)item);       // history and key head
    const int kt = item - rows_item * ntiles;
    const int batch = (int)a.by_heads.quotient((uint32_t)rows_item), kvh = rows_item - batch * a.kv_heads;
    const int c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int k0 = kt * kTile, wk0 = k0 + wave * 16, k = wk0 + c;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = prefix_of(a.prefix, batch, a.length);

    u32x4 kf[S::KK], vf[S::KK];
    const int kseg = k < a.length ? row_segment(seg, k, a.length) : kNoSegOwner;
    const bool live = kseg >= 0;
    load_owner<T, DP, UNIT>(kf, static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh + wk0 * a.k.sr, a.k.sr,
                            a.length - wk0, a.dim, live, lane);
    load_owner<T, DP, UNIT>(vf, static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh + wk0 * a.v.sr, a.v.sr,
                            a.length - wk0, a.dim, live, lane);
    const int own = live ? kseg : kNoSegOwner;
    const int t0 = a.causal && k0 >= prefix ? kt : 0;
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    if (tid < kMaxBorders) sh.border[tid] = kernel_borders()[tid];
    if (seg) mark_tiles(sh.marks, seg, a.length, kseg, k < a.length, t0, ntiles);
    const TileMarks* const mk = seg ? &sh.marks : nullptr;

    const Reader<T, DP> rd(lane);
    Feed<T, DP, UNIT> feed(tid);
    float row_lse = 0.f, row_delta = 0.f;
    const float z2 = a.scale * kLog2e, zc = CAP ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    int first = a.causal && k >= prefix ? k : 0;                  // queries from it to the history's end see the key, segments aside
    first = first < a.length ? first : a.length;
    // whether all pairs of the query tile with keys up to `row` are visible
    auto whole = [&](int t, int row, bool mixed) {
        const int q0 = t * kTile;
        return !mixed && q0 + kTile <= a.length && (!a.causal || q0 >= row || row < prefix);
    };
    auto query_rows = [&](const AttRows& r, int h, int t) {
        return static_cast<const T*>(r.data) + batch * r.sb + (kvh * a.group + h) * r.sh + t * kTile * r.sr;
    };
    auto load = [&](int h, int t) {
        feed.load(query_rows(a.q, h, t), a.q.sr, query_rows(a.dout, h, t), a.dout.sr, t * kTile, a.length, seg, a.dim);
        const int row = t * kTile + lane;
        const int64_t stat = ((int64_t)batch * a.heads + kvh * a.group + h) * a.length + (row < a.length ? row : a.length - 1);
        row_lse = a.lse[stat], row_delta = a.delta[stat];
    };

    f32x4 dk[S::DT], dv[S::DT];
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) dk[dt] = dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (tid < 4) (&sh.bad[0][0])[tid] = 0u;
    int parity = 0;
    struct Place {
        int h, t;                                                 // t = ntiles: behind the last
    };
    const int tfirst = next_tile(t0, ntiles, mk);
    auto after = [&](Place p) {
        p.t = next_tile(p.t + 1, ntiles, mk);
        if (p.t >= ntiles && p.h + 1 < a.group) p.h += 1, p.t = tfirst;
        return p;
    };
    Place round = {0, tfirst}, at = set ? after(round) : round;   // the first set's tile and this one's
    if (AHEAD && at.t < ntiles) load(at.h, at.t);
    while (round.t < ntiles) {
        const int h = at.h, t = at.t;
        const bool there = SPLIT == 1 || t < ntiles;
        if (!AHEAD && there) load(h, t);
        const bool mixed = there && tile_mixed(mk, t);
        const int q0 = t * kTile, lo = q0 - (k0 + kTile - 1); // the smallest distance of the block's pairs
        const int flat = a.bk.side ? uniform_bucket(a.bk, lo, lo + 2 * kTile - 2) : 0;
        const float* const table = a.table + (int64_t)(kvh * a.group + h) * buckets;
        __syncthreads();
        const bool masked = !whole(t, k0 + kTile - 1, mixed);
        bool far = false;                                     // some row of the tile is
        if (there) {
            feed.template put<false>(sh.q, sh.d, sh.seg, masked, sh.bad[parity]);
            far = __any(feed.seg != kNoSeg && far_lse(row_lse));
            if (wave == 0) {
                // a query that sees a non-finite value has NaN here, which masked pairs drop with their score
                float less = row_lse == -INFINITY || feed.seg == kNoSeg ? 0.f : to_log2(row_lse), dl = feed.seg == kNoSeg ? 0.f : row_delta;
                if (far) {
                    float low = 0.f;
                    if (feed.seg != kNoSeg && far_lse(row_lse)) {
                        const float* const two = a.far + 2 * (((int64_t)batch * a.heads + kvh * a.group + h) * a.length + q0 + lane);
                        less = two[0], low = two[1];
                    }
                    sh.low[lane] = low;
                }
                sh.less[lane] = less;
                sh.delta[lane] = dl;
                if (lane < 2) sh.bad[parity ^ 1][lane] = 0u;          // last read before the barrier above
            }
            if (flat < 0 && tid < 2 * kTile - 1)
                sh.bias[tid] = to_log2(table[bucket_of(a.bk, sh.border, lo + tid)]);
        }
        round = after(SPLIT > 1 ? after(round) : round);
        at = set ? after(round) : round;
        if (AHEAD && at.t < ntiles) load(at.h, at.t);
        __syncthreads();
        const bool sees = there && wk0 < a.length && !(a.causal && q0 + kTile - 1 < wk0 && wk0 >= prefix);
        auto pairs = [&](auto far) {
            f32x4 s[4], dp[4], slope[CAP ? 4 : 1];
            first_product<T, DP>(s, kf, rd, sh.q);
            to_scores<CAP>(s, slope, zc, cap2, z2, a.bk.side && flat >= 0 ? to_log2(table[flat]) : 0.f);
            if (flat < 0) add_bias(s, &sh.bias[4 * g - (k - k0) + kTile - 1]);
#pragma unroll
            for (int n = 0; n < 4; ++n) s[n] -= *reinterpret_cast<const f32x4*>(&sh.less[16 * n + 4 * g]);
            if (masked || far) {
                if (far) {
#pragma unroll
                    for (int n = 0; n < 4; ++n) s[n] -= *reinterpret_cast<const f32x4*>(&sh.low[16 * n + 4 * g]);
                }
                // rows are marked for the block: also where this wave's keys are visible to the whole tile
                if (sh.bad[parity][0] | sh.bad[parity][1]) spoil_rows(s, sh.bad[parity], g);
                if (mixed) mask_scores<true, true>(s, sh.seg, own, first - q0, lane, a.length - first);
                else mask_scores<false, true>(s, sh.seg, own, first - q0, lane, a.length - first);
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[n][r] = __builtin_amdgcn_exp2f(s[n][r]);
            first_product<T, DP>(dp, vf, rd, sh.d);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const f32x4 dl = *reinterpret_cast<const f32x4*>(&sh.delta[16 * n + 4 * g]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dp[n][r] = weighed(s[n][r], dp[n][r] - dl[r]);
                    if constexpr (CAP) dp[n][r] = weighed(dp[n][r], slope[n][r]);
                }
            }
            second_product<T, DP>(dv, s, rd, sh.d);
            second_product<T, DP>(dk, dp, rd, sh.q);
        };
        // Rows of 512 bytes spill registers: the rare case apart keeps its own out of the usual one's way (256 x 200, 8 heads of 128, the
        // whole backward pass 2.10 ms and 2.18).  Others only run out of instruction cache by it (1024 x 200: 2.76 and 1.80).
        if constexpr (S::RB <= 256) {
            if (sees) pairs(far);
        } else if (sees) {
            if (far) pairs(std::true_type{});
            else pairs(std::false_type{});
        }
        parity ^= 1;
    }
    __syncthreads();
    if constexpr (SPLIT > 1) {
        if (set) {
            hand_over(sets[1].q, dk, wave, lane);                 // and the rows of do behind
            hand_over(sets[0].q, dv, wave, lane);
        }
        __syncthreads();
        if (!set) {
            take_over(sets[1].q, dk, 1.f, 1.f, wave, lane);
            take_over(sets[0].q, dv, 1.f, 1.f, wave, lane);
        }
        __syncthreads();
        if (set) return;
    }
    if (wk0 < a.length) {
        T* const dkp = static_cast<T*>(a.dk.data) + batch * a.dk.sb + kvh * a.dk.sh + wk0 * a.dk.sr;
        T* const dvp = static_cast<T*>(a.dv.data) + batch * a.dv.sb + kvh * a.dv.sh + wk0 * a.dv.sr;
        unsigned char* const room = sh.q + wave * 16 * S::RB;
        store_rows<T, DP, UNIT>(room, dk, a.scale, dkp, a.dk.sr, a.length - wk0, a.dim, lane);
        store_rows<T, DP, UNIT>(room, dv, 1.f, dvp, a.dv.sr, a.length - wk0, a.dim, lane);
    }
}

}  // namespace

void attend_backward_keys(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s)
{
    a.items = a.batch * a.kv_heads * att_blocks(a.length, kTile);
    a.by_tiles = FastDiv::of(att_blocks(a.length, kTile)), a.by_heads = FastDiv::of(a.kv_heads);
    by_shape_and_cap(c, unit, [&](auto type, auto dp, auto u, auto cap) {
        constexpr int DP = decltype(dp)::value;
        constexpr int WAVES = Shape<decltype(type), DP>::RB <= 128 ? 3 : 2;
        auto go = [&](auto split) {
            constexpr int SPLIT = decltype(split)::value;
            k_attend_dkv<decltype(type), DP, decltype(u)::value, decltype(cap)::value, (SPLIT > 1 ? 2 : WAVES), SPLIT>
                <<<att_grid(a.items), dim3(kBlock * SPLIT), 0, s>>>(a);
        };
        if constexpr (Shape<decltype(type), DP>::RB <= 256)
            if (two_sets(a)) return go(std::integral_constant<int, 2>{});
        go(std::integral_constant<int, 1>{});
    });
}

}  // namespace gram
