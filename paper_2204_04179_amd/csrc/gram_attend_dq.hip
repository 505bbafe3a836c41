// Attention over item histories, backward pass over the queries: dq and the gradient of the table (notation of
// gram_attend_fwd.hip).
//
//   dp_ij = do_i.v_j   delta_i = sum_j p_ij dp_ij   ds_ij = p_ij (dp_ij - delta_i)   dz_ij = ds_ij (1 - (c_ij / cap)^2)
//   dq_i = scale sum_j dz_ij k_j       dtable[head, b] = sum of ds over the pairs of bucket b
//
// delta is summed in float32 from the weights, not do.o, which knows o to as many bits as it was stored in: the table's
// gradient is a sum over whole batches in which an error of delta does not average out.  (float32 without a table takes do.o.)
//
// 1024 x 200 positions, 8 heads of 128, causal, bf16: 1.04 ms with the table's gradient, 0.75 without; 0.45 would move q, k, v, do and
// dq once.  Registers allow two waves per SIMD, which wait half of the time.  8 x 2000: 0.22 ms without; float32, 1024 x 200, 8 heads of
// 64: 1.82 ms with.
#include "gram_attend.h"

namespace gram {

namespace {


template <typename T, int DP> struct DqShared {
    __attribute__((aligned(1024))) unsigned char k[Shape<T, DP>::TILE], v[Shape<T, DP>::TILE];
    __attribute__((aligned(16))) int seg[kTile];
    float bias[2 * kTile];
    float table[kMaxBorders];
    int border[kMaxBorders];
    float base[kTile];                             // of rows whose lse is far from zero
    float strip[kWavesPerBlock][4][kStrip];        // see table_near
    float bucket[kWavesPerBlock][kMaxBorders];     // sums of ds by bucket, each wave's own
    TileMarks marks;
};

// One block: 64 queries of one head.  Dynamic LDS: kWavesPerBlock rows of 2 kNear + 1 sums of ds by distance.
// KEEP > 0: histories of at most KEEP tiles; weights and products of the first walk stay in registers, and the second walk
// loads the keys alone (queries of 1024 x 200, 8 heads of 128: 1.43 ms without).
// TABLE: the table's gradient is wanted, and with it ds itself, so that delta_i = sum_j p_ij dp_ij comes first.  Otherwise one
// walk does: bf16 rows take delta from dO . O, which knows O to 8 bits, sum p dp and p k on the way, and set dq right by
// (dO . O - sum p dp) p k at the end; the products with p read no more of the tile.  float32 rows need none of that.
template <typename T, int DP, int UNIT, bool CAP, int WAVES, bool TABLE, int KEEP, int SPLIT>
__global__ __launch_bounds__(kBlock * SPLIT, WAVES) void k_attend_dq(const AttArgs a)
{
    using S = Shape<T, DP>;
    constexpr bool AHEAD = S::RB <= 256 && KEEP == 0, MEND = !TABLE && sizeof(T) == 2;
    extern __shared__ float dist[];
    __shared__ DqShared<T, DP> sets[SPLIT];
    const int set = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kBlock) : 0;
    DqShared<T, DP>& sh = sets[set];
    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int tid = threadIdx.x % kBlock, lane = lane_id();
    const int nqt = (a.length + kTile - 1) / kTile;
    const int rows_item = (int)a.by_tiles.quotient((uint32_t)item);       // history and head
    const int qt = nqt - 1 - (item - rows_item * nqt);
    const int batch = (int)a.by_heads.quotient((uint32_t)rows_item), head = rows_item - batch * a.heads;
    const int kvh = (int)a.by_group.quotient((uint32_t)head);
    const int c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int q0 = qt * kTile, wq0 = q0 + wave * 16, q = wq0 + c;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = prefix_of(a.prefix, batch, a.length);
    const T* const kp = static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh;
    const T* const vp = static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh;
    const int64_t stat = ((int64_t)batch * a.heads + head) * a.length + (q < a.length ? q : a.length - 1);

    u32x4 qf[S::KK], df[S::KK];
    const int qseg = q < a.length ? row_segment(seg, q, a.length) : kNoSegOwner;
    const bool live = qseg >= 0;
    load_owner<T, DP, UNIT>(qf, static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh + wq0 * a.q.sr, a.q.sr,
                            a.length - wq0, a.dim, live, lane);
    load_owner<T, DP, UNIT>(df, static_cast<const T*>(a.dout.data) + batch * a.dout.sb + head * a.dout.sh + wq0 * a.dout.sr,
                            a.dout.sr, a.length - wq0, a.dim, live, lane);
    float delta = 0.f;
    if constexpr (!TABLE) {
        u32x4 of[S::KK];
        load_owner<T, DP, UNIT>(of, static_cast<const T*>(a.o.data) + batch * a.o.sb + head * a.o.sh + wq0 * a.o.sr, a.o.sr,
                                a.length - wq0, a.dim, live, lane);
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) delta += dot_chunk<T>(df[kk], of[kk]);
        delta = group_sum(delta);
    }
    const float lse = a.lse[stat];
    // whether any row is far, of the wave or, where its waves have to agree, of the block
    float any_lse = lse;
    if (KEEP == 0) any_lse = a.lse[((int64_t)batch * a.heads + head) * a.length + (q0 + lane < a.length ? q0 + lane : a.length - 1)];
    const bool far = __any(far_lse(any_lse));
    if (KEEP == 0 && far && tid < kTile) sh.base[tid] = 0.f;
    float less = lse == -INFINITY ? 0.f : to_log2(lse);           // a row that sees nothing: all its pairs are masked
    const int own = live ? qseg : kNoSegOwner;
    const int ntiles = (a.length + kTile - 1) / kTile;
    int t1 = ntiles;
    if (a.causal) {
        t1 = qt + 1;
        const int pt = (prefix + kTile - 1) / kTile;
        t1 = pt > t1 ? pt : t1;
        t1 = t1 < ntiles ? t1 : ntiles;
    }
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    if (tid < buckets) sh.table[tid] = to_log2(a.table[(int64_t)head * buckets + tid]);
    if (tid < kMaxBorders) sh.border[tid] = kernel_borders()[tid];
    if (seg) mark_tiles(sh.marks, seg, a.length, qseg, q < a.length, 0, t1);
    const TileMarks* const mk = seg ? &sh.marks : nullptr;
    constexpr int kRows = kWavesPerBlock * SPLIT;                 // of sums by distance
    float* const my_dist = dist + (set * kWavesPerBlock + wave) * (2 * kNear + 1) + kNear;

    const Reader<T, DP> rd(lane);
    Feed<T, DP, UNIT> feed(tid);
    const float z2 = a.scale * kLog2e, zc = CAP ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    int last = a.length;
    if (a.causal) {
        last = q + 1 > prefix ? q + 1 : prefix;
        last = last < a.length ? last : a.length;
    }
    if (q >= a.length) last = 0;                                  // the table's gradient is summed over rows
    const bool full_rows = wq0 + 16 <= a.length;
    auto whole = [&](int t, int row, bool mixed) {
        const int k1 = t * kTile + kTile;
        return !mixed && k1 <= a.length && (!a.causal || k1 - 1 <= row || k1 <= prefix);
    };
    auto load = [&](int t) {
        const int k0 = t * kTile;
        feed.load(kp + k0 * a.k.sr, a.k.sr, vp + k0 * a.v.sr, a.v.sr, k0, a.length, seg, a.dim);
    };
    const int tfirst = next_tile(0, t1, mk);
    constexpr bool EARLY = KEEP > 2;                 // the next tile's loads on their way: 1.03 ms and 1.09; two tiles would lose a
    bool loaded = false;                             // wave per SIMD to it (1024 x 100, heads of 64: 15 us and 14)
    const bool one_tile = TABLE && next_tile(tfirst + 1, t1, mk) >= t1;

    f32x4 dq[MEND ? 2 : 1][S::DT];                                // ds k, p k
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) dq[0][dt] = dq[MEND ? 1 : 0][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float seen = less - less;                                     // sum p dp; NaN if the statistics are not finite
    // the distances that the block's pairs can have (table_near touches 76 below a pair of tiles), within kNear
    const int near_lo = q0 - (t1 - 1) * kTile - 76 > -kNear ? q0 - (t1 - 1) * kTile - 76 : -kNear;
    const int near_hi = q0 + kTile - 1 < kNear ? q0 + kTile - 1 : kNear;
    int flat_bucket = -1;
    float flat_sum = 0.f;
    if constexpr (TABLE) {
        for (int n = near_lo + tid; n <= near_hi; n += kBlock)
#pragma unroll
            for (int w = set * kWavesPerBlock; w < (set + 1) * kWavesPerBlock; ++w) dist[w * (2 * kNear + 1) + kNear + n] = 0.f;
        for (int i = tid; i < kWavesPerBlock * 4 * kStrip; i += kBlock) (&sh.strip[0][0][0])[i] = 0.f;
        if (tid < kMaxBorders)
            for (int w = 0; w < kWavesPerBlock; ++w) sh.bucket[w][tid] = 0.f;
        delta = 0.f;
    }
    auto flat_of = [&](int t) {
        const int hi = q0 + kTile - 1 - t * kTile;
        return a.bk.side ? uniform_bucket(a.bk, hi - 2 * kTile + 2, hi) : 0;
    };
    auto sees = [&](int t) { return wq0 < a.length && !(a.causal && t * kTile > wq0 + 15 && t * kTile >= prefix); };
    // scores of a tile in LDS
    auto score = [&](int t, bool mixed, f32x4 (&s)[4], f32x4 (&slope)[CAP ? 4 : 1]) {
        const int k0 = t * kTile, flat = flat_of(t);
        first_product<T, DP>(s, qf, rd, sh.k);
        to_scores<CAP>(s, slope, zc, cap2, z2, a.bk.side && flat >= 0 ? sh.table[flat] : 0.f);
        if (flat < 0) add_bias(s, &sh.bias[4 * g - (q - q0) + kTile - 1]);
        if (!whole(t, wq0, mixed) || !full_rows || (KEEP == 0 && far)) {
            if (KEEP == 0 && far) {                               // weights are 2^(s - base - less)
                const float base = sh.base[wave * 16 + c];
#pragma unroll
                for (int n = 0; n < 4; ++n) s[n] -= base;
            }
            if (mixed) mask_scores<true, false>(s, sh.seg, own, last - k0, lane);
            else mask_scores<false, false>(s, sh.seg, own, last - k0, lane);
        }
    };
    // weights and dp of a tile in LDS
    auto weigh = [&](int t, bool mixed, f32x4 (&s)[4], f32x4 (&dp)[4], f32x4 (&slope)[CAP ? 4 : 1]) {
        score(t, mixed, s, slope);
        first_product<T, DP>(dp, df, rd, sh.v);
        if (KEEP > 0 && far) {                                    // weights follow when all tiles have been seen
#pragma unroll
            for (int n = 0; n < 4; ++n) s[n] -= less;
            return;
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[n][r] = __builtin_amdgcn_exp2f(s[n][r] - less);
    };
    auto add_seen = [&](const f32x4 (&s)[4], const f32x4 (&dp)[4]) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) seen += weighed(s[n][r], dp[n][r]);
    };
    // ds in place of the weights, and what they add to the table's gradient
    auto table_sums = [&](int t, f32x4 (&s)[4], const f32x4 (&dp)[4]) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[n][r] = weighed(s[n][r], dp[n][r] - delta);
        if constexpr (!TABLE) return;
        const int flat = flat_of(t);
        if (flat >= 0) {
            if (flat != flat_bucket) {
                if (flat_bucket >= 0) add_bucket(sh.bucket[wave], flat_bucket, flat_sum, lane);
                flat_bucket = flat, flat_sum = 0.f;
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) flat_sum += (s[n][0] + s[n][1]) + (s[n][2] + s[n][3]);
        } else {
            table_near(a, s, wq0 - t * kTile, sh.strip[wave], my_dist, sh.bucket[wave], sh.border, lane);
        }
    };
    auto put_bias = [&](int t) {
        const int hi = q0 + kTile - 1 - t * kTile;
        if (flat_of(t) < 0 && tid < 2 * kTile - 1) sh.bias[tid] = sh.table[bucket_of(a.bk, sh.border, hi - tid)];
    };
    // DELTA: only sum p dp; else the gradients, with that sum on the way where the one tile holds it all
    auto walk = [&](auto delta_only) {
        constexpr bool DELTA = decltype(delta_only)::value;
        auto after = [&](int t) { return next_tile(t + 1, t1, mk); };
        int round = tfirst, t = set ? after(round) : round;       // the first set's tile and this one's
        if (AHEAD && !loaded && t < t1) load(t);
        loaded = false;
        while (round < t1) {
            const bool there = SPLIT == 1 || t < t1, mixed = there && tile_mixed(mk, t);
            if (!AHEAD && there) load(t);
            __syncthreads();
            if (there) {
                feed.template put<false>(sh.k, sh.v, sh.seg, !whole(t, q0, mixed), nullptr);
                put_bias(t);
            }
            round = after(SPLIT > 1 ? after(round) : round);
            const int tn = set ? after(round) : round;
            if (AHEAD && tn < t1) load(tn);
            __syncthreads();
            if (there && sees(t)) {
                f32x4 s[MEND && !DELTA ? 2 : 1][4], dp[4], slope[CAP ? 4 : 1];
                weigh(t, mixed, s[0], dp, slope);
                if (DELTA || MEND || one_tile) add_seen(s[0], dp);
                if constexpr (!DELTA) {
                    if (one_tile) delta = group_sum(seen);
                    if constexpr (MEND) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) s[1][n] = s[0][n];
                    }
                    table_sums(t, s[0], dp);
                    if constexpr (CAP) {
#pragma unroll
                        for (int m = 0; m <= (MEND ? 1 : 0); ++m)
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int r = 0; r < 4; ++r) s[m][n][r] = weighed(s[m][n][r], slope[n][r]);
                    }
                    second_products<T, DP>(dq, s, rd, sh.k);
                }
            }
            t = tn;
        }
        if constexpr (DELTA) {
            delta = group_sum(seen);
            if constexpr (SPLIT > 1) {
                __syncthreads();                                  // the bias has been read
                sh.bias[wave * 16 + c] = delta;
                __syncthreads();
                delta = sets[0].bias[wave * 16 + c] + sets[1].bias[wave * 16 + c];
            }
        }
    };
    auto load_first = [&] {
        const int t = set ? next_tile(tfirst + 1, t1, mk) : tfirst;
        if (AHEAD || EARLY) load(t < t1 ? t : 0), loaded = true;
    };
    load_first();
    if (KEEP == 0 && far) {                          // a walk over the keys for the maximum and sum of rows that are far
        float top = -INFINITY, sum = 0.f;
        for (int t = tfirst; t < t1; t = next_tile(t + 1, t1, mk)) {
            const bool mixed = tile_mixed(mk, t);
            load(t);
            __syncthreads();
            feed.template put<false>(sh.k, sh.v, sh.seg, !whole(t, q0, mixed), nullptr);
            put_bias(t);
            __syncthreads();
            if (!sees(t)) continue;
            f32x4 s[4], slope[CAP ? 4 : 1];
            score(t, mixed, s, slope);
            float most = top;
#pragma unroll
            for (int n = 0; n < 4; ++n) most = fmaxf(most, fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])));
            most = group_max(most);
            const float from = most == -INFINITY ? 0.f : most;
            sum *= __builtin_amdgcn_exp2f(top - from);
            top = most;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(s[n][r] - from);
        }
        sum = group_sum(sum);
        if (live && far_lse(lse)) {
            less = __builtin_amdgcn_logf(sum);
            if (g == 0) sh.base[wave * 16 + c] = top;
            if (g == 0 && set == 0) a.far[2 * stat] = top, a.far[2 * stat + 1] = less;
        }
        __syncthreads();
        load_first();
    }
    if constexpr (KEEP > 0) {
        f32x4 s[KEEP][4], dp[KEEP][4], none[1];
        int tile[KEEP];
        int t = tfirst;
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            tile[i] = t;
            if (t < t1) {
                const bool mixed = tile_mixed(mk, t);
                const int tn = next_tile(t + 1, t1, mk);
                if (!EARLY) load(t);
                __syncthreads();
                feed.template put<false>(sh.k, sh.v, sh.seg, !whole(t, q0, mixed), nullptr);
                put_bias(t);
                if (EARLY && i + 1 < KEEP && tn < t1) load(tn);
                __syncthreads();
                if (sees(t)) {
                    weigh(t, mixed, s[i], dp[i], none);
                    if (!far) add_seen(s[i], dp[i]);
                }
                t = tn;
            }
        }
        if (far) {                                   // s are scores less the rounded lse: what is left of a row's maximum, and its sum
            const bool mine = live && far_lse(lse);
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (tile[i] < t1 && sees(tile[i]))
#pragma unroll
                    for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(fmaxf(s[i][n][0], s[i][n][1]), fmaxf(s[i][n][2], s[i][n][3])));
            top = group_max(top);
            top = mine ? top : 0.f;
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (tile[i] < t1 && sees(tile[i]))
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        s[i][n] -= top;
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(s[i][n][r]);
                    }
            sum = group_sum(sum);
            const float low = mine ? __builtin_amdgcn_logf(sum) : 0.f;
            if (mine && g == 0) a.far[2 * stat] = less + top, a.far[2 * stat + 1] = low;
#pragma unroll
            for (int i = 0; i < KEEP; ++i)
                if (tile[i] < t1 && sees(tile[i])) {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[i][n][r] = __builtin_amdgcn_exp2f(s[i][n][r] - low);
                    add_seen(s[i], dp[i]);
                }
        }
        delta = group_sum(seen);
        auto load_keys = [&](int n) {
            feed.template load<false>(kp + n * kTile * a.k.sr, a.k.sr, kp, a.k.sr, n * kTile, a.length, seg, a.dim);
        };
        bool there = true;                           // the keys of the last tile are in LDS still
#pragma unroll
        for (int i = KEEP - 1; i >= 0; --i) {
            if (tile[i] >= t1) continue;
            if (!there) {
                if (!EARLY) load_keys(tile[i]);
                __syncthreads();
                feed.template put<false, false>(sh.k, sh.v, sh.seg, !whole(tile[i], q0, tile_mixed(mk, tile[i])), nullptr);
                __syncthreads();
            }
            there = false;
            if (EARLY && i > 0) load_keys(tile[i - 1]);
            if (sees(tile[i])) {
                table_sums(tile[i], s[i], dp[i]);
                second_product<T, DP>(dq[0], s[i], rd, sh.k);
            }
        }
    } else {
        if constexpr (TABLE) {
            if (!one_tile) walk(std::true_type{});
        }
        walk(std::false_type{});
        if constexpr (SPLIT > 1) {
            __syncthreads();
            if (set) {
                hand_over(sets[1].k, dq[0], wave, lane);          // and the values behind
                if constexpr (MEND) {
                    hand_over(sets[0].k, dq[1], wave, lane);
                    seen = group_sum(seen);
                    sets[1].bias[wave * 16 + c] = seen;
                }
            }
            __syncthreads();
            if (!set) {
                take_over(sets[1].k, dq[0], 1.f, 1.f, wave, lane);
                if constexpr (MEND) take_over(sets[0].k, dq[1], 1.f, 1.f, wave, lane);
            }
        }
        if constexpr (MEND) {
            seen = group_sum(seen) + (SPLIT > 1 ? sets[SPLIT - 1].bias[wave * 16 + c] : 0.f);
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) dq[0][dt] += (delta - seen) * dq[1][dt];
            delta = seen;
        }
    }
    __syncthreads();
    if (set == 0 && wq0 < a.length) {
        T* const dqp = static_cast<T*>(a.dq.data) + batch * a.dq.sb + head * a.dq.sh + wq0 * a.dq.sr;
        store_rows<T, DP, UNIT>(sh.k + wave * 16 * S::RB, dq[0], a.scale, dqp, a.dq.sr, a.length - wq0, a.dim, lane);
        if (g == 0 && q < a.length) a.delta[stat] = delta;
    }
    if constexpr (TABLE) {
        if (flat_bucket >= 0) add_bucket(sh.bucket[wave], flat_bucket, flat_sum, lane);
        __syncthreads();
        // bucket b of a side: the distances from its border to the next one's, eight lanes to a bucket; keys after the
        // query count as distance 0 where there is one side
        const float* const row = dist + kNear;
        constexpr int W = 2 * kNear + 1;
        auto at = [&](int n) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kRows; w += 4) sum += (row[w * W + n] + row[(w + 1) * W + n]) + (row[(w + 2) * W + n] + row[(w + 3) * W + n]);
            return sum;
        };
        for (int b = threadIdx.x >> 3; b < buckets; b += kBlock * SPLIT / 8) {
            const int sub = tid & 7;
            const bool after = b >= a.bk.side;
            const int i = (after ? b - a.bk.side : b) - a.bk.exact, most = after ? -near_lo : near_hi;
            int from = i < 0 ? i + a.bk.exact : i == 0 ? a.bk.exact : sh.border[i - 1];
            int to = i < 0 ? from + 1 : i < a.bk.borders ? sh.border[i] : kNear + 1;
            to = to < most + 1 ? to : most + 1;
            if (after && from == 0) from = 1;
            float sum = sub < kRows ? sets[sub / kWavesPerBlock].bucket[sub % kWavesPerBlock][b] : 0.f;
            for (int n = from + sub; n < to; n += 8) sum += at(after ? -n : n);
            if (b == 0 && !a.bk.two_sided)
                for (int n = 1 + sub; n <= -near_lo; n += 8) sum += at(-n);
            sum = eight_lanes_total(sum);
            if (sub == 0) a.part[((int64_t)head * a.parts + batch * nqt + qt) * buckets + b] = sum;
        }
    }
}

}  // namespace

void attend_backward_queries(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s)
{
    a.items = a.batch * a.heads * att_blocks(a.length, kTile);
    a.by_tiles = FastDiv::of(att_blocks(a.length, kTile)), a.by_heads = FastDiv::of(a.heads), a.by_group = FastDiv::of(a.group);
    const bool few = two_sets(a);
    by_shape_and_cap(c, unit, [&](auto type, auto dp, auto u, auto cap) {
        constexpr int DP = decltype(dp)::value;
        constexpr int WAVES = Shape<decltype(type), DP>::RB <= 128 ? 3 : 2;
        auto go = [&](auto table, auto keep, auto split) {
            constexpr int KEEP = decltype(keep)::value, SPLIT = decltype(split)::value;
            const size_t dist = a.part ? SPLIT * kWavesPerBlock * (2 * kNear + 1) * sizeof(float) : 0;
            k_attend_dq<decltype(type), DP, decltype(u)::value, decltype(cap)::value, (KEEP > 2 || SPLIT > 1 ? 2 : WAVES),
                        decltype(table)::value, KEEP, SPLIT><<<att_grid(a.items), dim3(kBlock * SPLIT), dist, s>>>(a);
        };
        const std::integral_constant<int, 0> none;
        const std::integral_constant<int, 1> one;
        if constexpr (Shape<decltype(type), DP>::RB <= 256) {
            const std::integral_constant<int, 2> two;
            if (few) return a.part ? go(std::true_type{}, none, two) : go(std::false_type{}, none, two);
        }
        if (!a.part) return go(std::false_type{}, none, one);
        // kept are the tiles of histories of up to 256 positions, where there are no slopes to keep as well and registers
        // for it all: rows of 512 bytes leave none
        if constexpr (!decltype(cap)::value && Shape<decltype(type), DP>::RB <= 256) {
            const int tiles = att_blocks(a.length, kTile);
            if (tiles == 2) return go(std::true_type{}, std::integral_constant<int, 2>{}, one);
            if (tiles == 3 || tiles == 4) return go(std::true_type{}, std::integral_constant<int, 4>{}, one);
        }
        go(std::true_type{}, none, one);
    });
}

}  // namespace gram
