// Attention over item histories of at most 64 positions, the whole backward pass in one launch (notation of
// gram_attend_fwd.hip and gram_attend_dq.hip).
//
// A block takes one history and key head: queries, keys, values and dout of a head lie in LDS as one tile each, scores and
// weights are worked out once (the passes of longer histories do so up to three times), by waves that own 16 queries; the
// weights and their gradients then change hands through LDS to waves that own 16 keys.  delta comes from the tile itself.
//
// 128 x 55, 20 heads of 20, bf16, a table: 30 us, 34 MB at 1.1 TB/s; bound by one tile's chain of loads, products and exchanges,
// which up to four blocks per CU overlap.  1024 x 50, 4 heads of 64: 70 us, of that the table's gradient 14.
#include "gram_attend.h"

namespace gram {

namespace {

constexpr int kShortDist = 80;      // distances of one tile's pairs lie within (table_near touches 76 below the first)

template <typename T, int DP> struct ShortShared {
    using S = Shape<T, DP>;
    using P = Shape<T, kTile>;
    __attribute__((aligned(1024))) unsigned char q[S::TILE], d[S::TILE], k[S::TILE], v[S::TILE];
    __attribute__((aligned(1024))) unsigned char w[P::TILE], dz[P::TILE];      // weights and dz, [query][key]
    __attribute__((aligned(16))) int seg[kTile];
    uint32_t bad[2];
    float bias[2 * kTile];
    float table[kMaxBorders];
    int border[kMaxBorders];
    float bucket[kWavesPerBlock][kMaxBorders];
    float dist[kWavesPerBlock][2 * kShortDist + 1];
};

// A wave's strips of table_near lie in its own rows of the tile of weights, which are written after them.
template <typename T> __device__ __forceinline__ float (*strips(unsigned char* weights, int wave))[kStrip]
{
    static_assert(4 * kStrip * sizeof(float) <= 16 * Shape<T, kTile>::RB, "four strips in sixteen rows");
    return reinterpret_cast<float (*)[kStrip]>(weights + wave * 16 * Shape<T, kTile>::RB);
}

// Columns c of a first product (queries) as rows of a [query][key] tile.
template <typename T> __device__ __forceinline__ void put_weights(unsigned char* tile, const f32x4 (&w)[4], int row, int g)
{
    using P = Shape<T, kTile>;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        if constexpr (sizeof(T) == 2) {
            const u32x2 h = {pack_bf16x2(w[n][0], w[n][1]), pack_bf16x2(w[n][2], w[n][3])};
            *reinterpret_cast<u32x2*>(tile + row * P::RB + (((2 * n + (g >> 1)) ^ swz<T, P::NCH>(row)) * 16) + (g & 1) * 8) = h;
        } else {
            *reinterpret_cast<f32x4*>(tile + row * P::RB + (((4 * n + g) ^ swz<T, P::NCH>(row)) * 16)) = w[n];
        }
    }
}

// acc[dt] += (tile of rows)^T . (sixteen columns of the [query][key] tile, which lie at `col`)
template <typename T, int DP>
__device__ __forceinline__ void over_queries(f32x4 (&acc)[DP / 16], const Reader<T, DP>& rd, const unsigned char* rows,
                                             const unsigned char* weights, int col)
{
    constexpr int STEPS = sizeof(T) == 2 ? 2 : 4;
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        u32x4 b;
        if constexpr (sizeof(T) == 2) b = Reader<T, kTile>::column_frag2(weights, n, col);
        else b = Reader<T, kTile>::column_frag1(weights, n, col);
#pragma unroll
        for (int dt = 0; dt < DP / 16; ++dt) {
            if constexpr (sizeof(T) == 2) acc[dt] = mma<T>(rd.col_frag2(rows, n, dt), b, acc[dt]);
            else acc[dt] = mma<T>(rd.col_frag1(rows, n, dt), b, acc[dt]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Blocks per CU: LDS holds four where rows have 64 bytes, three at 128 (bf16), two or one beyond.  Registers for four are
// worth a few spilled ones (1024 x 50, 8 heads of 32: 80 us and 86 with three) unless the cap's slopes stand in them too (2048
// x 50: 148 us with three, 165 with four); the compiler's choice at 128 bytes beats a limit for three (74 and 87 us, heads of 64).
template <typename T, int DP, int UNIT, bool CAP>
__global__ __launch_bounds__(kBlock, (Shape<T, DP>::RB > 64 ? 2 : CAP ? 3 : 4)) void k_attend_short(const AttArgs a)
{
    using S = Shape<T, DP>;
    __shared__ ShortShared<T, DP> sh;
    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int tid = threadIdx.x, lane = lane_id();
    const int batch = (int)a.by_heads.quotient((uint32_t)item), kvh = item - batch * a.kv_heads;
    const int c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int w0 = wave * 16, row = w0 + c;                     // the wave's rows, as queries and as keys
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = prefix_of(a.prefix, batch, a.length);
    const int rseg = row < a.length ? row_segment(seg, row, a.length) : kNoSegOwner;
    const int own = rseg < 0 ? kNoSegOwner : rseg;
    const bool want_table = a.part != nullptr;
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    if (tid < kMaxBorders) sh.border[tid] = kernel_borders()[tid];
    if (tid < 2) sh.bad[tid] = 0u;
    int last = a.length;
    if (a.causal) {
        last = row + 1 > prefix ? row + 1 : prefix;
        last = last < a.length ? last : a.length;
    }
    if (row >= a.length) last = 0;
    const int flat = a.bk.side ? uniform_bucket(a.bk, 1 - kTile, kTile - 1) : 0;

    Feed<T, DP, UNIT> feed(tid);
    feed.load(static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh, a.k.sr,
              static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh, a.v.sr, 0, a.length, seg, a.dim);
    Feed<T, DP, UNIT> queries(tid);                             // of the first head, on their way with the keys
    float lse_ahead = 0.f;
    auto load_queries = [&](int h) {
        const int head = kvh * a.group + h;
        queries.load(static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh, a.q.sr,
                     static_cast<const T*>(a.dout.data) + batch * a.dout.sb + head * a.dout.sh, a.dout.sr, 0, a.length, seg, a.dim);
        lse_ahead = a.lse[((int64_t)batch * a.heads + head) * a.length + (row < a.length ? row : a.length - 1)];
    };
    load_queries(0);
    // whether any pair is masked, by the forward pass's rule: where none is, it has left non-finite values of k and v in place and
    // what they reach is not finite; elsewhere they are zeros here, and the rows that see them have NaN for their lse
    const int one = __builtin_amdgcn_readfirstlane(feed.seg);
    const bool masked = one == kNoSeg || !__all(feed.seg == one) || (a.causal && prefix < kTile);
    feed.template put<false>(sh.k, sh.v, sh.seg, masked, nullptr);

    const Reader<T, DP> rd(lane);
    const int own_keys = Reader<T, kTile>::column(lane, wave);   // the wave's columns of weights
    f32x4 dk[S::DT], dv[S::DT];
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) dk[dt] = dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float z2 = a.scale * kLog2e, zc = CAP ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;

    for (int h = 0; h < a.group; ++h) {
        const int head = kvh * a.group + h;
        const float lse = lse_ahead;
        if (tid < buckets) sh.table[tid] = to_log2(a.table[(int64_t)head * buckets + tid]);
        __syncthreads();                                        // the last head's tiles have been read; table and bad are set
        queries.template put<false>(sh.q, sh.d, sh.seg, masked, sh.bad);
        if (flat < 0 && tid < 2 * kTile - 1) sh.bias[tid] = sh.table[bucket_of(a.bk, sh.border, kTile - 1 - tid)];
        if (want_table) {
            for (int i = tid; i < kWavesPerBlock * (2 * kShortDist + 1); i += kBlock) (&sh.dist[0][0])[i] = 0.f;
            for (int i = lane; i < 4 * kStrip; i += kWave) strips<T>(sh.w, wave)[0][i] = 0.f;
            if (tid < kMaxBorders)
                for (int w = 0; w < kWavesPerBlock; ++w) sh.bucket[w][tid] = 0.f;
        }
        __syncthreads();
        // a query that holds a non-finite value, or sees one, has NaN for its statistics: the pairs that it sees are NaN
        float less = lse == -INFINITY ? 0.f : to_log2(lse);
        const bool spoilt = (sh.bad[w0 >> 5] >> (row & 31)) & 1;
        if (spoilt) less = NAN;
        f32x4 s[4], dp[4], slope[CAP ? 4 : 1];
        {
            u32x4 f[S::KK];
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) f[kk] = rd.row_frag(sh.q, wave, kk);
            first_product<T, DP>(s, f, rd, sh.k);
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) f[kk] = rd.row_frag(sh.d, wave, kk);
            first_product<T, DP>(dp, f, rd, sh.v);
        }
        to_scores<CAP>(s, slope, zc, cap2, z2, a.bk.side && flat >= 0 ? sh.table[flat] : 0.f);
        if (flat < 0) add_bias(s, &sh.bias[4 * g - row + kTile - 1]);
#pragma unroll
        for (int n = 0; n < 4; ++n) s[n] -= less;
        if (masked) mask_scores<true, false>(s, sh.seg, own, last, lane);
        const bool far = own >= 0 && far_lse(lse);
        if (__any(far)) {                                       // what is left of their maximum, and their sum
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])));
            top = group_max(top);
            top = far && !spoilt ? top : 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                s[n] -= top;
#pragma unroll
                for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(s[n][r]);
            }
            const float low = __builtin_amdgcn_logf(group_sum(sum));
#pragma unroll
            for (int n = 0; n < 4; ++n) s[n] -= far && !spoilt ? low : 0.f;
        }
        float delta = less - less;                              // NaN if the statistics are not finite
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[n][r] = __builtin_amdgcn_exp2f(s[n][r]);
                delta += weighed(s[n][r], dp[n][r]);
            }
        delta = group_sum(delta);
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) dp[n][r] = weighed(s[n][r], dp[n][r] - delta);
        if (want_table) {
            if (flat >= 0) {
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < 4; ++n) sum += (dp[n][0] + dp[n][1]) + (dp[n][2] + dp[n][3]);
                add_bucket(sh.bucket[wave], flat, sum, lane);
            } else {
                table_near(a, dp, w0, strips<T>(sh.w, wave), &sh.dist[wave][kShortDist], sh.bucket[wave], sh.border, lane);
            }
        }
        if constexpr (CAP) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) dp[n][r] = weighed(dp[n][r], slope[n][r]);
        }
        put_weights<T>(sh.w, s, row, g);
        put_weights<T>(sh.dz, dp, row, g);
        f32x4 dq[S::DT];
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) dq[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        second_product<T, DP>(dq, dp, rd, sh.k);
        __syncthreads();
        over_queries<T, DP>(dv, rd, sh.d, sh.w, own_keys);
        over_queries<T, DP>(dk, rd, sh.q, sh.dz, own_keys);
        if (want_table) {
            const float* const at0 = &sh.dist[0][kShortDist];
            constexpr int W = 2 * kShortDist + 1;
            auto at = [&](int n) { return (at0[n] + at0[W + n]) + (at0[2 * W + n] + at0[3 * W + n]); };
            for (int b = tid >> 3; b < buckets; b += kBlock / 8) {
                const int sub = tid & 7;
                const bool after = b >= a.bk.side;
                const int i = (after ? b - a.bk.side : b) - a.bk.exact;
                int from = i < 0 ? i + a.bk.exact : i == 0 ? a.bk.exact : sh.border[i - 1];
                int to = i < 0 ? from + 1 : i < a.bk.borders ? sh.border[i] : kTile;
                to = to < kTile ? to : kTile;
                if (after && from == 0) from = 1;
                float sum = sub < kWavesPerBlock ? sh.bucket[sub][b] : 0.f;
                for (int n = from + sub; n < to; n += 8) sum += at(after ? -n : n);
                if (b == 0 && !a.bk.two_sided)
                    for (int n = 1 + sub; n < kTile; n += 8) sum += at(-n);
                sum = eight_lanes_total(sum);
                if (sub == 0) a.part[((int64_t)head * a.parts + batch) * buckets + b] = sum;
            }
        }
        if (h + 1 < a.group) load_queries(h + 1);
        __syncthreads();                                        // the tiles have been read
        if (tid < 2) sh.bad[tid] = 0u;
        if (w0 < a.length) {
            T* const dqp = static_cast<T*>(a.dq.data) + batch * a.dq.sb + head * a.dq.sh + w0 * a.dq.sr;
            store_rows<T, DP, UNIT>(sh.q + wave * 16 * S::RB, dq, a.scale, dqp, a.dq.sr, a.length - w0, a.dim, lane);
        }
    }
    if (w0 < a.length) {
        T* const dkp = static_cast<T*>(a.dk.data) + batch * a.dk.sb + kvh * a.dk.sh + w0 * a.dk.sr;
        T* const dvp = static_cast<T*>(a.dv.data) + batch * a.dv.sb + kvh * a.dv.sh + w0 * a.dv.sr;
        unsigned char* const room = sh.d + wave * 16 * S::RB;
        store_rows<T, DP, UNIT>(room, dk, a.scale, dkp, a.dk.sr, a.length - w0, a.dim, lane);
        store_rows<T, DP, UNIT>(room, dv, 1.f, dvp, a.dv.sr, a.length - w0, a.dim, lane);
    }
}

}  // namespace

bool attend_backward_short(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s)
{
    // Four tiles of rows and two of weights have to fit a CU's LDS: float32 rows of more than 64 elements do not.  Against a launch
    // for the queries and one for the keys: 64 x 50, 4 heads of 128, 12 us and 17, with the table's gradient 17 and 21; 1024 x 60, 4
    // heads of 64 in float32, 205 and 221.
    if (a.length > kTile || (c.dtype == GRAM_F32 && c.head_dim > 64)) return false;
    // Rows of 256 bytes leave room for one block per CU, which a second one waits for: beyond that many blocks short histories, whose
    // tile is mostly empty, are faster in two launches, and so are most with the table's gradient, which the waves work out in
    // turn with their barriers.  1024 histories, 4 heads of 128, one launch and two, with that gradient and without: 20
    // positions 164 us and 123, 129 and 103; 50 positions 180 and 161, 145 and 148; 64 positions, 2 key heads for 8, 252 and 266 with it.
    if (c.head_dim > 64 && a.batch * a.kv_heads > kFewBlocks && (a.length <= 32 || (a.part && a.length <= 56))) return false;
    a.items = a.batch * a.kv_heads;
    a.by_heads = FastDiv::of(a.kv_heads);
    by_shape_and_cap(c, unit, [&](auto type, auto dp, auto u, auto cap) {
        using T = decltype(type);
        constexpr int DP = decltype(dp)::value;
        if constexpr (Shape<T, DP>::RB <= 256)
            k_attend_short<T, DP, decltype(u)::value, decltype(cap)::value><<<att_grid(a.items), dim3(kBlock), 0, s>>>(a);
    });
    return true;
}

}  // namespace gram
