// Attention over item histories, forward.
//
//   z_ij = scale q_i.k_j    c_ij = cap tanh(z_ij / cap) or z_ij    s_ij = c_ij + table[head, bucket(i - j)]
//   visible(i, j):  segment_i = segment_j >= 0  and  (not causal or j <= i or j < prefix)
//   o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - lse_i) over the visible j
//
// One pass over the keys with the running maximum and sum of the softmax; scores and weights stay in registers.
//
// 1024 x 200 positions, 8 heads of 128, causal, a table, bf16: 0.53 ms, where reading q, k, v and writing o would take 0.36 at a
// large copy's rate.  Half of a wave's life is waiting (barriers and LDS, three waves per SIMD), a fifth vector arithmetic.  float32, 8
// heads of 64 (as many bytes): 1.05 ms, of which the products over whole tiles would take 0.57 at a large product's rate; 256 x 200,
// 8 heads of 128: 0.53, and 0.28.
#include "gram_attend.h"

namespace gram {

namespace {

template <typename T, int DP> struct FwdShared {
    __attribute__((aligned(1024))) unsigned char k[Shape<T, DP>::TILE], v[Shape<T, DP>::TILE];
    __attribute__((aligned(16))) int seg[kTile];
    float bias[2 * kTile];
    float table[kMaxBorders];
    int border[kMaxBorders];
    TileMarks marks;
};

// One block: 64 queries of one head, 16 to a wave.
template <typename T, int DP, int UNIT, bool CAP, int WAVES, int SPLIT>
__global__ __launch_bounds__(kBlock * SPLIT, WAVES) void k_attend(const AttArgs a)
{
    using S = Shape<T, DP>;
    // the next tile's loads under way while this one is worked on; at 256 bytes a row the registers for it spill (1024 x 200, 8
    // heads of 128: 0.81 ms, and 0.53 without)
    constexpr bool AHEAD = S::RB < 256;
    __shared__ FwdShared<T, DP> sets[SPLIT];
    const int set = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kBlock) : 0;
    FwdShared<T, DP>& sh = sets[set];
    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int tid = threadIdx.x % kBlock, lane = lane_id();
    const int nqt = (a.length + kTile - 1) / kTile;
    const int rows_item = (int)a.by_tiles.quotient((uint32_t)item);       // history and head
    const int qt = nqt - 1 - (item - rows_item * nqt);                 // the longest rows of a causal mask first
    const int batch = (int)a.by_heads.quotient((uint32_t)rows_item), head = rows_item - batch * a.heads;
    const int kvh = (int)a.by_group.quotient((uint32_t)head);
    const int c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int q0 = qt * kTile, wq0 = q0 + wave * 16, q = wq0 + c;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = prefix_of(a.prefix, batch, a.length);
    const T* const kp = static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh;
    const T* const vp = static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh;

    u32x4 qf[S::KK];
    const int qseg = q < a.length ? row_segment(seg, q, a.length) : kNoSegOwner;
    load_owner<T, DP, UNIT>(qf, static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh + wq0 * a.q.sr, a.q.sr,
                            a.length - wq0, a.dim, qseg >= 0, lane);
    const int own = qseg < 0 ? kNoSegOwner : qseg;
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

    const Reader<T, DP> rd(lane);
    Feed<T, DP, UNIT> feed(tid);
    const float z2 = a.scale * kLog2e, zc = CAP ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    int last = a.length;                                 // keys before it are in sight, segments aside
    if (a.causal) {
        last = q + 1 > prefix ? q + 1 : prefix;
        last = last < a.length ? last : a.length;
    }
    // whether all pairs of the tile with rows from `row` on are visible
    auto whole = [&](int t, int row, bool mixed) {
        const int k1 = t * kTile + kTile;
        return !mixed && k1 <= a.length && (!a.causal || k1 - 1 <= row || k1 <= prefix);
    };
    auto load = [&](int t) {
        const int k0 = t * kTile;
        feed.load(kp + k0 * a.k.sr, a.k.sr, vp + k0 * a.v.sr, a.v.sr, k0, a.length, seg, a.dim);
    };

    f32x4 o[S::DT];
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto after = [&](int t) { return next_tile(t + 1, t1, mk); };
    int round = next_tile(0, t1, mk), t = set ? after(round) : round;     // the first set's tile and this one's
    if (AHEAD && t < t1) load(t);
    while (round < t1) {
        const bool there = SPLIT == 1 || t < t1, mixed = there && tile_mixed(mk, t);
        const int k0 = t * kTile, hi = q0 + kTile - 1 - k0;   // the largest distance of the block's pairs
        const int flat = a.bk.side ? uniform_bucket(a.bk, hi - 2 * kTile + 2, hi) : 0;
        if (!AHEAD && there) load(t);
        __syncthreads();                                      // the tile before has been read
        if (there) {
            feed.template put<true>(sh.k, sh.v, sh.seg, !whole(t, q0, mixed), nullptr);
            if (flat < 0 && tid < 2 * kTile - 1)
                sh.bias[tid] = sh.table[bucket_of(a.bk, sh.border, hi - tid)];
        }
        round = after(SPLIT > 1 ? after(round) : round);
        const int tn = set ? after(round) : round;
        if (AHEAD && tn < t1) load(tn);
        __syncthreads();
        if (there && wq0 < a.length && !(a.causal && k0 > wq0 + 15 && k0 >= prefix)) {
            f32x4 s[4], slope[CAP ? 4 : 1];
            first_product<T, DP>(s, qf, rd, sh.k);
            to_scores<CAP>(s, slope, zc, cap2, z2, a.bk.side && flat >= 0 ? sh.table[flat] : 0.f);
            if (flat < 0) add_bias(s, &sh.bias[4 * g - (q - q0) + kTile - 1]);
            if (!whole(t, wq0, mixed)) {
                if (mixed) mask_scores<true, false>(s, sh.seg, own, last - k0, lane);
                else mask_scores<false, false>(s, sh.seg, own, last - k0, lane);
            }
            float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
            for (int n = 1; n < 4; ++n) mx = fmaxf(mx, fmaxf(fmaxf(s[n][0], s[n][1]), fmaxf(s[n][2], s[n][3])));
            mx = group_max(mx);
            if (__any(mx > top)) {
                const float nt = fmaxf(mx, top);
                const float shrink = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - nt);
                top = nt;
                total *= shrink;
#pragma unroll
                for (int dt = 0; dt < S::DT; ++dt) o[dt] *= shrink;
            }
            const float base = top == -INFINITY ? 0.f : top;  // a row that has seen nothing so far
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][r] = __builtin_amdgcn_exp2f(s[n][r] - base);
                    total += s[n][r];
                }
            second_product<T, DP>(o, s, rd, sh.v);
        }
        t = tn;
    }
    total = group_sum(total);
    __syncthreads();                                              // the tiles have been read
    if constexpr (SPLIT > 1) {
        unsigned char* const room = sets[1].k;                    // and the values behind
        float* const stats = &sets[1].bias[2 * (wave * 16 + c)];
        if (set) {
            hand_over(room, o, wave, lane);
            stats[0] = top, stats[1] = total;
        }
        __syncthreads();
        if (set) return;
        const float other = stats[0], most = fmaxf(top, other);
        const float mine = top == most ? 1.f : __builtin_amdgcn_exp2f(top - most);
        const float theirs = other == most ? 1.f : __builtin_amdgcn_exp2f(other - most);
        take_over(room, o, mine, theirs, wave, lane);
        total = total * mine + stats[1] * theirs;
        top = most;
    }
    if (wq0 < a.length) {
        const bool empty = top == -INFINITY && total == 0.f;
        T* const op = static_cast<T*>(a.o.data) + batch * a.o.sb + head * a.o.sh + wq0 * a.o.sr;
        store_rows<T, DP, UNIT>(sh.k + wave * 16 * S::RB, o, empty ? 0.f : 1.f / total, op, a.o.sr, a.length - wq0, a.dim, lane);
        if (a.lse && g == 0 && q < a.length)
            a.lse[((int64_t)batch * a.heads + head) * a.length + q] = empty ? -INFINITY : row_lse(top, total);
    }
}

}  // namespace

void attend_forward(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s)
{
    a.items = a.batch * a.heads * att_blocks(a.length, kTile);
    a.by_tiles = FastDiv::of(att_blocks(a.length, kTile)), a.by_heads = FastDiv::of(a.heads), a.by_group = FastDiv::of(a.group);
    by_shape_and_cap(c, unit, [&](auto type, auto dp, auto u, auto cap) {
        constexpr int DP = decltype(dp)::value;
        // blocks per CU that registers allow: accumulators, fragments and the tile under way grow with the row's bytes
        constexpr int WAVES = Shape<decltype(type), DP>::RB <= 128 ? 4 : Shape<decltype(type), DP>::RB <= 256 ? 3 : 2;
        auto go = [&](auto split) {
            constexpr int SPLIT = decltype(split)::value;
            k_attend<decltype(type), DP, decltype(u)::value, decltype(cap)::value, (SPLIT > 1 ? 2 : WAVES), SPLIT>
                <<<att_grid(a.items), dim3(kBlock * SPLIT), 0, s>>>(a);
        };
        if constexpr (Shape<decltype(type), DP>::RB <= 256)
            if (two_sets(a)) return go(std::integral_constant<int, 2>{});
        go(std::integral_constant<int, 1>{});
    });
}

}  // namespace gram
