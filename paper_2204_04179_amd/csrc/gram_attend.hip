// Attention over item histories, forward and backward.
//
//   z_ij = scale q_i.k_j    c_ij = cap tanh(z_ij / cap) or z_ij    s_ij = c_ij + table[head, bucket(i - j)]
//   visible(i, j):  segment_i = segment_j >= 0  and  (not causal or j <= i or j < prefix)
//   p_ij = exp(s_ij - lse_i) over the visible j,  o_i = sum_j p_ij v_j
//   dp_ij = do_i.v_j   delta_i = sum_j p_ij dp_ij   ds_ij = p_ij (dp_ij - delta_i)   dz_ij = ds_ij (1 - (c_ij / cap)^2)
//   dq_i = scale sum_j dz_ij k_j   dk_j = scale sum_i dz_ij q_i   dv_j = sum_i p_ij do_i
//   dtable[head, b] = sum of ds over the pairs of bucket b
//
// One pass over the keys with the running maximum and sum of the softmax; scores, weights and their gradients stay in
// registers.  No sum goes through an atomic whose order could change: a row of every result has one writer.
#include <math.h>

#include "gram_attend.h"

namespace gram {

namespace {

// Work item of a block: the blocks of one head of one history share its keys, so neighbours in this order go to one XCD
// (blocks are dealt to the 8 XCDs in turn).
__device__ __forceinline__ int xcd_item(int items)
{
    const int each = (items + 7) / 8;
    const int item = (int)(blockIdx.x & 7) * each + (int)(blockIdx.x >> 3);
    return (int)(blockIdx.x >> 3) < each && item < items ? item : -1;
}

struct TileMarks {
    uint32_t active[kAttMaxTiles / 32], mixed[kAttMaxTiles / 32];
    int lo, hi, same;
};

// Marks the tiles [t0, t1) of streamed rows that hold a row of a segment in the owner rows' range, and among them those
// with any row that is not of the one segment all owner rows have.  own: this lane's segments of its owner rows that exist.
template <int N>
__device__ __forceinline__ void mark_tiles(TileMarks& mk, const int* __restrict__ seg, int length, const int (&own)[N],
                                           const bool (&own_there)[N], int t0, int t1, int* s_red)
{
    int lo = 0x7fffffff, hi = -1, bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!own_there[i]) continue;
        if (own[i] < 0) bad = 1;
        else lo = own[i] < lo ? own[i] : lo, hi = own[i] > hi ? own[i] : hi;
    }
    lo = wave_min(lo), hi = wave_max_i(hi), bad = __any(bad);
    if (lane_id() == 0) s_red[wave_id()] = lo, s_red[4 + wave_id()] = hi, s_red[8 + wave_id()] = bad;
    for (int i = t0 / 32 + threadIdx.x; i <= t1 / 32; i += kBlock)
        if (i < kAttMaxTiles / 32) mk.active[i] = 0u, mk.mixed[i] = 0u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) {
        lo = s_red[w] < lo ? s_red[w] : lo;
        hi = s_red[4 + w] > hi ? s_red[4 + w] : hi;
        bad |= s_red[8 + w];
    }
    const bool one = lo == hi && !bad;
    for (int t = t0 + wave_id(); t < t1; t += kWavesPerBlock) {
        const int row = t * kTile + lane_id();
        const int v = row < length ? seg[row] : -1;
        const bool touch = __any(v >= lo && v <= hi);
        const bool plain = one && __all(v == lo);
        if (lane_id() == 0) {
            if (touch) atomicOr(&mk.active[t >> 5], 1u << (t & 31));
            if (!plain) atomicOr(&mk.mixed[t >> 5], 1u << (t & 31));
        }
    }
    __syncthreads();
}

// The streamed operands: two tiles, loaded to registers while the tile before is worked on, then written to LDS.
template <typename T, int DP> struct Feed {
    using S = Shape<T, DP>;
    u32x4 a[S::NC], b[S::NC];

    __device__ __forceinline__ void load(const T* __restrict__ pa, int64_t sa, const T* __restrict__ pb, int64_t sb, int row0,
                                         int length, const int* __restrict__ seg, int dim, int unit)
    {
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            const int idx = threadIdx.x + i * kBlock, ch = idx % S::NCH;
            const int row = row0 + idx / S::NCH;
            const int at = row < length ? row : length - 1;
            a[i] = load_chunk(pa + at * sa, ch, dim, unit);
            b[i] = load_chunk(pb + at * sb, ch, dim, unit);
            // padding contributes nothing, whatever it holds
            if (row >= length || (seg && seg[at] < 0)) a[i] = b[i] = u32x4{0u, 0u, 0u, 0u};
        }
    }
    // clean_a / clean_b: the operand that enters a second product, where masked pairs may face it
    template <bool A, bool B> __device__ __forceinline__ void put(unsigned char* ta, unsigned char* tb, bool guard, uint32_t* flags)
    {
        if (guard) {
            bool any = false;
#pragma unroll
            for (int i = 0; i < S::NC; ++i) {
                if (A) any |= clean_chunk<T>(a[i]);
                if (B) any |= clean_chunk<T>(b[i]);
            }
            any = __any(any);
            if (lane_id() == 0) flags[wave_id()] = any;
        } else if (lane_id() == 0) {
            flags[wave_id()] = 0u;
        }
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            const int idx = threadIdx.x + i * kBlock, row = idx / S::NCH, ch = idx % S::NCH;
            const int at = row * S::RB + ((ch ^ swz<S::NCH>(row)) * 16);
            *reinterpret_cast<u32x4*>(ta + at) = a[i];
            *reinterpret_cast<u32x4*>(tb + at) = b[i];
        }
    }
};

__device__ __forceinline__ int next_tile(int t, int t1, const TileMarks* mk)
{
    if (mk)
        while (t < t1) {
            const uint32_t rest = mk->active[t >> 5] >> (t & 31);
            if (rest) {
                t += __builtin_ctz(rest);
                break;
            }
            t = (t | 31) + 1;
        }
    return __builtin_amdgcn_readfirstlane(t < t1 ? t : t1);
}

__device__ __forceinline__ int row_segment(const int* __restrict__ seg, int row, int length)
{
    if (row >= length) return kNoSeg;
    const int v = seg ? seg[row] : 0;
    return v < 0 ? kNoSeg : v;
}

// ---- forward ----------------------------------------------------------------------------------------------

template <typename T, int DP, int QB>
__global__ __launch_bounds__(kBlock, 2) void k_attend(const AttArgs a)
{
    using S = Shape<T, DP>;
    constexpr int NBUF = 4 * S::TILE <= 65536 ? 2 : 1;
    constexpr int QROWS = 64 * QB, SPAN = QROWS + kTile;
    __shared__ __attribute__((aligned(1024))) unsigned char s_k[NBUF][S::TILE], s_v[NBUF][S::TILE];
    __shared__ int s_seg[NBUF][kTile];
    __shared__ uint32_t s_flags[NBUF][4];
    __shared__ float s_bias[NBUF][SPAN];
    __shared__ float s_table[kMaxBorders];
    __shared__ int s_red[12];
    __shared__ TileMarks s_marks;

    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int nqt = (a.length + QROWS - 1) / QROWS;
    const int qt = nqt - 1 - item % nqt;                 // the longest rows of a causal mask first
    const int head = (item / nqt) % a.heads, batch = item / nqt / a.heads, kvh = head / a.group;
    const int c = lane_id() & 15, g = lane_id() >> 4;
    const int q0 = qt * QROWS, wq0 = q0 + wave_id() * 16 * QB;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = a.prefix ? a.prefix[batch] : 0;
    const T* const qp = static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh;
    const T* const kp = static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh;
    const T* const vp = static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh;

    u32x4 qf[QB][S::KK];
    int qseg[QB];
    bool there[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int q = wq0 + 16 * i + c, at = q < a.length ? q : a.length - 1;
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) qf[i][kk] = load_chunk(qp + at * a.q.sr, g + 4 * kk, a.dim, a.unit);
        there[i] = q < a.length;
        qseg[i] = !there[i] ? kNoSegOwner : seg ? seg[at] : 0;
        if (qseg[i] < 0) qseg[i] = kNoSegOwner;
    }
    const int ntiles = (a.length + kTile - 1) / kTile;
    int t1 = ntiles;
    if (a.causal) {
        t1 = (q0 + QROWS - 1) / kTile + 1;
        const int pt = (prefix + kTile - 1) / kTile;
        t1 = pt > t1 ? pt : t1;
        t1 = t1 < ntiles ? t1 : ntiles;
    }
    if (seg) mark_tiles(s_marks, seg, a.length, qseg, there, 0, t1, s_red);
    const TileMarks* const mk = seg ? &s_marks : nullptr;

    const Reader<T, DP> rd;
    Feed<T, DP> feed;
    f32x4 o[QB][S::DT];
    float top[QB], total[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        top[i] = -INFINITY, total[i] = 0.f;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) o[i][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float z2 = a.scale * kLog2e, zc = a.cap > 0.f ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    if ((int)threadIdx.x < buckets) s_table[threadIdx.x] = a.table[(int64_t)head * buckets + threadIdx.x] * kLog2e;
    __syncthreads();
    int row_seg = kNoSeg;

    // whether every pair of the tile with any of the rows [lo, hi] is visible
    auto whole = [&](int t, int lo) {
        const int k0 = t * kTile;
        if (k0 + kTile > a.length || (mk && ((mk->mixed[t >> 5] >> (t & 31)) & 1))) return false;
        return !a.causal || k0 + kTile - 1 <= lo || k0 + kTile <= prefix;
    };
    auto put = [&](int t, int buf) {
        const int k0 = t * kTile;
        feed.template put<false, true>(s_k[buf], s_v[buf], !whole(t, q0), s_flags[buf]);
        if (threadIdx.x < kTile) s_seg[buf][threadIdx.x] = row_seg;
        if (a.bk.side) {
            const int hi = q0 + QROWS - 1 - k0;                    // the largest distance of the block's pairs
            if (uniform_bucket(a.bk, hi - SPAN + 2, hi) < 0 && (int)threadIdx.x < SPAN - 1)
                s_bias[buf][threadIdx.x] = s_table[bucket_of(a.bk, hi - (int)threadIdx.x)];
        }
    };

    auto load = [&](int t) {
        feed.load(kp, a.k.sr, vp, a.v.sr, t * kTile, a.length, seg, a.dim, a.unit);
        if (threadIdx.x < kTile) row_seg = row_segment(seg, t * kTile + threadIdx.x, a.length);
    };

    int t = next_tile(0, t1, mk), buf = 0;
    if (t < t1) {
        load(t);
        put(t, 0);
    }
    __syncthreads();
    while (t < t1) {
        const int tn = next_tile(t + 1, t1, mk);
        if (tn < t1) load(tn);
        const int k0 = t * kTile;
        const bool none = wq0 >= a.length || (a.causal && k0 > wq0 + 16 * QB - 1 && k0 >= prefix);
        if (!none) {
            const bool all = whole(t, wq0);
            const bool odd = (s_flags[buf][0] | s_flags[buf][1] | s_flags[buf][2] | s_flags[buf][3]) != 0u;
            const int hi = q0 + QROWS - 1 - k0;
            const int flat = a.bk.side ? uniform_bucket(a.bk, hi - SPAN + 2, hi) : 0;
            const float flat2 = a.bk.side && flat >= 0 ? s_table[flat] : 0.f;
#pragma unroll
            for (int i = 0; i < QB; ++i) {
                f32x4 s[4];
                first_product<T, DP>(s, qf[i], rd, s_k[buf]);
                const int q = wq0 + 16 * i + c;
                if (a.cap > 0.f) {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][r] = tanh_f32(s[n][r] * zc) * cap2 + flat2;
                } else {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][r] = s[n][r] * z2 + flat2;
                }
                if (flat < 0) {
                    const float* const bias = &s_bias[buf][4 * g - (q - q0) + QROWS - 1];
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][r] += bias[16 * n + r];
                }
                uint32_t vis = 0xffffu;
                if (!all) {
                    vis = 0u;
                    const int last = a.causal ? (q + 1 > prefix ? q + 1 : prefix) : a.length;      // keys before it
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int key = 16 * n + 4 * g + r;
                            const bool see = s_seg[buf][key] == qseg[i] && k0 + key < last;
                            vis |= see ? 1u << (4 * n + r) : 0u;
                            s[n][r] = see ? s[n][r] : -INFINITY;
                        }
                }
                float mx = s[0][0];
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[n][r]);
                mx = group_max(mx);
                if (__any(mx > top[i])) {
                    const float nt = fmaxf(mx, top[i]);
                    const float shrink = top[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top[i] - nt);
                    top[i] = nt;
                    total[i] *= shrink;
#pragma unroll
                    for (int dt = 0; dt < S::DT; ++dt) o[i][dt] *= shrink;
                }
                const float base = top[i] == -INFINITY ? 0.f : top[i];       // a row that has seen nothing so far
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[n][r] = __builtin_amdgcn_exp2f(s[n][r] - base);
                        total[i] += s[n][r];
                    }
                second_product<T, DP>(o[i], s, rd, s_v[buf]);
                if (odd) add_nonfinite<T, DP>(o[i], s, vis, vp + k0 * a.v.sr, a.v.sr, a.length - k0, a.dim);
            }
        }
        if (NBUF == 1) __syncthreads();
        buf = NBUF == 1 ? 0 : buf ^ 1;
        if (tn < t1) put(tn, buf);
        __syncthreads();
        t = tn;
    }

    T* const op = static_cast<T*>(a.o.data) + batch * a.o.sb + head * a.o.sh;
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int q = wq0 + 16 * i + c;
        const float l = group_sum(total[i]);
        if (q >= a.length) continue;
        const bool empty = top[i] == -INFINITY && l == 0.f;
        const float inv = empty ? 0.f : 1.f / l;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) {
            f32x4 v = o[i][dt] * inv;
            if (empty) v = f32x4{0.f, 0.f, 0.f, 0.f};
            store4(op + q * a.o.sr, 16 * dt + 4 * g, a.dim, a.unit, v);
        }
        if (a.lse && g == 0)
            a.lse[((int64_t)batch * a.heads + head) * a.length + q] = empty ? -INFINITY : top[i] * kLn2 + logf(l);
    }
}

// ---- backward, queries ------------------------------------------------------------------------------------

// dq, and the gradient of the table: a wave owns queries and walks the keys, as the forward pass does.
// delta is dO.O where only dq, dk, dv are asked for, whose own rounding is coarser than that of O; for the table's float32
// gradient, sums over whole batches in which the rounding of O would not average out to float32 accuracy, a first walk
// sums p dp in float32.  The table's gradient: near tiles, whose distances lie in several buckets, add each ds to a
// histogram that is the thread's own (LDS, [bucket][thread]: no two threads share a word, so the order is the program's);
// tiles of one bucket add to a register.
template <typename T, int DP, int QB>
__global__ __launch_bounds__(kBlock, 2) void k_attend_dq(const AttArgs a)
{
    using S = Shape<T, DP>;
    constexpr int NBUF = 4 * S::TILE <= 32768 ? 2 : 1;
    constexpr int QROWS = 64 * QB, SPAN = QROWS + kTile;
    extern __shared__ float s_hist[];
    __shared__ __attribute__((aligned(1024))) unsigned char s_k[NBUF][S::TILE], s_v[NBUF][S::TILE];
    __shared__ int s_seg[NBUF][kTile];
    __shared__ uint32_t s_flags[NBUF][4];
    __shared__ float s_bias[NBUF][SPAN];
    __shared__ int s_bucket[NBUF][SPAN];
    __shared__ float s_table[kMaxBorders];
    __shared__ int s_red[12];
    __shared__ TileMarks s_marks;

    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int nqt = (a.length + QROWS - 1) / QROWS;
    const int qt = nqt - 1 - item % nqt;
    const int head = (item / nqt) % a.heads, batch = item / nqt / a.heads, kvh = head / a.group;
    const int c = lane_id() & 15, g = lane_id() >> 4;
    const int q0 = qt * QROWS, wq0 = q0 + wave_id() * 16 * QB;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = a.prefix ? a.prefix[batch] : 0;
    const T* const qp = static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh;
    const T* const op = static_cast<const T*>(a.o.data) + batch * a.o.sb + head * a.o.sh;
    const T* const dop = static_cast<const T*>(a.dout.data) + batch * a.dout.sb + head * a.dout.sh;
    const T* const kp = static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh;
    const T* const vp = static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh;
    const int64_t stat0 = ((int64_t)batch * a.heads + head) * a.length;
    const bool want_table = a.part != nullptr;

    u32x4 qf[QB][S::KK], df[QB][S::KK];
    int qseg[QB];
    bool there[QB];
    float lse2[QB], delta[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int q = wq0 + 16 * i + c, at = q < a.length ? q : a.length - 1;
        delta[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) {
            qf[i][kk] = load_chunk(qp + at * a.q.sr, g + 4 * kk, a.dim, a.unit);
            df[i][kk] = load_chunk(dop + at * a.dout.sr, g + 4 * kk, a.dim, a.unit);
            if (!want_table) delta[i] += dot_chunk<T>(df[i][kk], load_chunk(op + at * a.o.sr, g + 4 * kk, a.dim, a.unit));
        }
        there[i] = q < a.length;
        qseg[i] = !there[i] ? kNoSegOwner : seg ? seg[at] : 0;
        if (qseg[i] < 0) qseg[i] = kNoSegOwner;
        const float l = a.lse[stat0 + at];
        lse2[i] = l == -INFINITY ? 0.f : l * kLog2e;           // a row that sees nothing: all its pairs are masked
        delta[i] = group_sum(delta[i]);
    }
    const int ntiles = (a.length + kTile - 1) / kTile;
    int t1 = ntiles;
    if (a.causal) {
        t1 = (q0 + QROWS - 1) / kTile + 1;
        const int pt = (prefix + kTile - 1) / kTile;
        t1 = pt > t1 ? pt : t1;
        t1 = t1 < ntiles ? t1 : ntiles;
    }
    if (seg) mark_tiles(s_marks, seg, a.length, qseg, there, 0, t1, s_red);
    const TileMarks* const mk = seg ? &s_marks : nullptr;

    const Reader<T, DP> rd;
    Feed<T, DP> feed;
    f32x4 dq[QB][S::DT];
#pragma unroll
    for (int i = 0; i < QB; ++i)
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) dq[i][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float z2 = a.scale * kLog2e, zc = a.cap > 0.f ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    if ((int)threadIdx.x < buckets) s_table[threadIdx.x] = a.table[(int64_t)head * buckets + threadIdx.x] * kLog2e;
    if (want_table)
        for (int b = 0; b < buckets; ++b) s_hist[b * kBlock + threadIdx.x] = 0.f;
    __syncthreads();
    int row_seg = kNoSeg;
    int flat_bucket = -1;
    float flat_sum = 0.f;

    auto whole = [&](int t, int lo) {
        const int k0 = t * kTile;
        if (k0 + kTile > a.length || (mk && ((mk->mixed[t >> 5] >> (t & 31)) & 1))) return false;
        return !a.causal || k0 + kTile - 1 <= lo || k0 + kTile <= prefix;
    };
    auto load = [&](int t) {
        feed.load(kp, a.k.sr, vp, a.v.sr, t * kTile, a.length, seg, a.dim, a.unit);
        if (threadIdx.x < kTile) row_seg = row_segment(seg, t * kTile + threadIdx.x, a.length);
    };
    auto put = [&](int t, int buf) {
        const int k0 = t * kTile;
        feed.template put<true, false>(s_k[buf], s_v[buf], !whole(t, q0), s_flags[buf]);
        if (threadIdx.x < kTile) s_seg[buf][threadIdx.x] = row_seg;
        if (a.bk.side) {
            const int hi = q0 + QROWS - 1 - k0;
            if (uniform_bucket(a.bk, hi - SPAN + 2, hi) < 0 && (int)threadIdx.x < SPAN - 1) {
                const int b = bucket_of(a.bk, hi - (int)threadIdx.x);
                s_bias[buf][threadIdx.x] = s_table[b];
                s_bucket[buf][threadIdx.x] = b * kBlock;
            }
        }
    };

    for (int walk = want_table ? 0 : 1; walk < 2; ++walk) {
        int t = next_tile(0, t1, mk), buf = 0;
        if (t < t1) {
            load(t);
            put(t, 0);
        }
        __syncthreads();
        while (t < t1) {
            const int tn = next_tile(t + 1, t1, mk);
            if (tn < t1) load(tn);
            const int k0 = t * kTile;
            const bool none = wq0 >= a.length || (a.causal && k0 > wq0 + 16 * QB - 1 && k0 >= prefix);
            if (!none) {
                // rows behind the history are masked here: the table's gradient is summed over rows
                const bool all = whole(t, wq0) && wq0 + 16 * QB <= a.length;
                const bool odd = (s_flags[buf][0] | s_flags[buf][1] | s_flags[buf][2] | s_flags[buf][3]) != 0u;
                const int hi = q0 + QROWS - 1 - k0;
                const int flat = a.bk.side ? uniform_bucket(a.bk, hi - SPAN + 2, hi) : 0;
                const float flat2 = a.bk.side && flat >= 0 ? s_table[flat] : 0.f;
                if (want_table && walk == 1 && flat >= 0 && flat != flat_bucket) {
                    if (flat_bucket >= 0) unsafeAtomicAdd(&s_hist[flat_bucket * kBlock + threadIdx.x], flat_sum);
                    flat_bucket = flat, flat_sum = 0.f;
                }
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    const int q = wq0 + 16 * i + c;
                    f32x4 s[4], dp[4], slope[4];
                    first_product<T, DP>(s, qf[i], rd, s_k[buf]);
                    first_product<T, DP>(dp, df[i], rd, s_v[buf]);
                    if (a.cap > 0.f) {
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const float th = tanh_f32(s[n][r] * zc);
                                slope[n][r] = 1.f - th * th;
                                s[n][r] = th * cap2 + flat2;
                            }
                    } else {
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][r] = s[n][r] * z2 + flat2, slope[n][r] = 1.f;
                    }
                    const int e0 = 4 * g - (q - q0) + QROWS - 1;
                    if (flat < 0) {
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][r] += s_bias[buf][e0 + 16 * n + r];
                    }
                    uint32_t vis = 0xffffu;
                    if (!all) {
                        vis = 0u;
                        const int last = a.causal ? (q + 1 > prefix ? q + 1 : prefix) : a.length;
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int key = 16 * n + 4 * g + r;
                                if (s_seg[buf][key] == qseg[i] && k0 + key < last) vis |= 1u << (4 * n + r);
                            }
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const bool see = (vis >> (4 * n + r)) & 1;
                            const float p = __builtin_amdgcn_exp2f(s[n][r] - lse2[i]);
                            if (walk == 0) delta[i] += see ? p * dp[n][r] : 0.f;
                            else s[n][r] = see ? p * (dp[n][r] - delta[i]) : 0.f;
                        }
                    if (walk == 0) continue;
                    if (want_table) {
                        if (flat >= 0) {
#pragma unroll
                            for (int n = 0; n < 4; ++n) flat_sum += (s[n][0] + s[n][1]) + (s[n][2] + s[n][3]);
                        } else {
#pragma unroll
                            for (int n = 0; n < 4; ++n)
#pragma unroll
                                for (int r = 0; r < 4; ++r)
                                    unsafeAtomicAdd(&s_hist[s_bucket[buf][e0 + 16 * n + r] + threadIdx.x], s[n][r]);
                        }
                    }
                    if (a.cap > 0.f) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) s[n] *= slope[n];
                    }
                    second_product<T, DP>(dq[i], s, rd, s_k[buf]);
                    if (odd) add_nonfinite<T, DP>(dq[i], s, vis, kp + k0 * a.k.sr, a.k.sr, a.length - k0, a.dim);
                }
            }
            if (NBUF == 1) __syncthreads();
            buf = NBUF == 1 ? 0 : buf ^ 1;
            if (tn < t1) put(tn, buf);
            __syncthreads();
            t = tn;
        }
        if (walk == 0) {
#pragma unroll
            for (int i = 0; i < QB; ++i) delta[i] = group_sum(delta[i]);
        }
    }

    T* const dqp = static_cast<T*>(a.dq.data) + batch * a.dq.sb + head * a.dq.sh;
#pragma unroll
    for (int i = 0; i < QB; ++i) {
        const int q = wq0 + 16 * i + c;
        if (q >= a.length) continue;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) store4(dqp + q * a.dq.sr, 16 * dt + 4 * g, a.dim, a.unit, dq[i][dt] * a.scale);
        if (g == 0) a.delta[stat0 + q] = delta[i];
    }
    if (want_table) {
        if (flat_bucket >= 0) unsafeAtomicAdd(&s_hist[flat_bucket * kBlock + threadIdx.x], flat_sum);
        __syncthreads();
        for (int b = wave_id(); b < buckets; b += kWavesPerBlock) {
            const float* const h = &s_hist[b * kBlock + lane_id()];
            const float sum = wave_total((h[0] + h[64]) + (h[128] + h[192]));
            if (lane_id() == 0) a.part[((int64_t)head * a.parts + batch * nqt + qt) * buckets + b] = sum;
        }
    }
}

// ---- backward, keys ---------------------------------------------------------------------------------------

// dk and dv: a wave owns keys and walks the queries of every head that shares them.
template <typename T, int DP, int KB>
__global__ __launch_bounds__(kBlock, 2) void k_attend_dkv(const AttArgs a)
{
    using S = Shape<T, DP>;
    constexpr int NBUF = 4 * S::TILE <= 32768 ? 2 : 1;
    constexpr int KROWS = 64 * KB, SPAN = KROWS + kTile;
    __shared__ __attribute__((aligned(1024))) unsigned char s_q[NBUF][S::TILE], s_d[NBUF][S::TILE];
    __shared__ int s_seg[NBUF][kTile];
    __shared__ float s_lse[NBUF][kTile], s_delta[NBUF][kTile];
    __shared__ uint32_t s_flags[NBUF][4];
    __shared__ float s_bias[NBUF][SPAN];
    __shared__ int s_red[12];
    __shared__ TileMarks s_marks;

    const int item = xcd_item(a.items);
    if (item < 0) return;
    const int nkt = (a.length + KROWS - 1) / KROWS;
    const int kt = item % nkt;
    const int kvh = (item / nkt) % a.kv_heads, batch = item / nkt / a.kv_heads;
    const int c = lane_id() & 15, g = lane_id() >> 4;
    const int k0 = kt * KROWS, wk0 = k0 + wave_id() * 16 * KB;
    const int* const seg = a.seg ? a.seg + (int64_t)batch * a.length : nullptr;
    const int prefix = a.prefix ? a.prefix[batch] : 0;
    const T* const kp = static_cast<const T*>(a.k.data) + batch * a.k.sb + kvh * a.k.sh;
    const T* const vp = static_cast<const T*>(a.v.data) + batch * a.v.sb + kvh * a.v.sh;

    u32x4 kf[KB][S::KK], vf[KB][S::KK];
    int kseg[KB];
    bool there[KB];
#pragma unroll
    for (int i = 0; i < KB; ++i) {
        const int k = wk0 + 16 * i + c, at = k < a.length ? k : a.length - 1;
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) {
            kf[i][kk] = load_chunk(kp + at * a.k.sr, g + 4 * kk, a.dim, a.unit);
            vf[i][kk] = load_chunk(vp + at * a.v.sr, g + 4 * kk, a.dim, a.unit);
        }
        there[i] = k < a.length;
        kseg[i] = !there[i] ? kNoSegOwner : seg ? seg[at] : 0;
        if (kseg[i] < 0) kseg[i] = kNoSegOwner;
    }
    const int ntiles = (a.length + kTile - 1) / kTile;
    const int t0 = a.causal && k0 >= prefix ? k0 / kTile : 0;
    if (seg) mark_tiles(s_marks, seg, a.length, kseg, there, t0, ntiles, s_red);
    const TileMarks* const mk = seg ? &s_marks : nullptr;

    const Reader<T, DP> rd;
    Feed<T, DP> feed;
    f32x4 dk[KB][S::DT], dv[KB][S::DT];
#pragma unroll
    for (int i = 0; i < KB; ++i)
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) dk[i][dt] = dv[i][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float z2 = a.scale * kLog2e, zc = a.cap > 0.f ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    int row_seg = kNoSeg;
    float row_lse = 0.f, row_delta = 0.f;

    // whether every pair of query tile t with any key up to `hi` is visible
    auto whole = [&](int t, int hi) {
        const int q0 = t * kTile;
        if (q0 + kTile > a.length || (mk && ((mk->mixed[t >> 5] >> (t & 31)) & 1))) return false;
        return !a.causal || q0 >= hi || hi < prefix;
    };
    auto load = [&](int h, int t) {
        const int head = kvh * a.group + h;
        feed.load(static_cast<const T*>(a.q.data) + batch * a.q.sb + head * a.q.sh, a.q.sr,
                  static_cast<const T*>(a.dout.data) + batch * a.dout.sb + head * a.dout.sh, a.dout.sr, t * kTile, a.length,
                  seg, a.dim, a.unit);
        if (threadIdx.x < kTile) {
            const int row = t * kTile + threadIdx.x, at = row < a.length ? row : a.length - 1;
            const int64_t stat = ((int64_t)batch * a.heads + head) * a.length + at;
            row_seg = row_segment(seg, row, a.length);
            row_lse = a.lse[stat];
            row_delta = a.delta[stat];
        }
    };
    auto put = [&](int h, int t, int buf) {
        const int q0 = t * kTile;
        feed.template put<true, true>(s_q[buf], s_d[buf], !whole(t, k0 + KROWS - 1), s_flags[buf]);
        if (threadIdx.x < kTile) {
            s_seg[buf][threadIdx.x] = row_seg;
            s_lse[buf][threadIdx.x] = row_lse == -INFINITY ? 0.f : row_lse * kLog2e;
            s_delta[buf][threadIdx.x] = row_delta;
        }
        if (a.bk.side) {
            const int lo = q0 - (k0 + KROWS - 1);                  // the smallest distance of the block's pairs
            if (uniform_bucket(a.bk, lo, lo + SPAN - 2) < 0 && (int)threadIdx.x < SPAN - 1)
                s_bias[buf][threadIdx.x] =
                    a.table[(int64_t)(kvh * a.group + h) * buckets + bucket_of(a.bk, lo + (int)threadIdx.x)] * kLog2e;
        }
    };

    int h = 0, t = next_tile(t0, ntiles, mk), buf = 0;
    if (t < ntiles) {
        load(0, t);
        put(0, t, 0);
    }
    __syncthreads();
    while (t < ntiles) {
        int hn = h, tn = next_tile(t + 1, ntiles, mk);
        if (tn >= ntiles && h + 1 < a.group) hn = h + 1, tn = next_tile(t0, ntiles, mk);
        if (tn < ntiles) load(hn, tn);
        const int q0 = t * kTile;
        const bool none = wk0 >= a.length || (a.causal && q0 + kTile - 1 < wk0 && wk0 >= prefix);
        if (!none) {
            const bool all = whole(t, wk0 + 16 * KB - 1);
            const bool odd = (s_flags[buf][0] | s_flags[buf][1] | s_flags[buf][2] | s_flags[buf][3]) != 0u;
            const int lo = q0 - (k0 + KROWS - 1);
            const int flat = a.bk.side ? uniform_bucket(a.bk, lo, lo + SPAN - 2) : 0;
            const float flat2 = a.bk.side && flat >= 0 ? a.table[(int64_t)(kvh * a.group + h) * buckets + flat] * kLog2e : 0.f;
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                const int k = wk0 + 16 * i + c;
                f32x4 s[4], dp[4], slope[4];
                first_product<T, DP>(s, kf[i], rd, s_q[buf]);
                if (a.cap > 0.f) {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float th = tanh_f32(s[n][r] * zc);
                            slope[n][r] = 1.f - th * th;
                            s[n][r] = th * cap2 + flat2;
                        }
                } else {
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][r] = s[n][r] * z2 + flat2, slope[n][r] = 1.f;
                }
                if (flat < 0) {
                    const float* const bias = &s_bias[buf][4 * g - (k - k0) + KROWS - 1];
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[n][r] += bias[16 * n + r];
                }
                uint32_t vis = 0xffffu;
                if (!all) {
                    vis = 0u;
                    const int first = a.causal && k >= prefix ? k : 0;      // queries from it on
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = 16 * n + 4 * g + r;
                            if (s_seg[buf][row] == kseg[i] && q0 + row >= first) vis |= 1u << (4 * n + r);
                        }
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const f32x4 l = *reinterpret_cast<const f32x4*>(&s_lse[buf][16 * n + 4 * g]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p = __builtin_amdgcn_exp2f(s[n][r] - l[r]);
                        s[n][r] = (vis >> (4 * n + r)) & 1 ? p : 0.f;
                    }
                }
                second_product<T, DP>(dv[i], s, rd, s_d[buf]);
                const T* const qt = static_cast<const T*>(a.q.data) + batch * a.q.sb + (kvh * a.group + h) * a.q.sh + q0 * a.q.sr;
                const T* const dt =
                    static_cast<const T*>(a.dout.data) + batch * a.dout.sb + (kvh * a.group + h) * a.dout.sh + q0 * a.dout.sr;
                if (odd) add_nonfinite<T, DP>(dv[i], s, vis, dt, a.dout.sr, a.length - q0, a.dim);
                first_product<T, DP>(dp, vf[i], rd, s_d[buf]);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const f32x4 dl = *reinterpret_cast<const f32x4*>(&s_delta[buf][16 * n + 4 * g]);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[n][r] = (vis >> (4 * n + r)) & 1 ? s[n][r] * (dp[n][r] - dl[r]) * slope[n][r] : 0.f;
                }
                second_product<T, DP>(dk[i], s, rd, s_q[buf]);
                if (odd) add_nonfinite<T, DP>(dk[i], s, vis, qt, a.q.sr, a.length - q0, a.dim);
            }
        }
        if (NBUF == 1) __syncthreads();
        buf = NBUF == 1 ? 0 : buf ^ 1;
        if (tn < ntiles) put(hn, tn, buf);
        __syncthreads();
        h = hn, t = tn;
    }

    T* const dkp = static_cast<T*>(a.dk.data) + batch * a.dk.sb + kvh * a.dk.sh;
    T* const dvp = static_cast<T*>(a.dv.data) + batch * a.dv.sb + kvh * a.dv.sh;
#pragma unroll
    for (int i = 0; i < KB; ++i) {
        const int k = wk0 + 16 * i + c;
        if (k >= a.length) continue;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) {
            store4(dkp + k * a.dk.sr, 16 * dt + 4 * g, a.dim, a.unit, dk[i][dt] * a.scale);
            store4(dvp + k * a.dv.sr, 16 * dt + 4 * g, a.dim, a.unit, dv[i][dt]);
        }
    }
}

// dtable[head, b] = the sum of the blocks' partial rows, strand by strand in a fixed order.
__global__ __launch_bounds__(kBlock) void k_attend_dtable(const float* __restrict__ part, int parts, int buckets,
                                                          float* __restrict__ dtable)
{
    __shared__ double s[kBlock];
    const int head = blockIdx.y, b = blockIdx.x * 16 + threadIdx.x % 16, strand = threadIdx.x / 16;
    double sum = 0.0;
    if (b < buckets)
        for (int p = strand; p < parts; p += 16) sum += (double)part[((int64_t)head * parts + p) * buckets + b];
    s[threadIdx.x] = sum;
    __syncthreads();
    if (strand == 0 && b < buckets) {
        for (int k = 1; k < 16; ++k) sum += s[k * 16 + threadIdx.x];
        dtable[(int64_t)head * buckets + b] = (float)sum;
    }
}

// ---- host -------------------------------------------------------------------------------------------------

// Borders of one side: bucket exact + i begins at the smallest n with (n / exact)^(side - exact) >= (far / exact)^i.
// The power is a whole number only where it is one exactly: a value within 1e-15 of a whole number, forty times the error
// of the extended-precision power, is that number.
void make_buckets(const gram_attention_config& c, AttBuckets* bk)
{
    *bk = AttBuckets{};
    if (c.buckets == 0) return;
    bk->two_sided = c.two_sided != 0;
    bk->side = bk->two_sided ? c.buckets / 2 : c.buckets;
    bk->exact = bk->side / 2;
    if (bk->side == 1) return;
    const int wide = bk->side - bk->exact;
    for (int i = 1; i < wide; ++i) {
        const long double x = bk->exact * powl((long double)c.max_distance / bk->exact, (long double)i / wide);
        const long double near = roundl(x);
        const long double n = fabsl(x - near) <= 1e-15L * x ? near : ceill(x);
        bk->border[bk->borders++] = (int)n;
    }
}

const char* check_config(const gram_attention_config* c)
{
    if (!c) return "cfg is NULL";
    if (c->heads < 1 || c->kv_heads < 1 || c->heads > 65535 || c->heads % c->kv_heads != 0)
        return "heads must be a positive multiple of kv_heads, at most 65535";
    if (c->head_dim < 1 || c->head_dim > 128) return "head_dim must be in [1, 128]";
    if (c->dtype != GRAM_F32 && c->dtype != GRAM_BF16) return "dtype must be GRAM_F32 or GRAM_BF16";
    if (!(fabsf(c->scale) <= 1e30f)) return "scale must be finite";
    if (!(c->cap >= 0.f && c->cap <= 1e30f)) return "cap must be finite and >= 0 (0: none)";
    if (c->buckets < 0 || c->buckets > GRAM_ATTENTION_MAX_BUCKETS) return "buckets must be in [0, 64]";
    if (c->buckets > 0) {
        if (c->two_sided && c->buckets % 2 != 0) return "two-sided buckets must be an even number";
        const int side = c->two_sided ? c->buckets / 2 : c->buckets;
        if (c->max_distance < 1 || c->max_distance <= side / 2 || c->max_distance > (1 << 30))
            return "max_distance must be larger than half the buckets of a side, at most 2^30";
    }
    return nullptr;
}

const char* check_sizes(const gram_attention_config* c, int32_t batch, int32_t length)
{
    if (const char* why = check_config(c)) return why;
    if (batch < 0 || length < 0) return "batch and length must be >= 0";
    if (length > GRAM_ATTENTION_MAX_LENGTH) return "length must be at most 262144";
    if ((int64_t)batch * c->heads * ((length + kTile - 1) / kTile) > kAttMaxBlocks)
        return "batch * heads * ceil(length / 64) must be at most 2^23";
    return nullptr;
}

// Bytes per global access that addresses and strides of every operand allow: 16, 8 (bf16), or one element.
struct UnitFinder {
    uint64_t bits = 0;
    bool null = false;
    AttRows add(const gram_rows* r, int es)
    {
        AttRows out{};
        if (!r || !r->data) {
            null = true;
            return out;
        }
        out.data = r->data, out.sb = r->batch_stride, out.sr = r->row_stride, out.sh = r->head_stride;
        bits |= reinterpret_cast<uintptr_t>(r->data) | (uint64_t)(out.sb * es) | (uint64_t)(out.sr * es) | (uint64_t)(out.sh * es);
        return out;
    }
    int unit(int dim, int es) const
    {
        const uint64_t all = bits | (uint64_t)(dim * es);
        return (all & 15) == 0 ? 16 : es == 2 && (all & 7) == 0 ? 8 : es;
    }
    bool aligned(int es) const { return (bits & (uint64_t)(es - 1)) == 0; }
};

int elem_size(const gram_attention_config& c) { return c.dtype == GRAM_BF16 ? 2 : 4; }

void fill(AttArgs& a, const gram_attention_config& c, int32_t batch, int32_t length)
{
    a.batch = batch, a.length = length, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
    a.dim = c.head_dim, a.causal = c.causal != 0, a.scale = c.scale, a.cap = c.cap;
    make_buckets(c, &a.bk);
}

dim3 grid_of(int items) { return dim3((unsigned)((items + 7) / 8 * 8)); }

template <typename F> void by_shape(const gram_attention_config& c, F&& go)
{
    auto width = [&](auto type) {
        if (c.head_dim <= 32) go(type, std::integral_constant<int, 32>{});
        else if (c.head_dim <= 64) go(type, std::integral_constant<int, 64>{});
        else go(type, std::integral_constant<int, 128>{});
    };
    if (c.dtype == GRAM_BF16) width(Bf16{});
    else width(float{});
}

int blocks_of(int length, int rows) { return (length + rows - 1) / rows; }

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

}  // namespace gram

using namespace gram;

extern "C" {

int32_t gram_distance_bucket(const gram_attention_config* cfg, int32_t distance)
{
    if (check_config(cfg) || cfg->buckets == 0 || distance == INT32_MIN) return -1;
    AttBuckets bk;
    make_buckets(*cfg, &bk);
    if (distance < 0 && !bk.two_sided) return 0;
    const int n = distance < 0 ? -distance : distance;
    int b = n < bk.exact ? n : bk.exact;
    if (n >= bk.exact)
        for (int i = 0; i < bk.borders; ++i) b += n >= bk.border[i];
    return distance < 0 ? bk.side + b : b;
}

int gram_attention(const gram_attention_config* cfg, int32_t batch, int32_t length, const gram_rows* q, const gram_rows* k,
                   const gram_rows* v, const gram_rows* o, const int32_t* segments, const int32_t* prefix,
                   const float* table, float* lse, void* stream)
{
    if (const char* why = check_sizes(cfg, batch, length)) return fail_call(GRAM_ERR_ARG, "gram_attention: %s", why);
    if (prefix && !cfg->causal) return fail_call(GRAM_ERR_ARG, "gram_attention: a prefix needs the causal mask");
    if (batch == 0 || length == 0) return GRAM_OK;
    const int es = elem_size(*cfg);
    AttArgs a{};
    UnitFinder u;
    a.q = u.add(q, es), a.k = u.add(k, es), a.v = u.add(v, es), a.o = u.add(o, es);
    if (u.null || (cfg->buckets > 0 && !table)) return fail_call(GRAM_ERR_ARG, "gram_attention: NULL pointer");
    if (!u.aligned(es)) return fail_call(GRAM_ERR_ARG, "gram_attention: an operand is not aligned to its elements");
    fill(a, *cfg, batch, length);
    a.unit = u.unit(a.dim, es);
    a.seg = segments, a.prefix = prefix, a.table = table, a.lse = lse;
    hipStream_t s = static_cast<hipStream_t>(stream);
    by_shape(*cfg, [&](auto type, auto dp) {
        using T = decltype(type);
        constexpr int DP = decltype(dp)::value;
        a.items = batch * cfg->heads * blocks_of(length, 64);
        k_attend<T, DP, 1><<<grid_of(a.items), dim3(kBlock), 0, s>>>(a);
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention: %s", hipGetErrorString(e));
}

int64_t gram_attention_backward_bytes(const gram_attention_config* cfg, int32_t batch, int32_t length)
{
    if (check_sizes(cfg, batch, length)) return 0;
    const int64_t rows = (int64_t)batch * cfg->heads;
    return up256(rows * length * (int64_t)sizeof(float)) +
           up256(rows * blocks_of(length, 64) * cfg->buckets * (int64_t)sizeof(float)) + 256;
}

int gram_attention_backward(const gram_attention_config* cfg, int32_t batch, int32_t length, const gram_rows* q,
                            const gram_rows* k, const gram_rows* v, const gram_rows* o, const float* lse,
                            const gram_rows* dout, const gram_rows* dq, const gram_rows* dk, const gram_rows* dv,
                            const int32_t* segments, const int32_t* prefix, const float* table, float* dtable, void* work,
                            void* stream)
{
    if (const char* why = check_sizes(cfg, batch, length))
        return fail_call(GRAM_ERR_ARG, "gram_attention_backward: %s", why);
    if (prefix && !cfg->causal) return fail_call(GRAM_ERR_ARG, "gram_attention_backward: a prefix needs the causal mask");
    if (dtable && cfg->buckets == 0)
        return fail_call(GRAM_ERR_ARG, "gram_attention_backward: dtable without buckets");
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool none = batch == 0 || length == 0;
    const int es = elem_size(*cfg);
    AttArgs a{};
    if (!none) {
        UnitFinder u;
        a.q = u.add(q, es), a.k = u.add(k, es), a.v = u.add(v, es), a.o = u.add(o, es), a.dout = u.add(dout, es);
        a.dq = u.add(dq, es), a.dk = u.add(dk, es), a.dv = u.add(dv, es);
        if (u.null || !lse || !work || (cfg->buckets > 0 && !table))
            return fail_call(GRAM_ERR_ARG, "gram_attention_backward: NULL pointer");
        if (!u.aligned(es))
            return fail_call(GRAM_ERR_ARG, "gram_attention_backward: an operand is not aligned to its elements");
        if ((reinterpret_cast<uintptr_t>(work) & 15) != 0)
            return fail_call(GRAM_ERR_ARG, "gram_attention_backward: work must be 16-byte aligned");
        a.unit = u.unit(cfg->head_dim, es);
        fill(a, *cfg, batch, length);
        a.seg = segments, a.prefix = prefix, a.table = table, a.lse = const_cast<float*>(lse);
        a.delta = static_cast<float*>(work);
        a.part = dtable ? reinterpret_cast<float*>(static_cast<unsigned char*>(work) +
                                                   up256((int64_t)batch * cfg->heads * length * (int64_t)sizeof(float)))
                        : nullptr;
        a.parts = batch * blocks_of(length, 64);
        by_shape(*cfg, [&](auto type, auto dp) {
            using T = decltype(type);
            constexpr int DP = decltype(dp)::value;
            a.items = batch * cfg->heads * blocks_of(length, 64);
            k_attend_dq<T, DP, 1><<<grid_of(a.items), dim3(kBlock), dtable ? cfg->buckets * kBlock * sizeof(float) : 0, s>>>(a);
            a.items = batch * cfg->kv_heads * blocks_of(length, 64);
            k_attend_dkv<T, DP, 1><<<grid_of(a.items), dim3(kBlock), 0, s>>>(a);
        });
    }
    if (dtable)
        k_attend_dtable<<<dim3((unsigned)((cfg->buckets + 15) / 16), (unsigned)cfg->heads), dim3(kBlock), 0, s>>>(
            a.part, none ? 0 : a.parts, cfg->buckets, dtable);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention_backward: %s", hipGetErrorString(e));
}

int64_t gram_attention_step_bytes(const gram_attention_config* cfg, int32_t batch, int32_t capacity)
{
    if (check_config(cfg) || batch < 0 || capacity < 1) return 0;
    return (batch ? step_part_bytes(*cfg, batch, capacity) : 0) + 256;
}

int gram_attention_step(const gram_attention_config* cfg, int32_t batch, int32_t capacity, const gram_rows* q,
                        const gram_rows* k_new, const gram_rows* v_new, const gram_rows* k_cache, const gram_rows* v_cache,
                        const int32_t* lengths, const int32_t* first, const float* table, const gram_rows* o, void* work,
                        void* stream)
{
    if (const char* why = check_config(cfg)) return fail_call(GRAM_ERR_ARG, "gram_attention_step: %s", why);
    if (batch < 0 || capacity < 1) return fail_call(GRAM_ERR_ARG, "gram_attention_step: batch must be >= 0 and capacity >= 1");
    if (batch == 0) return GRAM_OK;
    const int es = elem_size(*cfg);
    UnitFinder u;
    const AttRows rq = u.add(q, es), rkn = u.add(k_new, es), rvn = u.add(v_new, es), rkc = u.add(k_cache, es),
                  rvc = u.add(v_cache, es), ro = u.add(o, es);
    if (u.null || !lengths || (cfg->buckets > 0 && !table) || (!work && step_part_bytes(*cfg, batch, capacity) > 0))
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: NULL pointer");
    if (!u.aligned(es)) return fail_call(GRAM_ERR_ARG, "gram_attention_step: an operand is not aligned to its elements");
    if ((reinterpret_cast<uintptr_t>(work) & 15) != 0)
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: work must be 16-byte aligned");
    AttBuckets bk;
    make_buckets(*cfg, &bk);
    if (!step_launch(*cfg, bk, batch, capacity, rq, rkn, rvn, rkc, rvc, ro, lengths, first, table, work,
                     u.unit(cfg->head_dim, es), static_cast<hipStream_t>(stream)))
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: batch * heads must be at most 2^23");
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention_step: %s", hipGetErrorString(e));
}

}  // extern "C"
