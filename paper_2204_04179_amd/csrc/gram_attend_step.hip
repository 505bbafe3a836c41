// Attention of one new item per history over a cache of keys and values, the serving form of gram_attend.hip.
//
// The cache is read once and that read is what bounds the call: a row of dim elements lies on dim * size / 16 lanes of a
// wave, 16 bytes each, so a load covers whole rows, and dot products and weighted sums are vector arithmetic (matrix
// instructions would have 16 columns for the few query heads of a key head).  Every lane keeps the running maximum, sum and
// weighted row of the keys that its lanes have seen; they are joined once at the end, within the wave, the block, and, when
// few histories would leave most CUs idle, between the blocks that took parts of one history (k_step_join).
#include "gram_attend.h"

namespace gram {

namespace {

constexpr int kStepUnroll = 4;        // row groups in flight per wave: 4 of keys and 4 of values

struct StepArgs {
    AttRows q, kn, vn, kc, vc, o;
    const int* lengths;
    const int* first;
    const float* table;
    float* part;                      // [batch, heads, splits, dim + 2] when splits > 1
    int batch, capacity, heads, kv_heads, group, chunks, dim, splits;
    float scale, cap;
    AttBuckets bk;
};

// Sum over the LPK lanes that hold one row, the same bits in each.
template <int LPK> __device__ __forceinline__ float row_lanes_sum(float v)
{
    auto dpp = [](float x, auto ctrl) {
        return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = dpp(v, std::integral_constant<int, 0xB1>{});                        // lane ^ 1
    v = dpp(v, std::integral_constant<int, 0x4E>{});                        // lane ^ 2
    if constexpr (LPK >= 8) v = dpp(v, std::integral_constant<int, 0x141>{});   // the other four of eight
    if constexpr (LPK >= 16) v = dpp(v, std::integral_constant<int, 0x140>{});  // the other eight of sixteen
    if constexpr (LPK >= 32) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v);
        const auto b = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        v = as_f32(b[0]) + as_f32(b[1]);
    }
    return v;
}

template <typename T> __device__ __forceinline__ void unpack(u32x4 x, float* v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
            v[2 * e] = __builtin_bit_cast(float, x[e] << 16);
            v[2 * e + 1] = __builtin_bit_cast(float, x[e] & 0xffff0000u);
        } else {
            v[e] = as_f32(x[e]);
        }
    }
}

template <typename T, int DP, int UNIT, int GC>
__global__ __launch_bounds__(kBlock) void k_step(const StepArgs a)
{
    constexpr int EPC = 16 / sizeof(T), LPK = DP / EPC, KPI = kWave / LPK, U = kStepUnroll;
    __shared__ float s_acc[kWavesPerBlock][GC][DP];
    __shared__ float s_top[kWavesPerBlock][GC], s_total[kWavesPerBlock][GC];
    __shared__ float s_table[GC][kMaxBorders];
    __shared__ int s_border[kMaxBorders];

    const int split = blockIdx.x % a.splits;
    const int chunk = (blockIdx.x / a.splits) % a.chunks;
    const int kvh = (blockIdx.x / a.splits / a.chunks) % a.kv_heads;
    const int b = blockIdx.x / a.splits / a.chunks / a.kv_heads;
    const int ch = lane_id() % LPK, sub = lane_id() / LPK;
    const int heads_here = a.group - chunk * GC < GC ? a.group - chunk * GC : GC;
    const int head0 = kvh * a.group + chunk * GC;

    const int n = a.lengths[b];
    const bool live = n >= 0 && n < a.capacity;
    int first = a.first ? a.first[b] : 0;
    first = first < 0 ? 0 : first;
    first = first > n ? n : first;
    const int rows = live ? n + 1 - first : 0;                       // the new item is the last of them
    const int per = ((rows + a.splits - 1) / a.splits + kTile - 1) / kTile * kTile;
    const int64_t lo64 = (int64_t)split * per;
    const int lo = first + (int)(lo64 < rows ? lo64 : rows), hi = first + (int)(lo64 + per < rows ? lo64 + per : rows);

    const T* const kc = static_cast<const T*>(a.kc.data) + b * a.kc.sb + kvh * a.kc.sh;
    const T* const vc = static_cast<const T*>(a.vc.data) + b * a.vc.sb + kvh * a.vc.sh;
    const T* const kn = static_cast<const T*>(a.kn.data) + b * a.kn.sb + kvh * a.kn.sh;
    const T* const vn = static_cast<const T*>(a.vn.data) + b * a.vn.sb + kvh * a.vn.sh;

    float q[GC][EPC], acc[GC][EPC], top[GC], total[GC], far2[GC];
    const RowSource ks = row_source(kn, 0, 1, a.dim), vs = row_source(vn, 0, 1, a.dim);
    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
#pragma unroll
    for (int h = 0; h < GC; ++h) {
        const int head = head0 + (h < heads_here ? h : 0);
        unpack<T>(load_chunk<T, UNIT>(row_source(static_cast<const T*>(a.q.data) + b * a.q.sb + head * a.q.sh, 0, 1, a.dim), 0u, ch,
                                      a.dim), q[h]);
        far2[h] = a.bk.side ? a.table[(int64_t)head * buckets + a.bk.side - 1] * kLog2e : 0.f;
        if ((int)threadIdx.x < buckets) s_table[h][threadIdx.x] = a.table[(int64_t)head * buckets + threadIdx.x] * kLog2e;
        top[h] = -INFINITY, total[h] = 0.f;
#pragma unroll
        for (int e = 0; e < EPC; ++e) acc[h][e] = 0.f;
    }
    const float z2 = a.scale * kLog2e, zc = a.cap > 0.f ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;

    if (threadIdx.x < kMaxBorders) s_border[threadIdx.x] = a.bk.border[threadIdx.x];
    __syncthreads();

    for (int base = lo + __builtin_amdgcn_readfirstlane(wave_id()) * (U * KPI); base < hi; base += kWavesPerBlock * U * KPI) {
        u32x4 kx[U], vx[U];
        bool in[U];
        const int held = (hi < n ? hi : n) - base;                   // rows of the round that the cache holds
        const RowSource kr = row_source(kc + base * a.kc.sr, a.kc.sr, held, a.dim), vr = row_source(vc + base * a.vc.sr, a.vc.sr, held, a.dim);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = u * KPI + sub;
            in[u] = base + row < hi;
            kx[u] = load_chunk<T, UNIT>(kr, row < held ? (uint32_t)row * kr.stride : kNowhere - 256u, ch, a.dim);
            vx[u] = load_chunk<T, UNIT>(vr, row < held ? (uint32_t)row * vr.stride : kNowhere - 256u, ch, a.dim);
        }
        if (base + U * KPI > n) {                                    // the new item, from its own rows
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (base + u * KPI + sub == n) {
                    kx[u] = load_chunk<T, UNIT>(ks, 0u, ch, a.dim);
                    vx[u] = load_chunk<T, UNIT>(vs, 0u, ch, a.dim);
                }
        }
        float s[U][GC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float k[EPC];
            unpack<T>(kx[u], k);
#pragma unroll
            for (int h = 0; h < GC; ++h) {
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < EPC; ++e) dot += q[h][e] * k[e];
                dot = row_lanes_sum<LPK>(dot);
                s[u][h] = a.cap > 0.f ? tanh_f32(dot * zc) * cap2 : dot * z2;
            }
        }
        if (a.bk.side) {
            if (n - (base + U * KPI - 1) >= a.bk.last) {                  // every key of the round in the last bucket
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int h = 0; h < GC; ++h) s[u][h] += far2[h];
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int away = n - (base + u * KPI + sub);
                    const int bucket = bucket_side(a.bk, s_border, away < 0 ? 0 : away);
#pragma unroll
                    for (int h = 0; h < GC; ++h)
                        s[u][h] += s_table[h][bucket];
                }
            }
        }
#pragma unroll
        for (int h = 0; h < GC; ++h) {
            float mx = top[h];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s[u][h] = in[u] ? s[u][h] : -INFINITY;
                mx = fmaxf(mx, s[u][h]);
            }
            const float from = mx == -INFINITY ? 0.f : mx;
            const float shrink = __builtin_amdgcn_exp2f(top[h] - from);
            top[h] = mx;
            total[h] *= shrink;
#pragma unroll
            for (int e = 0; e < EPC; ++e) acc[h][e] *= shrink;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s[u][h] = __builtin_amdgcn_exp2f(s[u][h] - from);
                total[h] += s[u][h];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[EPC];
            unpack<T>(vx[u], v);
#pragma unroll
            for (int h = 0; h < GC; ++h)
#pragma unroll
                for (int e = 0; e < EPC; ++e) acc[h][e] += s[u][h] * v[e];
        }
    }

    // join the lane groups of the wave, then the waves
#pragma unroll
    for (int h = 0; h < GC; ++h) {
        float mx = top[h];
#pragma unroll
        for (int w = LPK; w < kWave; w *= 2) mx = fmaxf(mx, __shfl_xor(mx, w));
        const float mine = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top[h] - mx);
        // a lane group that has seen no key, or only scores of minus infinity, has zeros (or their NaN) to add
        const float f = top[h] == -INFINITY ? (mx == -INFINITY ? 1.f : 0.f) : mine;
        total[h] *= f;
#pragma unroll
        for (int e = 0; e < EPC; ++e) acc[h][e] *= f;
#pragma unroll
        for (int w = LPK; w < kWave; w *= 2) {
            total[h] += __shfl_xor(total[h], w);
#pragma unroll
            for (int e = 0; e < EPC; ++e) acc[h][e] += __shfl_xor(acc[h][e], w);
        }
        if (sub == 0) {
#pragma unroll
            for (int e = 0; e < EPC; ++e) s_acc[wave_id()][h][ch * EPC + e] = acc[h][e];
            if (ch == 0) s_top[wave_id()][h] = mx, s_total[wave_id()][h] = total[h];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < GC * DP; i += kBlock) {
        const int h = i / DP, d = i % DP;
        if (h >= heads_here || d >= a.dim) continue;
        float mx = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) mx = fmaxf(mx, s_top[w][h]);
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) {
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_top[w][h] - mx);
            sum += s_total[w][h] * f;
            x += s_acc[w][h][d] * f;
        }
        const int head = head0 + h;
        if (a.splits == 1) {
            T* const op = static_cast<T*>(a.o.data) + b * a.o.sb + head * a.o.sh + d;
            const float r = rows == 0 ? 0.f : x / sum;
            if constexpr (sizeof(T) == 2) op->bits = (uint16_t)pack_bf16x2(r, 0.f);
            else *op = r;
        } else {
            float* const p = a.part + (((int64_t)b * a.heads + head) * a.splits + split) * (a.dim + 2);
            p[d] = x;
            if (d == 0) p[a.dim] = mx, p[a.dim + 1] = sum;
        }
    }
    // the new item's rows enter the cache from the block that has attended to them; no other block reads that row
    if (chunk == 0 && rows > 0 && lo <= n && n < hi) {
        T* const ko = static_cast<T*>(a.kc.data) + b * a.kc.sb + kvh * a.kc.sh + n * a.kc.sr;
        T* const vo = static_cast<T*>(a.vc.data) + b * a.vc.sb + kvh * a.vc.sh + n * a.vc.sr;
        if ((int)threadIdx.x < a.dim) ko[threadIdx.x] = kn[threadIdx.x];
        else if ((int)threadIdx.x >= 128 && (int)threadIdx.x - 128 < a.dim) vo[threadIdx.x - 128] = vn[threadIdx.x - 128];
    }
}

// Joins the parts of a history and head: out = sum_s part_s 2^(top_s - top) / sum_s total_s 2^(top_s - top).
template <typename T> __global__ __launch_bounds__(128) void k_step_join(const StepArgs a)
{
    const int head = blockIdx.x % a.heads, b = blockIdx.x / a.heads, d = threadIdx.x;
    if (d >= a.dim) return;
    const float* const p = a.part + ((int64_t)b * a.heads + head) * a.splits * (a.dim + 2);
    float mx = -INFINITY, sum = 0.f, x = 0.f;
    for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, p[s * (a.dim + 2) + a.dim]);
    for (int s = 0; s < a.splits; ++s) {
        const float* const ps = p + s * (a.dim + 2);
        const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ps[a.dim] - mx);
        sum += ps[a.dim + 1] * f;
        x += ps[d] * f;
    }
    const int n = a.lengths[b];
    const float r = n >= 0 && n < a.capacity ? x / sum : 0.f;
    T* const op = static_cast<T*>(a.o.data) + b * a.o.sb + head * a.o.sh + d;
    if constexpr (sizeof(T) == 2) op->bits = (uint16_t)pack_bf16x2(r, 0.f);
    else *op = r;
}

// Query heads per block: all that share a key head, up to eight, so that the cache is read once for them.
int step_heads(int group) { return group >= 5 ? 8 : group >= 3 ? 4 : group; }

// Parts per history: enough for four blocks on each CU, none of fewer than 256 rows of the cache's capacity.
int step_splits(const gram_attention_config& c, int32_t batch, int32_t capacity)
{
    const int group = c.heads / c.kv_heads, gc = step_heads(group);
    const int64_t blocks = (int64_t)batch * c.kv_heads * ((group + gc - 1) / gc);
    const int64_t want = (1024 + blocks - 1) / blocks, most = (capacity + 255) / 256;
    return (int)(want < most ? want : most);
}

}  // namespace

int64_t step_part_bytes(const gram_attention_config& c, int32_t batch, int32_t capacity)
{
    const int s = step_splits(c, batch, capacity);
    return s > 1 ? (int64_t)batch * c.heads * s * (c.head_dim + 2) * (int64_t)sizeof(float) : 0;
}

bool step_launch(const gram_attention_config& c, const AttBuckets& bk, int32_t batch, int32_t capacity, const AttRows& q,
                 const AttRows& kn, const AttRows& vn, const AttRows& kc, const AttRows& vc, const AttRows& o,
                 const int* lengths, const int* first, const float* table, void* work, int unit, hipStream_t s)
{
    StepArgs a{};
    a.q = q, a.kn = kn, a.vn = vn, a.kc = kc, a.vc = vc, a.o = o;
    a.lengths = lengths, a.first = first, a.table = table, a.part = static_cast<float*>(work);
    a.batch = batch, a.capacity = capacity, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
    a.dim = c.head_dim, a.scale = c.scale, a.cap = c.cap, a.bk = bk;
    const int gc = step_heads(a.group);
    a.chunks = (a.group + gc - 1) / gc;
    a.splits = step_splits(c, batch, capacity);
    const int64_t blocks = (int64_t)batch * c.kv_heads * a.chunks * a.splits;
    if (blocks > kAttMaxBlocks || (int64_t)batch * c.heads > kAttMaxBlocks) return false;
    by_shape(c, unit, [&](auto type, auto dp, auto u) {
        using T = decltype(type);
        constexpr int DP = decltype(dp)::value, UNIT = decltype(u)::value;
        const dim3 grid((unsigned)blocks);
        if (gc == 1) k_step<T, DP, UNIT, 1><<<grid, dim3(kBlock), 0, s>>>(a);
        else if (gc == 2) k_step<T, DP, UNIT, 2><<<grid, dim3(kBlock), 0, s>>>(a);
        else if (gc == 4) k_step<T, DP, UNIT, 4><<<grid, dim3(kBlock), 0, s>>>(a);
        else k_step<T, DP, UNIT, 8><<<grid, dim3(kBlock), 0, s>>>(a);
        if (a.splits > 1) k_step_join<T><<<dim3((unsigned)(batch * c.heads)), dim3(128), 0, s>>>(a);
    });
    return true;
}

}  // namespace gram
