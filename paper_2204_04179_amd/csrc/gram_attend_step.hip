// Attention of one new item per history over a cache of keys and values, the serving form of gram_attend.hip.
//
// The cache is read once and that read is what bounds the call.  The query heads that share a key head are the 16 columns
// of the matrix instructions (unused ones cost nothing that counts), 32 rows of the cache at a time and wave are the other
// side: keys go from memory straight to the operand registers, values through the wave's own rows of LDS, which the
// transposing read needs.  Each score is so worked out by one lane.  (With a row of the cache spread over lanes and the
// products in vector arithmetic, every lane of a row repeated its tanh and exponential: 98 us in place of 56, which
// are 4.8 TB/s, on 64 caches of up to 8192 rows, 8 heads of 128 on 2 key heads, capped.  float32, tuned for nothing so far:
// 375 us, 1.4 TB/s.)  Every wave keeps the running maximum, sum and weighted row; they are joined once at the end, in the block
// and, when few histories would leave most CUs idle, between the blocks that took parts of one history (k_step_join).
#include "gram_attend.h"

namespace gram {

namespace {

constexpr int kStepRows = 32;         // rows of the cache per wave and round
constexpr int kStepHeads = 16;        // query heads per block

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

// Zero where nothing was seen (an idle history) or only scores of minus infinity.
__device__ __forceinline__ float step_result(float x, float top, float sum) { return top == -INFINITY && sum == 0.f ? x * 0.f : x / sum; }

template <typename T, int DP, int UNIT>
__global__ __launch_bounds__(kBlock, (Shape<T, DP>::RB <= 128 ? 3 : 2)) void k_step(const StepArgs a)
{
    using S = Shape<T, DP>;
    constexpr int NV = kStepRows * S::NCH / kWave;                   // chunks of values per lane and round
    constexpr int RPP = kWave / S::NCH;                              // rows of values per load of a wave
    // values of a round, each wave's own; afterwards the waves' weighted rows, [wave][head][DP] in float32
    constexpr int ROOM = kStepRows * S::RB > kStepHeads * DP * 4 ? kStepRows * S::RB : kStepHeads * DP * 4;
    __shared__ __attribute__((aligned(1024))) unsigned char s_v[kWavesPerBlock][ROOM];
    __shared__ float s_top[kWavesPerBlock][kStepHeads], s_total[kWavesPerBlock][kStepHeads];
    __shared__ float s_table[kStepHeads][kMaxBorders];
    __shared__ int s_border[kMaxBorders];

    const int split = blockIdx.x % a.splits;
    const int chunk = (blockIdx.x / a.splits) % a.chunks;
    const int kvh = (blockIdx.x / a.splits / a.chunks) % a.kv_heads;
    const int b = blockIdx.x / a.splits / a.chunks / a.kv_heads;
    const int lane = lane_id(), c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int head0 = kvh * a.group + chunk * kStepHeads;
    const int heads_here = a.group - chunk * kStepHeads < kStepHeads ? a.group - chunk * kStepHeads : kStepHeads;

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

    const int buckets = a.bk.two_sided ? 2 * a.bk.side : a.bk.side;
    for (int i = threadIdx.x; i < heads_here * buckets; i += kBlock)
        s_table[i / buckets][i % buckets] = to_log2(a.table[(int64_t)head0 * buckets + i]);
    if (threadIdx.x < kMaxBorders) s_border[threadIdx.x] = a.bk.border[threadIdx.x];

    u32x4 qf[S::KK];
    {
        // head stride in place of a row stride
        const RowSource src = row_source(static_cast<const T*>(a.q.data) + b * a.q.sb + head0 * a.q.sh, a.q.sh, heads_here, a.dim);
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk)
            qf[kk] = load_chunk<T, UNIT>(src, c < heads_here ? (uint32_t)c * src.stride : kNowhere - 1024u, g + 4 * kk, a.dim);
    }
    u32x4 kx[2][S::KK], vx[NV];
    const RowSource kns = row_source(kn, 0, 1, a.dim), vns = row_source(vn, 0, 1, a.dim);
    auto load_keys = [&](int base) {
        const int held = (hi < n ? hi : n) - base;                   // rows of the round that the cache holds
        const RowSource src = row_source(kc + base * a.kc.sr, a.kc.sr, held, a.dim);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk)
                kx[t][kk] = load_chunk<T, UNIT>(src, 16 * t + c < held ? (uint32_t)(16 * t + c) * src.stride : kNowhere - 1024u, g + 4 * kk, a.dim);
        if (base + kStepRows > n)                                    // the new item, from its own row
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int kk = 0; kk < S::KK; ++kk)
                    if (base + 16 * t + c == n) kx[t][kk] = load_chunk<T, UNIT>(kns, 0u, g + 4 * kk, a.dim);
    };
    auto load_values = [&](int base) {
        const int held = (hi < n ? hi : n) - base;
        const RowSource src = row_source(vc + base * a.vc.sr, a.vc.sr, held, a.dim);
        const int r0 = lane / S::NCH, ch = lane % S::NCH;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            vx[i] = load_chunk<T, UNIT>(src, r0 + i * RPP < held ? (uint32_t)(r0 + i * RPP) * src.stride : kNowhere - 1024u, ch, a.dim);
        if (base + kStepRows > n)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (base + r0 + i * RPP == n) vx[i] = load_chunk<T, UNIT>(vns, 0u, ch, a.dim);
    };
    constexpr int STRIDE = kWavesPerBlock * kStepRows;
    int base = lo + wave * kStepRows;
    if (base < hi) {
        load_keys(base);
        load_values(base);
    }
    __syncthreads();

    const Reader<T, DP> rd(lane);
    f32x4 o[S::DT];
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float z2 = a.scale * kLog2e, zc = a.cap > 0.f ? a.scale / a.cap : 0.f, cap2 = a.cap * kLog2e;
    const float far2 = a.bk.side ? s_table[c < heads_here ? c : 0][a.bk.side - 1] : 0.f;

    for (; base < hi; base += STRIDE) {
        f32x4 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < S::KK; ++kk) s[t] = mma<T>(kx[t][kk], qf[kk], s[t]);
        }
        unsigned char* const room = s_v[wave];
        {
            const int r0 = lane / S::NCH, ch = lane % S::NCH;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int row = r0 + i * RPP;
                *reinterpret_cast<u32x4*>(room + row * S::RB + ((ch ^ swz<T, S::NCH>(row)) * 16)) = vx[i];
            }
        }
        if (base + STRIDE < hi) {
            load_keys(base + STRIDE);
            load_values(base + STRIDE);
        }
        const bool far = n - (base + kStepRows - 1) >= a.bk.last;    // every row of the round in the last bucket
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = base + 16 * t + 4 * g + r;
                float x = a.cap > 0.f ? tanh_f32(s[t][r] * zc) * cap2 : s[t][r] * z2;
                if (a.bk.side) {
                    float bias = far2;
                    if (!far) bias = s_table[c < heads_here ? c : 0][bucket_side(a.bk, s_border, n > row ? n - row : 0)];
                    x += bias;
                }
                s[t][r] = row < hi ? x : -INFINITY;
                mx = fmaxf(mx, s[t][r]);
            }
        mx = group_max(mx);
        if (__any(mx > top)) {
            const float nt = fmaxf(mx, top);
            const float shrink = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - nt);
            top = nt;
            total *= shrink;
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) o[dt] *= shrink;
        }
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - from);
                total += s[t][r];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if constexpr (sizeof(T) == 2) {
            // the matrix cores take bf16: a weight goes in as its rounding and the rounding of what that left, 16 bits in
            // all, which costs nothing beside the read of the cache
            u32x4 w, left;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; r += 2) {
                    const uint32_t hi2 = pack_bf16x2(s[t][r], s[t][r + 1]);
                    w[2 * t + r / 2] = hi2;
                    left[2 * t + r / 2] = pack_bf16x2(s[t][r] - as_f32(hi2 << 16), s[t][r + 1] - as_f32(hi2 & 0xffff0000u));
                }
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) {
                const u32x4 v = rd.col_frag2(room, 0, dt);
                o[dt] = mma<T>(v, w, o[dt]);
                o[dt] = mma<T>(v, left, o[dt]);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int dt = 0; dt < S::DT; ++dt) o[dt] = mma<T>(rd.col_frag1(room, t, dt), __builtin_bit_cast(u32x4, s[t]), o[dt]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // join the waves
    total = group_sum(total);
    float* const mine = reinterpret_cast<float*>(s_v[wave]);
    if (c < heads_here) {
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) *reinterpret_cast<f32x4*>(mine + c * DP + 16 * dt + 4 * g) = o[dt];
        if (g == 0) s_top[wave][c] = top, s_total[wave][c] = total;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < heads_here * DP; i += kBlock) {
        const int h = i / DP, d = i % DP;
        if (d >= a.dim) continue;
        float mx = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) mx = fmaxf(mx, s_top[w][h]);
#pragma unroll
        for (int w = 0; w < kWavesPerBlock; ++w) {
            // a wave that has seen no row, or only scores of minus infinity, has zeros (or their NaN) to add
            const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_top[w][h] - mx);
            sum += s_total[w][h] * f;
            x += reinterpret_cast<const float*>(s_v[w])[i] * f;
        }
        const int head = head0 + h;
        if (a.splits == 1) {
            T* const op = static_cast<T*>(a.o.data) + b * a.o.sb + head * a.o.sh + d;
            const float r = step_result(x, mx, sum);
            if constexpr (sizeof(T) == 2) op->bits = (uint16_t)pack_bf16x2(r, 0.f);
            else *op = r;
        } else {
            float* const p = a.part + (((int64_t)b * a.heads + head) * a.splits + split) * (a.dim + 2);
            p[d] = x;
            if (d == 0) p[a.dim] = mx, p[a.dim + 1] = sum;
        }
    }
    // the new item's rows enter the cache from the block that has attended to them; no block reads that row of the cache
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
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, p[s * (a.dim + 2) + a.dim]);
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
        const float* const ps = p + s * (a.dim + 2);
        const float f = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ps[a.dim] - mx);
        sum += ps[a.dim + 1] * f;
        x += ps[d] * f;
    }
    const float r = step_result(x, mx, sum);
    T* const op = static_cast<T*>(a.o.data) + b * a.o.sb + head * a.o.sh + d;
    if constexpr (sizeof(T) == 2) op->bits = (uint16_t)pack_bf16x2(r, 0.f);
    else *op = r;
}

// Parts per history: enough for four blocks on each CU, none of fewer than 256 rows of the cache's capacity.
int step_splits(const gram_attention_config& c, int32_t batch, int32_t capacity)
{
    const int64_t blocks = (int64_t)batch * c.kv_heads * ((c.heads / c.kv_heads + kStepHeads - 1) / kStepHeads);
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
    a.chunks = (a.group + kStepHeads - 1) / kStepHeads;
    a.splits = step_splits(c, batch, capacity);
    const int64_t blocks = (int64_t)batch * c.kv_heads * a.chunks * a.splits;
    if (blocks > kAttMaxBlocks || (int64_t)batch * c.heads > kAttMaxBlocks) return false;
    by_shape(c, unit, [&](auto type, auto dp, auto u) {
        using T = decltype(type);
        constexpr int DP = decltype(dp)::value, UNIT = decltype(u)::value;
        const dim3 grid((unsigned)blocks);
        k_step<T, DP, UNIT><<<grid, dim3(kBlock), 0, s>>>(a);
        if (a.splits > 1) k_step_join<T><<<dim3((unsigned)(batch * c.heads)), dim3(128), 0, s>>>(a);
    });
    return true;
}

}  // namespace gram
