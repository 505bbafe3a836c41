// What the attention kernels share: the argument block, tiles in LDS, matrix-core fragments, masks and the bias by
// distance.  Not part of the public ABI.
//
// Every product of the forward and backward pass is written so that the accumulator of one is the operand of the next
// without leaving the registers.  A wave owns 16 rows (queries, or keys in the pass over keys) per "owner block"; the
// other side is streamed through LDS in tiles of 64 rows.  A first product has the streamed rows as its 16 accumulator
// rows and the owner as its 16 columns: lane (c, g), c = lane % 16, g = lane / 16, then holds owner c and streamed rows
// 16 t + 4 g + r, r = 0..3.  In the second product the streamed rows are summed over: the order of the terms is free as
// long as both operands use the same one, so those registers are the B operand as they are (rounded to the operands'
// type), and the A operand, the streamed tile transposed, is read from LDS in that order.
#pragma once

#include "gram_internal.h"

namespace gram {

constexpr int kTile = 64;                     // streamed rows per tile
constexpr int kAttMaxTiles = GRAM_ATTENTION_MAX_LENGTH / kTile;
constexpr int kMaxBorders = 64;
constexpr int64_t kAttMaxBlocks = 1 << 23;    // blocks of a launch (256 threads each; a grid holds fewer than 2^32 threads)
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kNoSeg = -1, kNoSegOwner = -2;  // a streamed row that is not there, an owner row that is not there: never equal

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef s16x4 __attribute__((address_space(3))) lds_s16x4;

struct Bf16 { uint16_t bits; };

// Division of work items by a number of the launch: floor(n / d) = (n * mul) >> (32 + shift) for n below 2^31, with mul =
// ceil(2^(32 + shift) / d), shift = ceil(log2 d) - 1 (d = 1: no multiplication).
struct FastDiv {
    uint32_t d, mul, shift;
    __host__ static FastDiv of(uint32_t d)
    {
        uint32_t s = 0;
        while ((1u << (s + 1)) < d && s < 30) ++s;
        return {d, d == 1 ? 0u : (uint32_t)((((uint64_t)1 << (32 + s)) + d - 1) / d), s};
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

// One operand: element (b, row, head, 0) is at data + b * sb + row * sr + head * sh.
struct AttRows {
    void* data;
    int64_t sb, sr, sh;
};

// Distance -> bucket of one side: n < exact: n; else exact + (number of borders <= n).
struct AttBuckets {
    int side;                // buckets of one side (0: no bias)
    int exact;
    int two_sided;
    int borders;             // side - 1 - exact of them, ascending
    int last;                // from this distance on: bucket side - 1
    float inv_exact, per_log2;      // the bucket is near exact + per_log2 log2(n inv_exact)
    int border[kMaxBorders];
};

struct AttArgs {
    AttRows q, k, v, o, dout, dq, dk, dv;
    const int* seg;
    const int* prefix;
    const float* table;
    float* lse;
    float* delta;            // [batch, heads, length]
    float* far;              // [batch, heads, length, 2]: maximum and log2 of the sum of rows whose lse is far from zero
    float* part;             // partial gradients of the table: [heads, parts, buckets]
    int batch, length, heads, kv_heads, group, dim;
    int causal;
    int items, parts;
    FastDiv by_tiles, by_heads, by_group;      // tiles of a history; heads or key heads; heads that share a key head
    float scale, cap;
    AttBuckets bk;
};

// For kernels whose one parameter is an AttArgs: its borders where the arguments lie in memory (a lane's own index into the
// parameter would make a copy of it).
__device__ __forceinline__ const int* kernel_borders()
{
    return (const int*)((const char*)__builtin_amdgcn_kernarg_segment_ptr() + __builtin_offsetof(AttArgs, bk.border));
}

// By value: a bit cast applied to an element of a vector yields the vector's first element.
__device__ __forceinline__ float as_f32(uint32_t bits) { return __builtin_bit_cast(float, bits); }

template <typename T, int DP> struct Shape {
    static constexpr int ES = sizeof(T);
    static constexpr int RB = DP * ES;             // bytes of a row in LDS
    static constexpr int NCH = RB / 16;            // 16-byte chunks of a row
    static constexpr int KK = RB / 64;             // fragments along a row: 4 lane groups of 16 bytes
    static constexpr int DT = DP / 16;             // 16-column blocks of a row
    static constexpr int NC = NCH / 4;             // chunks of a tile per thread
    static constexpr int TILE = kTile * RB;
};

// 16-byte chunk `ch` of row `row` lies at chunk ch ^ swz(row), against reads of a tile that meet a bank twice: 64 banks hold
// one row of 16 chunks, two of 8, four of 4.  A fragment along rows takes the same chunk of 16 rows.  A transposed one of bf16 takes two
// neighbouring chunks of four neighbouring rows (hence the shift by one chunk), of float32 four neighbouring chunks of rows 4
// apart.  Counted one access at a time (SQ_LDS_BANK_CONFLICT beside SQ_LDS_IDX_ACTIVE): all of float32's reads, the transposed ones of
// bf16 rows of 128 and 256 bytes, the stores of tiles, the bias and the statistics have no conflicts.  bf16 fragments along rows
// take 8 cycles in place of 4, and so do transposed ones of 64-byte rows (4 for 2): these are the 22 to 33 % of conflicts that the
// kernels show.
template <typename T, int NCH> __device__ __forceinline__ int swz(int row)
{
    if constexpr (sizeof(T) == 2)
        return NCH >= 16 ? ((row & 7) << 1) | ((row >> 3) & 1) : NCH == 8 ? (row & 6) | ((row >> 3) & 1) : (row >> 2) & 3;
    else
        return NCH >= 16 ? row & 15 : row & 7;
}

// ---- global rows ------------------------------------------------------------------------------------------

// Rows [0, rows) of an operand, `stride` bytes apart, through a buffer descriptor: what lies behind the last of them
// reads as zero.  The host keeps stride below 2^26, so that 64 rows stay within the descriptor's 32-bit offsets.
constexpr uint32_t kAttBufferFlags = 0x00027000;     // 32-bit elements, no swizzle
constexpr uint32_t kNowhere = 0xffffff00u;        // an offset behind every descriptor's end
constexpr int64_t kAttMaxRowBytes = (int64_t)1 << 26;

struct RowSource {
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t stride;
};
template <typename T> __device__ __forceinline__ RowSource row_source(const T* base, int64_t sr, int rows, int dim)
{
    const uint32_t stride = (uint32_t)sr * (uint32_t)sizeof(T);
    const uint32_t bytes = rows > 0 ? (uint32_t)((rows < kTile ? rows : kTile) - 1) * stride + (uint32_t)dim * (uint32_t)sizeof(T) : 0u;
    return {__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, kAttBufferFlags), stride};
}

// The 16-byte chunk `ch` of a row that begins at byte `off`, zeros behind its `dim` elements.  UNIT: the bytes per load that
// the alignment of all operands allows (16; 8 with bf16; one element).
template <typename T, int UNIT> __device__ __forceinline__ u32x4 load_chunk(const RowSource& src, uint32_t off, int ch, int dim)
{
    constexpr int EPC = 16 / sizeof(T);
    const int at = ch * EPC;
    const uint32_t byte = off + (uint32_t)ch * 16u;
    if constexpr (UNIT == 16) {
        return __builtin_amdgcn_raw_buffer_load_b128(src.rsrc, at < dim ? byte : kNowhere, 0, 0);
    } else if constexpr (UNIT == 8) {
        const u32x2 lo = __builtin_amdgcn_raw_buffer_load_b64(src.rsrc, at < dim ? byte : kNowhere, 0, 0);
        const u32x2 hi = __builtin_amdgcn_raw_buffer_load_b64(src.rsrc, at + 4 < dim ? byte + 8u : kNowhere, 0, 0);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
        u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            const uint32_t where = at + e < dim ? byte + (uint32_t)(e * sizeof(T)) : kNowhere;
            if constexpr (sizeof(T) == 2)
                v[e / 2] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(src.rsrc, where, 0, 0) << (16 * (e & 1));
            else
                v[e] = __builtin_amdgcn_raw_buffer_load_b32(src.rsrc, where, 0, 0);
        }
        return v;
    }
}

__device__ __forceinline__ bool nonfinite_bits(uint32_t f32_bits) { return (f32_bits & 0x7f800000u) == 0x7f800000u; }

// ---- fragments --------------------------------------------------------------------------------------------

// C += A . B over one 64-byte piece of the summed dimension: 32 elements of bf16 in one matrix instruction, 16 of float32
// in four (instruction e takes element e of every lane's four).
template <typename T> __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[e], fb[e], c, 0, 0, 0);
        return c;
    }
}

// Offsets of this lane's reads from a tile, the same for every 16-row block of it.
template <typename T, int DP> struct Reader {
    using S = Shape<T, DP>;
    int direct[S::KK];       // rows c of a block, chunk g + 4 kk
    int trans[S::DT];        // bf16: the transposing read's piece; float32: row 4 g of a block, column 16 dt + c

    __device__ __forceinline__ explicit Reader(int lane)
    {
        const int c = lane & 15, g = lane >> 4;
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) direct[kk] = c * S::RB + (((g + 4 * kk) ^ swz<T, S::NCH>(c)) * 16);
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) trans[dt] = column(lane, dt);
    }
    // columns 16 dt .. + 15
    static __device__ __forceinline__ int column(int lane, int dt)
    {
        const int c = lane & 15, g = lane >> 4;
        if constexpr (sizeof(T) == 2) {
            // group g reads rows 4 g .. 4 g + 3 of a block: lane j of it supplies row j / 4, columns 4 (j % 4) .. + 3 and
            // receives column j of the four rows
            const int row = 4 * g + (c >> 2);
            return row * S::RB + (((2 * dt + ((c & 3) >> 1)) ^ swz<T, S::NCH>(row)) * 16) + (c & 1) * 8;
        } else {
            return 4 * g * S::RB + (((4 * dt + (c >> 2)) ^ swz<T, S::NCH>(4 * g)) * 16) + (c & 3) * 4;
        }
    }
    __device__ __forceinline__ u32x4 row_frag(const unsigned char* tile, int t, int kk) const
    {
        return *reinterpret_cast<const u32x4*>(tile + t * 16 * S::RB + direct[kk]);
    }
    // bf16: sixteen columns of the 32 rows from 32 tp on, as the A operand of a product over those rows
    __device__ __forceinline__ u32x4 col_frag2(const unsigned char* tile, int tp, int dt) const { return column_frag2(tile, tp, trans[dt]); }
    static __device__ __forceinline__ u32x4 column_frag2(const unsigned char* tile, int tp, int at)
    {
        const unsigned char* p = tile + tp * 32 * S::RB + at;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(uint32_t)(uintptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(uint32_t)(uintptr_t)(p + 16 * S::RB));
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // float32: the same over the 16 rows from 16 t on (row 4 g + e: the low bits of the swizzle change with e)
    __device__ __forceinline__ u32x4 col_frag1(const unsigned char* tile, int t, int dt) const { return column_frag1(tile, t, trans[dt]); }
    static __device__ __forceinline__ u32x4 column_frag1(const unsigned char* tile, int t, int at)
    {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = *reinterpret_cast<const uint32_t*>(tile + t * 16 * S::RB + e * S::RB + (at ^ (e * 16)));
        return v;
    }
};

// acc[m][dt] += (streamed tile transposed) . w[m], the w of a first product's layout, for M sets of weights that share the
// tile.  Fragments are read one group ahead of the products that take them; the barriers keep the compiler from reading all
// of them at once, for want of registers.
template <typename T, int DP, int M>
__device__ __forceinline__ void second_products(f32x4 (&acc)[M][DP / 16], const f32x4 (&w)[M][4], const Reader<T, DP>& rd,
                                                const unsigned char* tile)
{
    using S = Shape<T, DP>;
    constexpr int STEPS = sizeof(T) == 2 ? 2 : 4;              // pieces of the 64 rows
    constexpr int G = S::DT < 4 ? S::DT : 4, PER = S::DT / G, N = STEPS * PER;
    u32x4 f[2][G];
    auto read = [&](int n, u32x4 (&to)[G]) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if constexpr (sizeof(T) == 2) to[i] = rd.col_frag2(tile, n / PER, (n % PER) * G + i);
            else to[i] = rd.col_frag1(tile, n / PER, (n % PER) * G + i);
        }
    };
    read(0, f[0]);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n + 1 < N) read(n + 1, f[(n + 1) & 1]);
        const int step = n / PER;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            u32x4 b;
            // bf16: rounded to nearest even, to as many bits as the other operand has and the matrix instruction takes.  The rounding's
            // rest as a second operand would double these products, half of all and more; the outputs, rounded to bf16 themselves (0.17 %),
            // are off by 0.19 % for the weights and 0.24 % for their gradients in place of that.
            if constexpr (sizeof(T) == 2)
                b = u32x4{pack_bf16x2(w[m][2 * step][0], w[m][2 * step][1]), pack_bf16x2(w[m][2 * step][2], w[m][2 * step][3]),
                          pack_bf16x2(w[m][2 * step + 1][0], w[m][2 * step + 1][1]),
                          pack_bf16x2(w[m][2 * step + 1][2], w[m][2 * step + 1][3])};
            else
                b = __builtin_bit_cast(u32x4, w[m][step]);
#pragma unroll
            for (int i = 0; i < G; ++i) acc[m][(n % PER) * G + i] = mma<T>(f[n & 1][i], b, acc[m][(n % PER) * G + i]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}
template <typename T, int DP>
__device__ __forceinline__ void second_product(f32x4 (&acc)[DP / 16], const f32x4 (&w)[4], const Reader<T, DP>& rd,
                                               const unsigned char* tile)
{
    second_products<T, DP, 1>(reinterpret_cast<f32x4 (&)[1][DP / 16]>(acc), reinterpret_cast<const f32x4 (&)[1][4]>(w), rd, tile);
}

// first[t] = streamed tile . owner, all 64 rows; the four blocks of rows side by side, since each is one chain of products.
template <typename T, int DP>
__device__ __forceinline__ void first_product(f32x4 (&first)[4], const u32x4 (&own)[DP * sizeof(T) / 64], const Reader<T, DP>& rd,
                                              const unsigned char* tile)
{
    using S = Shape<T, DP>;
    u32x4 f[2][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        first[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        f[0][t] = rd.row_frag(tile, t, 0);
    }
#pragma unroll
    for (int kk = 0; kk < S::KK; ++kk) {
        if (kk + 1 < S::KK) {
#pragma unroll
            for (int t = 0; t < 4; ++t) f[(kk + 1) & 1][t] = rd.row_frag(tile, t, kk + 1);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) first[t] = mma<T>(f[kk & 1][t], own[kk], first[t]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Dot product of two chunks.
template <typename T> __device__ __forceinline__ float dot_chunk(u32x4 x, u32x4 y)
{
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
            sum += __builtin_bit_cast(float, x[e] << 16) * __builtin_bit_cast(float, y[e] << 16);
            sum += __builtin_bit_cast(float, x[e] & 0xffff0000u) * __builtin_bit_cast(float, y[e] & 0xffff0000u);
        } else {
            sum += as_f32(x[e]) * as_f32(y[e]);
        }
    }
    return sum;
}

// Product with a weight: zero where either is, whatever the other.  A masked pair has weight zero, and the product beside it may have
// overflowed although all values are finite.
__device__ float mul_zero(float, float) __asm("llvm.amdgcn.fmul.legacy");       // v_mul_legacy_f32
__device__ __forceinline__ float weighed(float weight, float x) { return mul_zero(weight, x); }

// ---- lanes ------------------------------------------------------------------------------------------------

// Over the four lane groups (lanes c, c + 16, c + 32, c + 48): rows are swapped between two copies of the register.
__device__ __forceinline__ float group_max(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t t = __builtin_bit_cast(uint32_t, fmaxf(as_f32(a[0]), as_f32(a[1])));
    const auto b = __builtin_amdgcn_permlane16_swap(t, t, false, false);
    return fmaxf(as_f32(b[0]), as_f32(b[1]));
}
__device__ __forceinline__ float group_sum(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t t = __builtin_bit_cast(uint32_t, as_f32(a[0]) + as_f32(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(t, t, false, false);
    return as_f32(b[0]) + as_f32(b[1]);
}
// Over all 64 lanes, the same bits in every lane.
__device__ __forceinline__ float wave_total(float v)
{
    auto ror = [](float x, auto ctrl) {
        return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = ror(v, std::integral_constant<int, 0x128>{});       // row_ror:8, 4, 2, 1
    v = ror(v, std::integral_constant<int, 0x124>{});
    v = ror(v, std::integral_constant<int, 0x122>{});
    v = ror(v, std::integral_constant<int, 0x121>{});
    return group_sum(v);
}
// Over eight neighbouring lanes.
__device__ __forceinline__ float eight_lanes_total(float v)
{
    auto dpp = [](float x, auto ctrl) {
        return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = dpp(v, std::integral_constant<int, 0xB1>{});        // lane ^ 1
    v = dpp(v, std::integral_constant<int, 0x4E>{});        // lane ^ 2
    return dpp(v, std::integral_constant<int, 0x141>{});    // the other four of eight
}
__device__ __forceinline__ int wave_max_i(int v)
{
    return __builtin_amdgcn_readlane(wave_incl_scan_op(v, (int)0x80000000, [](int a, int b) { return a > b ? a : b; }), kWave - 1);
}

// ---- scores -----------------------------------------------------------------------------------------------

// tanh: near zero by its series (what is left out is at most 6.0e-8 of the value, at 0.4: half a step of float32), else
// 1 - 2 / (e^2x + 1), whose error of 1.2e-7 is small beside values of at least tanh 0.4.
__device__ __forceinline__ float tanh_f32(float x)
{
    const float y = x * x;
    float s = -1382.f / 155925.f;
    s = s * y + 62.f / 2835.f;
    s = s * y - 17.f / 315.f;
    s = s * y + 2.f / 15.f;
    s = s * y - 1.f / 3.f;
    s = s * y * x + x;
    const float t = __builtin_amdgcn_exp2f(x * (2.f * kLog2e));
    const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(t + 1.f);
    return fabsf(x) < 0.4f ? s : far;
}

// A bias or lse in units of log 2, rounded by itself wherever it is used, so that a pair has the same score in every pass.  Finite ones
// stay finite, with room for a product beside them: the lowest number of the type hides a pair from rows that see others, and
// no more than that.
constexpr float kMostScore = 3e38f;
__device__ __forceinline__ float to_log2(float x)
{
#pragma clang fp contract(off)
    const float y = x * kLog2e;
    return fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(y, -kMostScore, kMostScore) : y;
}
// And back: the log of a row's sum.  At the end of the range it is the end of the type.
__device__ __forceinline__ float row_lse(float top, float total)
{
    const float lse = top * kLn2 + logf(total);
    return fabsf(top) >= kMostScore && fabsf(lse) < INFINITY ? copysignf(3.402823466e38f, top) : lse;
}

// A tile's products to scores in units of log 2: scaled, capped, with the bias `flat2` of the whole tile; slope (capped
// scores only): d score / d product over the scale.  The groups are kept apart, or the compiler works on all 16 at once and runs
// out of registers.
template <bool CAP, int N>
__device__ __forceinline__ void to_scores(f32x4 (&s)[N], f32x4 (&slope)[CAP ? N : 1], float zc, float cap2, float z2, float flat2)
{
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if constexpr (CAP) {
                const float th = tanh_f32(s[n][r] * zc);
                slope[n][r] = 1.f - th * th;
                s[n][r] = th * cap2 + flat2;
            } else {
                s[n][r] = s[n][r] * z2 + flat2;
            }
        }
        if constexpr (CAP) __builtin_amdgcn_sched_barrier(0);
    }
}

// bias: at the lane's first row of the tile.
__device__ __forceinline__ void add_bias(f32x4 (&s)[4], const float* bias)
{
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[n][r] += bias[16 * n + r];
}

// border: the borders in LDS.  The logarithm gives the bucket or one beside it.
__device__ __forceinline__ int bucket_side(const AttBuckets& bk, const int* border, int n)
{
    int i = (int)(__builtin_amdgcn_logf((float)n * bk.inv_exact) * bk.per_log2);
    i = i < 0 ? 0 : i > bk.borders ? bk.borders : i;
    const int below = border[i > 0 ? i - 1 : 0], above = border[i];
    if (i > 0 && n < below) --i;
    else if (i < bk.borders && n >= above) ++i;
    return n < bk.exact ? n : bk.exact + i;
}
__device__ __forceinline__ int bucket_of(const AttBuckets& bk, const int* border, int n)
{
    const int b = bucket_side(bk, border, n < 0 ? -n : n);
    return n >= 0 ? b : bk.two_sided ? bk.side + b : 0;
}
// The one bucket of all distances in [lo, hi], or -1 (several, or not looked for).
__device__ __forceinline__ int uniform_bucket(const AttBuckets& bk, int lo, int hi)
{
    if (lo >= bk.last) return bk.side - 1;
    if (hi < 0 && !bk.two_sided) return 0;
    if (hi < 0 && -hi >= bk.last) return 2 * bk.side - 1;
    return -1;
}

// The backward pass has 2^(s - lse) for weights, and lse is one float32: far from zero the log of a row's sum is lost beside its
// largest score, and the rounding alone is a factor (a power of two and more from 1e8 on, where programs mask with a
// bias).  Rows beyond this |lse| are given their maximum and sum again, as two numbers; up to it a weight is off by less than 2^-15.
// Looking for such rows costs 1 to 4 % of a backward pass; where all rows are, 1024 x 200, 8 heads of 128, takes 2.38 ms and 2.18
// without, 8 x 2000 809 us and 611, one-tile histories (1024 x 50, 4 heads of 64) 73 and 70.
constexpr float kFarLse = 256.f;
__device__ __forceinline__ bool far_lse(float lse) { return fabsf(lse) > kFarLse && fabsf(lse) < INFINITY; }

// ---- non-finite values ------------------------------------------------------------------------------------
//
// A masked pair has weight zero, and zero times an infinity or a NaN of the streamed tile is not zero: a product over the
// tile's rows would carry such a value to owner rows that do not see it.  In tiles with masked pairs a chunk that holds one
// goes to LDS as zeros, and the row that it belongs to is marked instead: its scores become NaN where they are visible.
template <typename T> __device__ __forceinline__ bool chunk_nonfinite(u32x4 v)
{
    if constexpr (sizeof(T) == 2) {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 most = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = v[e] & 0x7f807f80u;
            most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x));
        }
        return most[0] == 0x7f80 || most[1] == 0x7f80;
    } else {
        uint32_t most = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t x = v[e] & 0x7f800000u;
            most = most > x ? most : x;
        }
        return most == 0x7f800000u;
    }
}

// ---- walking the streamed rows ----------------------------------------------------------------------------

// Work item of a block: the blocks of one head of one history share its rows, so neighbours in this order go to one XCD
// (blocks are dealt to the 8 XCDs in turn).
__device__ __forceinline__ int xcd_item(int items)
{
    const int each = (items + 7) / 8;
    const int item = (int)(blockIdx.x & 7) * each + (int)(blockIdx.x >> 3);
    return (int)(blockIdx.x >> 3) < each && item < items ? item : -1;
}

__device__ __forceinline__ int row_segment(const int* __restrict__ seg, int row, int length)
{
    if (row >= length) return kNoSeg;
    const int v = seg ? seg[row] : 0;
    return v < 0 ? kNoSeg : v;
}

// A history's prefix, clipped to its length: sums with it stay in range whatever the entry holds.
__device__ __forceinline__ int prefix_of(const int* __restrict__ prefix, int batch, int length)
{
    const int p = prefix ? prefix[batch] : 0;
    return p < length ? p : length;
}

struct TileMarks {
    uint32_t active[kAttMaxTiles / 32], mixed[kAttMaxTiles / 32];
    int red[12];
};

// Marks the tiles [t0, t1) of streamed rows that hold a row of a segment in the owner rows' range, and among them those
// with any row that is not of the one segment all owner rows have.  own: this lane's segment of its owner row, if there.
__device__ __forceinline__ void mark_tiles(TileMarks& mk, const int* __restrict__ seg, int length, int own, bool there, int t0, int t1)
{
    const int lane = lane_id(), tid = threadIdx.x % kBlock, wave = tid / kWave;
    int lo = there && own >= 0 ? own : 0x7fffffff, hi = there && own >= 0 ? own : -1;
    lo = wave_min(lo), hi = wave_max_i(hi);
    int bad = __any(there && own < 0);
    if (lane == 0) mk.red[wave] = lo, mk.red[4 + wave] = hi, mk.red[8 + wave] = bad;
    for (int i = t0 / 32 + tid; i <= t1 / 32; i += kBlock)
        if (i < kAttMaxTiles / 32) mk.active[i] = 0u, mk.mixed[i] = 0u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) {
        lo = mk.red[w] < lo ? mk.red[w] : lo;
        hi = mk.red[4 + w] > hi ? mk.red[4 + w] : hi;
        bad |= mk.red[8 + w];
    }
    const bool one = lo == hi && !bad;
    for (int t = t0 + wave; t < t1; t += kWavesPerBlock) {
        const int v = row_segment(seg, t * kTile + lane, length);
        const bool touch = __any(v >= lo && v <= hi);
        const bool plain = one && __all(v == lo);
        if (lane == 0) {
            if (touch) atomicOr(&mk.active[t >> 5], 1u << (t & 31));
            if (!plain) atomicOr(&mk.mixed[t >> 5], 1u << (t & 31));
        }
    }
    __syncthreads();
}

// Launches of no more blocks than there are CUs leave each SIMD with one wave, whose loads, products and
// exponentials wait for one another.  There a block takes twice the waves: SPLIT sets of four share the owner rows, each
// walks every SPLIT-th of the tiles in LDS of its own, and the first joins what they found, always in the same order.
// 1 x 1500 queries in 4 heads of 64: 21 us with two sets and 28 with one, gradients 56 and 73; 4 x 100 the same with both.
// Up to two blocks per CU the last rows of long causal histories keep the launch waiting: 2 x 2048, 8 heads of 64, takes 34 us
// and 42, its gradients 90 and 122 (float32: 99 and 155, 308 and 479).  Without the causal mask, whose blocks are alike, they
// would take 143 us, and 16 x 200, 8 heads of 128, in as many blocks 16 us in place of 11.  Rows of 512 bytes (float32, more than 64
// elements) stay with one set: two of the queries' gradients do not fit a CU's LDS (72 KB of tiles and strips each, 24 of sums), and
// the others gain little (2 x 1003, 4 heads of 128: 91 us and 96, gradients 582 and 623; 4 x 200: 24 and 24, 85 and 84).
constexpr int kFewBlocks = 256, kLongTiles = 32;

// What the second set found, handed over through LDS that held tiles (all waves behind a barrier): lane by lane.
template <int DT> __device__ __forceinline__ void hand_over(unsigned char* room, const f32x4 (&acc)[DT], int wave, int lane)
{
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) reinterpret_cast<f32x4*>(room)[(wave * DT + dt) * kWave + lane] = acc[dt];
}
template <int DT> __device__ __forceinline__ void take_over(const unsigned char* room, f32x4 (&acc)[DT], float mine, float theirs,
                                                            int wave, int lane)
{
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
        acc[dt] = acc[dt] * mine + reinterpret_cast<const f32x4*>(room)[(wave * DT + dt) * kWave + lane] * theirs;
}

// mk NULL: every tile is active and none is mixed.
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
__device__ __forceinline__ bool tile_mixed(const TileMarks* mk, int t)
{
    return mk && __builtin_amdgcn_readfirstlane((mk->mixed[t >> 5] >> (t & 31)) & 1);
}

// The streamed operands: a tile of each, loaded to registers while the tile before is worked on, then written to LDS.
template <typename T, int DP, int UNIT> struct Feed {
    using S = Shape<T, DP>;
    static constexpr int STEP = kBlock / S::NCH;      // rows between a thread's chunks
    const int tid;
    u32x4 a[S::NC], b[S::NC];
    int seg;                                          // of row (lane) of the tile

    __device__ __forceinline__ explicit Feed(int thread) : tid(thread), seg(kNoSeg) {}
    // pa, pb: row row0 of the operands; BOTH false: a alone
    template <bool BOTH = true>
    __device__ __forceinline__ void load(const T* pa, int64_t sa, const T* pb, int64_t sb, int row0, int length,
                                         const int* __restrict__ segments, int dim)
    {
        const RowSource ra = row_source(pa, sa, length - row0, dim), rb = row_source(pb, sb, length - row0, dim);
        const uint32_t row = (uint32_t)tid / S::NCH;
        const int ch = (uint32_t)tid % S::NCH;
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            a[i] = load_chunk<T, UNIT>(ra, (row + i * STEP) * ra.stride, ch, dim);
            if constexpr (BOTH) b[i] = load_chunk<T, UNIT>(rb, (row + i * STEP) * rb.stride, ch, dim);
            else b[i] = u32x4{0u, 0u, 0u, 0u};
        }
        seg = row_segment(segments, row0 + (tid & (kWave - 1)), length);
    }
    // masked: the tile has masked pairs.  MARK_A: the mark of a row is a NaN among its elements of a (the operand of the first
    // product only); else its bit in bad[].
    template <bool MARK_A, bool BOTH = true>
    __device__ __forceinline__ void put(unsigned char* ta, unsigned char* tb, int* s_seg, bool masked, uint32_t* bad)
    {
        const int row = (uint32_t)tid / S::NCH, ch = (uint32_t)tid % S::NCH;
        const uint64_t there = __ballot(seg != kNoSeg);
        if (~there) {                                 // padding contributes nothing, whatever it holds
#pragma unroll
            for (int i = 0; i < S::NC; ++i)
                if (!((there >> (row + i * STEP)) & 1)) a[i] = b[i] = u32x4{0u, 0u, 0u, 0u};
        }
        if (masked) {
#pragma unroll
            for (int i = 0; i < S::NC; ++i) {
                const bool odd_a = chunk_nonfinite<T>(a[i]), odd_b = chunk_nonfinite<T>(b[i]);
                if (odd_a || odd_b) {
                    if (odd_a) a[i] = u32x4{0u, 0u, 0u, 0u};
                    if (odd_b) b[i] = u32x4{0u, 0u, 0u, 0u};
                    if (MARK_A) a[i][0] = sizeof(T) == 2 ? 0x7fc0u : 0x7fc00000u;
                    else if (bad) atomicOr(&bad[(row + i * STEP) >> 5], 1u << ((row + i * STEP) & 31));
                }
            }
        }
        if ((tid >> 6) == 0) s_seg[(tid & (kWave - 1))] = seg;
#pragma unroll
        for (int i = 0; i < S::NC; ++i) {
            const int at = (row + i * STEP) * S::RB + ((ch ^ swz<T, S::NCH>(row + i * STEP)) * 16);
            *reinterpret_cast<u32x4*>(ta + at) = a[i];
            if constexpr (BOTH) *reinterpret_cast<u32x4*>(tb + at) = b[i];
        }
    }
};

// A tile's masked scores: minus infinity where the row of the tile is not in the owner's segment (SEGMENTS; else only the
// place counts) or not below `edge` (FROM: among the `span` rows from `edge` on).
template <bool SEGMENTS, bool FROM>
__device__ __forceinline__ void mask_scores(f32x4 (&s)[4], const int* s_seg, int own, int edge, int lane, int span = 0)
{
    const int g4 = 4 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        typedef int i32x4 __attribute__((ext_vector_type(4)));
        i32x4 sg = {0, 0, 0, 0};
        if (SEGMENTS) sg = *reinterpret_cast<const i32x4*>(s_seg + 16 * n + g4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const bool in = FROM ? (uint32_t)(16 * n + r + (g4 - edge)) < (uint32_t)span : 16 * n + r < edge - g4;
            const bool see = (!SEGMENTS || sg[r] == own) && in;
            s[n][r] = see ? s[n][r] : -INFINITY;
        }
    }
}

// Owner fragments: row c of the wave's 16, zeros where the row is padding or not there.
template <typename T, int DP, int UNIT>
__device__ __forceinline__ void load_owner(u32x4 (&f)[DP * sizeof(T) / 64], const T* base, int64_t sr, int rows, int dim, bool live,
                                           int lane)
{
    const RowSource src = row_source(base, sr, rows < 16 ? rows : 16, dim);
    const int c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int kk = 0; kk < Shape<T, DP>::KK; ++kk) {
        f[kk] = load_chunk<T, UNIT>(src, (uint32_t)c * src.stride, g + 4 * kk, dim);
        if (!live) f[kk] = u32x4{0u, 0u, 0u, 0u};
    }
}

// A wave's 16 owner rows (lane (c, g): row c, columns 16 dt + 4 g + r) times `scale`, to memory.  They pass through the
// wave's own rows of LDS, so that a store covers whole rows: straight from the accumulators it would write 32 bytes (bf16) of
// 16 rows, which took the pass over the keys a quarter longer (1.32 against 1.06 ms without stores on 1024 x 200, 8 heads of
// 128).  room: 16 rows of LDS that no wave reads any more.
template <typename T, int DP, int UNIT>
__device__ __forceinline__ void store_rows(unsigned char* room, const f32x4 (&acc)[DP / 16], float scale, T* base, int64_t sr, int rows, int dim,
                                           int lane)
{
    using S = Shape<T, DP>;
    const int c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) {
        const f32x4 v = acc[dt] * scale;
        if constexpr (sizeof(T) == 2) {
            const u32x2 h = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            *reinterpret_cast<u32x2*>(room + c * S::RB + (((2 * dt + (g >> 1)) ^ swz<T, S::NCH>(c)) * 16) + (g & 1) * 8) = h;
        } else {
            *reinterpret_cast<f32x4*>(room + c * S::RB + (((4 * dt + g) ^ swz<T, S::NCH>(c)) * 16)) = v;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    constexpr int EPC = 16 / sizeof(T), ROWS = kWave / S::NCH;             // rows per pass of the wave
#pragma unroll
    for (int i = 0; i < 16 / ROWS; ++i) {
        const int row = i * ROWS + lane / S::NCH, ch = lane % S::NCH, at = ch * EPC;
        const u32x4 v = *reinterpret_cast<const u32x4*>(room + row * S::RB + ((ch ^ swz<T, S::NCH>(row)) * 16));
        if (row >= rows || at >= dim) continue;
        T* const to = base + row * sr + at;
        if constexpr (UNIT == 16) {
            *reinterpret_cast<u32x4*>(to) = v;
        } else if constexpr (UNIT == 8) {
            *reinterpret_cast<u32x2*>(to) = u32x2{v[0], v[1]};
            if (at + 4 < dim) *reinterpret_cast<u32x2*>(to + 4) = u32x2{v[2], v[3]};
        } else {
#pragma unroll
            for (int e = 0; e < EPC; ++e)
                if (at + e < dim) {
                    if constexpr (sizeof(T) == 2) to[e].bits = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
                    else to[e] = as_f32(v[e]);
                }
        }
    }
    __builtin_amdgcn_wave_barrier();
}

// ---- the gradient of the table ----------------------------------------------------------------------------

constexpr int kNear = 383;       // distances that have a sum of their own
constexpr int kStrip = 92;       // distances of a wave's 16 queries and a tile's 64 keys, each group's row of them

// The table's gradient.  A tile of one bucket adds its ds to a register of each lane.  A tile of several adds along its
// diagonals, which are the distances: lane (c, g) holds queries c and keys 16 n + 4 g + r, distance (a number of the tile)
// + c - 4 g - r - 16 n.  Shifting the registers r = 1..3 by r lanes within their row of 16 brings equal distances
// together; what is shifted out belongs to the same lanes' distances of n + 1.  That leaves five values a lane, distance
// + c - 4 g - 16 n, n = 0..4; the four groups are joined through LDS, where the sum of a distance is added to the wave's
// own `dist` row (distances within kNear) or, farther out where buckets are wide, bucket by bucket.  No word has two
// writers, so every sum has one order.
template <int SHIFT> __device__ __forceinline__ float row_shift(float v)        // lane i gets lane i + SHIFT's, 0 from outside
{
    constexpr int CTRL = SHIFT > 0 ? 0x100 | SHIFT : 0x110 | -SHIFT;            // row_shl, row_shr
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ void add_bucket(float* bucket, int b, float lane_sums, int lane)
{
    const float sum = wave_total(lane_sums);
    if (lane == 0) bucket[b] += sum;
}

// top: the distance of the wave's first query and the tile's first key.
__device__ __forceinline__ void table_near(const AttArgs& a, const f32x4 (&ds)[4], int top, float (*strip)[kStrip], float* dist,
                                           float* bucket, const int* border, int lane)
{
    const int c = lane & 15, g = lane >> 4;
    float spill = 0.f;
    // distance top + c - 4 g - 16 n lies at place c - 4 g - 16 n + 76 of its group's row
    float* const at = &strip[g][c - 4 * g + 76];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        at[-16 * n] = ds[n][0] + row_shift<1>(ds[n][1]) + row_shift<2>(ds[n][2]) + row_shift<3>(ds[n][3]) + spill;
        spill = row_shift<-15>(ds[n][1]) + row_shift<-14>(ds[n][2]) + row_shift<-13>(ds[n][3]);
    }
    at[-64] = spill;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float sum[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int place = lane + 64 * h;
        sum[h] = 0.f;
        if (place < kStrip) sum[h] = (strip[0][place] + strip[1][place]) + (strip[2][place] + strip[3][place]);
    }
    __builtin_amdgcn_wave_barrier();
    const int n0 = top - 76;                                   // distance of place 0
    if (n0 >= -kNear && n0 + kStrip - 1 <= kNear) {
        dist[n0 + lane] += sum[0];
        if (lane + 64 < kStrip) dist[n0 + 64 + lane] += sum[1];
    } else {
        const int b0 = bucket_of(a.bk, border, n0 + lane), b1 = bucket_of(a.bk, border, n0 + 64 + lane);
        uint64_t left0 = ~0ull, left1 = __ballot(lane + 64 < kStrip);
        while (left0 | left1) {
            const int b = left0 ? __builtin_amdgcn_readlane(b0, __builtin_ctzll(left0)) : __builtin_amdgcn_readlane(b1, __builtin_ctzll(left1));
            const bool m0 = b0 == b, m1 = lane + 64 < kStrip && b1 == b;
            add_bucket(bucket, b, (m0 ? sum[0] : 0.f) + (m1 ? sum[1] : 0.f), lane);
            left0 &= ~__ballot(m0), left1 &= ~__ballot(m1);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// ---- launches ---------------------------------------------------------------------------------------------
// unit: bytes per global access (template argument UNIT): 16, 8 (bf16 only), or the size of an element
template <typename F> inline void by_shape(const gram_attention_config& c, int unit, F&& go)
{
    auto width = [&](auto type, auto u) {
        if (c.head_dim <= 32) go(type, std::integral_constant<int, 32>{}, u);
        else if (c.head_dim <= 64) go(type, std::integral_constant<int, 64>{}, u);
        else go(type, std::integral_constant<int, 128>{}, u);
    };
    if (c.dtype == GRAM_BF16) {
        if (unit == 16) width(Bf16{}, std::integral_constant<int, 16>{});
        else if (unit == 8) width(Bf16{}, std::integral_constant<int, 8>{});
        else width(Bf16{}, std::integral_constant<int, 2>{});
    } else {
        if (unit == 16) width(float{}, std::integral_constant<int, 16>{});
        else width(float{}, std::integral_constant<int, 4>{});
    }
}
template <typename F> inline void by_shape_and_cap(const gram_attention_config& c, int unit, F&& go)
{
    by_shape(c, unit, [&](auto type, auto dp, auto u) {
        if (c.cap > 0.f) go(type, dp, u, std::true_type{});
        else go(type, dp, u, std::false_type{});
    });
}
inline dim3 att_grid(int items) { return dim3((unsigned)((items + 7) / 8 * 8)); }
constexpr int att_blocks(int length, int rows) { return (length + rows - 1) / rows; }
inline bool two_sets(const AttArgs& a)
{
    const int tiles = att_blocks(a.length, kTile);
    return tiles > 1 && (a.items <= kFewBlocks || (a.causal && a.items <= 2 * kFewBlocks && tiles >= kLongTiles));
}

void attend_forward(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s);      // gram_attend_fwd.hip
// Histories of one tile: all gradients in one launch.  False: not for this shape.
bool attend_backward_short(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s);       // gram_attend_short.hip
void attend_backward_queries(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s);     // gram_attend_dq.hip
void attend_backward_keys(const gram_attention_config& c, AttArgs a, int unit, hipStream_t s);        // gram_attend_dkv.hip

// ---- gram_attend_step.hip ---------------------------------------------------------------------------------
int64_t step_part_bytes(const gram_attention_config& c, int32_t batch, int32_t capacity);
bool step_launch(const gram_attention_config& c, const AttBuckets& bk, int32_t batch, int32_t capacity, const AttRows& q,
                 const AttRows& kn, const AttRows& vn, const AttRows& kc, const AttRows& vc, const AttRows& o,
                 const int* lengths, const int* first, const float* table, void* work, int unit, hipStream_t s);

}  // namespace gram
