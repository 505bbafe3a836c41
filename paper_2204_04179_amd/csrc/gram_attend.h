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
    int border[kMaxBorders];
};

struct AttArgs {
    AttRows q, k, v, o, dout, dq, dk, dv;
    const int* seg;
    const int* prefix;
    const float* table;
    float* lse;
    float* delta;            // [batch, heads, length]
    float* part;             // partial gradients of the table: [heads, parts, buckets]
    int batch, length, heads, kv_heads, group, dim;
    int causal, unit;        // unit: bytes per global load and store of an operand row (16, 8, or one element)
    int items, parts;
    float scale, cap;
    AttBuckets bk;
};

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

// 16-byte chunk `ch` of row `row` lies at chunk ch ^ swz(row): the 16 rows of a fragment read start in different banks.
template <int NCH> __device__ __forceinline__ int swz(int row)
{
    return NCH >= 16 ? row & 15 : NCH == 8 ? row & 7 : (row >> 1) & 3;
}

// ---- global rows ------------------------------------------------------------------------------------------

// One 16-byte chunk of a row of `dim` elements, zeros behind them.  unit: what alignment allows per load.
template <typename T> __device__ __forceinline__ u32x4 load_chunk(const T* __restrict__ row, int ch, int dim, int unit)
{
    constexpr int EPC = 16 / sizeof(T);
    const int at = ch * EPC;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (unit == 16) {
        if (at < dim) v = *reinterpret_cast<const u32x4*>(row + at);
    } else if (sizeof(T) == 2 && unit == 8) {
        if (at < dim) {
            const u32x2 t = *reinterpret_cast<const u32x2*>(row + at);
            v[0] = t[0], v[1] = t[1];
        }
        if (at + 4 < dim) {
            const u32x2 t = *reinterpret_cast<const u32x2*>(row + at + 4);
            v[2] = t[0], v[3] = t[1];
        }
    } else {
#pragma unroll
        for (int e = 0; e < EPC; ++e)
            if (at + e < dim) {
                if constexpr (sizeof(T) == 2) v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[at + e] << (16 * (e & 1));
                else v[e] = reinterpret_cast<const uint32_t*>(row)[at + e];
            }
    }
    return v;
}

// Four neighbouring elements at column `at`.
template <typename T> __device__ __forceinline__ void store4(T* __restrict__ row, int at, int dim, int unit, f32x4 v)
{
    if (unit >= 8) {                 // rows are whole groups of four elements
        if (at < dim) {
            if constexpr (sizeof(T) == 2) {
                const u32x2 t = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                *reinterpret_cast<u32x2*>(row + at) = t;
            } else {
                *reinterpret_cast<f32x4*>(row + at) = v;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < dim) {
                if constexpr (sizeof(T) == 2) row[at + e].bits = (uint16_t)pack_bf16x2(v[e], 0.f);
                else row[at + e] = v[e];
            }
    }
}

__device__ __forceinline__ bool nonfinite_bits(uint32_t f32_bits) { return (f32_bits & 0x7f800000u) == 0x7f800000u; }

// Replaces non-finite elements of a chunk by zero; true if there was one.
template <typename T> __device__ __forceinline__ bool clean_chunk(u32x4& v)
{
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
            if ((v[e] & 0x7f80u) == 0x7f80u) any = true, v[e] &= 0xffff0000u;
            if (nonfinite_bits(v[e])) any = true, v[e] &= 0x0000ffffu;
        } else {
            if (nonfinite_bits(v[e])) any = true, v[e] = 0u;
        }
    }
    return any;
}

template <typename T> __device__ __forceinline__ float load_elem(const T* p)
{
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, (uint32_t)p->bits << 16);
    else return *p;
}

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

    __device__ __forceinline__ Reader()
    {
        const int c = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) direct[kk] = c * S::RB + (((g + 4 * kk) ^ swz<S::NCH>(c)) * 16);
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) {
            if constexpr (sizeof(T) == 2) {
                // group g reads rows 4 g .. 4 g + 3 of a block: lane j of it supplies row j / 4, columns 4 (j % 4) .. + 3
                // and receives column j of the four rows
                const int row = 4 * g + (c >> 2);
                trans[dt] = row * S::RB + (((2 * dt + ((c & 3) >> 1)) ^ swz<S::NCH>(row)) * 16) + (c & 1) * 8;
            } else {
                trans[dt] = 4 * g * S::RB + (((4 * dt + (c >> 2)) ^ swz<S::NCH>(4 * g)) * 16) + (c & 3) * 4;
            }
        }
    }
    __device__ __forceinline__ u32x4 row_frag(const unsigned char* tile, int t, int kk) const
    {
        return *reinterpret_cast<const u32x4*>(tile + t * 16 * S::RB + direct[kk]);
    }
    // bf16: columns 16 dt .. + 15 of the 32 rows from 32 tp on, as the A operand of a product over those rows
    __device__ __forceinline__ u32x4 col_frag2(const unsigned char* tile, int tp, int dt) const
    {
        const unsigned char* p = tile + tp * 32 * S::RB + trans[dt];
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(uint32_t)(uintptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(uint32_t)(uintptr_t)(p + 16 * S::RB));
        return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // float32: the same over the 16 rows from 16 t on (row 4 g + e: the low bits of the swizzle change with e)
    __device__ __forceinline__ u32x4 col_frag1(const unsigned char* tile, int t, int dt) const
    {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = *reinterpret_cast<const uint32_t*>(tile + t * 16 * S::RB + e * S::RB + (trans[dt] ^ (e * 16)));
        return v;
    }
};

// acc[dt] += (streamed tile transposed) . w, the w of a first product's layout.
template <typename T, int DP>
__device__ __forceinline__ void second_product(f32x4 (&acc)[DP / 16], const f32x4 (&w)[4], const Reader<T, DP>& rd,
                                               const unsigned char* tile)
{
    using S = Shape<T, DP>;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int tp = 0; tp < 2; ++tp) {
            // rounded to nearest even as they enter the matrix cores, whose other operand has as few bits
            const u32x4 b = {pack_bf16x2(w[2 * tp][0], w[2 * tp][1]), pack_bf16x2(w[2 * tp][2], w[2 * tp][3]),
                             pack_bf16x2(w[2 * tp + 1][0], w[2 * tp + 1][1]), pack_bf16x2(w[2 * tp + 1][2], w[2 * tp + 1][3])};
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) acc[dt] = mma<T>(rd.col_frag2(tile, tp, dt), b, acc[dt]);
        }
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u32x4 b = __builtin_bit_cast(u32x4, w[t]);
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) acc[dt] = mma<T>(rd.col_frag1(tile, t, dt), b, acc[dt]);
        }
    }
}

// first[t] = streamed tile . owner, all 64 rows.
template <typename T, int DP>
__device__ __forceinline__ void first_product(f32x4 (&first)[4], const u32x4 (&own)[DP * sizeof(T) / 64], const Reader<T, DP>& rd,
                                              const unsigned char* tile)
{
    using S = Shape<T, DP>;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        first[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < S::KK; ++kk) first[t] = mma<T>(rd.row_frag(tile, t, kk), own[kk], first[t]);
    }
}

// What second_product leaves out where a tile holds non-finite elements and some pairs of it are masked: the tile went to
// LDS with zeros in their place, since a zero weight times them would not be zero, and the pairs that are visible take
// them here from memory.  Rare, so written to be small.
template <typename T, int DP>
__device__ __forceinline__ void add_nonfinite(f32x4 (&acc)[DP / 16], const f32x4 (&w)[4], uint32_t vis,
                                              const T* __restrict__ base, int64_t sr, int rows, int dim)
{
    const int c = lane_id() & 15, g = lane_id() >> 4;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
        float wi = w[0][0];
#pragma unroll
        for (int s = 1; s < 16; ++s) wi = s == i ? w[s >> 2][s & 3] : wi;
        const int vi = (vis >> i) & 1;
#pragma unroll 1
        for (int g2 = 0; g2 < 4; ++g2) {
            const int row = 16 * (i >> 2) + 4 * g2 + (i & 3);
            const float wk = __shfl(wi, g2 * 16 + c);
            const int vk = __shfl(vi, g2 * 16 + c);
            if (row >= rows) continue;
#pragma unroll
            for (int dt = 0; dt < Shape<T, DP>::DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int col = 16 * dt + 4 * g + e;
                    if (col < dim && vk) {
                        const float x = load_elem(base + row * sr + col);
                        if (nonfinite_bits(__builtin_bit_cast(uint32_t, x))) acc[dt][e] += wk * x;
                    }
                }
        }
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
__device__ __forceinline__ int wave_max_i(int v)
{
    return __builtin_amdgcn_readlane(wave_incl_scan_op(v, (int)0x80000000, [](int a, int b) { return a > b ? a : b; }), kWave - 1);
}

// ---- scores -----------------------------------------------------------------------------------------------

// tanh: near zero by its series (next term below 3e-8 of the value at 0.4), else 1 - 2 / (e^2x + 1), whose error of 1.2e-7
// is small beside values of at least tanh 0.4.
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

__device__ __forceinline__ int bucket_side(const AttBuckets& bk, int n)
{
    if (n < bk.exact) return n;
    int b = bk.exact;
    for (int i = 0; i < bk.borders; ++i) b += n >= bk.border[i];
    return b;
}
__device__ __forceinline__ int bucket_of(const AttBuckets& bk, int n)
{
    if (n >= 0) return bucket_side(bk, n);
    return bk.two_sided ? bk.side + bucket_side(bk, -n) : 0;
}
// The one bucket of all distances in [lo, hi], or -1 (several, or not looked for).
__device__ __forceinline__ int uniform_bucket(const AttBuckets& bk, int lo, int hi)
{
    const int last = bk.borders ? bk.border[bk.borders - 1] : bk.exact;      // from here on: bucket side - 1
    if (lo >= last) return bk.side - 1;
    if (hi < 0 && !bk.two_sided) return 0;
    if (-hi >= last && hi < 0) return 2 * bk.side - 1;
    return -1;
}

// ---- gram_attend_step.hip ---------------------------------------------------------------------------------
int64_t step_part_bytes(const gram_attention_config& c, int32_t batch, int32_t capacity);
bool step_launch(const gram_attention_config& c, const AttBuckets& bk, int32_t batch, int32_t capacity, const AttRows& q,
                 const AttRows& kn, const AttRows& vn, const AttRows& kc, const AttRows& vc, const AttRows& o,
                 const int* lengths, const int* first, const float* table, void* work, int unit, hipStream_t s);

}  // namespace gram
