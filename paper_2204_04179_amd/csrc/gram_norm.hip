// Layer norm of the positions' representations and its backward pass.
//
//   mu = mean(x)   var = mean((x - mu)^2)   r = (var + eps)^(-1/2)   xh = (x - mu) r   y = xh w + b
//   g = dy w       dx = r (g - mean(g) - xh mean(g xh)) [+ add]
//   dw = sum over rows of dy xh             db = sum over rows of dy
//
// A row stays in the registers of LPR lanes from its one read to its one write: the mean first, then the centred
// squares, so no two nearly equal numbers are subtracted.  All sums are float32; lanes are added by a butterfly, rows in
// a fixed order, so results are the same bits run to run.  What bounds both passes is HBM: each operand is touched once.
// 204,800 x 1024: float32 to bf16 207 us (6.1 TB/s), bf16 to bf16 156 us; backward of that with a float32 gradient added 466 us
// (5.4 TB/s).  51,200 x 4096, bf16: 215 us (3.9 TB/s) and 502 (5.0); 25,600 x 8192: 195 and 490, in float32 339 (5.0 TB/s) and 644
// (5.2).  7,040 x 400: 5.7 and 9.5 us, and 4.0 us for the last sum of 1.4 MB, of which a launch with nothing to add takes 2.5; 1,024
// partial rows of 8192 columns (67 MB) take it 24.
#include "gram_internal.h"

namespace gram {

namespace {

constexpr int kNormMaxParts = 1024;     // blocks of the backward pass: four per CU, each with its partial dw and db
constexpr int kNormPartRows = 16;       // rows per block at least,
constexpr int kNormWideRows = 4;        // where a block takes one row at a time

typedef float nf32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t nu32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t nu32x4 __attribute__((ext_vector_type(4)));

struct bf16_t { uint16_t bits; };

// VEC neighbouring elements as they lie in memory: 16 bytes per load, 8 for four of bf16.
template <typename T, int VEC> struct Raw {
    static constexpr int WORDS = VEC * (int)sizeof(T) / 4 > 0 ? VEC * (int)sizeof(T) / 4 : 1;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (VEC == 1) {
            if constexpr (sizeof(T) == 2) w[0] = p->bits;
            else w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (WORDS == 2) {
            const nu32x2 t = *reinterpret_cast<const nu32x2*>(p);
            w[0] = t[0], w[1] = t[1];
        } else {
#pragma unroll
            for (int q = 0; q < WORDS / 4; ++q) {
                const nu32x4 t = reinterpret_cast<const nu32x4*>(p)[q];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * q + e] = t[e];
            }
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) w[q] = 0u;
    }
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        else return __builtin_bit_cast(float, w[e]);
    }
};
template <int VEC, typename T> __device__ __forceinline__ void load_vec(const T* p, float* v)
{
    Raw<T, VEC> r;
    r.load(p);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = r.get(e);
}

template <int VEC> __device__ __forceinline__ void store_vec(float* p, const float* v)
{
    if constexpr (VEC == 1) {
        *p = v[0];
    } else {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
            const nf32x4 t = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            __builtin_nontemporal_store(t, reinterpret_cast<nf32x4*>(p) + q);
        }
    }
}

template <int VEC> __device__ __forceinline__ void store_vec(bf16_t* p, const float* v)
{
    if constexpr (VEC == 1) {
        p->bits = (uint16_t)pack_bf16x2(v[0], 0.f);
    } else if constexpr (VEC == 4) {
        const nu32x2 t = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        __builtin_nontemporal_store(t, reinterpret_cast<nu32x2*>(p));
    } else {
        const nu32x4 t = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        __builtin_nontemporal_store(t, reinterpret_cast<nu32x4*>(p));
    }
}

// Sum over the LPR lanes of a row (16: a DPP row; 64: a wave; 256: a block), the same bits in every lane.
template <int CTRL> __device__ __forceinline__ float add_dpp(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

template <int LPR, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float* s_red)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = add_dpp<0x128>(v[i]);    // row_ror:8
        v[i] = add_dpp<0x124>(v[i]);
        v[i] = add_dpp<0x122>(v[i]);
        v[i] = add_dpp<0x121>(v[i]);
        if constexpr (LPR > 16) {
            v[i] += __shfl_xor(v[i], 16);
            v[i] += __shfl_xor(v[i], 32);
        }
    }
    if constexpr (LPR > 64) {
        __syncthreads();                // the last row's sums have been read
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane_id() == 0) s_red[i * kWavesPerBlock + wave_id()] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (s_red[i * kWavesPerBlock] + s_red[i * kWavesPerBlock + 1]) +
                   (s_red[i * kWavesPerBlock + 2] + s_red[i * kWavesPerBlock + 3]);
    }
}

// One row per group of LPR lanes, VEC neighbouring columns per lane and chunk, CPL chunks.  x and y may be the same rows.
template <typename TX, typename TY, int VEC, int CPL, int LPR>
__global__ __launch_bounds__(kBlock) void k_layer_norm(const TX* x, const float* __restrict__ w,
                                                       const float* __restrict__ b, const int* __restrict__ seg, int64_t m,
                                                       int d, float inv_d, float eps, TY* y, float* __restrict__ stats)
{
    __shared__ float s_red[kWavesPerBlock];
    constexpr int RPB = kBlock / LPR;
    const int lr = threadIdx.x % LPR;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR; row < m; row += (int64_t)gridDim.x * RPB) {
        const bool live = !seg || seg[row] >= 0;
        float v[CPL * VEC];
        float sum[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int col = (c * LPR + lr) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[c * VEC + e] = 0.f;
            if (live && col < d) load_vec<VEC>(x + row * d + col, v + c * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[0] += v[c * VEC + e];
        }
        row_sum<LPR>(sum, s_red);
        const float mean = sum[0] * inv_d;
        sum[0] = 0.f;
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const bool in = (c * LPR + lr) * VEC < d;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[c * VEC + e] -= mean;
                sum[0] += in ? v[c * VEC + e] * v[c * VEC + e] : 0.f;
            }
        }
        row_sum<LPR>(sum, s_red);
        const float rstd = 1.f / sqrtf(sum[0] * inv_d + eps);
        if (stats && lr == 0) {
            stats[2 * row] = live ? mean : 0.f;
            stats[2 * row + 1] = live ? rstd : 0.f;
        }
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int col = (c * LPR + lr) * VEC;
            if (col < d) {
                float wv[VEC], bv[VEC];
                load_vec<VEC>(w + col, wv);
                load_vec<VEC>(b + col, bv);
#pragma unroll
                for (int e = 0; e < VEC; ++e) wv[e] = live ? v[c * VEC + e] * rstd * wv[e] + bv[e] : 0.f;
                store_vec<VEC>(y + row * d + col, wv);
            }
        }
    }
}

// Backward: the block walks rows blockIdx, blockIdx + gridDim, ... (times RPB) and keeps its share of dw and db in
// registers; at the end the groups of the block are added in order and the block writes one partial row of each.
template <typename TX, typename TY, int VEC, int CPL, int LPR>
__global__ __launch_bounds__(kBlock) void k_layer_norm_bwd(const TX* __restrict__ x, const float* __restrict__ w,
                                                           const float* __restrict__ stats, const TY* __restrict__ dy,
                                                           const int* __restrict__ seg, const float* add, int64_t m, int d,
                                                           float inv_d, float* dx, float* __restrict__ part)
{
    constexpr int RPB = kBlock / LPR;
    __shared__ float s_red[2 * kWavesPerBlock];
    __shared__ float s_part[RPB > 1 ? kBlock * VEC * CPL : 1];
    const int lr = threadIdx.x % LPR;
    float dwa[CPL * VEC], dba[CPL * VEC], wv[CPL * VEC];
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
        const int col = (c * LPR + lr) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) dwa[c * VEC + e] = dba[c * VEC + e] = wv[c * VEC + e] = 0.f;
        if (col < d) load_vec<VEC>(w + col, wv + c * VEC);
    }
    // a row is loaded while the one before it is worked on
    Raw<TX, VEC> rx[CPL];
    Raw<TY, VEC> ry[CPL];
    Raw<float, VEC> ra[CPL];
    float mean = 0.f, rstd = 0.f;
    bool live = false;
    auto fetch = [&](int64_t row) {
        live = !seg || seg[row] >= 0;
        mean = stats[2 * row], rstd = stats[2 * row + 1];
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int col = (c * LPR + lr) * VEC;
            rx[c].clear(), ry[c].clear(), ra[c].clear();
            if (col < d) {
                rx[c].load(x + row * d + col);
                ry[c].load(dy + row * d + col);
                if (add) ra[c].load(add + row * d + col);
            }
        }
    };
    const int64_t first = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
    if (first < m) fetch(first);
    for (int64_t row = first; row < m; row += (int64_t)gridDim.x * RPB) {
        const bool live_now = live;
        const float mean_now = mean, rstd_now = rstd;
        float xh[CPL * VEC], g[CPL * VEC], ad[CPL * VEC];
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const bool in = (c * LPR + lr) * VEC < d && live_now;      // padding is not used, whatever it holds
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                xh[c * VEC + e] = in ? (rx[c].get(e) - mean_now) * rstd_now : 0.f;
                g[c * VEC + e] = in ? ry[c].get(e) : 0.f;
                ad[c * VEC + e] = ra[c].get(e);
            }
        }
        if (row + (int64_t)gridDim.x * RPB < m) fetch(row + (int64_t)gridDim.x * RPB);
#pragma unroll
        for (int i = 0; i < CPL * VEC; ++i) {
            dwa[i] += g[i] * xh[i];
            dba[i] += g[i];
            g[i] *= wv[i];
            sum[0] += g[i];
            sum[1] += g[i] * xh[i];
        }
        row_sum<LPR>(sum, s_red);
        const float mg = sum[0] * inv_d, mgx = sum[1] * inv_d;
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
            const int col = (c * LPR + lr) * VEC;
            if (col < d) {
                float o[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int i = c * VEC + e;
                    o[e] = live_now ? rstd_now * (g[i] - mg - xh[i] * mgx) + ad[i] : 0.f;
                }
                store_vec<VEC>(dx + row * d + col, o);
            }
        }
    }
    float* const out = part + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float* const mine = half ? dba : dwa;
        if constexpr (RPB > 1) {
            __syncthreads();
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    s_part[(threadIdx.x / LPR) * (LPR * VEC * CPL) + (c * LPR + lr) * VEC + e] = mine[c * VEC + e];
            __syncthreads();
            for (int col = threadIdx.x; col < d; col += kBlock) {
                float t = 0.f;
#pragma unroll
                for (int r = 0; r < RPB; ++r) t += s_part[r * (LPR * VEC * CPL) + col];
                out[half * d + col] = t;
            }
        } else {
#pragma unroll
            for (int c = 0; c < CPL; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int col = (c * LPR + lr) * VEC + e;
                    if (col < d) out[half * d + col] = mine[c * VEC + e];
                }
        }
    }
}

// dw and db from the partial rows: 16 columns per block, 64 strands of rows each, added in a fixed order.
__global__ __launch_bounds__(1024) void k_layer_norm_parts(const float* __restrict__ part, int parts, int d,
                                                           float* __restrict__ dw, float* __restrict__ db)
{
    __shared__ float s[1024];
    const int col = blockIdx.x * 16 + threadIdx.x % 16, strand = threadIdx.x / 16;
    float sum = 0.f;
    if (col < 2 * d) {
        const float* const p = part + col;
#pragma unroll 8
        for (int i = strand; i < parts; i += 64) sum += p[(int64_t)i * 2 * d];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 256) s[threadIdx.x] = (s[threadIdx.x] + s[threadIdx.x + 256]) + (s[threadIdx.x + 512] + s[threadIdx.x + 768]);
    __syncthreads();
    if (strand == 0 && col < 2 * d) {
        sum = 0.f;
#pragma unroll
        for (int t = 0; t < 16; ++t) sum += s[t * 16 + threadIdx.x];
        if (col < d) dw[col] = sum;
        else db[col - d] = sum;
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int norm_parts(int64_t m, int rows)
{
    const int64_t p = (m + rows - 1) / rows;
    return (int)(p > kNormMaxParts ? kNormMaxParts : p);
}

// Lanes per row and chunks per lane by the width: the narrowest group of lanes that holds a row in registers (a row of
// 32 columns in a whole wave would leave 60 lanes without work; 1001 in the 32 chunks of a block that the widest rows need
// took five times as long as in 16 chunks of a wave).  `vec` columns travel per load: 16 bytes of bf16 where width and addresses
// allow it.  Blocks, and with them parts, of one row at a time only beyond 512 columns (gram_layer_norm_work_bytes).
template <typename F> bool norm_shape(int vec, int d, F&& go)
{
#define GRAM_NORM(V, C, L) return go(std::integral_constant<int, V>{}, std::integral_constant<int, C>{}, std::integral_constant<int, L>{})
    if (vec == 8) {
        if (d <= 128) GRAM_NORM(8, 1, 16);
        if (d <= 512) GRAM_NORM(8, 1, 64);
        if (d <= 1024) GRAM_NORM(8, 2, 64);
        if (d <= 2048) GRAM_NORM(8, 4, 64);
        GRAM_NORM(8, 4, 256);
    }
    if (vec == 4) {
        if (d <= 64) GRAM_NORM(4, 1, 16);
        if (d <= 256) GRAM_NORM(4, 1, 64);
        if (d <= 1024) GRAM_NORM(4, 4, 64);
        if (d <= 2048) GRAM_NORM(4, 8, 64);
        GRAM_NORM(4, 8, 256);
    }
    if (d <= 64) GRAM_NORM(1, 4, 16);
    if (d <= 512) GRAM_NORM(1, 8, 64);
    if (d <= 1024) GRAM_NORM(1, 16, 64);
    if (d <= 2048) GRAM_NORM(1, 8, 256);
    GRAM_NORM(1, 32, 256);
#undef GRAM_NORM
}

template <typename F> bool norm_types(int xt, int yt, F&& go)
{
    if (xt == GRAM_F32) return yt == GRAM_F32 ? go((float*)nullptr, (float*)nullptr) : go((float*)nullptr, (bf16_t*)nullptr);
    return yt == GRAM_F32 ? go((bf16_t*)nullptr, (float*)nullptr) : go((bf16_t*)nullptr, (bf16_t*)nullptr);
}

const char* norm_args(int64_t m, int32_t d, int32_t xt, int32_t yt)
{
    if (m < 0) return "m < 0";
    if (d < 1 || d > GRAM_LAYER_NORM_MAX_WIDTH) return "d must be in [1, 8192]";
    if ((xt != GRAM_F32 && xt != GRAM_BF16) || (yt != GRAM_F32 && yt != GRAM_BF16))
        return "x_dtype and y_dtype must be GRAM_F32 or GRAM_BF16";
    return nullptr;
}

}  // namespace

}  // namespace gram

using namespace gram;

extern "C" {

int64_t gram_layer_norm_work_bytes(int64_t m, int32_t d)
{
    if (norm_args(m, d, GRAM_F32, GRAM_F32)) return 0;
    const int parts = norm_parts(m, d > 512 ? kNormWideRows : kNormPartRows);    // of any alignment
    return (int64_t)(parts > 0 ? parts : 1) * 2 * d * (int64_t)sizeof(float);
}

int gram_layer_norm(const void* x, int32_t x_dtype, const float* weight, const float* bias, const int32_t* segments,
                    int64_t m, int32_t d, float eps, void* y, int32_t y_dtype, float* stats, void* stream)
{
    if (const char* why = norm_args(m, d, x_dtype, y_dtype)) return fail_call(GRAM_ERR_ARG, "gram_layer_norm: %s", why);
    if (!(eps >= 0.f) || eps > 1e30f) return fail_call(GRAM_ERR_ARG, "gram_layer_norm: eps must be finite and >= 0");
    if (m == 0) return GRAM_OK;
    if (!x || !weight || !bias || !y) return fail_call(GRAM_ERR_ARG, "gram_layer_norm: NULL pointer");
    const bool al = aligned16(x) && aligned16(weight) && aligned16(bias) && aligned16(y);
    const int vec = !al ? 1 : d % 8 == 0 ? 8 : d % 4 == 0 ? 4 : 1;
    norm_types(x_dtype, y_dtype, [&](auto* tx, auto* ty) {
        return norm_shape(vec, d, [&](auto V, auto C, auto L) {
            constexpr int RPB = kBlock / decltype(L)::value;
            using TX = std::remove_pointer_t<decltype(tx)>;
            using TY = std::remove_pointer_t<decltype(ty)>;
            const int64_t blocks = (m + RPB - 1) / RPB;
            k_layer_norm<TX, TY, decltype(V)::value, decltype(C)::value, decltype(L)::value>
                <<<dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20))), dim3(kBlock), 0, static_cast<hipStream_t>(stream)>>>(
                    static_cast<const TX*>(x), weight, bias, segments, m, d, 1.f / (float)d, eps, static_cast<TY*>(y), stats);
            return true;
        });
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_layer_norm: %s", hipGetErrorString(e));
}

int gram_layer_norm_backward(const void* x, int32_t x_dtype, const float* weight, const float* stats, const void* dy,
                             int32_t y_dtype, const int32_t* segments, const float* add, int64_t m, int32_t d, float* dx,
                             float* dweight, float* dbias, void* work, void* stream)
{
    if (const char* why = norm_args(m, d, x_dtype, y_dtype))
        return fail_call(GRAM_ERR_ARG, "gram_layer_norm_backward: %s", why);
    if (!dweight || !dbias || (m > 0 && (!x || !weight || !stats || !dy || !dx || !work)))
        return fail_call(GRAM_ERR_ARG, "gram_layer_norm_backward: NULL pointer");
    if ((reinterpret_cast<uintptr_t>(work) & 3) != 0)
        return fail_call(GRAM_ERR_ARG, "gram_layer_norm_backward: work must be 4-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    int parts = 0;
    float* const part = static_cast<float*>(work);
    if (m > 0) {
        const bool al = aligned16(x) && aligned16(weight) && aligned16(dy) && aligned16(dx) && (!add || aligned16(add));
        const int vec = !al ? 1 : d % 8 == 0 ? 8 : d % 4 == 0 ? 4 : 1;
        norm_types(x_dtype, y_dtype, [&](auto* tx, auto* ty) {
            return norm_shape(vec, d, [&](auto V, auto C, auto L) {
                using TX = std::remove_pointer_t<decltype(tx)>;
                using TY = std::remove_pointer_t<decltype(ty)>;
                parts = norm_parts(m, decltype(L)::value == 256 ? kNormWideRows : kNormPartRows);
                k_layer_norm_bwd<TX, TY, decltype(V)::value, decltype(C)::value, decltype(L)::value>
                    <<<dim3((unsigned)parts), dim3(kBlock), 0, s>>>(static_cast<const TX*>(x), weight, stats,
                                                                    static_cast<const TY*>(dy), segments, add, m, d,
                                                                    1.f / (float)d, dx, part);
                return true;
            });
        });
    }
    k_layer_norm_parts<<<dim3((unsigned)((2 * d + 15) / 16)), dim3(1024), 0, s>>>(part, parts, d, dweight, dbias);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_layer_norm_backward: %s", hipGetErrorString(e));
}

}  // extern "C"
