// Attention over item histories: the C entry points, their checks, and the last sum of the table's gradient.  The kernels
// are in gram_attend_fwd.hip, gram_attend_dq.hip, gram_attend_dkv.hip, gram_attend_short.hip and gram_attend_step.hip.
#include <math.h>

#include "gram_attend.h"

namespace gram {

namespace {

// dtable[head, b] = the sum of the blocks' partial rows, strand by strand in a fixed order.
__global__ __launch_bounds__(1024) void k_attend_dtable(const float* __restrict__ part, int parts, int buckets,
                                                        float* __restrict__ dtable)
{
    __shared__ double s[1024];
    const int head = blockIdx.y, b = blockIdx.x * 16 + threadIdx.x % 16, strand = threadIdx.x / 16;
    double sum = 0.0;
    if (b < buckets) {
        const float* const p = part + (int64_t)head * parts * buckets + b;
#pragma unroll 8
        for (int i = strand; i < parts; i += 64) sum += (double)p[(int64_t)i * buckets];
    }
    s[threadIdx.x] = sum;
    __syncthreads();
    if (strand < 8) {
#pragma unroll
        for (int k = 1; k < 8; ++k) sum += s[k * 128 + threadIdx.x];
        s[threadIdx.x] = sum;
    }
    __syncthreads();
    if (strand == 0 && b < buckets) {
#pragma unroll
        for (int k = 1; k < 8; ++k) sum += s[k * 16 + threadIdx.x];
        dtable[(int64_t)head * buckets + b] = (float)sum;
    }
}

// ---- host -------------------------------------------------------------------------------------------------

// Borders of one side: bucket exact + i begins at the smallest n with (n / exact)^(side - exact) >= (far / exact)^i.
// The power is a whole number only where it is one exactly: a value within 1e-15 of a whole number, twenty-five times the
// error of the product of up to 32 extended-precision roots, is that number.  One root per call and products of it, since
// a small batch is bound by the host: a power per border took 6.6 us of a cached step's 16.8.
void make_buckets(const gram_attention_config& c, AttBuckets* bk)
{
    *bk = AttBuckets{};
    if (c.buckets == 0) return;
    bk->two_sided = c.two_sided != 0;
    bk->side = bk->two_sided ? c.buckets / 2 : c.buckets;
    bk->exact = bk->side / 2;
    bk->last = bk->exact;
    if (bk->side == 1) return;
    const int wide = bk->side - bk->exact;
    bk->inv_exact = 1.f / (float)bk->exact;
    bk->per_log2 = (float)(wide / log2((double)c.max_distance / bk->exact));
    const long double root = powl((long double)c.max_distance / bk->exact, 1.0L / wide);
    long double x = bk->exact;
    for (int i = 1; i < wide; ++i) {
        x *= root;
        const long double near = roundl(x);
        const long double n = fabsl(x - near) <= 1e-15L * x ? near : ceill(x);
        bk->border[bk->borders++] = (int)n;
        bk->last = (int)n;
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
    int es, dim;
    int64_t batch;
    uint64_t bits = 0;
    bool null = false, far = false, shared = false;
    UnitFinder(const gram_attention_config& c, int32_t batch) : es(c.dtype == GRAM_BF16 ? 2 : 4), dim(c.head_dim), batch(batch) {}
    AttRows add(const gram_rows* r, int64_t rows, int64_t heads, bool written = false)
    {
        AttRows out{};
        if (!r || !r->data) {
            null = true;
            return out;
        }
        out.data = r->data;
        out.sb = stride(r->batch_stride, batch, INT64_MAX, written);
        out.sr = stride(r->row_stride, rows, kAttMaxRowBytes / es, written);
        out.sh = stride(r->head_stride, heads, INT64_MAX, written);
        bits |= reinterpret_cast<uintptr_t>(r->data) | (uint64_t)((out.sb | out.sr | out.sh) * es);
        return out;
    }
    // a stride of something that there is one of has no meaning
    int64_t stride(int64_t s, int64_t count, int64_t end, bool written)
    {
        if (count <= 1) return 0;
        far |= s < 0 || s >= end;
        shared |= written && s < dim;
        return s;
    }
    int unit() const
    {
        const uint64_t all = bits | (uint64_t)(dim * es);
        return (all & 15) == 0 ? 16 : es == 2 && (all & 7) == 0 ? 8 : es;
    }
    const char* refusal() const
    {
        if (null) return "NULL pointer";
        if (bits & (uint64_t)(es - 1)) return "an operand is not aligned to its elements";
        if (far) return "strides must be >= 0 and rows less than 64 MiB apart";
        if (shared) return "rows of an operand that is written must not overlap";
        return nullptr;
    }
};

void fill(AttArgs& a, const gram_attention_config& c, int32_t batch, int32_t length)
{
    a.batch = batch, a.length = length, a.heads = c.heads, a.kv_heads = c.kv_heads, a.group = c.heads / c.kv_heads;
    a.dim = c.head_dim, a.causal = c.causal != 0, a.scale = c.scale, a.cap = c.cap;
    make_buckets(c, &a.bk);
}

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
    AttArgs a{};
    UnitFinder u(*cfg, batch);
    const int64_t H = cfg->heads, KV = cfg->kv_heads;
    a.q = u.add(q, length, H), a.k = u.add(k, length, KV), a.v = u.add(v, length, KV), a.o = u.add(o, length, H, true);
    if (const char* why = cfg->buckets > 0 && !table ? "NULL pointer" : u.refusal())
        return fail_call(GRAM_ERR_ARG, "gram_attention: %s", why);
    fill(a, *cfg, batch, length);
    a.seg = segments, a.prefix = prefix, a.table = table, a.lse = lse;
    attend_forward(*cfg, a, u.unit(), static_cast<hipStream_t>(stream));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention: %s", hipGetErrorString(e));
}

int64_t gram_attention_backward_bytes(const gram_attention_config* cfg, int32_t batch, int32_t length)
{
    if (check_sizes(cfg, batch, length)) return 0;
    const int64_t rows = (int64_t)batch * cfg->heads;
    return up256(rows * length * (int64_t)sizeof(float)) + up256(rows * length * 2 * (int64_t)sizeof(float)) +
           up256(rows * att_blocks(length, 64) * cfg->buckets * (int64_t)sizeof(float)) + 256;
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
    AttArgs a{};
    if (!none) {
        UnitFinder u(*cfg, batch);
        const int64_t H = cfg->heads, KV = cfg->kv_heads;
        a.q = u.add(q, length, H), a.k = u.add(k, length, KV), a.v = u.add(v, length, KV), a.o = u.add(o, length, H);
        a.dout = u.add(dout, length, H);
        a.dq = u.add(dq, length, H, true), a.dk = u.add(dk, length, KV, true), a.dv = u.add(dv, length, KV, true);
        if (const char* why = !lse || !work || (cfg->buckets > 0 && !table) ? "NULL pointer" : u.refusal())
            return fail_call(GRAM_ERR_ARG, "gram_attention_backward: %s", why);
        if ((reinterpret_cast<uintptr_t>(work) & 15) != 0)
            return fail_call(GRAM_ERR_ARG, "gram_attention_backward: work must be 16-byte aligned");
        fill(a, *cfg, batch, length);
        a.seg = segments, a.prefix = prefix, a.table = table, a.lse = const_cast<float*>(lse);
        const int64_t rows = (int64_t)batch * cfg->heads * length;
        unsigned char* at = static_cast<unsigned char*>(work);
        a.delta = reinterpret_cast<float*>(at), at += up256(rows * (int64_t)sizeof(float));
        a.far = reinterpret_cast<float*>(at), at += up256(rows * 2 * (int64_t)sizeof(float));
        a.part = dtable ? reinterpret_cast<float*>(at) : nullptr;
        a.parts = batch * att_blocks(length, kTile);
        const int unit = u.unit();
        if (!attend_backward_short(*cfg, a, unit, s)) {
            attend_backward_queries(*cfg, a, unit, s);  // also leaves delta and far for the pass over the keys
            attend_backward_keys(*cfg, a, unit, s);
        }
    }
    if (dtable)
        k_attend_dtable<<<dim3((unsigned)((cfg->buckets + 15) / 16), (unsigned)cfg->heads), dim3(1024), 0, s>>>(
            a.part, none ? 0 : a.parts, cfg->buckets, dtable);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention_backward: %s", hipGetErrorString(e));
}

int64_t gram_attention_step_bytes(const gram_attention_config* cfg, int32_t batch, int32_t capacity)
{
    if (check_config(cfg) || batch < 0 || capacity < 1 || capacity > GRAM_ATTENTION_MAX_CAPACITY) return 0;
    return (batch ? step_part_bytes(*cfg, batch, capacity) : 0) + 256;
}

int gram_attention_step(const gram_attention_config* cfg, int32_t batch, int32_t capacity, const gram_rows* q,
                        const gram_rows* k_new, const gram_rows* v_new, const gram_rows* k_cache, const gram_rows* v_cache,
                        const int32_t* lengths, const int32_t* first, const float* table, const gram_rows* o, void* work,
                        void* stream)
{
    if (const char* why = check_config(cfg)) return fail_call(GRAM_ERR_ARG, "gram_attention_step: %s", why);
    if (batch < 0 || capacity < 1 || capacity > GRAM_ATTENTION_MAX_CAPACITY)
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: batch must be >= 0 and capacity in [1, 2^30]");
    if (batch == 0) return GRAM_OK;
    UnitFinder u(*cfg, batch);
    const int64_t H = cfg->heads, KV = cfg->kv_heads;
    const AttRows rq = u.add(q, 1, H), rkn = u.add(k_new, 1, KV), rvn = u.add(v_new, 1, KV),
                  rkc = u.add(k_cache, capacity, KV, true), rvc = u.add(v_cache, capacity, KV, true), ro = u.add(o, 1, H, true);
    const bool null = !lengths || (cfg->buckets > 0 && !table) || (!work && step_part_bytes(*cfg, batch, capacity) > 0);
    if (const char* why = null ? "NULL pointer" : u.refusal()) return fail_call(GRAM_ERR_ARG, "gram_attention_step: %s", why);
    if (rq.sh >= kAttMaxRowBytes / u.es)    // the heads of a query are the rows of an operand
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: the heads of q must be less than 64 MiB apart");
    if ((reinterpret_cast<uintptr_t>(work) & 15) != 0)
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: work must be 16-byte aligned");
    AttBuckets bk;
    make_buckets(*cfg, &bk);
    if (!step_launch(*cfg, bk, batch, capacity, rq, rkn, rvn, rkc, rvc, ro, lengths, first, table, work,
                     u.unit(), static_cast<hipStream_t>(stream)))
        return fail_call(GRAM_ERR_ARG, "gram_attention_step: batch * heads must be at most 2^23");
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? GRAM_OK : fail_call(GRAM_ERR_HIP, "gram_attention_step: %s", hipGetErrorString(e));
}

}  // extern "C"
