// Attention inside the sets of a ragged batch: the C entry points.
#include "attention.h"

namespace lcn {

static bool attention_desc_fits(const lcn_attention_desc *d)
{
    if (!d || d->num_sets < 0 || d->num_sets > (1 << 24) || d->total_q < 0 || d->total_q > MAX_ROWS || d->total_k < 0 ||
        d->total_k > MAX_ROWS || d->max_q < 0 || d->heads < 1 || d->heads > 1024 || d->kv_heads < 1 || d->heads % d->kv_heads ||
        d->head_dim < 1 || d->head_dim > 128 || (d->dtype != LCN_F32 && d->dtype != LCN_BF16))
        return false;
    if (d->clear != 0 && d->clear != 1) return false;
    if (!(d->scale - d->scale == 0.f) || !(d->cap >= 0.f) || !(d->cap - d->cap == 0.f)) return false;
    const int64_t strides[6] = {d->q_token, d->q_head, d->k_token, d->k_head, d->v_token, d->v_head};
    for (int i = 0; i < 6; ++i)
        if (strides[i] < 0 || strides[i] > (1 << 22)) return false;
    // workgroups are numbered in 32 bits: one per tile of 64 tokens and head (split only where there are few), or a wavefront per token and head
    if ((d->total_q / 64 + d->num_sets) * (int64_t)d->heads > 0x7fffffff || d->total_q * d->heads / 4 > 0x7ffffff0) return false;
    if ((d->total_k / 64 + d->num_sets) * (int64_t)d->heads > 0x7fffffff) return false;
    return d->num_sets == 0 || (d->q_off && d->k_off);
}

static AttentionArgs args_of(const lcn_attention_desc *d, const void *q, const void *k, const void *v)
{
    AttentionArgs a{};
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_off = d->q_off;
    a.k_off = d->k_off;
    a.prefix = d->causal ? d->prefix : nullptr;
    a.slopes = d->slopes;
    a.q_head = d->q_head ? d->q_head : d->head_dim;
    a.k_head = d->k_head ? d->k_head : d->head_dim;
    a.v_head = d->v_head ? d->v_head : d->head_dim;
    a.q_token = d->q_token ? d->q_token : (int64_t)d->heads * d->head_dim;
    a.k_token = d->k_token ? d->k_token : (int64_t)d->kv_heads * d->head_dim;
    a.v_token = d->v_token ? d->v_token : (int64_t)d->kv_heads * d->head_dim;
    a.total_q = d->total_q;
    a.total_k = d->total_k;
    a.sets = d->num_sets;
    a.heads = d->heads;
    a.kv_heads = d->kv_heads;
    a.dim = d->head_dim;
    a.causal = d->causal != 0;
    a.scale = d->scale;
    a.cap = d->cap;
    a.clear = d->clear != 0;
    return a;
}

// Whether every row is whole 16-byte pieces from aligned addresses.
static bool pieces(const AttentionArgs &a, size_t e, const void *const *more, int count)
{
    uintptr_t all = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
    for (int i = 0; i < count; ++i) all |= (uintptr_t)more[i];
    const long long strides = a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head | a.dim;
    return (all & 15) == 0 && (strides & (long long)(16 / e - 1)) == 0;
}

static int shape_of(const AttentionArgs &a)
{
    if (a.slopes || !(a.scale > 0.f)) return SHAPED;
    return a.cap == 0.f ? PLAIN : a.cap <= MOST_CAP ? CAPPED : SHAPED;
}

// Rows of a set's chunks: no set has more queries than there are.
static int64_t chunk_rows(const lcn_attention_desc *d)
{
    return (d->max_q < d->total_q ? d->max_q : d->total_q) * (d->heads / d->kv_heads);
}
// Where a set has few queries, its keys are split over workgroups: up to 32 rows (queries times the heads that share a key
// head) fit a wavefront.  Chunks of keys are so long that there are some eight workgroups per compute unit, from 128 keys (a
// step of a workgroup's wavefronts) to 2048.  0: not split, as also where a set has less than 128 keys on average.
// One query, 32 heads on 8, for 32 sets of 4000 keys: bf16 130 us (not split 319), float 313 (1637); eight queries, 8 heads on 2, for 32
// sets of 1000 keys: 22 (21), 38 (41); one query for 256 sets of 128 keys: 15 (16), 28 (54).
static int chunk_of(const lcn_attention_desc *d)
{
    const int64_t rows = chunk_rows(d);
    if (d->max_q == 0 || rows > 32 || d->total_k < 128LL * d->num_sets) return 0;
    const int64_t keys = d->total_k * d->kv_heads / 2048;
    const int64_t chunk = (keys + 127) / 128 * 128;
    return (int)(chunk < 128 ? 128 : chunk > 2048 ? 2048 : chunk);
}
// Into how many workgroups a tile's other side is split so that there are some 512 of them, or 1024 where tiles have 64 tokens
// instead of 128: `tiles` of 128 there are, `length` is the
// average length of a set's other side, and a share has at least 256 of it (4 sets of 145 queries and 4300 keys, 2 float
// heads of 32, forward and all gradients: 119 us, with whole tiles 556 us).
static int shares(int64_t tiles, int64_t length)
{
    const int64_t wanted = tiles > 0 ? (512 + tiles - 1) / tiles : 1, most = length / 256;
    const int64_t n = wanted < most ? wanted : most;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}
static int key_splits(const lcn_attention_desc *d)
{
    if (d->num_sets == 0) return 1;
    const int64_t tiles = (d->total_q / 128 + d->num_sets) * d->heads;
    return shares(tiles, d->total_k / d->num_sets);
}
// dk and dv: twice as many, since the query heads of a key head are its other side as well, and a causal set's first
// keys have twice the average length
static int query_splits(const lcn_attention_desc *d)
{
    if (d->num_sets == 0) return 1;
    const int64_t tiles = (d->total_k / 128 + d->num_sets) * d->kv_heads;
    return shares((tiles + 1) / 2, d->total_q / d->num_sets * (d->heads / d->kv_heads));
}

// -inf for the lse of queries where there is no set at all
__global__ __launch_bounds__(256) void no_key_kernel(float *lse, long long count)
{
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < count; i += (long long)gridDim.x * 256) lse[i] = minus_infinity();
}
static hipError_t clear_all(void *out, long long values, int32_t dtype, float *lse, long long rows, hipStream_t s)
{
    const hipError_t e = launch_zero(out, (size_t)values * (dtype == LCN_F32 ? 4 : 2), s);
    if (e != hipSuccess || !lse || rows == 0) return e;
    const long long groups = (rows + 255) / 256;
    hipLaunchKernelGGL(no_key_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, lse, rows);
    return hipGetLastError();
}

struct ForwardSpace {
    int chunk, rows, key_splits;
    float *part;
    float2 *part_top;
    size_t bytes;
};
static ForwardSpace forward_space(char *ws, const lcn_attention_desc *d)
{
    Carver c{ws};
    ForwardSpace f{};
    f.chunk = chunk_of(d);
    f.key_splits = 1;
    size_t n = 0;
    if (f.chunk) {
        f.rows = (int)chunk_rows(d);
        n = (size_t)(d->total_k / f.chunk + d->num_sets) * d->kv_heads * f.rows;
    } else if ((f.key_splits = key_splits(d)) > 1) {
        n = (size_t)f.key_splits * d->total_q * d->heads;
    }
    f.part = (float *)c.take(n * d->head_dim * 4);
    f.part_top = (float2 *)c.take(n * 8);
    f.bytes = c.used;
    return f;
}
struct GradSpace {
    float *delta, *part;   // part: for dq, then for dk and dv
    int key_splits, splits;
    size_t bytes;
};
static GradSpace grad_space(char *ws, const lcn_attention_desc *d)
{
    Carver c{ws};
    GradSpace f;
    f.delta = (float *)c.take((size_t)d->heads * (size_t)d->total_q * 4);
    f.key_splits = key_splits(d);
    f.splits = query_splits(d);
    const size_t q = f.key_splits > 1 ? (size_t)f.key_splits * d->total_q * d->heads : 0;
    const size_t k = f.splits > 1 ? (size_t)f.splits * 2 * d->total_k * d->kv_heads : 0;
    f.part = (float *)c.take((q > k ? q : k) * d->head_dim * 4);
    f.bytes = c.used;
    return f;
}

}  // namespace lcn

using namespace lcn;

extern "C" {

lcn_status lcn_attention_workspace_bytes(const lcn_attention_desc *desc, int32_t backward, size_t *bytes)
{
    if (!bytes || !attention_desc_fits(desc)) return LCN_ERR_INVALID_ARG;
    *bytes = backward ? grad_space(nullptr, desc).bytes : forward_space(nullptr, desc).bytes;
    return LCN_OK;
}

lcn_status lcn_attention(const lcn_attention_desc *desc, const void *q, const void *k, const void *v, void *o, float *lse,
                         void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!attention_desc_fits(desc)) return LCN_ERR_INVALID_ARG;
    if (desc->total_q == 0 || (desc->num_sets == 0 && !desc->clear)) return LCN_OK;
    if (!q || !o || !lse || (desc->total_k > 0 && (!k || !v))) return LCN_ERR_INVALID_ARG;
    if (desc->num_sets == 0) {
        const int64_t rows = desc->total_q * desc->heads;
        OPCHK(clear_all(o, rows * desc->head_dim, desc->dtype, lse, rows, (hipStream_t)hip_stream));
        return LCN_OK;
    }
    AttentionArgs a = args_of(desc, q, k, v);
    a.o = o;
    a.lse = lse;
    const void *more[1] = {o};
    const bool vec = pieces(a, desc->dtype == LCN_F32 ? 4 : 2, more, 1);
    const int shape = shape_of(a);
    const ForwardSpace f = forward_space((char *)workspace, desc);
    if (f.bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < f.bytes)) return LCN_ERR_ALLOC;
    a.key_splits = f.key_splits;
    if (f.chunk) {
        a.chunk = f.chunk;
        a.rows = f.rows;
        a.part = f.part;
        a.part_top = f.part_top;
        if (desc->dtype == LCN_F32)
            OPCHK(attention_by_chunks<float>(a, vec, shape, (hipStream_t)hip_stream));
        else
            OPCHK(attention_by_chunks<__bf16>(a, vec, shape, (hipStream_t)hip_stream));
        return LCN_OK;
    }
    a.part = f.part;
    a.part_top = f.part_top;
    if (desc->dtype == LCN_F32)
        OPCHK(attention_forward<float>(a, vec, shape, (hipStream_t)hip_stream));
    else
        OPCHK(attention_forward<__bf16>(a, vec, shape, (hipStream_t)hip_stream));
    return LCN_OK;
}

lcn_status lcn_attention_backward(const lcn_attention_desc *desc, const void *q, const void *k, const void *v, const void *o,
                                  const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *workspace,
                                  size_t workspace_bytes, void *hip_stream)
{
    if (!attention_desc_fits(desc) || !dk != !dv) return LCN_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)hip_stream;
    if ((!dq && !dk) || (desc->num_sets == 0 && !desc->clear)) return LCN_OK;
    if (desc->num_sets == 0) {
        const int64_t rows_q = desc->total_q * desc->heads, rows_k = desc->total_k * desc->kv_heads;
        if (dq) OPCHK(clear_all(dq, rows_q * desc->head_dim, desc->dtype, nullptr, 0, s));
        if (dk) OPCHK(clear_all(dk, rows_k * desc->head_dim, desc->dtype, nullptr, 0, s));
        if (dv) OPCHK(clear_all(dv, rows_k * desc->head_dim, desc->dtype, nullptr, 0, s));
        return LCN_OK;
    }
    if (desc->total_q > 0 && (!q || !o || !lse || !d_o)) return LCN_ERR_INVALID_ARG;
    if (desc->total_k > 0 && (!k || !v)) return LCN_ERR_INVALID_ARG;
    const GradSpace f = grad_space((char *)workspace, desc);
    if (f.bytes && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < f.bytes)) return LCN_ERR_ALLOC;
    AttentionArgs a = args_of(desc, q, k, v);
    a.d_o = d_o;
    a.o = const_cast<void *>(o);
    a.lse_in = lse;
    a.delta = f.delta;
    a.key_splits = f.key_splits;
    a.splits = f.splits;
    a.part = f.part;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    const void *more[5] = {o, d_o, dq, dk, dv};
    const bool vec = pieces(a, desc->dtype == LCN_F32 ? 4 : 2, more, 5);
    const int shape = shape_of(a);
    if (desc->dtype == LCN_F32)
        OPCHK(attention_backward<float>(a, vec, shape, s));
    else
        OPCHK(attention_backward<__bf16>(a, vec, shape, s));
    return LCN_OK;
}

}  // extern "C"
