// dd_attention_forward / dd_attention_backward: arguments, tensor maps and launches.  Forward: the plan (with
// offsets) and one launch.  Backward: the plan and delta = d_o . o in one, dq, then dk and dv.
#include <cmath>

#include "dd_args.h"
#include "dd_attention.cuh"

namespace ddm {

static int encode_heads(dd_ctx *ctx, CUtensorMap *map, const dd_heads &x, uint64_t tokens, uint64_t heads, uint64_t dim)
{
    const cuuint64_t dims[3] = {dim, heads, tokens}, strides[2] = {x.ld_head * 2, x.ld_token * 2};
    const cuuint32_t box[3] = {64, 1, kTile}, step[3] = {1, 1, 1};
    const EncodeTiled fn = tensor_map_encoder();
    if (!fn || fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, x.data, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
        snprintf(ctx->cuda_err, sizeof ctx->cuda_err, "cuTensorMapEncodeTiled failed");
        return DD_ERR_CUDA;
    }
    return DD_OK;
}

static int check_attention(const dd_attention &a)
{
    if (a.heads < 1 || a.kv_heads < 1 || a.dim < 8 || a.dim % 8 || a.heads % a.kv_heads) return DD_ERR_INVALID_ARG;
    if (a.tokens >= (1ull << 31) || a.heads >= (1ull << 16) || a.dim > 128) return DD_ERR_TOO_LARGE;
    if (!std::isfinite(a.scale) || a.scale <= 0.0f) return DD_ERR_INVALID_ARG;
    if (a.flags & ~(uint32_t)DD_DEBUG_EXPIRE_WAIT) return DD_ERR_INVALID_ARG;
    if (a.offsets) {
        if (a.sequences >= (1ull << 24)) return DD_ERR_TOO_LARGE;
        if ((uintptr_t)a.offsets & 3u) return DD_ERR_ALIGNMENT;
    }
    if ((a.tokens / kTile + (a.offsets ? a.sequences : 0) + 1) * a.heads >= (1ull << 28)) return DD_ERR_TOO_LARGE;      // a grid of clusters
    return DD_OK;
}

// Strides of a tensor that the TMA engine and 16-byte accesses can use; strides over a single token or head
// do not matter and are set to what an encoder takes.
static int check_tensor(dd_heads &x, const dd_attention &a, uint64_t heads)
{
    const int rc = check_heads(x, a.tokens, heads, a.dim);
    if (rc != DD_OK) return rc;
    if (heads == 1) x.ld_head = a.dim;
    if (a.tokens <= 1) x.ld_token = heads * x.ld_head;
    return (uintptr_t)x.data % 16 || x.ld_head % 8 || x.ld_token % 8 ? DD_ERR_ALIGNMENT : DD_OK;
}

// Most tiles of `rows` tokens that a launch may have.
static uint64_t most_tiles(const dd_attention &a, unsigned rows)
{
    return a.offsets ? a.tokens / rows + a.sequences : (a.tokens + rows - 1) / rows;
}

static uint64_t round16(uint64_t n) { return (n + 15) / 16 * 16; }
static uint64_t plan_bytes(const dd_attention &a, unsigned rows) { return a.offsets ? 16 + 16 * most_tiles(a, rows) : 0; }

static PlanArgs plan_args(const dd_attention &a, unsigned rows, Plan *plan, int32_t *status)
{
    return {a.offsets, (unsigned)a.sequences, (unsigned)a.tokens, rows, plan, status};
}

template <int DP>
static int launch_forward(dd_ctx *ctx, const dd_attention &b, const AttnArgs &a, cudaStream_t stream)
{
    static std::atomic<bool> done[64];
    const int rc = allow_smem(ctx, attention_forward_kernel<DP>, fwd_smem_bytes(DP), done);
    if (rc != DD_OK) return rc;
    return launch_after(ctx, attention_forward_kernel<DP>, most_tiles(b, 2 * kTile) * b.heads, 32 * (kFwdWarps + 4), fwd_smem_bytes(DP), stream, a);
}

// CTAs that share a tile of keys: those that end first by an estimate in tiles of queries.  A CTA's own costs are two
// of them, with others to wait for and add up with three and half the cluster's size more; the GPU ends after its
// SMs' mean, or after the CTA of a sequence's first keys, which all queries of all heads of the group read.  (Lengths
// are not known here: one sequence.)  Measured with 1 / 2 / 4 CTAs: 8192 tokens, 8 heads on 2 578 / 384 / 413 us, 4096
// tokens, 8 on 8 121 / 141 / 189, 915 tokens, 6 on 3 43 / 36 / 34 (each time the least is taken).
static unsigned dkv_cluster(const dd_ctx *ctx, const dd_attention &b)
{
    const double n = (double)((b.tokens + kTile - 1) / kTile), all = b.heads * (b.causal ? n * (n + 1) / 2 : n * n), first = n * (double)(b.heads / b.kv_heads);
    unsigned best = 1;
    double least = 0;
    for (unsigned c = 1; c <= 8; c *= 2) {
        const double own = c > 1 ? 5 + c / 2 - 1 : 2, mean = (all + n * b.kv_heads * c * own) / ctx->sm_count, longest = first / c + own;
        const double time = mean > longest ? mean : longest;
        if (c == 1 || time < least) {
            least = time;
            best = c;
        }
    }
    return best;
}

template <int DP>
static int launch_backward(dd_ctx *ctx, const dd_attention &b, AttnArgs &a, const DeltaArgs &d, const PlanArgs &plan, cudaStream_t stream)
{
    static std::atomic<bool> done_q[64], done_kv[64];
    int rc = allow_smem(ctx, attention_dq_kernel<DP>, bwd_smem_bytes(DP), done_q);
    if (rc == DD_OK) rc = allow_smem(ctx, attention_dkv_kernel<DP>, bwd_smem_bytes(DP), done_kv);
    constexpr int lanes = DP / 8;
    if (rc == DD_OK) rc = launch_after(ctx, attention_delta_kernel<lanes>, (b.tokens * b.heads * lanes + 255) / 256 + (plan.plan ? 1 : 0), 256, 0, stream, d, plan);
    const uint64_t tiles = most_tiles(b, kTile);
    if (rc == DD_OK) rc = launch_after(ctx, attention_dq_kernel<DP>, tiles * b.heads, 32 * (kBwdWarps + 4), bwd_smem_bytes(DP), stream, a);
    a.cluster = dkv_cluster(ctx, b);
    if (rc == DD_OK)
        rc = launch_clusters(ctx, attention_dkv_kernel<DP>, tiles * b.kv_heads * a.cluster, 32 * (kBwdWarps + 4), bwd_smem_bytes(DP), a.cluster, stream, a);
    return rc;
}

static AttnArgs attention_args(const dd_attention &b, unsigned rows, const Plan *plan, int32_t *status)
{
    AttnArgs a;
    std::memset(&a, 0, sizeof a);
    a.plan = plan;
    a.tokens = (unsigned)b.tokens;
    a.tiles = blocks_of(b.tokens, rows);
    a.heads = (unsigned)b.heads;
    a.group = (unsigned)(b.heads / b.kv_heads);
    a.dim = (unsigned)b.dim;
    a.scale = b.scale;
    a.causal = b.causal != 0;
    a.expire = b.flags != 0;
    a.status = status;
    return a;
}

static HeadRows rows_of(const dd_heads &x) { return {static_cast<__nv_bfloat16 *>(x.data), x.ld_token, x.ld_head}; }

}  // namespace ddm

using namespace ddm;

extern "C" uint64_t dd_attention_scratch_bytes(const dd_attention *attention, int backward)
{
    if (!attention || check_attention(*attention) != DD_OK) return 0;
    const dd_attention &a = *attention;
    return backward ? round16(a.tokens * a.heads * 4) + plan_bytes(a, kTile) : plan_bytes(a, 2 * kTile);
}

extern "C" int dd_attention_forward(dd_ctx *ctx, const dd_attention *attention, const dd_heads *q_, const dd_heads *k_, const dd_heads *v_,
                                    const dd_heads *o_, float *lse, void *scratch, int32_t *status, void *cuda_stream)
{
    if (!ctx || !attention || !q_ || !k_ || !v_ || !o_) return DD_ERR_INVALID_ARG;
    const dd_attention &b = *attention;
    dd_heads q = *q_, k = *k_, v = *v_, o = *o_;
    int rc = check_attention(b);
    if (rc == DD_OK) rc = check_tensor(q, b, b.heads);
    if (rc == DD_OK) rc = check_tensor(k, b, b.kv_heads);
    if (rc == DD_OK) rc = check_tensor(v, b, b.kv_heads);
    if (rc == DD_OK) rc = check_tensor(o, b, b.heads);
    if (rc == DD_OK) rc = check_aligned({scratch});
    if (rc != DD_OK) return rc;
    if ((uintptr_t)status & 3u || (uintptr_t)lse & 3u) return DD_ERR_ALIGNMENT;
    const size_t bytes = plan_bytes(b, 2 * kTile);
    const uint64_t T = b.tokens;
    rc = check_alias({heads_extent(o, T, b.heads, b.dim), extent(lse, 1, T * b.heads, T * b.heads, 4), extent(scratch, 1, bytes, bytes, 1)},
                     {heads_extent(q, T, b.heads, b.dim), heads_extent(k, T, b.kv_heads, b.dim), heads_extent(v, T, b.kv_heads, b.dim),
                      extent(b.offsets, 1, b.sequences + 1, b.sequences + 1, 4)});
    if (rc != DD_OK) return rc;
    if (T == 0 || (b.offsets && b.sequences == 0)) return DD_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    if (!scratch && bytes) {
        rc = ensure_decoder_scratch(ctx, bytes);
        if (rc != DD_OK) return rc;
        scratch = ctx->decoder_scratch;
    }
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    Plan *plan = b.offsets ? static_cast<Plan *>(scratch) : nullptr;
    AttnArgs a = attention_args(b, 2 * kTile, plan, status);
    rc = encode_heads(ctx, &a.q, q, T, b.heads, b.dim);
    if (rc == DD_OK) rc = encode_heads(ctx, &a.k, k, T, b.kv_heads, b.dim);
    if (rc == DD_OK) rc = encode_heads(ctx, &a.v, v, T, b.kv_heads, b.dim);
    a.o = rows_of(o);
    a.lse = lse;
    if (rc == DD_OK && plan) rc = launch_after(ctx, attention_plan_kernel, 1, kPlanThreads, 0, stream, plan_args(b, 2 * kTile, plan, status));
    if (rc != DD_OK) return rc;
    return b.dim <= 64 ? launch_forward<64>(ctx, b, a, stream) : launch_forward<128>(ctx, b, a, stream);
}

extern "C" int dd_attention_backward(dd_ctx *ctx, const dd_attention *attention, const dd_heads *q_, const dd_heads *k_, const dd_heads *v_,
                                     const dd_heads *o_, const float *lse, const dd_heads *d_o_, const dd_heads *dq_, const dd_heads *dk_,
                                     const dd_heads *dv_, void *scratch, int32_t *status, void *cuda_stream)
{
    if (!ctx || !attention || !q_ || !k_ || !v_ || !o_ || !d_o_ || !dq_ || !dk_ || !dv_) return DD_ERR_INVALID_ARG;
    const dd_attention &b = *attention;
    dd_heads q = *q_, k = *k_, v = *v_, o = *o_, d_o = *d_o_, dq = *dq_, dk = *dk_, dv = *dv_;
    const uint64_t T = b.tokens;
    int rc = check_attention(b);
    for (dd_heads *x : {&q, &o, &d_o, &dq})
        if (rc == DD_OK) rc = check_tensor(*x, b, b.heads);
    for (dd_heads *x : {&k, &v, &dk, &dv})
        if (rc == DD_OK) rc = check_tensor(*x, b, b.kv_heads);
    if (rc == DD_OK) rc = check_aligned({scratch});
    if (rc != DD_OK) return rc;
    if (T > 0 && !lse) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)status & 3u || (uintptr_t)lse & 3u) return DD_ERR_ALIGNMENT;
    const size_t delta_bytes = round16(T * b.heads * 4), bytes = delta_bytes + plan_bytes(b, kTile);
    rc = check_alias({heads_extent(dq, T, b.heads, b.dim), heads_extent(dk, T, b.kv_heads, b.dim), heads_extent(dv, T, b.kv_heads, b.dim),
                      extent(scratch, 1, bytes, bytes, 1)},
                     {heads_extent(q, T, b.heads, b.dim), heads_extent(k, T, b.kv_heads, b.dim), heads_extent(v, T, b.kv_heads, b.dim),
                      heads_extent(o, T, b.heads, b.dim), heads_extent(d_o, T, b.heads, b.dim), extent(lse, 1, T * b.heads, T * b.heads, 4),
                      extent(b.offsets, 1, b.sequences + 1, b.sequences + 1, 4)});
    if (rc != DD_OK) return rc;
    if (T == 0 || (b.offsets && b.sequences == 0)) return DD_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    if (!scratch) {
        rc = ensure_decoder_scratch(ctx, bytes);
        if (rc != DD_OK) return rc;
        scratch = ctx->decoder_scratch;
    }
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    float *delta = static_cast<float *>(scratch);
    Plan *plan = b.offsets ? reinterpret_cast<Plan *>(static_cast<char *>(scratch) + delta_bytes) : nullptr;
    AttnArgs a = attention_args(b, kTile, plan, status);
    rc = encode_heads(ctx, &a.q, q, T, b.heads, b.dim);
    if (rc == DD_OK) rc = encode_heads(ctx, &a.k, k, T, b.kv_heads, b.dim);
    if (rc == DD_OK) rc = encode_heads(ctx, &a.v, v, T, b.kv_heads, b.dim);
    if (rc == DD_OK) rc = encode_heads(ctx, &a.d_o, d_o, T, b.heads, b.dim);
    if (rc != DD_OK) return rc;
    a.q_rows = rows_of(q);
    a.k_rows = rows_of(k);
    a.v_rows = rows_of(v);
    a.do_rows = rows_of(d_o);
    a.dq = rows_of(dq);
    a.dk = rows_of(dk);
    a.dv = rows_of(dv);
    a.lse = const_cast<float *>(lse);
    a.delta = delta;
    const DeltaArgs d = {static_cast<const __nv_bfloat16 *>(o.data), static_cast<const __nv_bfloat16 *>(d_o.data), o.ld_token, o.ld_head,
                         d_o.ld_token, d_o.ld_head, delta, (unsigned)T, (unsigned)b.heads, (unsigned)b.dim};
    const PlanArgs p = plan_args(b, kTile, plan, status);
    return b.dim <= 64 ? launch_backward<64>(ctx, b, a, d, p, stream) : launch_backward<128>(ctx, b, a, d, p, stream);
}
