// Host side of the tensor-core products: tensor maps, problems, splits and launches, for the entry points that
// are built on them.
#pragma once

#include "dd_args.h"
#include "dd_ffn_stream.cuh"

namespace ddm {

constexpr unsigned long long kFfnMax = 1ull << 30;

struct Matrix {
    const void *data;
    unsigned long long rows, cols, ld;      // bf16 elements
};

inline int encode(dd_ctx *ctx, CUtensorMap *map, const Matrix &m, unsigned box_rows = 64)
{
    const cuuint64_t dims[2] = {m.cols, m.rows}, strides[1] = {m.ld * 2};
    const cuuint32_t box[2] = {64, box_rows}, step[2] = {1, 1};
    const EncodeTiled fn = tensor_map_encoder();
    if (!fn || fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(m.data), dims, strides, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
        snprintf(ctx->cuda_err, sizeof ctx->cuda_err, "cuTensorMapEncodeTiled failed");
        return DD_ERR_CUDA;
    }
    return DD_OK;
}

// Adds a problem of m x n outputs in tiles of 256 x cols with its K blocks; the rest is set by the caller.
inline GemmProblem &add_problem(GemmArgs &a, unsigned long long m, unsigned long long n, int cols, unsigned k1, unsigned k2 = 0,
                                unsigned splits = 1)
{
    GemmProblem &p = a.prob[a.nprob++];
    std::memset(&p, 0, sizeof p);
    p.m = (unsigned)m;
    p.n = (unsigned)n;
    p.tiles_m = blocks_of(m, 2 * kBM);
    p.tiles_n = blocks_of(n, cols);
    p.kblocks[0] = k1;
    p.kblocks[1] = k2;
    p.splits = splits;
    p.split_rows = p.tiles_m * 2 * kBM;
    a.tiles += p.tiles_m * p.tiles_n * splits;
    p.tile_end = a.tiles;
    return p;
}

// Float32 slabs of split products: 256 KB for each of two tiles per pair of SMs.
inline size_t slab_bytes(const dd_ctx *ctx) { return (size_t)ctx->sm_count * (2 * kBM) * 256 * 4; }

// Splits of a launch's first problem: `tiles` tiles of `blocks` K blocks, beside `other` K blocks of
// further problems.  Alone, the number that makes the fewest waves of the shortest units (a unit's
// epilogue counts as 10 blocks, the launch that adds the splits up as 8); with others to fill the
// gaps, the smallest one whose units are no longer than what each pair has to do anyway.
inline unsigned choose_splits(const dd_ctx *ctx, unsigned tiles, unsigned blocks, unsigned long long other, unsigned most = kMaxSplits)
{
    const unsigned pairs = (unsigned)ctx->sm_count / 2;
    const unsigned long long share = ((unsigned long long)tiles * blocks + other) / pairs + 1;
    unsigned best = 1;
    unsigned long long least = ~0ull;
    for (unsigned s = 1; s <= most && (s == 1 || (tiles * s <= 2 * pairs && blocks >= 4 * s)); ++s) {
        if (other) {
            best = s;
            if (blocks / s <= share) break;
            continue;
        }
        const unsigned long long cost = (unsigned long long)blocks_of(tiles * s, pairs) * (blocks_of(blocks, s) + 10) + (s > 1 ? 8 : 0);
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    return best;
}

// K blocks that a unit's epilogue takes as long as (256 x 256 outputs: 2.7 us): with fewer, the schedule counts these.
// (One token, d 2048, 32000 columns of the vocabulary, whose gradient has one K block a tile: the backward pass 224 us without, 111 with.
// The block's backward pass, 321 / 448 tokens, d 2048, f 8192, bf16 gradients 104 / 108 us without, 101 / 105 with, float32 169 / 165
// and 157 / 159; 1000 tokens, 256 x 1024 40 and 38, float32 44 and 40.)
constexpr unsigned kEpilogueBlocks = 8;
inline unsigned unit_blocks(unsigned blocks) { return blocks > kEpilogueBlocks ? blocks : kEpilogueBlocks; }

template <int EPI, int BN, int ACT, bool SUM = false>
inline int launch_gemm_act(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
{
    constexpr size_t smem = gemm_smem_bytes(EPI, BN);
    static std::atomic<bool> done[64];
    const int rc = allow_smem(ctx, ffn_gemm_kernel<EPI, BN, ACT, SUM>, smem, done);
    if (rc != DD_OK) return rc;
    const unsigned most = (unsigned)ctx->sm_count / 2, pairs = a.tiles < most ? a.tiles : most;
    const GemmProblem &p = a.prob[0];
    a.first = p.tile_end;
    a.rest = a.first % pairs;
    a.extra = 0;
    if (a.rest && a.nprob > 1) {
        const GemmProblem &q = a.prob[1];
        // a unit costs its K blocks, or its epilogue, which runs under the next unit's, where that is longer
        const unsigned one = unit_blocks((p.kblocks[0] + p.kblocks[1]) / p.splits), next = unit_blocks(blocks_of(q.kblocks[0] + q.kblocks[1], q.splits));
        a.extra = (one + next / 2) / next;
        const unsigned room = (a.tiles - a.first) / (pairs - a.rest);
        if (a.extra > room) a.extra = room;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * pairs);
    cfg.blockDim = dim3(kGemmThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, ffn_gemm_kernel<EPI, BN, ACT, SUM>, a));
    return DD_OK;
}

template <int EPI, int BN>
inline int launch_gemm(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
{
    if constexpr (EPI == kEpiStore) {
        for (int i = 0; i < a.nprob; ++i)
            if (a.prob[i].out_f32 == kOutSum) return launch_gemm_act<EPI, BN, DD_ACT_SILU, true>(ctx, a, stream);
        return launch_gemm_act<EPI, BN, DD_ACT_SILU>(ctx, a, stream);
    } else {
        return a.e.activation == DD_ACT_GELU_TANH ? launch_gemm_act<EPI, BN, DD_ACT_GELU_TANH>(ctx, a, stream)
                                                  : launch_gemm_act<EPI, BN, DD_ACT_SILU>(ctx, a, stream);
    }
}

// Slabs handed out so far, and what becomes of them.
struct Splits {
    size_t used = 0;                  // floats
    ReduceArgs r;
};

// Output of problem `p`, out (ld_out) [+ addend]: directly, or by way of its splits' slabs.
inline void set_output(const dd_ctx *ctx, GemmProblem &p, Splits &sp, void *out, uint64_t ld_out, bool f32, const void *addend,
                       uint64_t ld_addend, bool addend_f32)
{
    if (p.splits == 1) {
        p.out = out;
        p.ld_out = ld_out;
        p.out_f32 = f32 ? kOutF32 : addend && addend_f32 ? kOutSum : kOutBf16;
        p.addend = addend;
        p.ld_addend = ld_addend;
        return;
    }
    const unsigned ld = (p.n + 7) / 8 * 8;
    p.out = ctx->ffn_slabs + sp.used;
    p.ld_out = ld;
    p.out_f32 = 1;
    const unsigned long long slab = (unsigned long long)p.split_rows * ld;
    ReduceJob &j = sp.r.job[sp.r.count];
    const unsigned long long before = sp.r.count ? sp.r.job[sp.r.count - 1].end : 0;
    j = {ctx->ffn_slabs + sp.used, p.splits, p.m, p.n, ld, slab, before + (unsigned long long)p.m * (ld / 8), out, addend, ld_out, ld_addend,
         f32, addend_f32};
    ++sp.r.count;
    sp.used += p.splits * slab;
}

// The slabs, with the first call of either direction: no later call allocates them.
inline int ensure_ffn_slabs(dd_ctx *ctx)
{
    if (ctx->ffn_slabs) return DD_OK;
    DD_CUDA(ctx, cudaMalloc(&ctx->ffn_slabs, slab_bytes(ctx)));
    return DD_OK;
}

inline int set_stride(uint64_t &ld, uint64_t cols)
{
    if (ld == 0) ld = cols;
    if (ld < cols) return DD_ERR_INVALID_ARG;
    if (ld >= kFfnMax) return DD_ERR_TOO_LARGE;
    return ld % 8 ? DD_ERR_ALIGNMENT : DD_OK;
}

// ---- few tokens ----------------------------------------------------------------------------

// Up to here the weight-streaming kernel is ahead of the 256-row tiles of the pairs, forward with gate and up kept / backward:
// 160 tokens, d 2048, f 8192 37 / 84 us (42 / 92), 300 tokens, 1024 x 4096 28 / 48 us (30 / 50); behind at 384 tokens, 2048 x 8192:
// 66 / 120 us (64 / 116).
constexpr unsigned long long kStreamMaxTokens = 320;

// Ring of a CTA: two CTAs share an SM.
constexpr unsigned kStreamRing = 96 * 1024;

template <int EPI, int ACT>
inline int launch_stream_act(dd_ctx *ctx, const StreamArgs &a, unsigned grid, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kStreamThreads);
    cfg.dynamicSmemBytes = stream_smem_bytes(a.cols, a.stages);
    cfg.stream = stream;
    static std::atomic<bool> done[64];
    const int rc = allow_smem(ctx, ffn_stream_kernel<EPI, ACT>, kStreamRing + 2048, done);
    if (rc != DD_OK) return rc;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)a.cluster, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, ffn_stream_kernel<EPI, ACT>, a));
    return DD_OK;
}

// Shape and launch: the tokens in equal tiles of at most 128, K over as many CTAs as give every SM
// one, each with two K blocks at least; x: the token matrices of the K segments.
template <int EPI>
inline int launch_stream(dd_ctx *ctx, StreamArgs &a, std::initializer_list<Matrix> x, cudaStream_t stream)
{
    const unsigned rows = blocks_of(a.m, stream_features(EPI)), blocks = a.kblocks[0] + a.kblocks[1], sms = (unsigned)ctx->sm_count;
    a.tiles_n = blocks_of(a.n, kStreamMaxCols);
    const auto cluster = [&] {
        unsigned s = 1;
        while (s < kStreamMaxCluster && rows * a.tiles_n * s < sms && blocks >= 4 * s) s *= 2;
        return s;
    };
    unsigned s = cluster();
    while (rows * a.tiles_n * s < sms && a.n / a.tiles_n >= 64) {
        a.tiles_n *= 2;
        s = cluster();
    }
    a.cols = blocks_of(blocks_of(a.n, a.tiles_n), 16) * 16;
    a.tiles_n = blocks_of(a.n, a.cols);
    a.cluster = (int)s;
    const unsigned stages = kStreamRing / stream_stage_bytes(a.cols);
    a.stages = (int)(stages > kStreamMaxStages ? kStreamMaxStages : stages);
    int i = 0;
    for (const Matrix &m : x) {
        const int rc = encode(ctx, &a.x[i++], m, a.cols);
        if (rc != DD_OK) return rc;
    }
    const unsigned grid = rows * a.tiles_n * s;
    constexpr bool kActs = EPI == kEpiGate || EPI == kEpiBack;
    return kActs && a.e.activation == DD_ACT_GELU_TANH ? launch_stream_act<EPI, kActs ? DD_ACT_GELU_TANH : DD_ACT_SILU>(ctx, a, grid, stream)
                                                       : launch_stream_act<EPI, DD_ACT_SILU>(ctx, a, grid, stream);
}

inline StreamArgs stream_args(const EpilogueArgs &e, uint64_t features, uint64_t tokens)
{
    StreamArgs a;
    std::memset(&a, 0, sizeof a);
    a.m = (unsigned)features;
    a.n = (unsigned)tokens;
    a.e = e;
    return a;
}

// ---- many tokens ----------------------------------------------------------------------------

// Launches of kEpiStore problems, in tiles of 256 or 512 columns, and of what adds their splits up (dd_ffn.cu).
int launch_store(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream);
int launch_reduce(dd_ctx *ctx, const Splits &sp, cudaStream_t stream);

}  // namespace ddm
