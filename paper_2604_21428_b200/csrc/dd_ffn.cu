// dd_gated_ffn_forward / dd_gated_ffn_backward: arguments, tensor maps and launches of the gated
// feed-forward block.  Forward: one launch for gate, up and their product, one for the way down.
// Backward: one launch for the gradients inside the block, one for dx and the three weights.
#include <atomic>
#include <cmath>
#include <cstring>

#include "dd_ctx.h"
#include "dd_ffn_stream.cuh"

namespace ddm {

constexpr unsigned long long kFfnMax = 1ull << 30;

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor map encoder, found through the runtime (the library does not link libcuda).
static EncodeTiled tensor_map_encoder()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            return (EncodeTiled) nullptr;
        }
        return (EncodeTiled)p;
    }();
    return fn;
}

struct Matrix {
    const void *data;
    unsigned long long rows, cols, ld;      // bf16 elements
};

static int encode(dd_ctx *ctx, CUtensorMap *map, const Matrix &m, unsigned box_rows = 64)
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

static unsigned blocks_of(unsigned long long n, unsigned b) { return (unsigned)((n + b - 1) / b); }

// Adds a problem of m x n outputs in tiles of 256 x cols with its K blocks; the rest is set by the caller.
static GemmProblem &add_problem(GemmArgs &a, unsigned long long m, unsigned long long n, int cols, unsigned k1, unsigned k2 = 0,
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
static size_t slab_bytes(const dd_ctx *ctx) { return (size_t)ctx->sm_count * (2 * kBM) * 256 * 4; }

// Splits of a launch's first problem: `tiles` tiles of `blocks` K blocks, beside `other` K blocks of
// further problems.  Alone, the number that makes the fewest waves of the shortest units (a unit's
// epilogue counts as 10 blocks, the launch that adds the splits up as 8); with others to fill the
// gaps, the smallest one whose units are no longer than what each pair has to do anyway.
static unsigned choose_splits(const dd_ctx *ctx, unsigned tiles, unsigned blocks, unsigned long long other)
{
    const unsigned pairs = (unsigned)ctx->sm_count / 2;
    const unsigned long long share = ((unsigned long long)tiles * blocks + other) / pairs + 1;
    unsigned best = 1;
    unsigned long long least = ~0ull;
    for (unsigned s = 1; s <= kMaxSplits && (s == 1 || (tiles * s <= 2 * pairs && blocks >= 4 * s)); ++s) {
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

// ---- few tokens ----------------------------------------------------------------------------

// Up to here the weight-streaming kernel is ahead of the 256-row tiles of the pairs, forward with gate and up kept / backward:
// 160 tokens, d 2048, f 8192 37 / 84 us (42 / 92), 300 tokens, 1024 x 4096 28 / 48 us (30 / 50); behind at 384 tokens, 2048 x 8192:
// 66 / 120 us (64 / 116).
constexpr unsigned long long kStreamMaxTokens = 320;

// Ring of a CTA: two CTAs share an SM.
constexpr unsigned kStreamRing = 96 * 1024;

// Kernels opt in to their shared memory once per process and device; contexts of several host threads may
// come by at the same time (opting in twice does no harm).
template <typename K>
static int allow_smem(dd_ctx *ctx, K kernel, size_t bytes, std::atomic<bool> (&done)[64])
{
    const int d = ctx->device;
    if (d < 64 && done[d]) return DD_OK;
    DD_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (d < 64) done[d] = true;
    return DD_OK;
}

// Whether a kEpiStore launch takes 256 x 512 tiles.  They read a quarter fewer operand bytes a product, but
// fill tensor memory, so that an epilogue has no product to run under, and there are half as many.  The
// estimate is in cycles: a K block 1060 against 620, the rest of a unit 6000 against 800; one problem
// runs in waves, several fill the gaps.  Measured, 256 x 256 / 256 x 512: 4096 tokens, d 2048, f 8192 backward
// 636 / 580 us, forward 317 / 302; 2048 tokens 327 / 307 and 159 / 181; 1024 tokens backward 174 / 212; 8192 tokens,
// 512 x 2048 123 / 130 (the smaller time is taken in each case).
static bool wide_tiles(const dd_ctx *ctx, const GemmArgs &a)
{
    const unsigned pairs = (unsigned)ctx->sm_count / 2;
    unsigned long long time[2];
    for (int w = 0; w < 2; ++w) {
        unsigned long long sum = 0, longest = 0, tiles = 0;
        for (int i = 0; i < a.nprob; ++i) {
            const GemmProblem &p = a.prob[i];
            if (p.splits > 1) return false;
            const unsigned long long unit = (unsigned long long)(p.kblocks[0] + p.kblocks[1]) * (w ? 1060 : 620) + (w ? 6000 : 800);
            tiles = (unsigned long long)p.tiles_m * blocks_of(p.n, w ? 512 : 256);
            sum += tiles * unit;
            longest = unit > longest ? unit : longest;
        }
        time[w] = a.nprob == 1 ? blocks_of(tiles, pairs) * longest : sum / pairs + longest / 8;
        if (time[w] < longest) time[w] = longest;
    }
    return time[1] < time[0];
}

template <int EPI, int BN, int ACT>
static int launch_gemm_act(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
{
    constexpr size_t smem = gemm_smem_bytes(EPI, BN);
    static std::atomic<bool> done[64];
    const int rc = allow_smem(ctx, ffn_gemm_kernel<EPI, BN, ACT>, smem, done);
    if (rc != DD_OK) return rc;
    const unsigned most = (unsigned)ctx->sm_count / 2, pairs = a.tiles < most ? a.tiles : most;
    const GemmProblem &p = a.prob[0];
    a.first = p.tile_end;
    a.rest = a.first % pairs;
    a.extra = 0;
    if (a.rest && a.nprob > 1) {
        const GemmProblem &q = a.prob[1];
        const unsigned one = (p.kblocks[0] + p.kblocks[1]) / p.splits, next = blocks_of(q.kblocks[0] + q.kblocks[1], q.splits);
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
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, ffn_gemm_kernel<EPI, BN, ACT>, a));
    return DD_OK;
}

template <int EPI, int BN>
static int launch_gemm(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
{
    return EPI != kEpiStore && a.e.activation == DD_ACT_GELU_TANH ? launch_gemm_act<EPI, BN, EPI == kEpiStore ? DD_ACT_SILU : DD_ACT_GELU_TANH>(ctx, a, stream)
                                                                  : launch_gemm_act<EPI, BN, DD_ACT_SILU>(ctx, a, stream);
}

static int launch_store(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
{
    if (!wide_tiles(ctx, a)) return launch_gemm<kEpiStore, 256>(ctx, a, stream);
    a.tiles = 0;
    for (int i = 0; i < a.nprob; ++i) {
        GemmProblem &p = a.prob[i];
        p.tiles_n = blocks_of(p.n, 512);
        a.tiles += p.tiles_m * p.tiles_n;
        p.tile_end = a.tiles;
    }
    return launch_gemm<kEpiStore, 512>(ctx, a, stream);
}

// Slabs handed out so far, and what becomes of them.
struct Splits {
    size_t used = 0;                  // floats
    ReduceArgs r;
};

// Output of problem `p`, out (ld_out) [+ addend]: directly, or by way of its splits' slabs.
static void set_output(const dd_ctx *ctx, GemmProblem &p, Splits &sp, void *out, uint64_t ld_out, bool f32, const void *addend,
                       uint64_t ld_addend, bool addend_f32)
{
    if (p.splits == 1) {
        p.out = out;
        p.ld_out = ld_out;
        p.out_f32 = f32;
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

static int launch_reduce(dd_ctx *ctx, const Splits &sp, cudaStream_t stream)
{
    if (!sp.r.count) return DD_OK;
    const unsigned long long blocks = (sp.r.job[sp.r.count - 1].end + 255) / 256, most = (unsigned long long)ctx->sm_count * 8;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks < most ? blocks : most));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, ffn_reduce_kernel, sp.r));
    return DD_OK;
}

template <int EPI, int ACT>
static int launch_stream_act(dd_ctx *ctx, const StreamArgs &a, unsigned grid, cudaStream_t stream)
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
static int launch_stream(dd_ctx *ctx, StreamArgs &a, std::initializer_list<Matrix> x, cudaStream_t stream)
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
    return EPI != kEpiStore && a.e.activation == DD_ACT_GELU_TANH
               ? launch_stream_act<EPI, EPI == kEpiStore ? DD_ACT_SILU : DD_ACT_GELU_TANH>(ctx, a, grid, stream)
               : launch_stream_act<EPI, DD_ACT_SILU>(ctx, a, grid, stream);
}

static StreamArgs stream_args(const EpilogueArgs &e, uint64_t features, uint64_t tokens)
{
    StreamArgs a;
    std::memset(&a, 0, sizeof a);
    a.m = (unsigned)features;
    a.n = (unsigned)tokens;
    a.e = e;
    return a;
}

// The slabs, with the first call of either direction: no later call allocates them.
static int ensure_ffn_slabs(dd_ctx *ctx)
{
    if (ctx->ffn_slabs) return DD_OK;
    DD_CUDA(ctx, cudaMalloc(&ctx->ffn_slabs, slab_bytes(ctx)));
    return DD_OK;
}

// Context-owned scratch for callers that bring none.
static int ensure_ffn_scratch(dd_ctx *ctx, size_t bytes)
{
    if (bytes <= ctx->ffn_scratch_cap) return DD_OK;
    DD_CUDA(ctx, cudaDeviceSynchronize());
    if (ctx->ffn_scratch) cudaFree(ctx->ffn_scratch);
    ctx->ffn_scratch = nullptr;
    ctx->ffn_scratch_cap = 0;
    DD_CUDA(ctx, cudaMalloc(&ctx->ffn_scratch, bytes));
    ctx->ffn_scratch_cap = bytes;
    return DD_OK;
}

// ---- arguments ---------------------------------------------------------------------------------

// Rows of a matrix in memory, in bytes; no rows: touches nothing.
struct Extent {
    const void *p;
    size_t rows, width, pitch;
};

static Extent extent(const void *p, unsigned long long rows, unsigned long long cols, unsigned long long ld, size_t elem = 2)
{
    return Extent{p, p ? (size_t)rows : 0, (size_t)cols * elem, (size_t)ld * elem};
}

// Whether two matrices share a byte.  Rows of one pitch may lie side by side (gate and up as halves of one
// buffer's rows); of different pitches whatever lies between the ends is taken.
static bool touches(const Extent &a, const Extent &b)
{
    if (!a.rows || !b.rows) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    if (y < x) return touches(b, a);
    if (y >= x + (a.rows - 1) * a.pitch + a.width) return false;
    if (a.pitch != b.pitch) return true;
    const size_t off = (y - x) % a.pitch;
    return off < a.width || off + b.width > a.pitch;
}

static int set_stride(uint64_t &ld, uint64_t cols)
{
    if (ld == 0) ld = cols;
    if (ld < cols) return DD_ERR_INVALID_ARG;
    if (ld >= kFfnMax) return DD_ERR_TOO_LARGE;
    return ld % 8 ? DD_ERR_ALIGNMENT : DD_OK;
}

// Validates the block and fills in its defaults; without gate and up their stride is not looked at.
static int check_block(const dd_ctx *ctx, dd_gated_ffn &b, bool with_gate)
{
    if (!ctx || b.d < 1 || b.f < 1) return DD_ERR_INVALID_ARG;
    if (b.activation != DD_ACT_SILU && b.activation != DD_ACT_GELU_TANH) return DD_ERR_INVALID_ARG;
    if (b.flags & ~(uint32_t)DD_DEBUG_EXPIRE_WAIT) return DD_ERR_INVALID_ARG;
    if (b.tokens >= kFfnMax || b.d >= kFfnMax || b.f >= kFfnMax) return DD_ERR_TOO_LARGE;
    struct { uint64_t *ld; uint64_t cols; } strides[] = {{&b.ld_x, b.d}, {&b.ld_y, b.d}, {&b.ld_gate, b.f}, {&b.ld_in, b.d}, {&b.ld_down, b.f}};
    for (auto &s : strides) {
        if (s.ld == &b.ld_gate && !with_gate) continue;
        const int rc = set_stride(*s.ld, s.cols);
        if (rc != DD_OK) return rc;
    }
    if (!b.w_gate || !b.w_up || !b.w_down) return DD_ERR_INVALID_ARG;
    return DD_OK;
}

static int check_aligned(std::initializer_list<const void *> ptrs)
{
    for (const void *p : ptrs)
        if ((uintptr_t)p & 15u) return DD_ERR_ALIGNMENT;
    return DD_OK;
}

// Outputs first: none may touch another output or an input.
static int check_alias(std::initializer_list<Extent> outs, std::initializer_list<Extent> ins)
{
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (auto q = outs.begin(); q != o; ++q)
            if (touches(*o, *q)) return DD_ERR_ALIAS;
        for (const Extent &i : ins)
            if (touches(*o, i)) return DD_ERR_ALIAS;
    }
    return DD_OK;
}

}  // namespace ddm

using namespace ddm;

extern "C" int dd_gated_ffn_forward(dd_ctx *ctx, const dd_gated_ffn *block, const void *x, const void *residual,
                                    void *gate, void *up, void *hidden, void *y, int32_t *status, void *cuda_stream)
{
    if (!block) return DD_ERR_INVALID_ARG;
    dd_gated_ffn b = *block;
    int rc = check_block(ctx, b, gate != nullptr);
    if (rc != DD_OK) return rc;
    if ((gate == nullptr) != (up == nullptr)) return DD_ERR_INVALID_ARG;
    if (b.tokens > 0 && (!x || !y)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)status & 3u) return DD_ERR_ALIGNMENT;
    rc = check_aligned({x, residual, gate, up, hidden, y, b.w_gate, b.w_up, b.w_down});
    if (rc != DD_OK) return rc;
    const uint64_t T = b.tokens, ldh = (b.f + 7) / 8 * 8;
    const Extent ex = extent(x, T, b.d, b.ld_x), ey = extent(y, T, b.d, b.ld_y), eg = extent(gate, T, b.f, b.ld_gate),
                 eu = extent(up, T, b.f, b.ld_gate), eh = extent(hidden, T, ldh, ldh), er = extent(residual, T, b.d, b.ld_y),
                 wg = extent(b.w_gate, b.f, b.d, b.ld_in), wu = extent(b.w_up, b.f, b.d, b.ld_in),
                 wd = extent(b.w_down, b.d, b.f, b.ld_down);
    rc = check_alias({ey, eg, eu, eh}, {ex, wg, wu, wd, y == residual ? Extent{} : er});
    if (rc == DD_OK && y == residual) rc = check_alias({eg, eu, eh}, {er});
    if (rc != DD_OK) return rc;
    if (T == 0) return DD_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    rc = ensure_ffn_slabs(ctx);
    if (rc != DD_OK) return rc;
    if (!hidden) {
        rc = ensure_ffn_scratch(ctx, (size_t)(T * ldh) * 2);
        if (rc != DD_OK) return rc;
        hidden = ctx->ffn_scratch;
    }
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    EpilogueArgs e;
    std::memset(&e, 0, sizeof e);
    e.activation = b.activation;
    e.expire = b.flags != 0;
    e.status = status;
    e.gate = (__nv_bfloat16 *)gate;
    e.up = (__nv_bfloat16 *)up;
    e.hidden = (__nv_bfloat16 *)hidden;
    e.ld_gate = b.ld_gate;
    e.ld_hidden = ldh;
    e.out = (__nv_bfloat16 *)y;
    e.residual = (const __nv_bfloat16 *)residual;
    e.ld_out = e.ld_residual = b.ld_y;
    const Matrix mx = {x, T, b.d, b.ld_x}, mg = {b.w_gate, b.f, b.d, b.ld_in}, mu = {b.w_up, b.f, b.d, b.ld_in},
                 md = {b.w_down, b.d, b.f, b.ld_down}, mh = {hidden, T, b.f, ldh};
    if (T <= kStreamMaxTokens) {
        StreamArgs a = stream_args(e, b.f, T);
        a.kblocks[0] = blocks_of(b.d, kBK);
        rc = encode(ctx, &a.w[0], mg);
        if (rc == DD_OK) rc = encode(ctx, &a.w[1], mu);
        if (rc == DD_OK) rc = launch_stream<kEpiGate>(ctx, a, {mx}, stream);
        if (rc != DD_OK) return rc;
        a.m = (unsigned)b.d;
        a.kblocks[0] = blocks_of(b.f, kBK);
        a.own_prior = 1;
        rc = encode(ctx, &a.w[0], md);
        return rc == DD_OK ? launch_stream<kEpiStore>(ctx, a, {mh}, stream) : rc;
    }
    GemmArgs a;
    std::memset(&a, 0, sizeof a);
    a.e = e;
    rc = encode(ctx, &a.maps[0], mx);
    if (rc == DD_OK) rc = encode(ctx, &a.maps[1], mg);
    if (rc == DD_OK) rc = encode(ctx, &a.maps[2], mu);
    if (rc != DD_OK) return rc;
    GemmProblem &p = add_problem(a, T, b.f, 128, blocks_of(b.d, kBK));
    p.b_map[0] = 1;
    p.b_map[1] = 2;
    rc = launch_gemm<kEpiGate, 256>(ctx, a, stream);
    if (rc != DD_OK) return rc;

    a.nprob = 0;
    a.tiles = 0;
    const unsigned kf = blocks_of(b.f, kBK);
    const unsigned splits = choose_splits(ctx, blocks_of(T, 2 * kBM) * blocks_of(b.d, 256), kf, 0);
    GemmProblem &q = add_problem(a, T, b.d, 256, kf, 0, splits);
    q.b_map[0] = 1;
    rc = encode(ctx, &a.maps[0], mh);
    if (rc == DD_OK) rc = encode(ctx, &a.maps[1], md);
    Splits sp;
    sp.r.count = 0;
    set_output(ctx, q, sp, y, b.ld_y, false, residual, b.ld_y, false);
    if (rc == DD_OK) rc = launch_store(ctx, a, stream);
    return rc == DD_OK ? launch_reduce(ctx, sp, stream) : rc;
}

extern "C" int dd_gated_ffn_backward(dd_ctx *ctx, const dd_gated_ffn *block, const void *x, const void *gate,
                                     const void *up, const void *dy, void *dx, void *dw_gate, void *dw_up,
                                     void *dw_down, dd_dtype grad_dtype, int accumulate, void *scratch,
                                     int32_t *status, void *cuda_stream)
{
    if (!block) return DD_ERR_INVALID_ARG;
    dd_gated_ffn b = *block;
    int rc = check_block(ctx, b, true);
    if (rc != DD_OK) return rc;
    if (grad_dtype != DD_F32 && grad_dtype != DD_BF16) return DD_ERR_INVALID_ARG;
    if (!dw_gate || !dw_up || !dw_down) return DD_ERR_INVALID_ARG;
    if (b.tokens > 0 && (!x || !gate || !up || !dy || !dx)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)status & 3u) return DD_ERR_ALIGNMENT;
    rc = check_aligned({x, gate, up, dy, dx, dw_gate, dw_up, dw_down, scratch, b.w_gate, b.w_up, b.w_down});
    if (rc != DD_OK) return rc;
    const uint64_t T = b.tokens, ldh = (b.f + 7) / 8 * 8;
    const size_t ge = grad_dtype == DD_BF16 ? 2 : 4;
    rc = check_alias({extent(dx, T, b.d, b.ld_x), extent(dw_gate, b.f, b.d, b.ld_in, ge), extent(dw_up, b.f, b.d, b.ld_in, ge),
                      extent(dw_down, b.d, b.f, b.ld_down, ge), extent(scratch, 3 * T, ldh, ldh)},
                     {extent(x, T, b.d, b.ld_x), extent(gate, T, b.f, b.ld_gate), extent(up, T, b.f, b.ld_gate),
                      extent(dy, T, b.d, b.ld_y), extent(b.w_gate, b.f, b.d, b.ld_in), extent(b.w_up, b.f, b.d, b.ld_in),
                      extent(b.w_down, b.d, b.f, b.ld_down)});
    if (rc != DD_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (T == 0) {                          // sums over no token
        if (accumulate) return DD_OK;
        DD_CUDA(ctx, cudaMemset2DAsync(dw_gate, b.ld_in * ge, 0, b.d * ge, b.f, stream));
        DD_CUDA(ctx, cudaMemset2DAsync(dw_up, b.ld_in * ge, 0, b.d * ge, b.f, stream));
        DD_CUDA(ctx, cudaMemset2DAsync(dw_down, b.ld_down * ge, 0, b.f * ge, b.d, stream));
        return DD_OK;
    }
    rc = ensure_ffn_slabs(ctx);
    if (rc != DD_OK) return rc;
    if (!scratch) {
        rc = ensure_ffn_scratch(ctx, (size_t)(3 * T * ldh) * 2);
        if (rc != DD_OK) return rc;
        scratch = ctx->ffn_scratch;
    }
    enum { kX, kDy, kWg, kWu, kWd, kDg, kDu, kH };
    __nv_bfloat16 *dg = (__nv_bfloat16 *)scratch, *du = dg + T * ldh, *h = du + T * ldh;
    const Matrix mats[kH + 1] = {{x, T, b.d, b.ld_x}, {dy, T, b.d, b.ld_y}, {b.w_gate, b.f, b.d, b.ld_in},
                                   {b.w_up, b.f, b.d, b.ld_in}, {b.w_down, b.d, b.f, b.ld_down},
                                   {dg, T, b.f, ldh}, {du, T, b.f, ldh}, {h, T, b.f, ldh}};
    GemmArgs a;
    std::memset(&a, 0, sizeof a);
    const bool few = T <= kStreamMaxTokens;
    for (int i = 0; i <= kH; ++i) {
        rc = encode(ctx, &a.maps[i], mats[i]);
        if (rc != DD_OK) return rc;
    }
    EpilogueArgs &e = a.e;
    e.activation = b.activation;
    e.expire = b.flags != 0;
    e.status = status;
    e.gate = (__nv_bfloat16 *)const_cast<void *>(gate);
    e.up = (__nv_bfloat16 *)const_cast<void *>(up);
    e.dgate = dg;
    e.dup = du;
    e.hidden = h;
    e.ld_gate = b.ld_gate;
    e.ld_hidden = ldh;
    // dh = dy w_down: [T, d] x [d, f], and the gradients inside the block in its epilogue
    if (few) {
        StreamArgs c = stream_args(e, b.f, T);
        c.e.out = (__nv_bfloat16 *)dx;
        c.e.ld_out = b.ld_x;
        c.kblocks[0] = blocks_of(b.d, kBK);
        c.w[0] = a.maps[kWd];
        c.w_mn = 1;
        rc = launch_stream<kEpiBack>(ctx, c, {mats[kDy]}, stream);
        if (rc != DD_OK) return rc;
        c.m = (unsigned)b.d;                              // dgate w_gate + dup w_up
        c.kblocks[0] = c.kblocks[1] = blocks_of(b.f, kBK);
        c.w[0] = a.maps[kWg];
        c.w[1] = a.maps[kWu];
        c.own_prior = c.late_trigger = a.late_wait = 1;
        rc = launch_stream<kEpiStore>(ctx, c, {mats[kDg], mats[kDu]}, stream);
        if (rc != DD_OK) return rc;
    } else {
        GemmArgs c = a;
        c.maps[0] = a.maps[kDy];
        c.maps[1] = a.maps[kWd];
        GemmProblem &p = add_problem(c, T, b.f, 256, blocks_of(b.d, kBK));
        p.b_map[0] = 1;
        p.b_mn = 1;
        rc = launch_gemm<kEpiBack, 256>(ctx, c, stream);
        if (rc != DD_OK) return rc;
    }
    const unsigned kt = blocks_of(T, kBK), kf = blocks_of(b.f, kBK), pairs = (unsigned)ctx->sm_count / 2;
    const unsigned wtiles = 3 * blocks_of(b.f, 2 * kBM) * blocks_of(b.d, 256);
    const unsigned xtiles = few ? 0 : blocks_of(T, 2 * kBM) * blocks_of(b.d, 256);
    Splits sp;
    sp.r.count = 0;
    if (!few) {                                           // dgate w_gate + dup w_up
        GemmProblem &p = add_problem(a, T, b.d, 256, kf, kf, choose_splits(ctx, xtiles, 2 * kf, (unsigned long long)wtiles * kt));
        p.a_map[0] = kDg;
        p.a_map[1] = kDu;
        p.b_map[0] = kWg;
        p.b_map[1] = kWu;
        p.b_mn = 1;
        set_output(ctx, p, sp, dx, b.ld_x, false, nullptr, 0, false);
    }
    // Few weights and many tokens: too few tiles for the pairs, so the tokens are split as well, as long
    // as all units make one wave and it shortens them by more than the reducing launch costs (8192 tokens,
    // d 256, f 512: 71 -> 39 us; with units left over for a second wave 2000 tokens, 504 x 1200 took 51, not 37)
    unsigned wsplits = 1;
    while (wsplits < kMaxSplits && a.tiles + wtiles * (wsplits + 1) <= pairs && kt >= 4 * (wsplits + 1)) ++wsplits;
    if (kt - kt / wsplits < 16) wsplits = 1;
    struct { int a, b; void *out; uint64_t m, n, ld; } weights[3] = {
        {kDg, kX, dw_gate, b.f, b.d, b.ld_in}, {kDu, kX, dw_up, b.f, b.d, b.ld_in}, {kDy, kH, dw_down, b.d, b.f, b.ld_down}};
    for (const auto &w : weights) {
        GemmProblem &q = add_problem(a, w.m, w.n, 256, kt, 0, wsplits);
        q.a_map[0] = (unsigned char)w.a;
        q.b_map[0] = (unsigned char)w.b;
        q.a_mn = q.b_mn = 1;
        set_output(ctx, q, sp, w.out, w.ld, grad_dtype == DD_F32, accumulate ? w.out : nullptr, w.ld, grad_dtype == DD_F32);
    }
    rc = launch_store(ctx, a, stream);
    return rc == DD_OK ? launch_reduce(ctx, sp, stream) : rc;
}
