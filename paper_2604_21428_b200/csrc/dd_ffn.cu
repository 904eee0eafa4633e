// dd_gated_ffn_forward / dd_gated_ffn_backward: arguments, tensor maps and launches of the gated
// feed-forward block.  Forward: one launch for gate, up and their product, one for the way down.
// Backward: one launch for the gradients inside the block, one for dx and the three weights.
#include <cmath>

#include "dd_gemm_launch.cuh"

namespace ddm {

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

int launch_store(dd_ctx *ctx, GemmArgs &a, cudaStream_t stream)
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

__global__ void __launch_bounds__(256)
ffn_reduce_kernel(const __grid_constant__ ReduceArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int k = 0;
    for (unsigned long long i = (unsigned long long)blockIdx.x * blockDim.x + threadIdx.x; i < a.job[a.count - 1].end;
         i += (unsigned long long)gridDim.x * blockDim.x) {
        while (i >= a.job[k].end) ++k;
        const ReduceJob &j = a.job[k];
        const unsigned long long at = i - (k ? a.job[k - 1].end : 0ull);
        const unsigned pieces = j.ld / 8, row = (unsigned)(at / pieces), col = (unsigned)(at % pieces) * 8;
        const unsigned cols = j.n - col < 8 ? j.n - col : 8;
        const float *src = j.slabs + (unsigned long long)row * j.ld + col;
        float x[2][4];
        for (unsigned s0 = 0; s0 < j.splits; s0 += kMaxSplits) {          // in split order, eight asked for at a time
            float4 v[kMaxSplits][2];
#pragma unroll
            for (int s = 0; s < kMaxSplits; ++s)
                if (s0 + s < j.splits) {
                    v[s][0] = __ldcg(reinterpret_cast<const float4 *>(src + (s0 + s) * j.slab));
                    v[s][1] = __ldcg(reinterpret_cast<const float4 *>(src + (s0 + s) * j.slab) + 1);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!s0) { x[h][0] = v[0][h].x; x[h][1] = v[0][h].y; x[h][2] = v[0][h].z; x[h][3] = v[0][h].w; }
                else { x[h][0] += v[0][h].x; x[h][1] += v[0][h].y; x[h][2] += v[0][h].z; x[h][3] += v[0][h].w; }
#pragma unroll
                for (int s = 1; s < kMaxSplits; ++s)
                    if (s0 + s < j.splits) { x[h][0] += v[s][h].x; x[h][1] += v[s][h].y; x[h][2] += v[s][h].z; x[h][3] += v[s][h].w; }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned c = col + 4 * h, live = cols > 4 * h ? cols - 4 * h : 0;
            if (!live) break;
            if (j.addend) {
                float add[4];
                const unsigned long long from = (unsigned long long)row * j.ld_addend + c;
                if (j.addend_f32) load4_f32(static_cast<const float *>(j.addend) + from, add, live);
                else load4(static_cast<const __nv_bfloat16 *>(j.addend) + from, add, live);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[h][q] += add[q];
            }
            const unsigned long long to = (unsigned long long)row * j.ld_out + c;
            if (j.out_f32) store4_f32(static_cast<float *>(j.out) + to, x[h], live);
            else store4(static_cast<__nv_bfloat16 *>(j.out) + to, x[h], live);
        }
    }
}

int launch_reduce(dd_ctx *ctx, const Splits &sp, cudaStream_t stream)
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
