// dd_vocab_loss_forward / dd_vocab_loss_backward.  Forward: one launch that forms the logits tile by tile
// and leaves each row's largest and sum of exponentials over 128 columns, one that joins those.  Backward, for each
// piece of the vocabulary: the logits once more, as their gradient in bf16; then the products of that with the
// weight and with the hidden rows, side by side.
//
// Bound by the products, 2 T d V of them forward, 6 T d V backward beside 2 T d V for the logits again: 8192 tokens,
// d 2048, 32000 columns 762 us forward in short runs and 865 sustained under the 1000 W cap (1410 and 1240 TFLOP/s), 2440 and
// 2795 us backward (1760 and 1540 TFLOP/s with the logits); float32 dweight 2465 and 2850, added to 2695 and
// 3065.  With few tokens by the weights' bytes, read once forward; backward reads them twice and writes as many (4 tokens: 39 us
// from a cold L2 and 97 from a warm one, of which the bytes need 20 and 40).
//
// The logits' gradient is rounded to bf16 because it is an operand of both products: in the results that is one rounding
// beside their own: 1.3-1.5 times the error of theirs alone in the mean.  A target's term is most of a row, and its rounding is
// the same in all of the row, so a few tokens do not average it out: 2.2 were seen with one token, 1.7 with eight, 1.6 with 32.
#include <cmath>

#include "dd_decoder.h"
#include "dd_gemm_launch.cuh"

namespace ddm {

// lse = log sum exp over the partial sums of a token, and the loss; 32 tokens a block, its 32 warps taking every
// 32nd of their partial sums, eight of them asked for at a time.
constexpr unsigned kJoinWarps = 32;

__global__ void __launch_bounds__(32 * kJoinWarps)
vocab_loss_join_kernel(const float2 *partial, unsigned parts, unsigned tokens, const long long *targets, long long vocab, float *loss, float *lse)
{
    constexpr float l = 1.4426950408889634f;
    __shared__ float2 share[kJoinWarps][33];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = blockIdx.x * 32 + lane;
    const auto join = [](float2 &a, const float2 &b) {
        const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.0f : m;
        a.y = a.y * exp2_fast((a.x - base) * l) + b.y * exp2_fast((b.x - base) * l);
        a.x = m;
    };
    float2 mine = make_float2(-INFINITY, 0.0f);
    for (unsigned p0 = warp; p0 < parts; p0 += 8 * kJoinWarps) {
        float2 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned p = p0 + i * kJoinWarps;
            x[i] = p < parts && t < tokens ? __ldcg(partial + (unsigned long long)p * tokens + t) : make_float2(-INFINITY, 0.0f);
        }
#pragma unroll
        for (int d = 1; d < 8; d *= 2)
#pragma unroll
            for (int i = 0; i < 8; i += 2 * d) join(x[i], x[i + d]);
        join(mine, x[0]);
    }
    share[warp][lane] = mine;
    __syncthreads();
    // now a warp has a token, its lanes the warps' shares
    const unsigned mt = blockIdx.x * 32 + warp;
    if (mt >= tokens) return;
    float2 x = share[lane][warp];
#pragma unroll
    for (int d = 16; d; d /= 2) {
        const float2 y = make_float2(__shfl_xor_sync(0xffffffffu, x.x, d), __shfl_xor_sync(0xffffffffu, x.y, d));
        join(x, y);
    }
    if (lane) return;
    const float z = x.x + logf(x.y);
    const long long target = targets[mt];
    lse[mt] = z;
    loss[mt] = target < 0 ? 0.0f : target >= vocab ? NAN : z - loss[mt];
}

// Splits of the sum over the vocabulary that makes dhidden: with few tokens it has few tiles and a long K (35 tokens,
// d 231, 8075 columns: 17 us for the second launch with 8 splits, 12 with more).
constexpr unsigned kLossSplits = 32;

// Tokens up to which the logits (forward), and with them dhidden (backward), are made by the kernel that streams weights
// past few tokens.  It reads the weights at 4.5 TB/s where the products' kernel reads them at 3.3, and its clusters split
// the sum over d, which the other kernel's epilogues cannot do; but it reads the tokens for every 128 columns and finishes
// a tile after its products.  So it goes furthest where the other kernel's tiles of 256 columns would leave three
// quarters of the pairs of SMs idle, and, forward, as far as one tile of tokens where its own tiles give every SM one
// without clusters.  us from a cold L2, this / the other kernel:
//   forward   2344 x 1643 (d x columns), 16 / 105 / 256 tokens 14 / 16 / 22 (23 / 26 / 28), 4096 x 3000 18 / 24 / 28 (33 / 35 / 35);
//             512 x 5000, 16 / 48 / 80 tokens 14 / 16 / 18 (16 all), 2048 x 8192 20 / 22 / 25 (25 / 25 / 26);
//             768 x 32000, 4 / 64 / 128 / 192 tokens 22 / 25 / 28 / 37 (27 / 31 / 29 / 29), 2048 x 32000 39 / 41 / 45 / 59 (49 / 46 / 47 / 47)
//   backward  2344 x 1643, 16 / 105 / 256 tokens 24 / 30 / 37 (38 / 41 / 43), 4096 x 3000 31 / 42 / 49 (51 / 55 / 57);
//             512 x 5000, 16 / 105 / 128 / 160 tokens 18 / 24 / 29 / 28 (25 / 29 / 29 / 29), 1024 x 16000 38 / 47 / 49 / 53 (47 / 49 / 49 / 50);
//             768 x 32000 from a warm L2, 4 / 64 / 96 tokens 48 / 56 / 63 (51 / 57 / 56)
static bool few_tokens(const dd_ctx *ctx, const dd_vocab_loss &l, bool backward)
{
    const unsigned sms = (unsigned)ctx->sm_count;
    const bool narrow = blocks_of(l.vocab, 256) * 4 <= sms / 2, wide = blocks_of(l.vocab, kBM) >= sms;
    return l.tokens <= (narrow ? 256 : backward ? (wide ? 80 : 128) : wide ? kStreamMaxCols : 48);
}

static uint64_t rows8(uint64_t n) { return (n + 7) / 8 * 8; }

// Columns of the vocabulary whose gradients are held at one time: as many as make 128 MB, so that what the
// first launch of a piece writes is still in L2 when the second reads it, but 2048 at least.
static uint64_t piece_columns(const dd_vocab_loss &l)
{
    const uint64_t most = (64ull << 20) / (l.tokens ? l.tokens : 1), cols = most < 2048 ? 2048 : most;
    const uint64_t pieces = (l.vocab + cols - 1) / cols, each = (l.vocab + pieces - 1) / pieces;
    return (each + 255) / 256 * 256 < l.vocab ? (each + 255) / 256 * 256 : l.vocab;
}

static uint64_t forward_bytes(const dd_vocab_loss &l) { return (l.vocab + 127) / 128 * l.tokens * sizeof(float2); }
static uint64_t piece_bytes(const dd_vocab_loss &l) { return l.tokens * rows8(piece_columns(l)) * 2; }
static uint64_t backward_bytes(const dd_vocab_loss &l)
{
    return piece_bytes(l) + (piece_columns(l) < l.vocab ? l.tokens * rows8(l.d) * 4 : 0);
}

static int check_loss(const dd_ctx *ctx, dd_vocab_loss &l)
{
    if (!ctx || l.d < 1 || l.vocab < 1) return DD_ERR_INVALID_ARG;
    if (l.tokens >= kFfnMax || l.d >= kFfnMax || l.vocab >= kFfnMax) return DD_ERR_TOO_LARGE;
    if (l.flags & ~(uint32_t)DD_DEBUG_EXPIRE_WAIT) return DD_ERR_INVALID_ARG;
    int rc = set_stride(l.ld_hidden, l.d);
    if (rc == DD_OK) rc = set_stride(l.ld_weight, l.d);
    if (rc != DD_OK) return rc;
    if (!l.weight || (l.tokens && !l.targets)) return DD_ERR_INVALID_ARG;
    return (uintptr_t)l.targets & 7u ? DD_ERR_ALIGNMENT : DD_OK;
}

// The logits' launch, with one of its two epilogues.
template <int EPI>
static int launch_logits(dd_ctx *ctx, GemmArgs &a, uint64_t tokens, uint64_t columns, uint64_t d, cudaStream_t stream)
{
    a.nprob = 0;
    a.tiles = 0;
    GemmProblem &p = add_problem(a, tokens, columns, 256, blocks_of(d, kBK));
    p.b_map[0] = 1;
    return launch_gemm_act<EPI, 256, DD_ACT_SILU>(ctx, a, stream);
}

// The same for few tokens, by the kernel that streams the weights past them.
template <int EPI>
static int launch_few_logits(dd_ctx *ctx, const EpilogueArgs &e, const Matrix &hidden, const Matrix &weight, cudaStream_t stream)
{
    StreamArgs a = stream_args(e, weight.rows, hidden.rows);
    a.kblocks[0] = blocks_of(weight.cols, kBK);
    const int rc = encode(ctx, &a.w[0], weight);
    return rc == DD_OK ? launch_stream<EPI>(ctx, a, {hidden}, stream) : rc;
}

static EpilogueArgs loss_epilogue(const dd_vocab_loss &l, int32_t *status)
{
    EpilogueArgs e;
    std::memset(&e, 0, sizeof e);
    e.expire = l.flags != 0;
    e.status = status;
    e.targets = reinterpret_cast<const long long *>(l.targets);
    e.vocab = (long long)l.vocab;
    return e;
}

static int own_scratch(dd_ctx *ctx, void *&scratch, size_t bytes)
{
    if (scratch) return DD_OK;
    const int rc = ensure_decoder_scratch(ctx, bytes);
    scratch = ctx->decoder_scratch;
    return rc;
}

}  // namespace ddm

using namespace ddm;

extern "C" uint64_t dd_vocab_loss_scratch_bytes(dd_ctx *ctx, const dd_vocab_loss *loss, int backward)
{
    if (!loss) return 0;
    dd_vocab_loss l = *loss;
    if (check_loss(ctx, l) != DD_OK) return 0;
    return backward ? backward_bytes(l) : forward_bytes(l);
}

extern "C" int dd_vocab_loss_forward(dd_ctx *ctx, const dd_vocab_loss *l_, const void *hidden, float *loss, float *lse, void *scratch,
                                     int32_t *status, void *cuda_stream)
{
    if (!l_) return DD_ERR_INVALID_ARG;
    dd_vocab_loss l = *l_;
    int rc = check_loss(ctx, l);
    if (rc != DD_OK) return rc;
    const uint64_t T = l.tokens, bytes = forward_bytes(l);
    if (T && (!hidden || !loss || !lse)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)status & 3u || (uintptr_t)loss & 3u || (uintptr_t)lse & 3u) return DD_ERR_ALIGNMENT;
    rc = check_aligned({hidden, l.weight, scratch});
    if (rc != DD_OK) return rc;
    rc = check_alias({extent(loss, T, 1, 1, 4), extent(lse, T, 1, 1, 4), extent(scratch, 1, bytes, bytes, 1)},
                     {extent(hidden, T, l.d, l.ld_hidden), extent(l.weight, l.vocab, l.d, l.ld_weight), extent(l.targets, T, 1, 1, 8)});
    if (rc != DD_OK || T == 0) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    rc = ensure_ffn_slabs(ctx);
    if (rc == DD_OK) rc = own_scratch(ctx, scratch, bytes);
    if (rc != DD_OK) return rc;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    GemmArgs a;
    std::memset(&a, 0, sizeof a);
    a.e = loss_epilogue(l, status);
    a.e.loss = loss;
    a.e.partial = static_cast<float2 *>(scratch);
    a.e.tokens = (unsigned)T;
    const Matrix h = {hidden, T, l.d, l.ld_hidden}, w = {l.weight, l.vocab, l.d, l.ld_weight};
    if (few_tokens(ctx, l, false)) {
        rc = launch_few_logits<kEpiLoss>(ctx, a.e, h, w, stream);
    } else {
        rc = encode(ctx, &a.maps[0], h);
        if (rc == DD_OK) rc = encode(ctx, &a.maps[1], w);
        if (rc == DD_OK) rc = launch_logits<kEpiLoss>(ctx, a, T, l.vocab, l.d, stream);
    }
    if (rc != DD_OK) return rc;
    return launch_after(ctx, vocab_loss_join_kernel, blocks_of(T, 32), 32 * kJoinWarps, 0, stream, a.e.partial, blocks_of(l.vocab, 128), (unsigned)T, a.e.targets,
                        a.e.vocab, loss, lse);
}

extern "C" int dd_vocab_loss_backward(dd_ctx *ctx, const dd_vocab_loss *l_, const void *hidden, const float *lse, const float *dloss,
                                      void *dhidden, void *dweight, dd_dtype grad_dtype, int accumulate, void *scratch, int32_t *status,
                                      void *cuda_stream)
{
    if (!l_) return DD_ERR_INVALID_ARG;
    dd_vocab_loss l = *l_;
    int rc = check_loss(ctx, l);
    if (rc != DD_OK) return rc;
    const uint64_t T = l.tokens, bytes = backward_bytes(l), ldd = rows8(l.d);
    if (grad_dtype != DD_F32 && grad_dtype != DD_BF16) return DD_ERR_INVALID_ARG;
    if (!dweight || (T && (!hidden || !lse || !dloss || !dhidden))) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)status & 3u || (uintptr_t)dloss & 3u || (uintptr_t)lse & 3u) return DD_ERR_ALIGNMENT;
    rc = check_aligned({hidden, l.weight, dhidden, dweight, scratch});
    if (rc != DD_OK) return rc;
    const size_t ge = grad_dtype == DD_BF16 ? 2 : 4;
    rc = check_alias({extent(dhidden, T, l.d, l.ld_hidden), extent(dweight, l.vocab, l.d, l.ld_weight, ge), extent(scratch, 1, bytes, bytes, 1)},
                     {extent(hidden, T, l.d, l.ld_hidden), extent(l.weight, l.vocab, l.d, l.ld_weight), extent(l.targets, T, 1, 1, 8),
                      extent(lse, T, 1, 1, 4), extent(dloss, T, 1, 1, 4)});
    if (rc != DD_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (T == 0) {                          // sums over no token
        if (!accumulate) DD_CUDA(ctx, cudaMemset2DAsync(dweight, l.ld_weight * ge, 0, l.d * ge, l.vocab, stream));
        return DD_OK;
    }
    rc = ensure_ffn_slabs(ctx);
    if (rc == DD_OK) rc = own_scratch(ctx, scratch, bytes);
    if (rc != DD_OK) return rc;
    const uint64_t cols = piece_columns(l), ldg = rows8(cols);
    __nv_bfloat16 *g = static_cast<__nv_bfloat16 *>(scratch);
    float *sums = reinterpret_cast<float *>(g + T * ldg);         // dhidden over the pieces so far
    GemmArgs a;
    std::memset(&a, 0, sizeof a);
    a.e = loss_epilogue(l, status);
    a.e.lse = lse;
    a.e.dloss = dloss;
    a.e.hidden = g;
    a.e.ld_hidden = ldg;
    const unsigned kt = blocks_of(T, kBK), pairs = (unsigned)ctx->sm_count / 2;
    const bool few = few_tokens(ctx, l, true) && cols == l.vocab;
    for (uint64_t first = 0; first < l.vocab; first += cols) {
        const uint64_t n = l.vocab - first < cols ? l.vocab - first : cols;
        const bool last = first + n == l.vocab;
        const Matrix w = {static_cast<const __nv_bfloat16 *>(l.weight) + first * l.ld_weight, n, l.d, l.ld_weight};
        a.e.first = (long long)first;
        rc = encode(ctx, &a.maps[0], {hidden, T, l.d, l.ld_hidden});
        if (rc == DD_OK) rc = encode(ctx, &a.maps[1], w);
        if (rc == DD_OK) rc = encode(ctx, &a.maps[2], {g, T, n, ldg});
        if (rc == DD_OK && few) {
            rc = launch_few_logits<kEpiSoft>(ctx, a.e, {hidden, T, l.d, l.ld_hidden}, w, stream);
            // dhidden by the same kernel; dweight beside it, as in the block's backward pass
            StreamArgs c = stream_args(a.e, l.d, T);
            c.e.out = static_cast<__nv_bfloat16 *>(dhidden);
            c.e.ld_out = l.ld_hidden;
            c.kblocks[0] = blocks_of(n, kBK);
            c.w[0] = a.maps[1];
            c.w_mn = c.own_prior = c.late_trigger = a.late_wait = 1;
            if (rc == DD_OK) rc = launch_stream<kEpiStore>(ctx, c, {{g, T, n, ldg}}, stream);
        } else if (rc == DD_OK) {
            rc = launch_logits<kEpiSoft>(ctx, a, T, n, l.d, stream);
        }
        if (rc != DD_OK) return rc;
        a.nprob = 0;
        a.tiles = 0;
        Splits sp;
        sp.r.count = 0;
        const unsigned wtiles = blocks_of(n, 2 * kBM) * blocks_of(l.d, 256), xtiles = blocks_of(T, 2 * kBM) * blocks_of(l.d, 256), kn = blocks_of(n, kBK);
        if (!few) {
            GemmProblem &x = add_problem(a, T, l.d, 256, kn, 0, choose_splits(ctx, xtiles, kn, (unsigned long long)wtiles * unit_blocks(kt), kLossSplits));
            x.a_map[0] = 2;
            x.b_map[0] = 1;
            x.b_mn = 1;
            if (last) set_output(ctx, x, sp, dhidden, l.ld_hidden, false, first ? sums : nullptr, ldd, true);
            else set_output(ctx, x, sp, sums, ldd, true, first ? sums : nullptr, ldd, true);
        }
        // few weights and many tokens: the tokens are split as well, as in the block's backward pass
        unsigned splits = 1;
        while (splits < kMaxSplits && a.tiles + wtiles * (splits + 1) <= pairs && kt >= 4 * (splits + 1)) ++splits;
        if (kt - kt / splits < 16) splits = 1;
        GemmProblem &y = add_problem(a, n, l.d, 256, kt, 0, splits);
        y.a_map[0] = 2;
        y.b_map[0] = 0;
        y.a_mn = y.b_mn = 1;
        void *dw = static_cast<char *>(dweight) + first * l.ld_weight * ge;
        set_output(ctx, y, sp, dw, l.ld_weight, grad_dtype == DD_F32, accumulate ? dw : nullptr, l.ld_weight, grad_dtype == DD_F32);
        rc = launch_store(ctx, a, stream);
        if (rc == DD_OK) rc = launch_reduce(ctx, sp, stream);
        if (rc != DD_OK) return rc;
    }
    return DD_OK;
}
