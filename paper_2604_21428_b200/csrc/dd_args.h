// What the entry points of the learner's operators share: the tensor map encoder, overlap and alignment
// checks of their arguments, and launch settings.
#pragma once

#include <atomic>
#include <cstring>
#include <initializer_list>

#include <cuda.h>

#include "dd_ctx.h"
#include "dd_decoder.h"

namespace ddm {

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor map encoder, found through the runtime (the library does not link libcuda).
inline EncodeTiled tensor_map_encoder()
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

inline unsigned blocks_of(unsigned long long n, unsigned b) { return (unsigned)((n + b - 1) / b); }

// Rows of a matrix in memory, in bytes; no rows: touches nothing.  A row may be a comb: pieces of `tooth` bytes every
// `step` of them (the heads of a token, what lies between belonging to others); step 0: all of it.
struct Extent {
    const void *p;
    size_t rows, width, pitch;
    size_t tooth, step;
};

inline Extent extent(const void *p, unsigned long long rows, unsigned long long cols, unsigned long long ld, size_t elem = 2)
{
    return Extent{p, p ? (size_t)rows : 0, (size_t)cols * elem, (size_t)ld * elem, (size_t)cols * elem, 0};
}

// Whether two matrices share a byte.  Rows of one pitch may lie side by side (gate and up as halves of one
// buffer's rows), and combs of one step between each other's teeth (queries, keys and values of a head side by side); otherwise
// whatever lies between the ends is taken.
inline bool touches(const Extent &a, const Extent &b)
{
    if (!a.rows || !b.rows) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    if (y < x) return touches(b, a);
    if (y >= x + (a.rows - 1) * a.pitch + a.width) return false;
    const auto between = [&](size_t off) { return off % a.step >= a.tooth && off % a.step + b.tooth <= a.step; };
    const bool combs = a.step && a.step == b.step;
    if (combs && a.pitch % a.step == 0 && b.pitch % a.step == 0 && between(y - x)) return false;      // all teeth at one place of a step
    if (a.pitch != b.pitch) return true;
    const size_t off = (y - x) % a.pitch;
    if (off + b.width > a.pitch) return true;
    return off < a.width && !(combs && between(off));
}

// Fills in a tensor's default strides.  Its rows of `dim` elements must not overlap, with the tokens' rows
// (all heads of one) following one another or the heads' (all tokens of one).
inline int check_heads(dd_heads &x, uint64_t tokens, uint64_t heads, uint64_t dim)
{
    if (tokens && !x.data) return DD_ERR_INVALID_ARG;
    if (!x.ld_head) x.ld_head = dim;
    if (!x.ld_token) x.ld_token = heads * dim;
    if (x.ld_head >= (1ull << 38) || x.ld_token >= (1ull << 38)) return DD_ERR_TOO_LARGE;
    const auto follow = [dim](uint64_t outer, uint64_t n_outer, uint64_t inner, uint64_t n_inner) {
        if (n_inner > 1 && inner < dim) return false;
        return n_outer <= 1 || outer >= (unsigned __int128)(n_inner - 1) * inner + dim;
    };
    if (!tokens || follow(x.ld_token, tokens, x.ld_head, heads) || follow(x.ld_head, heads, x.ld_token, tokens)) return DD_OK;
    return DD_ERR_INVALID_ARG;
}

inline Extent heads_extent(const dd_heads &x, uint64_t tokens, uint64_t heads, uint64_t dim, size_t elem = 2)
{
    if (!tokens) return Extent{};
    if (tokens == 1) return extent(x.data, heads, dim, x.ld_head, elem);
    if (heads == 1) return extent(x.data, tokens, dim, x.ld_token, elem);
    const bool heads_inside = x.ld_token >= x.ld_head;
    const uint64_t inner = heads_inside ? x.ld_head : x.ld_token, outer = heads_inside ? x.ld_token : x.ld_head, n = heads_inside ? heads : tokens;
    Extent e = extent(x.data, heads_inside ? tokens : heads, (n - 1) * inner + dim, outer, elem);
    e.tooth = dim * elem;
    e.step = inner * elem;
    return e;
}

inline int check_aligned(std::initializer_list<const void *> ptrs)
{
    for (const void *p : ptrs)
        if ((uintptr_t)p & 15u) return DD_ERR_ALIGNMENT;
    return DD_OK;
}

// Outputs first: none may touch another output or an input.
inline int check_alias(std::initializer_list<Extent> outs, std::initializer_list<Extent> ins)
{
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        for (auto q = outs.begin(); q != o; ++q)
            if (touches(*o, *q)) return DD_ERR_ALIAS;
        for (const Extent &i : ins)
            if (touches(*o, i)) return DD_ERR_ALIAS;
    }
    return DD_OK;
}

// Kernels opt in to their shared memory once per process and device; contexts of several host threads may
// come by at the same time (opting in twice does no harm).
template <typename K>
inline int allow_smem(dd_ctx *ctx, K kernel, size_t bytes, std::atomic<bool> (&done)[64])
{
    const int d = ctx->device;
    if (d < 64 && done[d]) return DD_OK;
    DD_CUDA(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (d < 64) done[d] = true;
    return DD_OK;
}

// Context-owned scratch of the decoder's operators, for callers that bring none.
inline int ensure_decoder_scratch(dd_ctx *ctx, size_t bytes)
{
    if (bytes <= ctx->decoder_scratch_cap) return DD_OK;
    DD_CUDA(ctx, cudaDeviceSynchronize());
    if (ctx->decoder_scratch) cudaFree(ctx->decoder_scratch);
    ctx->decoder_scratch = nullptr;
    ctx->decoder_scratch_cap = 0;
    DD_CUDA(ctx, cudaMalloc(&ctx->decoder_scratch, bytes));
    ctx->decoder_scratch_cap = bytes;
    return DD_OK;
}

// Launches that may begin while the one before them on the stream ends; the kernels wait for it themselves.
template <typename K, typename... A>
inline int launch_clusters(dd_ctx *ctx, K kernel, unsigned long long grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t stream,
                           const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {cluster, 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, args...));
    return DD_OK;
}

template <typename K, typename... A>
inline int launch_after(dd_ctx *ctx, K kernel, unsigned long long grid, unsigned threads, size_t smem, cudaStream_t stream, const A &...args)
{
    return launch_clusters(ctx, kernel, grid, threads, smem, 1, stream, args...);
}

}  // namespace ddm
