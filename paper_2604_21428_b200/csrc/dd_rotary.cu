// dd_rotary_apply: rotary positions of queries and keys in one launch.
//
// Bound by memory: every element is read and written once, and a block forms the angles of its few tokens
// once for all heads (float64 product and reduction to a part of a turn, float32 sine and cosine of that).
// 16384 tokens, 20 heads of 128, bf16: 31 us, 5.4 TB/s.  Loads issued before the angles took 45 us (fewer blocks
// an SM), blocks of 2048 to 8192 units 34-55.
#include <cmath>

#include "dd_args.h"
#include "dd_decoder.h"
#include "dd_tcgen05.cuh"

namespace ddm {

constexpr int kRotaryThreads = 256;
constexpr unsigned kRotaryUnits = 1024, kRotaryMaxUnits = 8192, kRotaryMaxAngles = 4096;

struct RotaryTensor {
    const char *in;
    char *out;
    unsigned long long in_token, in_head, out_token, out_head;      // bytes
    unsigned heads;
};

struct RotaryArgs {
    RotaryTensor x[2];
    const void *positions;
    const double *frequencies;
    unsigned long long tokens;
    unsigned block_tokens, block_heads;         // of both tensors together
    unsigned half, pairs, units;                // pairs of a head; its units of work that turn, and all of them
    unsigned by_units, by_heads;                // 2^32 / units and 2^32 / block_heads, rounded up
    float magnitude;
    int positions_64, inverse;
};

template <typename T, int N, int ALIGN>
struct alignas(ALIGN) Pack {
    T v[N];
};

// n / d for the m = ceil(2^32 / d) of a d: exact as long as n d < 2^32 (here n, d <= 2^13).
__device__ __forceinline__ unsigned quotient(unsigned n, unsigned m) { return m ? __umulhi(n, m) : n; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float &to, float x) { to = x; }
__device__ __forceinline__ void put(__nv_bfloat16 &to, float x) { to = __float2bfloat16_rn(x); }

// A unit is one piece of N neighbouring elements and, where pairs are split over the halves of the head, its
// partner piece (INTER: N / 2 pairs within the piece).  Units behind the last pair are copied, C elements each.
template <typename T, int N, int C, bool INTER>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a)
{
    typedef Pack<T, N, C * sizeof(T)> Piece;
    typedef Pack<T, C, C * sizeof(T)> Rest;
    extern __shared__ float2 turn[];            // [block_tokens][half]: magnitude x (cos, sin)
    __shared__ int live[kRotaryThreads];        // block_tokens is at most this
    const unsigned long long t0 = (unsigned long long)blockIdx.x * a.block_tokens;
    const unsigned nt = a.tokens - t0 < a.block_tokens ? (unsigned)(a.tokens - t0) : a.block_tokens;
    const unsigned h0 = blockIdx.y * a.block_heads, all = a.x[0].heads + a.x[1].heads;
    const unsigned nh = all - h0 < a.block_heads ? all - h0 : a.block_heads;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (unsigned i = threadIdx.x; i < nt * a.half; i += kRotaryThreads) {
        const unsigned t = i / a.half, j = i - t * a.half;
        const long long pos = a.positions_64 ? static_cast<const long long *>(a.positions)[t0 + t]
                                             : static_cast<const int *>(a.positions)[t0 + t];
        const double w = (double)pos * (a.frequencies[j] * 0.15915494309189533577);      // turns: 1 / (2 pi)
        const float part = (float)(w - rint(w));
        float s, c;
        sincospif(2.0f * part, &s, &c);
        turn[i] = make_float2(a.magnitude * c, a.magnitude * (a.inverse ? -s : s));
        if (j == 0) live[t] = pos >= 0;
    }
    __syncthreads();
    for (unsigned i = threadIdx.x; i < nt * a.block_heads * a.units; i += kRotaryThreads) {
        const unsigned row = quotient(i, a.by_units), u = i - row * a.units;
        const unsigned t = quotient(row, a.by_heads), hb = row - t * a.block_heads;
        if (hb >= nh || !live[t]) continue;
        unsigned h = h0 + hb;
        const bool second = h >= a.x[0].heads;
        const RotaryTensor &x = a.x[second];
        if (second) h -= a.x[0].heads;
        const T *in = reinterpret_cast<const T *>(x.in + (t0 + t) * x.in_token + h * x.in_head);
        T *out = reinterpret_cast<T *>(x.out + (t0 + t) * x.out_token + h * x.out_head);
        if (u >= a.pairs) {
            if (in == out) continue;
            const unsigned at = 2 * a.half + (u - a.pairs) * C;
            *reinterpret_cast<Rest *>(out + at) = *reinterpret_cast<const Rest *>(in + at);
        } else if (INTER) {
            Piece p = *reinterpret_cast<const Piece *>(in + u * N);
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                const float2 w = turn[t * a.half + u * (N / 2) + k];
                const float x0 = to_float(p.v[2 * k]), x1 = to_float(p.v[2 * k + 1]);
                put(p.v[2 * k], x0 * w.x - x1 * w.y);
                put(p.v[2 * k + 1], x1 * w.x + x0 * w.y);
            }
            *reinterpret_cast<Piece *>(out + u * N) = p;
        } else {
            Piece p = *reinterpret_cast<const Piece *>(in + u * N), q = *reinterpret_cast<const Piece *>(in + a.half + u * N);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float2 w = turn[t * a.half + u * N + k];
                const float x0 = to_float(p.v[k]), x1 = to_float(q.v[k]);
                put(p.v[k], x0 * w.x - x1 * w.y);
                put(q.v[k], x1 * w.x + x0 * w.y);
            }
            *reinterpret_cast<Piece *>(out + u * N) = p;
            *reinterpret_cast<Piece *>(out + a.half + u * N) = q;
        }
    }
}

template <typename T, int N, int C, bool INTER>
static int launch_rotary(dd_ctx *ctx, RotaryArgs &a, unsigned dim, cudaStream_t stream)
{
    a.pairs = INTER ? 2 * a.half / N : a.half / N;
    a.units = a.pairs + (dim - 2 * a.half) / C;
    const unsigned all = a.x[0].heads + a.x[1].heads, most = kRotaryMaxUnits / a.units;      // units <= 1024
    a.block_heads = all < most ? all : most;
    const unsigned row = a.block_heads * a.units;
    unsigned nt = row < kRotaryUnits ? kRotaryUnits / row : 1;
    const auto limit = [&](unsigned long long n) { if (nt > n) nt = n < 1 ? 1 : (unsigned)n; };
    limit(kRotaryThreads);
    limit(kRotaryMaxAngles / a.half);
    limit(a.tokens / (2 * ctx->sm_count));                  // few tokens: spread over the GPU
    a.block_tokens = nt;
    const auto inverse_of = [](unsigned d) { return d == 1 ? 0u : (unsigned)(((1ull << 32) + d - 1) / d); };
    a.by_units = inverse_of(a.units);
    a.by_heads = inverse_of(a.block_heads);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.tokens + nt - 1) / nt), blocks_of(all, a.block_heads));
    cfg.blockDim = dim3(kRotaryThreads);
    cfg.dynamicSmemBytes = (size_t)nt * a.half * sizeof(float2);
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, rotary_kernel<T, N, C, INTER>, a));
    return DD_OK;
}

template <typename T>
static int launch_rotary_type(dd_ctx *ctx, RotaryArgs &a, unsigned dim, bool inter, bool wide, cudaStream_t stream)
{
    constexpr int N = 16 / (int)sizeof(T);
    if (inter) return wide ? launch_rotary<T, N, N, true>(ctx, a, dim, stream) : launch_rotary<T, 2, 1, true>(ctx, a, dim, stream);
    return wide ? launch_rotary<T, N, N, false>(ctx, a, dim, stream) : launch_rotary<T, 1, 1, false>(ctx, a, dim, stream);
}

}  // namespace ddm

using namespace ddm;

extern "C" int dd_rotary_apply(dd_ctx *ctx, const dd_rotary *r, const dd_heads *q, const dd_heads *k, const dd_heads *q_out,
                               const dd_heads *k_out, const void *positions, const double *frequencies, void *cuda_stream)
{
    if (!ctx || !r || !q || !k || !q_out || !k_out) return DD_ERR_INVALID_ARG;
    if (r->dtype != DD_F32 && r->dtype != DD_BF16) return DD_ERR_INVALID_ARG;
    if (r->heads < 1 || r->dim < 1 || r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > r->dim) return DD_ERR_INVALID_ARG;
    if (r->tokens >= (1ull << 24) || r->heads >= (1ull << 16) || r->kv_heads >= (1ull << 16) || r->dim > 1024) return DD_ERR_TOO_LARGE;
    if (!std::isfinite(r->magnitude)) return DD_ERR_INVALID_ARG;
    if (r->tokens > 0 && (!positions || !frequencies)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)positions & (r->positions_64 ? 7u : 3u) || (uintptr_t)frequencies & 7u) return DD_ERR_ALIGNMENT;
    const size_t size = r->dtype == DD_BF16 ? 2 : 4;
    RotaryArgs a;
    std::memset(&a, 0, sizeof a);
    bool wide = r->dim * size % 16 == 0 && (r->interleaved ? r->rotary_dim : r->rotary_dim / 2) * size % 16 == 0 && r->rotary_dim * size % 16 == 0;
    Extent in[2] = {}, out[2] = {};
    bool same[2] = {false, false};
    for (int i = 0; i < 2; ++i) {
        const uint64_t heads = i ? r->kv_heads : r->heads;
        dd_heads x = i ? *k : *q, y = i ? *k_out : *q_out;
        if (heads == 0) continue;
        int rc = check_heads(x, r->tokens, heads, r->dim);
        if (rc == DD_OK) rc = check_heads(y, r->tokens, heads, r->dim);
        if (rc != DD_OK) return rc;
        if ((uintptr_t)x.data % size || (uintptr_t)y.data % size) return DD_ERR_ALIGNMENT;
        for (const dd_heads *z : {&x, &y})
            wide = wide && (uintptr_t)z->data % 16 == 0 && z->ld_token * size % 16 == 0 && z->ld_head * size % 16 == 0;
        same[i] = x.data == y.data;
        if (same[i] && r->tokens > 0 && ((r->tokens > 1 && x.ld_token != y.ld_token) || (heads > 1 && x.ld_head != y.ld_head))) return DD_ERR_ALIAS;
        in[i] = heads_extent(x, r->tokens, heads, r->dim, size);
        out[i] = heads_extent(y, r->tokens, heads, r->dim, size);
        a.x[i] = {static_cast<const char *>(x.data), static_cast<char *>(y.data), x.ld_token * size, x.ld_head * size,
                  y.ld_token * size, y.ld_head * size, (unsigned)heads};
    }
    const Extent at = extent(positions, r->tokens, 1, 1, r->positions_64 ? 8 : 4), fr = extent(frequencies, 1, r->rotary_dim / 2, r->rotary_dim / 2, 8);
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j) {
            if (!(i == j && same[i]) && touches(out[i], in[j])) return DD_ERR_ALIAS;
            if (i < j && touches(out[i], out[j])) return DD_ERR_ALIAS;
        }
    for (int i = 0; i < 2; ++i)
        if (touches(out[i], at) || touches(out[i], fr)) return DD_ERR_ALIAS;
    if (r->tokens == 0) return DD_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    a.positions = positions;
    a.frequencies = frequencies;
    a.tokens = r->tokens;
    a.half = (unsigned)r->rotary_dim / 2;
    a.magnitude = r->magnitude;
    a.positions_64 = r->positions_64 != 0;
    a.inverse = r->inverse != 0;
    const bool inter = r->interleaved != 0;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    return r->dtype == DD_BF16 ? launch_rotary_type<__nv_bfloat16>(ctx, a, (unsigned)r->dim, inter, wide, stream)
                               : launch_rotary_type<float>(ctx, a, (unsigned)r->dim, inter, wide, stream);
}
