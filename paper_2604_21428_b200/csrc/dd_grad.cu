// The learner's optimizer side: global gradient norm, clipping and the AdamW step over lists of
// tensors.  Every kernel walks one flat tile index over the whole list (persistent grid, tiles of
// 8192 elements handed out round-robin), so many small tensors cost no launches of their own.
#include <cmath>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "dd_ctx.h"
#include "dd_learner.h"

namespace ddm {

constexpr int kListThreads = 256;
constexpr int kListTile = 8192;              // elements: 32 per thread
constexpr int kListSmall = 32, kListMax = 256;
// CTAs of 256 threads launched per SM; registers let 6 / 5 / 5 of them run at a time (norm, scale, AdamW), the
// rest follow as those end.  Measured at 4 / 6 / 8: norm of 1.2e9 bf16 453 / 365 / 407 us, clip of 151M bf16
// 156 / 158 / 152 us, norm and AdamW on 151M fp32 876 / 912 / 828 us (one number for the three).
constexpr int kListCtasPerSm = 8;
constexpr unsigned char kNoVector = 255;
constexpr unsigned kKeepBytes = 64u << 20;   // of a list that is read twice, kept in L2 (126 MB) from the first time

// One launch's tensors, by value in the kernel parameters: no staging copy, and nothing for a
// stream capture to keep alive.  CAP = 32 keeps the parameters of short lists under 2 KB.
template <int NPTR, int CAP>
struct ListArgs {
    void *ptr[NPTR][CAP];
    unsigned long long n[CAP];
    unsigned tile_end[CAP];                  // one past the tensor's last flat tile
    unsigned char bf16[CAP];                 // type of the gradient
    unsigned char head[CAP];                 // elements before the first 16-byte boundary; kNoVector: pointers disagree
    unsigned tiles;
    int count;
};

struct NormTail {
    double *partials;                        // one per CTA of every launch of the call
    unsigned first, total;                   // this launch's offset; partials of the whole call
    unsigned *ticket;
    dd_grad_record *record;
    float max_norm;
    int last;                                // the call's last launch reduces
    unsigned keep_from;                      // AGAIN: first tile to keep in L2
};

struct AdamwConsts {
    float beta1, rest1, beta2, rest2, eps, decay, step_size, inv_c2;
    const dd_grad_record *clip;
};

__device__ __forceinline__ float lo_bf16(unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float load_elem(const void *p, bool bf16, unsigned long long e)
{
    return bf16 ? __uint_as_float((unsigned)static_cast<const unsigned short *>(p)[e] << 16)
                : static_cast<const float *>(p)[e];
}
__device__ __forceinline__ unsigned short round_bf16(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi)
{
    return (unsigned)round_bf16(lo) | ((unsigned)round_bf16(hi) << 16);
}

__device__ __forceinline__ double block_sum(double x, double *sm)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = x;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < kListThreads / 32; ++w) t += sm[w];
    __syncthreads();
    return t;
}

// The tensor that holds flat tile `tile`, between the candidates lo and hi (a scan of the table,
// some 40 cycles a step, took longer than the tiles themselves in lists of 200 tensors).
template <typename A>
__device__ __forceinline__ int find_tensor(const A &a, unsigned tile, int lo, int hi)
{
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (tile < a.tile_end[mid]) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Programmatic launch: the next launch on the stream may be set up under this one, and waits here
// before it touches memory.
__device__ __forceinline__ void after_prior_launch()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A tile's span within its tensor: vector pieces from `begin` (a boundary of all the tensor's
// pointers) to `end`; the tensor's first tile also has the `head` elements before.
struct Span {
    unsigned long long begin, end;
    unsigned head;
    bool vec;
};

template <typename A>
__device__ __forceinline__ Span span_of(const A &a, unsigned tile, int i)
{
    const unsigned first = i ? a.tile_end[i - 1] : 0u;
    const unsigned char h = a.head[i];
    Span s;
    s.vec = h != kNoVector;
    const unsigned head = s.vec ? h : 0u;
    s.begin = head + (unsigned long long)(tile - first) * kListTile;
    s.end = s.begin + kListTile < a.n[i] ? s.begin + kListTile : a.n[i];
    s.head = tile == first ? head : 0u;
    return s;
}

__device__ __forceinline__ float squares(const uint4 &w)
{
    const unsigned x[4] = {w.x, w.y, w.z, w.w};
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s = fmaf(lo_bf16(x[j]), lo_bf16(x[j]), s);
        s = fmaf(hi_bf16(x[j]), hi_bf16(x[j]), s);
    }
    return s;
}

__device__ __forceinline__ float squares(const float4 &w) { return fmaf(w.x, w.x, fmaf(w.y, w.y, fmaf(w.z, w.z, w.w * w.w))); }

__device__ __forceinline__ uint4 load_policy(const uint4 *p, unsigned long long policy)
{
    uint4 w;
    asm volatile("ld.global.L2::cache_hint.v4.b32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(p), "l"(policy) : "memory");
    return w;
}

__device__ __forceinline__ float4 load_policy(const float4 *p, unsigned long long policy)
{
    float4 w;
    asm volatile("ld.global.L2::cache_hint.v4.f32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=f"(w.x), "=f"(w.y), "=f"(w.z), "=f"(w.w) : "l"(p), "l"(policy) : "memory");
    return w;
}

// Sum of squares of this thread's part of a tile: V holds E elements.
template <typename V, int E, bool AGAIN>
__device__ __forceinline__ float tile_squares(const V *p, unsigned pieces, unsigned long long policy)
{
    constexpr int kSteps = kListTile / (E * kListThreads);
    float s = 0.0f;
    V w[kSteps];
    if (pieces == kSteps * kListThreads) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
            w[k] = AGAIN ? load_policy(p + threadIdx.x + k * kListThreads, policy) : p[threadIdx.x + k * kListThreads];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) s += squares(w[k]);
    } else {
        for (unsigned k = threadIdx.x; k < pieces; k += kListThreads) s += squares(p[k]);
    }
    return s;
}

// sum of g^2: fp32 over the 32 elements a thread takes of a tile (and up to 2 more at a tensor's ends),
// fp64 across tiles, threads and CTAs.  The CTA that draws the last ticket adds the partials in
// index order, so the result does not depend on which one that is.
// AGAIN: the clip reads everything once more, from the end.  The last 64 MB then keep L2's ordinary
// priority and the rest is marked to go first: 156 -> 152 us for 151M bf16 (without the marks, reading from
// the end gains nothing).  Marking the 64 MB to go last takes 150 but outlives the call: reading
// 88 MB four times took 110 us after such a clip, 88 after this one, 84 after a norm alone.
template <int CAP, bool AGAIN>
__global__ void __launch_bounds__(kListThreads)
grad_norm_kernel(const __grid_constant__ ListArgs<1, CAP> a, const __grid_constant__ NormTail t)
{
    __shared__ double sm[kListThreads / 32];
    __shared__ unsigned drawn;
    double acc = 0.0;
    int i = 0;
    unsigned long long keep = 0, drop = 0;
    if (AGAIN) {
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(keep));
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(drop));
    }
    after_prior_launch();
    for (unsigned tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        i = find_tensor(a, tile, i, a.count - 1);
        const Span sp = span_of(a, tile, i);
        const void *g = a.ptr[0][i];
        const bool bf16 = a.bf16[i];
        const unsigned cnt = (unsigned)(sp.end - sp.begin), per = bf16 ? 8 : 4, pieces = sp.vec ? cnt / per : 0;
        const unsigned long long policy = tile >= t.keep_from ? keep : drop;
        float s = 0.0f;
        if (bf16) s = tile_squares<uint4, 8, AGAIN>(reinterpret_cast<const uint4 *>(static_cast<const unsigned short *>(g) + sp.begin), pieces, policy);
        else s = tile_squares<float4, 4, AGAIN>(reinterpret_cast<const float4 *>(static_cast<const float *>(g) + sp.begin), pieces, policy);
        for (unsigned e = pieces * per + threadIdx.x; e < cnt; e += kListThreads) {
            const float x = load_elem(g, bf16, sp.begin + e);
            s = fmaf(x, x, s);
        }
        if (threadIdx.x < sp.head) {
            const float x = load_elem(g, bf16, threadIdx.x);
            s = fmaf(x, x, s);
        }
        acc += (double)s;
    }
    const double part = block_sum(acc, sm);
    if (threadIdx.x == 0) {
        t.partials[t.first + blockIdx.x] = part;
        __threadfence();
        drawn = t.last ? atomicAdd(t.ticket, 1u) : 0xffffffffu;
    }
    __syncthreads();
    if (drawn != gridDim.x - 1) return;
    __threadfence();
    double x = 0.0;
    for (unsigned k = threadIdx.x; k < t.total; k += kListThreads) x += __ldcg(t.partials + k);
    x = block_sum(x, sm);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(x);
        const bool ok = isfinite(norm);
        t.record->norm_sq = x;
        t.record->norm = norm;
        t.record->scale = ok ? fminf(1.0f, t.max_norm / (norm + 1e-6f)) : 1.0f;
        t.record->status = ok ? DD_STATUS_OK : DD_STATUS_NONFINITE;
        t.record->reserved = 0;
        *t.ticket = 0;
    }
}

__device__ __forceinline__ uint4 scaled(const uint4 &w, float c)
{
    return make_uint4(pack_bf16(c * lo_bf16(w.x), c * hi_bf16(w.x)), pack_bf16(c * lo_bf16(w.y), c * hi_bf16(w.y)),
                      pack_bf16(c * lo_bf16(w.z), c * hi_bf16(w.z)), pack_bf16(c * lo_bf16(w.w), c * hi_bf16(w.w)));
}

__device__ __forceinline__ float4 scaled(const float4 &w, float c) { return make_float4(c * w.x, c * w.y, c * w.z, c * w.w); }

template <typename V, int E>
__device__ __forceinline__ void tile_scale(const V *p, V *q, unsigned pieces, float c)
{
    constexpr int kSteps = kListTile / (E * kListThreads);
    V w[kSteps];
    if (pieces == kSteps * kListThreads) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) w[k] = p[threadIdx.x + k * kListThreads];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) q[threadIdx.x + k * kListThreads] = scaled(w[k], c);
    } else {
        for (unsigned k = threadIdx.x; k < pieces; k += kListThreads) q[k] = scaled(p[k], c);
    }
}

// out = scale * g, last tiles first: those the norm kept in L2.
template <int CAP>
__global__ void __launch_bounds__(kListThreads)
grad_scale_kernel(const __grid_constant__ ListArgs<2, CAP> a, const dd_grad_record *record, int in_place)
{
    after_prior_launch();
    const float scale = record->scale;
    if (record->status != DD_STATUS_OK || (in_place && scale == 1.0f)) return;
    int i = a.count - 1;
    for (unsigned step = blockIdx.x; step < a.tiles; step += gridDim.x) {
        const unsigned tile = a.tiles - 1 - step;
        i = find_tensor(a, tile, 0, i);
        const Span sp = span_of(a, tile, i);
        const void *g = a.ptr[0][i];
        void *o = a.ptr[1][i];
        const bool bf16 = a.bf16[i];
        const unsigned cnt = (unsigned)(sp.end - sp.begin), per = bf16 ? 8 : 4, pieces = sp.vec ? cnt / per : 0;
        if (bf16) tile_scale<uint4, 8>(reinterpret_cast<const uint4 *>(static_cast<const unsigned short *>(g) + sp.begin),
                                       reinterpret_cast<uint4 *>(static_cast<unsigned short *>(o) + sp.begin), pieces, scale);
        else tile_scale<float4, 4>(reinterpret_cast<const float4 *>(static_cast<const float *>(g) + sp.begin),
                                   reinterpret_cast<float4 *>(static_cast<float *>(o) + sp.begin), pieces, scale);
        const auto one = [&](unsigned long long e) {
            const float x = scale * load_elem(g, bf16, e);
            if (bf16) static_cast<unsigned short *>(o)[e] = round_bf16(x);
            else static_cast<float *>(o)[e] = x;
        };
        for (unsigned e = pieces * per + threadIdx.x; e < cnt; e += kListThreads) one(sp.begin + e);
        if (threadIdx.x < sp.head) one(threadIdx.x);
    }
}

__device__ __forceinline__ void adamw_elem(float &p, float &m, float &v, float g, const AdamwConsts &c)
{
    m = fmaf(c.beta1, m, c.rest1 * g);
    v = fmaf(c.beta2, v, c.rest2 * g * g);
    p = fmaf(p, c.decay, -c.step_size * (m / (sqrtf(v * c.inv_c2) + c.eps)));
}

// ptr: 0 p, 1 m, 2 v, 3 gradient, 4 bf16 copy (may be null).
template <int CAP>
__global__ void __launch_bounds__(kListThreads)
adamw_kernel(const __grid_constant__ ListArgs<5, CAP> a, const __grid_constant__ AdamwConsts c)
{
    after_prior_launch();
    float scale = 1.0f;
    if (c.clip) {
        if (c.clip->status != DD_STATUS_OK) return;
        scale = c.clip->scale;
    }
    const auto grad4 = [&](const void *g, bool bf16, unsigned long long e) {
        if (!bf16) return *reinterpret_cast<const float4 *>(static_cast<const float *>(g) + e);
        const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const unsigned short *>(g) + e);
        return make_float4(lo_bf16(w.x), hi_bf16(w.x), lo_bf16(w.y), hi_bf16(w.y));
    };
    int i = a.count - 1;
    for (unsigned step = blockIdx.x; step < a.tiles; step += gridDim.x) {
        const unsigned tile = a.tiles - 1 - step;
        i = find_tensor(a, tile, 0, i);
        const Span sp = span_of(a, tile, i);
        float *p = static_cast<float *>(a.ptr[0][i]), *m = static_cast<float *>(a.ptr[1][i]), *v = static_cast<float *>(a.ptr[2][i]);
        const void *g = a.ptr[3][i];
        unsigned short *o = static_cast<unsigned short *>(a.ptr[4][i]);
        const bool bf16 = a.bf16[i];
        const unsigned cnt = (unsigned)(sp.end - sp.begin), vec = sp.vec ? cnt & ~3u : 0u;
#pragma unroll 2
        for (unsigned k = 4 * threadIdx.x; k < vec; k += 4 * kListThreads) {
            const unsigned long long e = sp.begin + k;
            float4 P = *reinterpret_cast<const float4 *>(p + e), M = *reinterpret_cast<const float4 *>(m + e),
                   V = *reinterpret_cast<const float4 *>(v + e);
            const float4 G = grad4(g, bf16, e);
            adamw_elem(P.x, M.x, V.x, scale * G.x, c);
            adamw_elem(P.y, M.y, V.y, scale * G.y, c);
            adamw_elem(P.z, M.z, V.z, scale * G.z, c);
            adamw_elem(P.w, M.w, V.w, scale * G.w, c);
            *reinterpret_cast<float4 *>(p + e) = P;
            *reinterpret_cast<float4 *>(m + e) = M;
            *reinterpret_cast<float4 *>(v + e) = V;
            if (o) *reinterpret_cast<uint2 *>(o + e) = make_uint2(pack_bf16(P.x, P.y), pack_bf16(P.z, P.w));
        }
        const auto one = [&](unsigned long long e) {
            float P = p[e], M = m[e], V = v[e];
            adamw_elem(P, M, V, scale * load_elem(g, bf16, e), c);
            p[e] = P;
            m[e] = M;
            v[e] = V;
            if (o) o[e] = round_bf16(P);
        };
        for (unsigned k = vec + threadIdx.x; k < cnt; k += kListThreads) one(sp.begin + k);
        if (threadIdx.x < sp.head) one(threadIdx.x);
    }
}

// ---- host side ----------------------------------------------------------------------------

static bool ranges_overlap(const void *a, size_t abytes, const void *b, size_t bbytes)
{
    if (!a || !b || !abytes || !bbytes) return false;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + bbytes && y < x + abytes;
}

static int check_list(const dd_ctx *ctx, const uint64_t *sizes, const uint8_t *dtypes, int count)
{
    if (!ctx || count < 0 || (count > 0 && (!sizes || !dtypes))) return DD_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        if (dtypes[i] != DD_F32 && dtypes[i] != DD_BF16) return DD_ERR_INVALID_ARG;
        if (sizes[i] > kMaxFragmentElems) return DD_ERR_TOO_LARGE;
    }
    return DD_OK;
}

static int check_grads(const void *const *grads, const uint64_t *sizes, const uint8_t *dtypes, int count)
{
    if (count > 0 && !grads) return DD_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        if (!grads[i]) return DD_ERR_INVALID_ARG;
        if ((uintptr_t)grads[i] & (dtypes[i] == DD_BF16 ? 1u : 3u)) return DD_ERR_ALIGNMENT;
    }
    return DD_OK;
}

// Fills one launch's arguments with tensors [at, ...) and returns the index of the first tensor
// left over.  Tensors without elements take no tile and are left out.
template <int NPTR, int CAP, typename F>
static int fill_list(ListArgs<NPTR, CAP> &a, const uint64_t *sizes, const uint8_t *dtypes, int count, int at, F pointers)
{
    int k = 0;
    a.tiles = 0;
    for (; at < count && k < CAP; ++at) {
        if (sizes[at] == 0) continue;
        void *p[NPTR];
        const unsigned head = pointers(at, p);
        for (int j = 0; j < NPTR; ++j) a.ptr[j][k] = p[j];
        a.n[k] = sizes[at];
        a.bf16[k] = dtypes[at] == DD_BF16;
        a.head[k] = (unsigned char)(head != kNoVector && head > sizes[at] ? sizes[at] : head);
        const uint64_t body = sizes[at] - (head == kNoVector ? 0 : a.head[k]);
        a.tiles += body ? (unsigned)((body + kListTile - 1) / kListTile) : 1;
        a.tile_end[k++] = a.tiles;
    }
    a.count = k;
    return at;
}

// Elements from p to the next boundary of `elems` elements of `size` bytes.
static unsigned head_of(const void *p, unsigned size, unsigned elems)
{
    return (unsigned)((elems - (uintptr_t)p / size % elems) % elems);
}

static unsigned list_grid(const dd_ctx *ctx, unsigned tiles)
{
    const unsigned most = (unsigned)(ctx->sm_count * kListCtasPerSm);
    return tiles < 1 ? 1 : tiles < most ? tiles : most;
}

template <typename... P, typename... Q>
static int launch_list(dd_ctx *ctx, void (*kernel)(P...), unsigned grid, cudaStream_t stream, const Q &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kListThreads);
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    DD_CUDA(ctx, cudaLaunchKernelEx(&cfg, kernel, args...));
    return DD_OK;
}

// again: the tensors are read once more by a launch that starts from their end.
template <int CAP>
static int launch_norm(dd_ctx *ctx, const void *const *grads, const uint64_t *sizes, const uint8_t *dtypes,
                       int count, float max_norm, dd_grad_record *record, bool again, cudaStream_t stream)
{
    const size_t launches = count > CAP ? (size_t)(count + CAP - 1) / CAP : 1;
    int rc = ensure_workspace(ctx, 1, 1, launches);
    if (rc != DD_OK) return rc;
    // The launches of a list share the first workspace, so that no list makes it grow: from 34 launches
    // (8,449 tensors) on their grids shrink.
    const size_t share = first_workspace(ctx) / launches;
    const unsigned most = share < 1 ? 1 : share < 65536 ? (unsigned)share : 65536u;
    NormTail t;
    t.partials = ctx->partials;
    t.ticket = ctx->tickets;
    t.record = record;
    t.max_norm = max_norm;
    t.first = 0;
    t.keep_from = 0;
    int at = 0;
    do {
        ListArgs<1, CAP> a;
        at = fill_list(a, sizes, dtypes, count, at, [&](int i, void **p) {
            p[0] = const_cast<void *>(grads[i]);
            const unsigned eb = dtypes[i] == DD_BF16 ? 2 : 4;
            return head_of(p[0], eb, 16 / eb);
        });
        const unsigned wanted = list_grid(ctx, a.tiles), grid = wanted < most ? wanted : most;
        t.last = at >= count;
        t.total = t.first + grid;
        if (again) {
            unsigned long long bytes = 0;                  // from the end of this launch's tensors
            t.keep_from = a.tiles;
            for (int k = a.count - 1; k >= 0 && bytes < kKeepBytes && t.last; --k) {
                const unsigned tile_bytes = kListTile * (a.bf16[k] ? 2 : 4), first = k ? a.tile_end[k - 1] : 0u;
                const unsigned long long room = (kKeepBytes - bytes + tile_bytes - 1) / tile_bytes, n = a.tile_end[k] - first;
                t.keep_from -= (unsigned)(n < room ? n : room);
                bytes += n * tile_bytes;
            }
        }
        rc = again ? launch_list(ctx, grad_norm_kernel<CAP, true>, grid, stream, a, t)
                   : launch_list(ctx, grad_norm_kernel<CAP, false>, grid, stream, a, t);
        if (rc != DD_OK) return rc;
        t.first += grid;
    } while (at < count);
    return DD_OK;
}

template <int CAP>
static int launch_scale(dd_ctx *ctx, void *const *grads, void *const *outs, const uint64_t *sizes,
                        const uint8_t *dtypes, int count, const dd_grad_record *record, cudaStream_t stream)
{
    for (int at = 0; at < count;) {
        ListArgs<2, CAP> a;
        at = fill_list(a, sizes, dtypes, count, at, [&](int i, void **p) {
            p[0] = grads[i];
            p[1] = outs ? outs[i] : grads[i];
            const unsigned eb = dtypes[i] == DD_BF16 ? 2 : 4, h = head_of(p[0], eb, 16 / eb);
            return h == head_of(p[1], eb, 16 / eb) ? h : (unsigned)kNoVector;
        });
        if (!a.tiles) continue;
        const int rc = launch_list(ctx, grad_scale_kernel<CAP>, list_grid(ctx, a.tiles), stream, a, record,
                                   (int)(outs == nullptr));
        if (rc != DD_OK) return rc;
    }
    return DD_OK;
}

template <int CAP>
static int launch_adamw(dd_ctx *ctx, const AdamwConsts &c, float *const *params, const void *const *grads,
                        float *const *m, float *const *v, void *const *copies, const uint64_t *sizes,
                        const uint8_t *dtypes, int count, cudaStream_t stream)
{
    for (int at = 0; at < count;) {
        ListArgs<5, CAP> a;
        at = fill_list(a, sizes, dtypes, count, at, [&](int i, void **p) {
            p[0] = params[i];
            p[1] = m[i];
            p[2] = v[i];
            p[3] = const_cast<void *>(grads[i]);
            p[4] = copies ? copies[i] : nullptr;
            const unsigned h = head_of(p[0], 4, 4);
            const bool same = h == head_of(p[1], 4, 4) && h == head_of(p[2], 4, 4) && h == head_of(p[3], dtypes[i] == DD_BF16 ? 2 : 4, 4) &&
                              (!p[4] || h == head_of(p[4], 2, 4));
            return same ? h : (unsigned)kNoVector;
        });
        if (!a.tiles) continue;
        const int rc = launch_list(ctx, adamw_kernel<CAP>, list_grid(ctx, a.tiles), stream, a, c);
        if (rc != DD_OK) return rc;
    }
    return DD_OK;
}

static int check_norm_args(const dd_ctx *ctx, const void *const *grads, const uint64_t *sizes, const uint8_t *dtypes,
                           int count, float max_norm, const dd_grad_record *record)
{
    int rc = check_list(ctx, sizes, dtypes, count);
    if (rc != DD_OK) return rc;
    if (!record || !(max_norm >= 0.0f)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)record & 7u) return DD_ERR_ALIGNMENT;
    return check_grads(grads, sizes, dtypes, count);
}

}  // namespace ddm

using namespace ddm;

extern "C" int dd_grad_norm(dd_ctx *ctx, const void *const *grads, const uint64_t *sizes, const uint8_t *dtypes,
                            int count, float max_norm, dd_grad_record *record, void *cuda_stream)
{
    const int rc = check_norm_args(ctx, grads, sizes, dtypes, count, max_norm, record);
    if (rc != DD_OK) return rc;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    return count <= kListSmall ? launch_norm<kListSmall>(ctx, grads, sizes, dtypes, count, max_norm, record, false, stream)
                               : launch_norm<kListMax>(ctx, grads, sizes, dtypes, count, max_norm, record, false, stream);
}

extern "C" int dd_clip_gradients(dd_ctx *ctx, void *const *grads, void *const *outs, const uint64_t *sizes,
                                 const uint8_t *dtypes, int count, float max_norm, dd_grad_record *record,
                                 void *cuda_stream)
{
    int rc = check_norm_args(ctx, grads, sizes, dtypes, count, max_norm, record);
    if (rc != DD_OK) return rc;
    for (int i = 0; outs && i < count; ++i) {
        if (sizes[i] == 0) continue;
        const size_t eb = dtypes[i] == DD_BF16 ? 2 : 4;
        if (!outs[i]) return DD_ERR_INVALID_ARG;
        if ((uintptr_t)outs[i] & (eb - 1)) return DD_ERR_ALIGNMENT;
        if (outs[i] != grads[i] && ranges_overlap(outs[i], eb * sizes[i], grads[i], eb * sizes[i])) return DD_ERR_ALIAS;
    }
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    rc = count <= kListSmall ? launch_norm<kListSmall>(ctx, grads, sizes, dtypes, count, max_norm, record, true, stream)
                             : launch_norm<kListMax>(ctx, grads, sizes, dtypes, count, max_norm, record, true, stream);
    if (rc != DD_OK) return rc;
    return count <= kListSmall ? launch_scale<kListSmall>(ctx, grads, outs, sizes, dtypes, count, record, stream)
                               : launch_scale<kListMax>(ctx, grads, outs, sizes, dtypes, count, record, stream);
}

extern "C" int dd_adamw_step(dd_ctx *ctx, const dd_adamw *opt, float *const *params, const void *const *grads,
                             float *const *exp_avg, float *const *exp_avg_sq, void *const *copies,
                             const uint64_t *sizes, const uint8_t *dtypes, int count, const dd_grad_record *clip,
                             void *cuda_stream)
{
    int rc = check_list(ctx, sizes, dtypes, count);
    if (rc != DD_OK) return rc;
    if (!opt || opt->step < 1 || !std::isfinite(opt->lr) || !std::isfinite(opt->weight_decay) ||
        !(opt->beta1 >= 0.0 && opt->beta1 < 1.0) || !(opt->beta2 >= 0.0 && opt->beta2 < 1.0) ||
        !(opt->eps >= 0.0 && std::isfinite(opt->eps)))
        return DD_ERR_INVALID_ARG;
    if (count > 0 && (!params || !exp_avg || !exp_avg_sq)) return DD_ERR_INVALID_ARG;
    if ((uintptr_t)clip & 7u) return DD_ERR_ALIGNMENT;
    rc = check_grads(grads, sizes, dtypes, count);
    if (rc != DD_OK) return rc;
    for (int i = 0; i < count; ++i) {
        const size_t n = sizes[i];
        if (n == 0) continue;
        const void *p[5] = {params[i], exp_avg[i], exp_avg_sq[i], grads[i], copies ? copies[i] : nullptr};
        const size_t bytes[5] = {4 * n, 4 * n, 4 * n, (dtypes[i] == DD_BF16 ? 2 : 4) * n, 2 * n};
        if (!p[0] || !p[1] || !p[2]) return DD_ERR_INVALID_ARG;
        if ((((uintptr_t)p[0] | (uintptr_t)p[1] | (uintptr_t)p[2]) & 3u) || ((uintptr_t)p[4] & 1u)) return DD_ERR_ALIGNMENT;
        for (int x = 0; x < 5; ++x)
            for (int y = 0; y < x; ++y)
                if (ranges_overlap(p[x], bytes[x], p[y], bytes[y])) return DD_ERR_ALIAS;
    }
    AdamwConsts c;
    const double c1 = -std::expm1((double)opt->step * std::log(opt->beta1));     // 1 - beta1^step
    const double c2 = -std::expm1((double)opt->step * std::log(opt->beta2));
    c.beta1 = (float)opt->beta1;
    c.rest1 = (float)(1.0 - opt->beta1);
    c.beta2 = (float)opt->beta2;
    c.rest2 = (float)(1.0 - opt->beta2);
    c.eps = (float)opt->eps;
    c.decay = (float)(1.0 - opt->lr * opt->weight_decay);
    c.step_size = (float)(opt->lr / c1);
    c.inv_c2 = (float)(1.0 / c2);
    c.clip = clip;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return cuda_fail(ctx, cudaErrorInvalidDevice, "cudaSetDevice");
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    return count <= kListSmall
               ? launch_adamw<kListSmall>(ctx, c, params, grads, exp_avg, exp_avg_sq, copies, sizes, dtypes, count, stream)
               : launch_adamw<kListMax>(ctx, c, params, grads, exp_avg, exp_avg_sq, copies, sizes, dtypes, count, stream);
}
