// The block's products for few tokens: bound by streaming the weights, so the weights take the
// 128-row side of the tensor-core tile and the tokens its N side (16 to 128 columns).  Each weight is
// read once per tile of tokens: up to 128 of them, fewer where SMs would be idle otherwise (the second
// reading comes from L2).  Gate and up share a tile: 64 rows each.
//
// One CTA computes a tile over a share of K; the S CTAs of a cluster share one tile's K and add
// their float32 partial sums through distributed shared memory in rank order, each rank finishing
// the tokens it owns.  No workspace, no atomics, and with S up to 8 even a 2048 x 8192 matrix
// spreads over the whole GPU.
//
// The call's second launch starts early (programmatic launch): it fills its ring with weights, which
// the call's first launch does not write, and waits only before it reads activations.  The launch before
// the call may well write them -- an optimizer step that leaves the weights' bf16 copies -- so
// the first launch lets the second one start only once its own wait for that launch is over.
//
// d 2048, f 8192, gate and up kept: 1 / 64 / 128 tokens 24 / 28 / 35 us forward, of which the 100.7 MB of
// weights need 15.4; the rest is two launches' ramp, reduction and hand-over.  A ring of 64 KB took 27.0
// against 24.4 (1 token) and 45 against 38 (128), clusters up to 296 CTAs 25.4 against 22.4, L2 prefetch of
// what follows the ring 25.2 against 24.4.
#pragma once

#include "dd_ffn_gemm.cuh"

namespace ddm {

constexpr unsigned kRound = 64;                   // tokens reduced per round
constexpr int kStreamThreads = 192;
constexpr unsigned kStreamMaxStages = 8, kStreamMaxCluster = 8, kStreamMaxCols = 128;

__host__ __device__ constexpr int stream_features(int epi) { return epi == kEpiGate ? kBM / 2 : kBM; }
// n: tokens of a tile, a multiple of 16
__host__ __device__ constexpr unsigned stream_stage_bytes(unsigned n) { return (kBM + n) * kBK * 2; }
__host__ __device__ constexpr unsigned stream_round_bytes(unsigned n) { return (n < kRound ? n : kRound) * kBM * 4; }
// The reduction reuses the ring: one buffer per round, at most two.
__host__ __device__ constexpr unsigned stream_ring_bytes(unsigned n, unsigned stages)
{
    const unsigned ring = stages * stream_stage_bytes(n), rounds = (n > kRound ? 2 : 1) * stream_round_bytes(n);
    return ring > rounds ? ring : rounds;
}
__host__ __device__ constexpr unsigned stream_smem_bytes(unsigned n, unsigned stages) { return 1024 + stream_ring_bytes(n, stages); }

// What an epilogue reads for four features of a token, asked for before the sums are ready.
struct Aux {
    uint2 a, b;                       // kEpiBack: gate, up; kEpiStore: residual
    long long target;                 // kEpiLoss, kEpiSoft
    float lse, dloss;                 // kEpiSoft
};

__device__ __forceinline__ uint2 load4_raw(const __nv_bfloat16 *p, unsigned live)
{
    if (live >= 4) return *reinterpret_cast<const uint2 *>(p);
    const unsigned short *q = reinterpret_cast<const unsigned short *>(p);
    uint2 w = make_uint2(q[0], 0u);
    if (live > 1) w.x |= (unsigned)q[1] << 16;
    if (live > 2) w.y = q[2];
    return w;
}

__device__ __forceinline__ void unpack4(const uint2 &w, float (&x)[4])
{
    x[0] = __uint_as_float(w.x << 16);
    x[1] = __uint_as_float(w.x & 0xffff0000u);
    x[2] = __uint_as_float(w.y << 16);
    x[3] = __uint_as_float(w.y & 0xffff0000u);
}

template <int EPI>
__device__ __forceinline__ Aux load_aux(const EpilogueArgs &a, unsigned t, unsigned c, unsigned live)
{
    Aux r;
    r.a = r.b = make_uint2(0u, 0u);
    if (EPI == kEpiBack) {
        r.a = load4_raw(a.gate + (unsigned long long)t * a.ld_gate + c, live);
        r.b = load4_raw(a.up + (unsigned long long)t * a.ld_gate + c, live);
    } else if (EPI == kEpiLoss || EPI == kEpiSoft) {
        r.target = a.targets[t];
        if (EPI == kEpiSoft) {
            r.lse = a.lse[t];
            r.dloss = a.dloss[t];
        }
    } else if (EPI == kEpiStore && a.residual) {
        r.a = load4_raw(a.residual + (unsigned long long)t * a.ld_residual + c, live);
    }
    return r;
}

// Four features from c on of token t, from their finished sums (kEpiGate: x gate, u up).
template <int EPI, int ACT>
__device__ __forceinline__ void finish4(const EpilogueArgs &a, unsigned t, unsigned c, unsigned live, const Aux &aux, float (&x)[4],
                                        float (&u)[4])
{
    const unsigned long long at = (unsigned long long)t * a.ld_gate + c, to = (unsigned long long)t * a.ld_hidden + c;
    if (EPI == kEpiGate) {
        if (a.gate) {
            store4(a.gate + at, x, live);
            store4(a.up + at, u, live);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = activate<ACT, false>(x[i], nullptr) * u[i];
        store4(a.hidden + to, x, live);
    } else if (EPI == kEpiBack) {
        float g[4];
        unpack4(aux.a, g);
        unpack4(aux.b, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float dh = x[i];
            float slope;
            const float act = activate<ACT, true>(g[i], &slope);
            x[i] = dh * act;
            g[i] = dh * u[i] * slope;
            u[i] = act * u[i];
        }
        store4(a.dup + to, x, live);
        store4(a.dgate + to, g, live);
        store4(a.hidden + to, u, live);
    } else if (EPI == kEpiLoss) {             // the warp's 128 logits of the token
        constexpr float l = 1.4426950408889634f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= live) x[i] = -INFINITY;
            else if (aux.target == (long long)c + i) a.loss[t] = x[i];
        }
        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
#pragma unroll
        for (int d = 16; d; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float base = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += exp2_fast((x[i] - base) * l);
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (threadIdx.x % 32 == 0) a.partial[(unsigned long long)(c / 128) * a.tokens + t] = make_float2(top, sum);
    } else if (EPI == kEpiSoft) {
        constexpr float l = 1.4426950408889634f;
        const bool some = aux.target >= 0 && aux.target < a.vocab;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = exp2_fast(fmaf(x[i], l, some ? -aux.lse * l : -INFINITY));
            x[i] = (some && aux.target - a.first == (long long)c + i ? p - 1.0f : p) * (some ? aux.dloss : 0.0f);
        }
        store4(a.hidden + to, x, live);
    } else {
        float r[4];
        unpack4(aux.a, r);                // zeros without a residual
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += r[i];
        store4(a.out + (unsigned long long)t * a.ld_out + c, x, live);
    }
}

// N values of each lane, combined over the warp's 2 N lanes: lane l has the result of value l / 2.
template <int N, typename Op>
__device__ __forceinline__ float warp_combine(const float (&v)[N], unsigned lane, const Op &op)
{
    float half[N / 2];
    const bool up = lane & N;
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
        half[i] = op(up ? v[i + N / 2] : v[i], __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + N / 2], N));
    if constexpr (N > 2) return warp_combine<N / 2>(half, lane, op);
    else return op(half[0], __shfl_xor_sync(0xffffffffu, half[0], 1));
}

// kEpiLoss of a tile that one CTA has the sums of, by its first 128 threads (thread = feature, lane of tensor memory):
// largest and sum of exponentials of each token's 128 logits.  Over a warp's 32 features they come by halving, one
// shuffle for each token and not five, and from the four warps through `share`, 4.9 KB of shared memory (96 tokens, d
// 768, 32000 columns: 33 -> 27 us with the join).  `target`: of token n0 + threadIdx.x.
__device__ __forceinline__ void finish_loss(const EpilogueArgs &a, unsigned tmem, unsigned char *share, unsigned m0, unsigned m,
                                            unsigned n0, unsigned n, unsigned N, long long target)
{
    constexpr float l = 1.4426950408889634f;
    const unsigned thread = threadIdx.x, warp = thread >> 5, lane = thread & 31, feature = m0 + thread;
    float2 (*const sums)[kStreamMaxCols] = reinterpret_cast<float2 (*)[kStreamMaxCols]>(share);
    int *const targets = reinterpret_cast<int *>(share + 4 * sizeof *sums);           // as a feature of the tile, -1: not in it
    float *const tops = reinterpret_cast<float *>(targets + kStreamMaxCols) + warp * 16;
    const long long at = target - m0;
    targets[thread] = at >= 0 && at < kBM && thread < N && n0 + thread < n ? (int)at : -1;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    for (unsigned c = 0; c < N; c += 16) {
        unsigned r[16];
        float x[16], v[16];
        tmem_ld16(tmem + (warp * 32 << 16) + c, r);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int4 at4 = *reinterpret_cast<const int4 *>(targets + c + i);
            const int t[4] = {at4.x, at4.y, at4.z, at4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[i + k] = feature < m ? __uint_as_float(r[i + k]) : -INFINITY;
                if (t[k] == (int)thread && feature < m) a.loss[n0 + c + i + k] = x[i + k];
                v[i + k] = x[i + k];
            }
        }
        const float top = warp_combine<16>(v, lane, [](float p, float q) { return fmaxf(p, q); });
        if (!(lane & 1)) tops[lane / 2] = top;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float base = tops[i] == -INFINITY ? 0.0f : tops[i];
            v[i] = exp2_fast((x[i] - base) * l);
        }
        __syncwarp();
        const float sum = warp_combine<16>(v, lane, [](float p, float q) { return p + q; });
        if (!(lane & 1)) sums[warp][c + lane / 2] = make_float2(top, sum);
    }
    asm volatile("bar.sync 1, 128;" ::: "memory");
    if (thread >= N || n0 + thread >= n) return;
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sums[w][thread].x);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += sums[w][thread].y * exp2_fast((sums[w][thread].x - base) * l);
    a.partial[(unsigned long long)(m0 / kBM) * a.tokens + n0 + thread] = make_float2(top, sum);
}

// One launch.  Kept small: 1.5 KB more of parameters cost the host 0.7 us a launch.
struct StreamArgs {
    CUtensorMap w[2];                 // weights: kEpiGate gate and up, else the K segments
    CUtensorMap x[2];                 // token matrices of the K segments, boxes of `cols` rows
    unsigned m, n;                    // features (rows of the output's transpose), tokens
    unsigned tiles_n, cols;           // tiles along the tokens, tokens of a tile (a multiple of 16)
    unsigned kblocks[2];              // K blocks of the segments
    int w_mn;                         // 1: the features are the contiguous direction of the weights
    int cluster, stages;              // CTAs per tile, ring stages
    int own_prior;                    // the launch before is this call's own: the weights are not its results
    int late_trigger;                 // with own_prior: the next launch may start once that one has ended
    EpilogueArgs e;
};

// blockIdx.x = tile * cluster + rank.
template <int EPI, int ACT>
__global__ void __launch_bounds__(kStreamThreads, 2)
ffn_stream_kernel(const __grid_constant__ StreamArgs p)
{
    constexpr unsigned kABytes = kBM * kBK * 2;
    constexpr int kFeatures = stream_features(EPI), kQuads = kFeatures / 4, kTokensAtOnce = 128 / kQuads;

    extern __shared__ unsigned char smem_raw[];
    const unsigned smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    __shared__ alignas(8) unsigned long long bars[2 * kStreamMaxStages + 1];
    __shared__ int abort_flag;
    __shared__ unsigned tmem_base;
    const unsigned full = smem_addr(bars), empty = full + 8 * kStreamMaxStages, done = empty + 8 * kStreamMaxStages;
    volatile int *abort = &abort_flag;
    const int warp = threadIdx.x >> 5;
    const unsigned S = p.cluster, stages = p.stages, N = p.cols, stage_bytes = stream_stage_bytes(N);
    const unsigned tmem_cols = N <= 32 ? 32 : N <= 64 ? 64 : 128;
    const unsigned rank = blockIdx.x % S, tile = blockIdx.x / S;
    const unsigned m0 = tile / p.tiles_n * kFeatures, n0 = tile % p.tiles_n * N;   // tiles of the same weights are neighbours
    const unsigned blocks = p.kblocks[0] + p.kblocks[1];
    const unsigned kb0 = (unsigned)((unsigned long long)blocks * rank / S);
    const unsigned count = (unsigned)((unsigned long long)blocks * (rank + 1) / S) - kb0;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (unsigned s = 0; s < stages; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(full + 8 * s) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(empty + 8 * s) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(done) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&tmem_base)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = tmem_base;
    if (!p.own_prior) asm volatile("griddepcontrol.wait;" ::: "memory");      // before the trigger: see the top of the file
    if (!p.late_trigger) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    long long target = -1;
    if (warp == 4) {
        if (elect_one()) {
            const auto weights = [&](unsigned kb, unsigned s) {
                const int seg = kb >= p.kblocks[0], k0 = (int)(kb - (seg ? p.kblocks[0] : 0u)) * kBK;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const CUtensorMap *m = &p.w[EPI == kEpiGate ? c : seg];
                    const int row = (int)m0 + (EPI == kEpiGate ? 0 : 64 * c);
                    tma_load_2d(smem + s * stage_bytes + c * kChunkBytes, m, p.w_mn ? row : k0, p.w_mn ? k0 : row, full + 8 * s);
                }
            };
            const auto tokens = [&](unsigned kb, unsigned s) {
                const int seg = kb >= p.kblocks[0], k0 = (int)(kb - (seg ? p.kblocks[0] : 0u)) * kBK;
                tma_load_2d(smem + s * stage_bytes + kABytes, &p.x[seg], k0, (int)n0, full + 8 * s);
            };
            const unsigned first = count < stages ? count : stages;
            for (unsigned i = 0; i < first; ++i) {
                mbar_arrive_expect_tx(full + 8 * i, stage_bytes + (p.e.expire && i == 0 ? 16u : 0u));
                weights(kb0 + i, i);
            }
            if (p.own_prior) asm volatile("griddepcontrol.wait;" ::: "memory");
            for (unsigned i = 0; i < first; ++i) tokens(kb0 + i, i);
            unsigned it = first, s = 0, phase = 0;          // stage of copy `it`, parity of its previous use
            for (; it < count; ++it) {
                if (!gemm_wait(empty + 8 * s, phase, abort) || *abort) break;
                mbar_arrive_expect_tx(full + 8 * s, stage_bytes);
                weights(kb0 + it, s);
                tokens(kb0 + it, s);
                if (++s == stages) { s = 0; phase ^= 1; }
            }
            // no copy may be in flight when the ring is reused, whoever gave up
            for (unsigned j = it > stages ? it - stages : 0; j < it; ++j)
                mbar_wait_bounded(full + 8 * (j % stages), (j / stages) & 1);
        }
    } else if (warp == 5) {
        if (elect_one()) {
            const unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((unsigned)p.w_mn << 15) |
                                   ((N / 8) << 17) | ((kBM / 16) << 24);
            const unsigned astep = p.w_mn ? 2048 : 32;
            for (unsigned it = 0, s = 0, phase = 0; it < count; ++it) {
                if (!gemm_wait(full + 8 * s, phase, abort)) break;
                tc_fence_after();
                const unsigned sa = smem + s * stage_bytes, sb = sa + kABytes;
#pragma unroll
                for (int k = 0; k < kBK / 16; ++k)
                    umma_bf16(tmem, umma_desc(sa + k * astep, p.w_mn), umma_desc(sb + k * 32, false), idesc, it | k);
                umma_commit(empty + 8 * s);
                if (++s == stages) { s = 0; phase ^= 1; }
            }
            umma_commit(done);
            if (!mbar_wait_bounded(done, 0)) *abort = 1;
        }
    } else if (EPI == kEpiLoss && S == 1) {                      // (never the second launch)
        if (threadIdx.x < N && n0 + threadIdx.x < p.n) target = p.e.targets[n0 + threadIdx.x];
    } else if (p.own_prior) {
        asm volatile("griddepcontrol.wait;" ::: "memory");      // the epilogue may read what the prior launch wrote
        if (p.late_trigger) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();                      // every product is complete, no copy is in flight
    tc_fence_after();

    const bool whole = EPI == kEpiLoss && S == 1;
    if (EPI == kEpiLoss && whole && warp < 4) finish_loss(p.e, tmem, smem_raw + (smem - smem_addr(smem_raw)), m0, p.m, n0, p.n, N, target);

    // This rank's sums to shared memory as [token][128 rows], a round of up to 64 tokens at a time;
    // then every rank adds up, over the ranks in order, the tokens that it owns.
    const unsigned f4 = threadIdx.x % kQuads * 4, feature = m0 + f4, live = feature < p.m ? p.m - feature : 0;
#pragma unroll 1
    for (unsigned c = 0, round = 0; c < N && !whole; c += kRound, ++round) {
        const unsigned buf = smem + (round & 1) * stream_round_bytes(N), cols = N - c < kRound ? N - c : kRound;
        const unsigned owned = (cols + S - 1) / S, last = (rank + 1) * owned < cols ? (rank + 1) * owned : cols;
        const unsigned left = p.n > n0 + c ? p.n - n0 - c : 0, end = last < left ? last : left;      // tokens that exist
        unsigned j = rank * owned + threadIdx.x / kQuads;
        const bool mine = warp < 4 && (live || EPI == kEpiLoss);              // (whose warps stay together)
        Aux aux[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (mine && j + b * kTokensAtOnce < end) aux[b] = load_aux<EPI>(p.e, n0 + c + j + b * kTokensAtOnce, feature, live);
        __syncwarp();                     // lanes own different tokens and features; what follows is for whole warps
        if (warp < 4) {
            const unsigned col = tmem + ((unsigned)(warp * 32) << 16) + c, to = buf + threadIdx.x * 4;
#pragma unroll 1
            for (unsigned h = 0; h < cols; h += 16) {
                unsigned r[16];
                tmem_ld16(col + h, r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    asm volatile("st.shared.b32 [%0], %1;" :: "r"(to + (h + i) * kBM * 4), "r"(r[i]) : "memory");
            }
        }
        if (S > 1) cluster_sync();
        else __syncthreads();
        // two tokens at a time: the reads from all ranks are on their way together (one at a time, with what the
        // epilogue reads asked for in between, a round of 64 tokens took 7 us)
        for (; mine && j < end; j += 2 * kTokensAtOnce) {
            float4 vx[2][kStreamMaxCluster], vu[2][EPI == kEpiGate ? kStreamMaxCluster : 1];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < kStreamMaxCluster; ++r)
                    if (r < S && j + b * kTokensAtOnce < end) {
                        const unsigned from = buf + ((j + b * kTokensAtOnce) * kBM + f4) * 4;
                        vx[b][r] = ld_cluster4(from, r);
                        if (EPI == kEpiGate) vu[b][r] = ld_cluster4(from + kFeatures * 4, r);
                    }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const unsigned k = j + b * kTokensAtOnce;
                if (k >= end) break;
                const Aux now = aux[b];
                if (k + 2 * kTokensAtOnce < end) aux[b] = load_aux<EPI>(p.e, n0 + c + k + 2 * kTokensAtOnce, feature, live);
                float x[4] = {vx[b][0].x, vx[b][0].y, vx[b][0].z, vx[b][0].w}, u[4];
                if (EPI == kEpiGate) { u[0] = vu[b][0].x; u[1] = vu[b][0].y; u[2] = vu[b][0].z; u[3] = vu[b][0].w; }
#pragma unroll
                for (int r = 1; r < kStreamMaxCluster; ++r)
                    if (r < S) {
                        x[0] += vx[b][r].x; x[1] += vx[b][r].y; x[2] += vx[b][r].z; x[3] += vx[b][r].w;
                        if (EPI == kEpiGate) {
                            const float4 v = vu[b][EPI == kEpiGate ? r : 0];
                            u[0] += v.x; u[1] += v.y; u[2] += v.z; u[3] += v.w;
                        }
                    }
                finish4<EPI, ACT>(p.e, n0 + c + k, feature, live, now, x, u);
            }
        }
        __syncwarp();
    }
    if (S > 1) cluster_sync_relaxed();    // nobody leaves while its sums may still be read
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 5)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(tmem_cols) : "memory");
    if (threadIdx.x == 0 && abort_flag && p.e.status) *p.e.status = DD_STATUS_WAIT_LIMIT;
}

}  // namespace ddm
