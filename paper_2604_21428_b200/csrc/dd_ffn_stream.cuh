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

// Four floats at `addr` (a shared-memory address of this CTA) in the CTA of rank `rank`.
__device__ __forceinline__ float4 ld_cluster4(unsigned addr, unsigned rank)
{
    float4 x;
    asm volatile("{\n .reg .b32 r;\n mapa.shared::cluster.u32 r, %4, %5;\n ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [r];\n}"
                 : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr), "r"(rank) : "memory");
    return x;
}

__device__ __forceinline__ void tmem_ld16(unsigned addr, unsigned (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}

// What an epilogue reads for four features of a token, asked for before the sums are ready.
struct Aux {
    uint2 a, b;                       // kEpiBack: gate, up; kEpiStore: residual
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
    } else {
        float r[4];
        unpack4(aux.a, r);                // zeros without a residual
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += r[i];
        store4(a.out + (unsigned long long)t * a.ld_out + c, x, live);
    }
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
    } else if (p.own_prior) {
        asm volatile("griddepcontrol.wait;" ::: "memory");      // the epilogue may read what the prior launch wrote
        if (p.late_trigger) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();                      // every product is complete, no copy is in flight
    tc_fence_after();

    // This rank's sums to shared memory as [token][128 rows], a round of up to 64 tokens at a time;
    // then every rank adds up, over the ranks in order, the tokens that it owns.
    const unsigned f4 = threadIdx.x % kQuads * 4, feature = m0 + f4, live = feature < p.m ? p.m - feature : 0;
#pragma unroll 1
    for (unsigned c = 0, round = 0; c < N; c += kRound, ++round) {
        const unsigned buf = smem + (round & 1) * stream_round_bytes(N), cols = N - c < kRound ? N - c : kRound;
        const unsigned owned = (cols + S - 1) / S, last = (rank + 1) * owned < cols ? (rank + 1) * owned : cols;
        const unsigned left = p.n > n0 + c ? p.n - n0 - c : 0, end = last < left ? last : left;      // tokens that exist
        unsigned j = rank * owned + threadIdx.x / kQuads;
        const bool mine = warp < 4 && live;
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
