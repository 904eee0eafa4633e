// Tensor-core products of the gated feed-forward block: D = sum_s A_s B_s^T over one or two
// K segments, bf16 operands, float32 accumulators in tensor memory, epilogues of the block.
//
// A pair of SMs (a cluster of two CTAs) computes one 256 x BN tile with tcgen05.mma of
// cta_group::2: each CTA stages 128 rows of A and BN / 2 rows of B and keeps 128 rows of the
// accumulator, so that every operand byte in shared memory feeds twice the products that it would
// for one SM.  Persistent pairs walk the tiles of up to four problems.  In each CTA warp 8 (one lane)
// has the TMA engine fill a ring of stages of 64 K-elements (128-byte rows, 128-byte swizzle);
// warp 9 of the first CTA (one lane) issues the products for both; warps 0-7 turn finished
// accumulators into results.  With BN = 256 two accumulators alternate, so the epilogue of one tile runs
// under the products of the next; BN = 512 (long K only) reads fewer operand bytes a product instead.
// Operands are read where they lie in either order -- K contiguous, or M / N contiguous (the
// descriptor's "major" bit) -- so no product of the backward pass needs a transposed copy.
//
// What bounds it: at 8192 tokens, d 2048, f 8192 the operands come out of L2 at 10-13 TB/s (128 FLOP a
// byte with BN = 256) with the tensor pipe 68-77 % active, under the 1000 W cap.  Forward 606-624 us in short
// runs, 660-716 back to back for seconds; backward 1155-1196 and 1280-1370 (GPUs differ; the library's bare
// products 560 / 646 and 1130 / 1295 beside the larger of these).  With the loads taken out after the first
// ring the forward pass takes 473 us, with the products taken out 497 (short runs).
//
// Every wait is bounded: on giving up a role raises its CTA's abort flag, the roles leave their
// loops, copies and products in flight are awaited (again bounded), tensor memory is freed and
// the caller's status word says DD_STATUS_WAIT_LIMIT.
#pragma once

#include "dd_learner.h"
#include "dd_tcgen05.cuh"

namespace ddm {

constexpr int kBM = 128, kBK = 64;              // rows of one CTA, K elements of a stage
constexpr int kMaxMaps = 8, kMaxProblems = 4;
constexpr unsigned kTileGroup = 8;                // 4 / 8 / 16: forward 657 / 646 / 639 us, backward 1305 / 1309 / 1325 (8192 tokens)
constexpr int kMaxSplits = 8;
constexpr int kBoxBytes = 32 * 128;               // an epilogue box: 32 rows of 64 bf16 or 32 float32

enum GemmEpilogue { kEpiStore = 0, kEpiGate = 1, kEpiBack = 2, kEpiLoss = 3, kEpiSoft = 4 };

// What the epilogues read and write.  kEpiGate: gate and up (null when not kept) and hidden are outputs;
// kEpiBack: gate and up are inputs, dgate, dup and hidden outputs; kEpiStore: out = sums [+ residual].
// The sums as logits of tokens (rows) and a piece of the vocabulary (columns), of which nothing is stored:
// kEpiLoss leaves each row's largest and its sum of exponentials over 128 columns in `partial`, and the target's
// logit in `loss`; kEpiSoft the gradient dloss (exp(z - lse) - [target]) in hidden.
struct EpilogueArgs {
    __nv_bfloat16 *gate, *up, *dgate, *dup, *hidden, *out;
    const __nv_bfloat16 *residual;
    unsigned long long ld_gate, ld_hidden, ld_out, ld_residual;
    int *status;
    const long long *targets;         // by row; outside 0 .. vocab - 1: none
    const float *lse, *dloss;         // kEpiSoft, by row
    float *loss;                      // kEpiLoss
    float2 *partial;                  // [columns / 128][rows]: largest logit, sum of exp(z - largest)
    long long first, vocab;           // kEpiSoft: the piece's first column
    unsigned tokens;                  // kEpiLoss: row length of `partial`
    int activation;
    int expire;                       // test hook: the first stage waits for 16 bytes that no copy brings
};

enum { kOutBf16 = 0, kOutF32 = 1, kOutSum = 2 };

struct GemmProblem {
    unsigned m, n;                    // output rows and columns
    unsigned tiles_m, tiles_n, tile_end;
    unsigned kblocks[2];              // K blocks of the two segments (second may be 0)
    unsigned splits;                  // K is cut into this many units per tile, split s writing rows split_rows s + ...
    unsigned split_rows;
    unsigned char a_map[2], b_map[2]; // tensor maps of the segments; kEpiGate: b_map = {w_gate, w_up}
    unsigned char a_mn, b_mn;         // 1: M (N) is the contiguous direction in memory
    // kEpiStore: out = sums [+ addend of the output's type]; the addend may be the output itself
    unsigned char out_f32;            // kOutBf16, kOutF32, or kOutSum: bf16 with a float32 addend
    void *out;
    const void *addend;
    unsigned long long ld_out, ld_addend;
};

struct GemmArgs {
    CUtensorMap maps[kMaxMaps];       // 64 x 64 boxes of row-major bf16 matrices
    GemmProblem prob[kMaxProblems];
    int nprob;
    unsigned tiles;                   // units of all problems
    unsigned first, rest, extra;      // schedule: see unit_of
    // 1: nothing here depends on the launch before, which itself began after all that does; this launch runs beside
    // it and only ends after it
    int late_wait;
    EpilogueArgs e;                   // kEpiStore: the problems have their own outputs
};

constexpr int kEpiWarps = 8, kGemmThreads = 32 * kEpiWarps + 64;
// Boxes that a warp of the epilogue stages results in; kEpiBack also reads gate and up through its two.
__host__ __device__ constexpr int gemm_boxes(int epi) { return epi == kEpiLoss ? 0 : epi == kEpiStore || epi == kEpiSoft ? 1 : 2; }
__host__ __device__ constexpr unsigned gemm_epi_bytes(int epi) { return kEpiWarps * gemm_boxes(epi) * kBoxBytes; }
// A stage of one CTA: 128 rows of A and half of the tile's BN rows of B.
__host__ __device__ constexpr unsigned gemm_stage_bytes(int bn) { return (unsigned)(kBM + bn / 2) * kBK * 2; }
__host__ __device__ constexpr int gemm_stages(int epi, int bn) { return (int)((224 * 1024 - gemm_epi_bytes(epi)) / gemm_stage_bytes(bn)); }
__host__ __device__ constexpr unsigned gemm_smem_bytes(int epi, int bn) { return 1024 + gemm_stages(epi, bn) * gemm_stage_bytes(bn) + gemm_epi_bytes(epi); }

// ---- activation ---------------------------------------------------------------------------------

// Both activations are g sigmoid(s(g)); returns a(g) and sets its derivative.  The exponential and the
// reciprocal are the hardware's approximations (2 ulp and 1 ulp): their error is far below the bf16
// rounding of what they feed, and the epilogues are bound by their instruction count.  exp overflows
// to infinity and the sigmoid to 0 where it should.
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate(float g, float *slope)
{
    constexpr float k = 1.5957691216057308f, q = 0.044715f, l = -1.4426950408889634f;      // 2 sqrt(2 / pi), -log2(e)
    const float g2 = g * g;
    const float z = ACT == DD_ACT_SILU ? l * g : g * fmaf(l * k * q, g2, l * k);            // -s log2(e)
    float e, sg;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(sg) : "f"(1.0f + e));
    const float a = g * sg;
    if (SLOPE) {
        const float rest = 1.0f - sg;
        *slope = fmaf(a, ACT == DD_ACT_SILU ? rest : rest * fmaf(3.0f * k * q, g2, k), sg);
    }
    return a;
}

// Up to four consecutive bf16, `live` of them inside the row.
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float (&x)[4], unsigned live)
{
    if (live >= 4) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < live) p[i] = __float2bfloat16_rn(x[i]);
    }
}

__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&x)[4], unsigned live)
{
    if (live >= 4) {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        x[0] = __uint_as_float(w.x << 16);
        x[1] = __uint_as_float(w.x & 0xffff0000u);
        x[2] = __uint_as_float(w.y << 16);
        x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < live ? __bfloat162float(p[i]) : 0.0f;
    }
}

// Addends are read past L1 (here and in load_share): the launch that runs beside the one before it
// (GemmArgs::late_wait) adds to what an earlier launch wrote without a wait of its own, and a line that its
// SM still held from then would be old.
__device__ __forceinline__ void load4_f32(const float *p, float (&x)[4], unsigned live)
{
    if (live >= 4) {
        const float4 w = __ldcg(reinterpret_cast<const float4 *>(p));
        x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < live ? __ldcg(p + i) : 0.0f;
    }
}

__device__ __forceinline__ void store4_f32(float *p, const float (&x)[4], unsigned live)
{
    if (live >= 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < live) p[i] = x[i];
    }
}

// ---- tiles ----------------------------------------------------------------------------------------

struct TilePos {
    int p;                    // problem
    unsigned m0, n0;          // first output row and column
    unsigned split;
    unsigned kb0, kb1;        // K blocks, counted over both segments
};

// The it-th unit of a pair; a.tiles or more: none.  Units of the first problem go round the pairs and
// may be longer than the others: the `rest` pairs that got one more of them leave the other pairs
// `extra` units of the following problems to begin with, then those go round all pairs.
__device__ __forceinline__ unsigned unit_of(const GemmArgs &a, unsigned pair, unsigned pairs, unsigned it)
{
    const bool long_pair = pair < a.rest;
    const unsigned mine = (a.first - a.rest) / pairs + (long_pair ? 1 : 0);
    if (it < mine) return it * pairs + pair;
    const unsigned j = it - mine, early = a.extra * (pairs - a.rest);
    if (long_pair) return a.first + early + j * pairs + pair;
    return a.first + (j < a.extra ? j * (pairs - a.rest) + pair - a.rest : early + (j - a.extra) * pairs + pair);
}

// Neighbouring tiles (what the GPU holds at one time) cover a block of 8 tile rows, so that both
// operands of a wave stay in L2.
template <int COLS>
__device__ __forceinline__ TilePos tile_pos(const GemmArgs &a, unsigned t)
{
    TilePos r;
    r.p = 0;
    while (t >= a.prob[r.p].tile_end) ++r.p;
    const GemmProblem &p = a.prob[r.p];
    t -= r.p ? a.prob[r.p - 1].tile_end : 0u;
    const unsigned blocks = p.kblocks[0] + p.kblocks[1];
    r.split = 0;
    r.kb0 = 0;
    r.kb1 = blocks;
    if (p.splits > 1) {
        r.split = t % p.splits;
        t /= p.splits;
        r.kb0 = blocks * r.split / p.splits;
        r.kb1 = blocks * (r.split + 1) / p.splits;
    }
    const unsigned group = kTileGroup * p.tiles_n, g = t / group, first = kTileGroup * g;
    const unsigned rows = p.tiles_m - first < kTileGroup ? p.tiles_m - first : kTileGroup;
    t -= g * group;
    r.m0 = (first + t % rows) * 2 * kBM;
    r.n0 = (t / rows) * COLS;
    return r;
}

// Results leave a warp through a box in shared memory: in tensor memory a lane holds a row, in
// global memory eight lanes together write 128 bytes of one.  (Rows written lane by lane cost the
// load/store unit a pass per row; 64-byte boxes stored by the TMA engine took 1 us a box and warp.)
// 128-byte rows, the 16-byte piece j of row r at piece j ^ (r mod 8): free of bank conflicts both ways.
__device__ __forceinline__ unsigned box_piece(unsigned box, int row, int j) { return box + row * 128 + ((j ^ (row & 7)) << 4); }

__device__ __forceinline__ void st_shared(unsigned addr, unsigned a, unsigned b, unsigned c, unsigned d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ uint4 ld_shared(unsigned addr)
{
    uint4 w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(addr) : "memory");
    return w;
}

// 32 columns of the lane's row, packed bf16, as pieces 4 h .. 4 h + 3.
__device__ __forceinline__ void write_half(unsigned box, int lane, int h, const unsigned (&w)[16])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) st_shared(box_piece(box, lane, 4 * h + j), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}

__device__ __forceinline__ void pack32(const float (&x)[32], unsigned (&w)[16])
{
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack2(x[2 * j], x[2 * j + 1]);
}

// The box to rows row0.. and columns col.. of a bf16 matrix of m x n.
__device__ __forceinline__ void store_box(unsigned box, int lane, __nv_bfloat16 *out, unsigned long long ld, unsigned row0, unsigned col,
                                          unsigned m, unsigned n)
{
    const unsigned c = col + (lane & 7) * 8;
    uint4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = ld_shared(box_piece(box, 4 * i + (lane >> 3), lane & 7));
    __nv_bfloat16 *o = out + (unsigned long long)(row0 + (lane >> 3)) * ld + c;
    if (row0 + 32 <= m && col + 64 <= n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(o + 4 * i * ld) = w[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (row0 + 4 * i + (lane >> 3) >= m) break;
        if (c + 8 <= n) {
            *reinterpret_cast<uint4 *>(o + 4 * i * ld) = w[i];
        } else {
            const unsigned u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int k = 0; k < 7; ++k)
                if (c + k < n) reinterpret_cast<unsigned short *>(o + 4 * i * ld)[k] = (unsigned short)(u[k / 2] >> (16 * (k & 1)));
        }
    }
}

// 32 rows from row0 and 64 columns from col on of a bf16 matrix, a lane's share in the order of store_box;
// zeros past its end.
__device__ __forceinline__ void load_share(uint4 (&w)[8], int lane, const __nv_bfloat16 *in, unsigned long long ld, unsigned row0,
                                           unsigned col, unsigned m, unsigned n)
{
    const unsigned c = col + (lane & 7) * 8, live = c < n ? n - c : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned row = row0 + 4 * i + (lane >> 3);
        w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row >= m || !live) continue;
        const __nv_bfloat16 *src = in + (unsigned long long)row * ld + c;
        if (live >= 8) {
            w[i] = __ldcg(reinterpret_cast<const uint4 *>(src));
        } else {
            unsigned u[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < 7; ++k)
                if (k < live) u[k / 2] |= (unsigned)__ldcg(reinterpret_cast<const unsigned short *>(src) + k) << (16 * (k & 1));
            w[i] = make_uint4(u[0], u[1], u[2], u[3]);
        }
    }
}

// Rows row0.. and columns col.. of a bf16 matrix to the box; zeros past its end.
__device__ __forceinline__ void load_box(unsigned box, int lane, const __nv_bfloat16 *in, unsigned long long ld, unsigned row0, unsigned col,
                                         unsigned m, unsigned n)
{
    const unsigned c = col + (lane & 7) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        const unsigned bytes = row0 + r >= m || c >= n ? 0 : n - c < 8 ? 2 * (n - c) : 16;
        const __nv_bfloat16 *src = bytes ? in + (unsigned long long)(row0 + r) * ld + c : in;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(box_piece(box, r, lane & 7)), "l"(src), "r"(bytes) : "memory");
    }
}

// 32 float32 columns of the lane's row through the box to out [+ addend]; SUM (kOutSum) rounds what goes out.  The
// choice is made outside, and launches without such a problem have a kernel without it: made for every piece it holds the
// stores up (d 2048, f 8192, float32 gradients: 512 tokens backward 160 -> 181 us, 100 tokens 116 -> 129; d 256, f 1024, 321
// tokens forward 25 -> 28), and the longer kernel alone costs small blocks 1 us (d 512, f 2048, 512 tokens backward 40 -> 41).
template <bool SUM>
__device__ __forceinline__ void finish_f32(unsigned box, int lane, const float (&x)[32], const GemmProblem &p, unsigned row0, unsigned out_row0,
                                           unsigned col)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        st_shared(box_piece(box, lane, j), __float_as_uint(x[4 * j]), __float_as_uint(x[4 * j + 1]), __float_as_uint(x[4 * j + 2]),
                  __float_as_uint(x[4 * j + 3]));
    __syncwarp();
    const unsigned c = col + (lane & 7) * 4, live = c < p.n ? p.n - c : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        const uint4 w = ld_shared(box_piece(box, r, lane & 7));
        if (row0 + r >= p.m || !live) continue;
        float y[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)}, add[4];
        if (p.addend) {
            const unsigned long long at = (unsigned long long)(row0 + r) * p.ld_addend + c;
            load4_f32(static_cast<const float *>(p.addend) + at, add, live);
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] += add[k];
        }
        const unsigned long long at = (unsigned long long)(out_row0 + r) * p.ld_out + c;
        if (!SUM) store4_f32(static_cast<float *>(p.out) + at, y, live);
        else store4(static_cast<__nv_bfloat16 *>(p.out) + at, y, live);
    }
    __syncwarp();
}

// Chunks of WIDTH columns of a tile that an epilogue warp finishes: `half` of the tile's columns, as far
// as the output goes; none if the warp's rows are past its end.
template <int COLS, int WIDTH>
__device__ __forceinline__ unsigned chunks_of(const GemmProblem &p, const TilePos &pos, unsigned row0, unsigned half)
{
    const unsigned col = pos.n0 + half * (COLS / 2);
    if (pos.m0 + row0 >= p.m || col >= p.n) return 0;
    const unsigned c = (p.n - col + WIDTH - 1) / WIDTH;
    return c < COLS / 2 / WIDTH ? c : COLS / 2 / WIDTH;
}

// BN: accumulator columns of a pair's tile.  kEpiGate puts BN / 2 columns of gate (the first CTA's
// share of B) beside BN / 2 of up (the second's).  SUM: kEpiStore with a kOutSum problem.
template <int EPI, int BN, int ACT, bool SUM>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
ffn_gemm_kernel(const __grid_constant__ GemmArgs a)
{
    constexpr int kStages = gemm_stages(EPI, BN), kProducer = kEpiWarps, kIssuer = kEpiWarps + 1;
    constexpr unsigned kStageBytes = gemm_stage_bytes(BN), kABytes = kBM * kBK * 2;
    constexpr int kCols = EPI == kEpiGate ? BN / 2 : BN;      // output columns of a tile
    constexpr unsigned kTmemCols = 512, kSlots = kTmemCols / BN;   // accumulators that alternate
    static_assert(BN == 256 || (BN == 512 && EPI == kEpiStore), "one or two products of 256 columns a step");

    extern __shared__ unsigned char smem_raw[];
    const unsigned smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    __shared__ alignas(8) unsigned long long bars[2 * kStages + 5];
    __shared__ int abort_flag;
    __shared__ unsigned tmem_base;
    const unsigned full = smem_addr(bars), empty = full + 8 * kStages, tfull = empty + 8 * kStages, tempty = tfull + 16, drain = tempty + 16;
    volatile int *abort = &abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int s = 0; s < kStages; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(full + 8 * s) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(empty + 8 * s) : "memory");
        }
        for (int s = 0; s < 2; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(tfull + 8 * s) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(tempty + 8 * s), "r"(2 * kEpiWarps) : "memory");   // both CTAs' warps
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(drain) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const unsigned tmem = tmem_base;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!a.late_wait) asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp == kProducer) {
        if (elect_one()) {
            const unsigned full0 = cluster_addr(full, 0);      // the first CTA's barriers count both CTAs' bytes
            unsigned it = 0, s = 0, phase = 1;                 // copies so far, stage, parity of its previous use
            bool ok = true;
            for (unsigned u = 0, t; ok && (t = unit_of(a, pair, pairs, u)) < a.tiles; ++u) {
                const TilePos pos = tile_pos<kCols>(a, t);
                const GemmProblem &p = a.prob[pos.p];
                const int m0 = (int)(pos.m0 + rank * kBM), n0 = (int)(pos.n0 + (EPI == kEpiGate ? 0 : rank * 128));
                for (unsigned kb = pos.kb0; kb < pos.kb1; ++kb, ++it) {
                    if ((it >= kStages && !gemm_wait(empty + 8 * s, phase, abort)) || *abort) { ok = false; break; }
                    const int seg = kb >= p.kblocks[0], k0 = (int)(kb - (seg ? p.kblocks[0] : 0u)) * kBK;
                    const CUtensorMap *ma = &a.maps[p.a_map[seg]], *mb = &a.maps[p.b_map[EPI == kEpiGate ? rank : seg]];
                    const unsigned st = smem + s * kStageBytes, bar = full0 + 8 * s;
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * s, 2 * kStageBytes + (a.e.expire && it == 0 ? 16u : 0u));
#pragma unroll
                    for (int c = 0; c < kBM / 64; ++c)
                        tma_load_2d_pair(st + c * kChunkBytes, ma, p.a_mn ? m0 + 64 * c : k0, p.a_mn ? k0 : m0 + 64 * c, bar);
#pragma unroll
                    for (int c = 0; c < BN / 128; ++c) {              // this CTA's 128 of every 256 columns
                        const int n = n0 + c / 2 * 256 + 64 * (c & 1);
                        tma_load_2d_pair(st + kABytes + c * kChunkBytes, mb, p.b_mn ? n : k0, p.b_mn ? k0 : n, bar);
                    }
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
            }
            // no copy of either CTA may be in flight when the pair ends, whoever gave up
            if (rank == 0)
                for (unsigned j = it > kStages ? it - kStages : 0; j < it; ++j)
                    mbar_wait_bounded(full + 8 * (j % kStages), (j / kStages) & 1);
        }
    } else if (warp == kIssuer) {
        if (rank == 0 && elect_one()) {
            unsigned acc = 0, s = 0, phase = 0;                // tiles started, stage, its parity
            bool ok = true;
            for (unsigned t; ok && (t = unit_of(a, pair, pairs, acc)) < a.tiles; ++acc) {
                const TilePos pos = tile_pos<kCols>(a, t);
                const GemmProblem &p = a.prob[pos.p];
                const unsigned slot = acc % kSlots;
                if (acc >= kSlots && !gemm_wait(tempty + 8 * slot, (acc / kSlots - 1) & 1, abort)) { ok = false; break; }
                tc_fence_after();
                // float32 accumulators, bf16 x bf16, the operands' majors, N = 256, M = 256
                const unsigned idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((unsigned)p.a_mn << 15) |
                                       ((unsigned)p.b_mn << 16) | ((256u / 8) << 17) | ((2 * kBM / 16) << 24);
                const unsigned astep = p.a_mn ? 2048 : 32, bstep = p.b_mn ? 2048 : 32;     // bytes per 16 K elements
                for (unsigned kb = pos.kb0; kb < pos.kb1; ++kb) {
                    if (!gemm_wait(full + 8 * s, phase, abort)) { ok = false; break; }
                    tc_fence_after();
                    const unsigned sa = smem + s * kStageBytes, sb = sa + kABytes;
#pragma unroll
                    for (int k = 0; k < kBK / 16; ++k)
#pragma unroll
                        for (int h = 0; h < BN / 256; ++h)
                            umma_bf16_pair(tmem + slot * BN + 256 * h, umma_desc(sa + k * astep, p.a_mn),
                                           umma_desc(sb + h * 2 * kChunkBytes + k * bstep, p.b_mn), idesc, kb != pos.kb0 || k);
                    umma_commit_pair(empty + 8 * s, 3);
                    if (++s == kStages) { s = 0; phase ^= 1; }
                }
                if (ok) umma_commit_pair(tfull + 8 * slot, 3);
            }
            umma_commit_pair(drain, 1);   // no product may be in flight when tensor memory is freed
            mbar_wait_bounded(drain, 0);
        }
    } else {
        const unsigned tempty0 = cluster_addr(tempty, 0);
        const unsigned row0 = rank * kBM + (warp & 3) * 32, half = warp >> 2;
        const unsigned box = smem + kStages * kStageBytes + warp * gemm_boxes(EPI) * kBoxBytes, box2 = box + kBoxBytes;
        // kEpiBack: gate and up of a chunk, asked for before its products are complete
        const auto load_chunk = [&](const GemmProblem &p, const TilePos &pos, unsigned c) {
            const unsigned col = pos.n0 + half * (kCols / 2) + 64 * c;
            load_box(box, lane, a.e.gate, a.e.ld_gate, pos.m0 + row0, col, p.m, p.n);
            load_box(box2, lane, a.e.up, a.e.ld_gate, pos.m0 + row0, col, p.m, p.n);
        };
        unsigned acc = 0;
        for (unsigned t; (t = unit_of(a, pair, pairs, acc)) < a.tiles; ++acc) {
            const TilePos pos = tile_pos<kCols>(a, t);
            const GemmProblem &p = a.prob[pos.p];
            const unsigned slot = acc % kSlots, row = pos.m0 + row0;
            const unsigned chunks = chunks_of<kCols, 64>(p, pos, row0, half);
            if (EPI == kEpiBack && chunks) load_chunk(p, pos, 0);
            // kEpiStore to bf16 with a bf16 addend: its share of a chunk is asked for a chunk ahead
            const bool add = EPI == kEpiStore && p.addend && !p.out_f32;
            const auto load_addend = [&](uint4 (&w)[8], unsigned c) {
                load_share(w, lane, static_cast<const __nv_bfloat16 *>(p.addend), p.ld_addend, row, pos.n0 + half * (kCols / 2) + 64 * c, p.m, p.n);
            };
            uint4 share[EPI == kEpiStore ? 8 : 1];
            if constexpr (EPI == kEpiStore) {
                if (add && chunks) load_addend(share, 0);
            }
            long long target = -1;
            float soft_off = 0.0f, soft_by = 0.0f;
            if constexpr (EPI == kEpiLoss || EPI == kEpiSoft) {
                if (chunks && row + lane < p.m) target = a.e.targets[row + lane];
                if (EPI == kEpiSoft && target >= 0 && target < a.e.vocab) {
                    soft_off = -a.e.lse[row + lane] * 1.4426950408889634f;
                    soft_by = a.e.dloss[row + lane];
                } else if (EPI == kEpiSoft) {
                    soft_off = -INFINITY;                          // no gradient
                    target = -1;
                }
            }
            const bool ok = gemm_wait(tfull + 8 * slot, (acc / kSlots) & 1, abort);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const unsigned taddr = tmem + ((unsigned)((warp & 3) * 32) << 16) + slot * BN + half * (kCols / 2);
            const unsigned col0 = pos.n0 + half * (kCols / 2);
            const auto release = [&] {                             // this warp has read its part of the accumulator
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * slot);
            };
            if (!chunks) release();
            if constexpr (EPI == kEpiLoss) {
                constexpr float l = 1.4426950408889634f;
                float top = -INFINITY, sum = 0.0f;
#pragma unroll 1
                for (unsigned c = 0; c < 2 * chunks; ++c) {
                    unsigned r[32];
                    float x[32];
                    tmem_ld32(taddr + 32 * c, r);
                    tmem_ld_wait();
                    if (c + 1 == 2 * chunks) release();
                    const unsigned col = col0 + 32 * c, live = col < p.n ? p.n - col : 0;
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = live >= 32 || j < live ? __uint_as_float(r[j]) : -INFINITY;
                    float m = x[0];
#pragma unroll
                    for (int j = 1; j < 32; ++j) m = fmaxf(m, x[j]);
                    m = fmaxf(m, top);
                    const float base = m == -INFINITY ? 0.0f : m, off = -base * l;
                    float part[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < 32; ++j) part[j & 1] += exp2_fast(fmaf(x[j], l, off));
                    sum = fmaf(sum, exp2_fast((top - base) * l), part[0] + part[1]);
                    top = m;
                    const bool here = target >= col && target < (long long)col + 32;
                    if (__any_sync(0xffffffffu, here)) {
                        float z = 0.0f;
                        const int at = here ? (int)(target - col) : -1;
#pragma unroll
                        for (int j = 0; j < 32; ++j) z = at == j ? x[j] : z;
                        if (here) a.e.loss[row + lane] = z;
                    }
                }
                if (chunks && row + lane < p.m) a.e.partial[(unsigned long long)(col0 / 128) * p.m + row + lane] = make_float2(top, sum);
            } else if constexpr (EPI == kEpiSoft) {
                constexpr float l = 1.4426950408889634f;
#pragma unroll 1
                for (unsigned c = 0; c < chunks; ++c) {
                    const unsigned col = col0 + 64 * c;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        unsigned r[32], w[16];
                        float x[32];
                        tmem_ld32(taddr + 64 * c + 32 * h, r);
                        tmem_ld_wait();
                        if (h == 1 && c + 1 == chunks) release();
                        const long long rel = target - a.e.first - col - 32 * h;
                        const int at = rel >= 0 && rel < 32 ? (int)rel : -1;
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] = exp2_fast(fmaf(__uint_as_float(r[j]), l, soft_off)) * soft_by;
                        if (__any_sync(0xffffffffu, at >= 0)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = at == j ? (exp2_fast(fmaf(__uint_as_float(r[j]), l, soft_off)) - 1.0f) * soft_by : x[j];
                        }
                        pack32(x, w);
                        write_half(box, lane, h, w);
                    }
                    __syncwarp();
                    store_box(box, lane, a.e.hidden, a.e.ld_hidden, row, col, p.m, p.n);
                    __syncwarp();
                }
            } else if (EPI == kEpiStore && p.out_f32) {
#pragma unroll 1
                for (unsigned c = 0; c < 2 * chunks; ++c) {
                    unsigned r[32];
                    float x[32];
                    tmem_ld32(taddr + 32 * c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(r[j]);
                    if (c + 1 == 2 * chunks) release();
                    if (SUM && p.out_f32 == kOutSum) finish_f32<true>(box, lane, x, p, row, row, col0 + 32 * c);
                    else finish_f32<false>(box, lane, x, p, row, pos.split * p.split_rows + row, col0 + 32 * c);
                }
            } else if (EPI == kEpiStore) {
                unsigned r[2][32];
                if (chunks) {
                    tmem_ld32(taddr, r[0]);
                    tmem_ld32(taddr + 32, r[1]);
                }
#pragma unroll 1
                for (unsigned c = 0; c < chunks; ++c) {
                    tmem_ld_wait();
                    if (c + 1 == chunks) release();
                    if constexpr (EPI == kEpiStore) {
                        if (add) {                                 // the addend to rows, where the sums are
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                st_shared(box_piece(box, 4 * i + (lane >> 3), lane & 7), share[i].x, share[i].y, share[i].z, share[i].w);
                            __syncwarp();
                            if (c + 1 < chunks) load_addend(share, c + 1);
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const unsigned piece = box_piece(box, lane, 4 * h + j);
                            float x[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r[h][8 * j + i]);
                            if (add) {
                                const uint4 a4 = ld_shared(piece);
                                const unsigned u[4] = {a4.x, a4.y, a4.z, a4.w};
#pragma unroll
                                for (int i = 0; i < 8; ++i) x[i] += __uint_as_float(i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
                            }
                            st_shared(piece, pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
                        }
                    }
                    __syncwarp();
                    if (c + 1 < chunks) {                          // on their way while this chunk is stored
                        tmem_ld32(taddr + 64 * (c + 1), r[0]);
                        tmem_ld32(taddr + 64 * (c + 1) + 32, r[1]);
                    }
                    store_box(box, lane, static_cast<__nv_bfloat16 *>(p.out), p.ld_out, row, col0 + 64 * c, p.m, p.n);
                    __syncwarp();
                }
            } else if constexpr (EPI == kEpiGate || EPI == kEpiBack) {
#pragma unroll 1
                for (unsigned c = 0; c < chunks; ++c) {
                    const unsigned col = col0 + 64 * c, at = taddr + 64 * c;
                    unsigned w[16], held[2][16];
                    if (EPI == kEpiBack) {
                        asm volatile("cp.async.wait_all;" ::: "memory");
                        __syncwarp();
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        unsigned r[32];
                        float x[32];
                        tmem_ld32(at + 32 * h, r);
                        if (EPI == kEpiGate) {
                            unsigned r2[32];
                            float u[32];
                            tmem_ld32(at + BN / 2 + 32 * h, r2);
                            tmem_ld_wait();
                            if (h == 1 && c + 1 == chunks) release();
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                x[j] = __uint_as_float(r[j]);
                                u[j] = __uint_as_float(r2[j]);
                            }
                            if (a.e.gate) {
                                pack32(x, w);
                                write_half(box2, lane, h, w);
                                pack32(u, held[h]);                // up
                            }
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[j] = activate<ACT, false>(x[j], nullptr) * u[j];
                            pack32(x, w);
                            write_half(box, lane, h, w);           // hidden
                        } else {
                            tmem_ld_wait();
                            if (h == 1 && c + 1 == chunks) release();
#pragma unroll
                            for (int j = 0; j < 4; ++j) {          // a lane's own pieces: gate becomes dgate, up dup
                                const unsigned pg = box_piece(box, lane, 4 * h + j), pu = box_piece(box2, lane, 4 * h + j);
                                const uint4 g4 = ld_shared(pg), u4 = ld_shared(pu);
                                const unsigned gw[4] = {g4.x, g4.y, g4.z, g4.w}, uw[4] = {u4.x, u4.y, u4.z, u4.w};
                                float dg[8], du[8], hid[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const float g = __uint_as_float(i & 1 ? gw[i / 2] & 0xffff0000u : gw[i / 2] << 16);
                                    const float u = __uint_as_float(i & 1 ? uw[i / 2] & 0xffff0000u : uw[i / 2] << 16);
                                    const float dh = __uint_as_float(r[8 * j + i]);
                                    float slope;
                                    const float act = activate<ACT, true>(g, &slope);
                                    dg[i] = dh * u * slope;
                                    du[i] = dh * act;
                                    hid[i] = act * u;
                                }
                                st_shared(pg, pack2(dg[0], dg[1]), pack2(dg[2], dg[3]), pack2(dg[4], dg[5]), pack2(dg[6], dg[7]));
                                st_shared(pu, pack2(du[0], du[1]), pack2(du[2], du[3]), pack2(du[4], du[5]), pack2(du[6], du[7]));
#pragma unroll
                                for (int i = 0; i < 4; ++i) held[h][4 * j + i] = pack2(hid[2 * i], hid[2 * i + 1]);
                            }
                        }
                    }
                    __syncwarp();
                    if (EPI == kEpiGate) {
                        store_box(box, lane, a.e.hidden, a.e.ld_hidden, row, col, p.m, p.n);
                        if (a.e.gate) {
                            store_box(box2, lane, a.e.gate, a.e.ld_gate, row, col, p.m, p.n);
                            __syncwarp();
                            write_half(box, lane, 0, held[0]);
                            write_half(box, lane, 1, held[1]);
                            __syncwarp();
                            store_box(box, lane, a.e.up, a.e.ld_gate, row, col, p.m, p.n);
                        }
                    } else {
                        store_box(box, lane, a.e.dgate, a.e.ld_hidden, row, col, p.m, p.n);
                        store_box(box2, lane, a.e.dup, a.e.ld_hidden, row, col, p.m, p.n);
                        __syncwarp();
                        write_half(box, lane, 0, held[0]);
                        write_half(box, lane, 1, held[1]);
                        __syncwarp();
                        store_box(box, lane, a.e.hidden, a.e.ld_hidden, row, col, p.m, p.n);
                        __syncwarp();
                        if (c + 1 < chunks) load_chunk(p, pos, c + 1);
                    }
                    __syncwarp();
                }
            }
        }
        if (EPI == kEpiBack) asm volatile("cp.async.wait_all;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    cluster_sync_relaxed();               // both CTAs are done with each other's shared and tensor memory
    tc_fence_after();
    if (warp == kIssuer)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(kTmemCols) : "memory");
    if (threadIdx.x == 0 && abort_flag && a.e.status) *a.e.status = DD_STATUS_WAIT_LIMIT;
    if (a.late_wait) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Problems whose K was split: out = [addend +] sum of the splits' float32 slabs, in split order.
struct ReduceJob {
    const float *slabs;
    unsigned splits, m, n, ld;                   // ld: row length of a slab, whole eights
    unsigned long long slab;                     // elements from one split's slab to the next
    unsigned long long end;                      // one past the job's last piece of eight columns
    void *out;
    const void *addend;                          // the output's type, or bf16 (a residual)
    unsigned long long ld_out, ld_addend;
    int out_f32, addend_f32;
};

struct ReduceArgs {
    ReduceJob job[kMaxProblems];
    int count;
};

}  // namespace ddm
