// Attention over packed sequences on tcgen05: scores, weights and gradients of 128 x 128 tiles live in tensor
// memory and registers, nothing of a tile's size goes to global memory.
//
// Roles of a CTA: warps 0-7 (backward 0-15) compute on tiles (a thread owns a row of an accumulator, the lane of
// tensor memory that it can reach, or some columns of it).  Of the four warps behind them one (a lane) has the TMA
// engine fill rings of operand tiles, one (a lane) issues the products, one zeroes rows past a sequence's end, and
// all give registers to the others (a warpgroup does so as a whole).  An operand tile is 128 tokens of one head:
// one or two boxes of 64 elements a row (128-byte swizzle), columns past `dim` filled with zeros by the TMA
// engine.  Tiles may reach past their sequence: scores there are masked, and rows that a product sums over are
// zeroed in shared memory first, since a weight of 0 does not silence a NaN of the neighbour's.
//
// The weights p (and ds) go back into tensor memory as bf16 and are the A operand of the next product from
// there, so they never pass through shared memory.
//
// Every wait is bounded, as in the block's products: on giving up a role raises the abort flag, the roles leave
// their loops, copies and products in flight are awaited (again bounded), tensor memory is freed and the
// status word says DD_STATUS_WAIT_LIMIT.
#pragma once

#include "dd_decoder.h"
#include "dd_tcgen05.cuh"

namespace ddm {

constexpr int kTile = 128;                        // rows of a tile
constexpr int kBoxTile = kTile * 128;             // bytes of a box: 128 rows of 64 bf16
constexpr int kFwdWarps = 8, kBwdWarps = 16;      // that compute; four more follow
constexpr float kLog2e = 1.4426950408889634f;

// Tiles of all sequences, those with most work first.
struct PlanItem {
    unsigned start, len, tile, pad;               // the sequence's first token and length
};

struct Plan {
    unsigned count, pad[3];
    PlanItem item[1];
};

struct HeadRows {
    __nv_bfloat16 *data;
    unsigned long long ld_token, ld_head;
};

struct AttnArgs {
    CUtensorMap q, k, v, d_o;
    const Plan *plan;                             // null: one sequence of all tokens
    unsigned tokens, tiles;                       // tiles of that sequence
    unsigned heads, group, dim;                   // query heads, query heads per head of keys
    float scale;
    int causal, expire;
    unsigned cluster;                             // CTAs that share a tile of keys in the last kernel
    HeadRows o, dq, dk, dv;
    HeadRows q_rows, k_rows, v_rows, do_rows;     // inputs once more, for operands that are kept in tensor memory
    float *lse;                                   // [heads][tokens]
    float *delta;                                 // [heads][tokens]: sum_j p_ij dp_ij
    int *status;
};

// ---- instructions ------------------------------------------------------------------------------

__device__ __forceinline__ void tma_load_heads(unsigned dst, const CUtensorMap *map, int x, int head, int token, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(head), "r"(token), "r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_st16(unsigned addr, const unsigned (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
           "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void init_bar(unsigned bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void arrive_bar(unsigned bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}

// Descriptors of operand tiles: the upper half is the same for all (128-byte swizzle, groups of 8 rows every
// 1024 bytes), the lower half is the address and, where rows are K, the step to the next 64 columns (in a cluster
// an address has the CTA's rank in its upper bits, which do not belong there).  They are kept as halves, and
// everything they are made of is warp-uniform, because the products are fed from uniform registers: with 64-bit
// descriptors put together for each product from per-lane values, issuing one took 115 cycles and not the 64 that
// it runs for.
constexpr unsigned kDescUpper = (1024 / 16) | (1u << 14) | (2u << 29);

// K contiguous: step k covers elements 16 k .. of every row.
__device__ __forceinline__ unsigned desc_rows(unsigned tile, int k)
{
    return ((tile >> 4 & 0x3fff) | (1u << 16)) + (k >> 2) * (kBoxTile / 16) + (k & 3) * 2;
}

// Rows are K (the tile's columns are N): step k covers rows 16 k .., the next 64 columns are one box on.
__device__ __forceinline__ unsigned desc_cols(unsigned tile, int k)
{
    return ((tile >> 4 & 0x3fff) | ((unsigned)(kBoxTile / 16) << 16)) + k * 128;
}

// float32 accumulators, bf16 operands, M = 128; b_mn: B's rows are K.
__host__ __device__ constexpr unsigned attn_idesc(int n, bool b_mn)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? 1u << 16 : 0u) | ((unsigned)(n / 8) << 17) | ((unsigned)(kTile / 16) << 24);
}

// d (+)= A B^T over the tiles' DP columns.
template <int DP>
__device__ __forceinline__ void mma_rows(unsigned d, unsigned a, unsigned b)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        asm volatile("{\n .reg .pred p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %4};\n mov.b64 b, {%2, %4};\n setp.ne.b32 p, %5, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}"
                     :: "r"(d), "r"(desc_rows(a, k)), "r"(desc_rows(b, k)), "r"(attn_idesc(kTile, false)), "r"(kDescUpper), "r"(k ? 1u : 0u) : "memory");
}

// The same with A in tensor memory, two of a row's elements per column.  Both operands in shared memory ask for
// 8 KB a product of 64 cycles, all that it gives; B alone leaves room for the copies.
template <int DP>
__device__ __forceinline__ void mma_held(unsigned d, unsigned a, unsigned b)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        asm volatile("{\n .reg .pred p;\n .reg .b64 b;\n mov.b64 b, {%2, %4};\n setp.ne.b32 p, %5, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}"
                     :: "r"(d), "r"(a + k * 8), "r"(desc_rows(b, k)), "r"(attn_idesc(kTile, false)), "r"(kDescUpper), "r"(k ? 1u : 0u) : "memory");
}

// d (+)= A B with A (128 x 128 bf16, two of a row's elements per column) in tensor memory, every 32 of its columns
// STEP columns of it on, and B a tile's 128 rows of DP columns.
template <int DP, int STEP>
__device__ __forceinline__ void mma_weights(unsigned d, unsigned a, unsigned b, bool accumulate)
{
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k)
        asm volatile("{\n .reg .pred p;\n .reg .b64 b;\n mov.b64 b, {%2, %4};\n setp.ne.b32 p, %5, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}"
                     :: "r"(d), "r"(a + (k >> 1) * STEP + (k & 1) * 8), "r"(desc_cols(b, k)), "r"(attn_idesc(DP, true)), "r"(kDescUpper),
                        "r"(k ? 1u : (unsigned)accumulate) : "memory");
}

// One operand tile: tokens token .. token + 127 of a head.
template <int DP>
__device__ __forceinline__ void load_tile(unsigned dst, const CUtensorMap *map, int head, int token, unsigned bar)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c) tma_load_heads(dst + c * kBoxTile, map, 64 * c, head, token, bar);
}

// The whole warp's wait, with one answer for all.
__device__ __forceinline__ bool warp_wait(unsigned bar, unsigned parity, volatile int *abort)
{
    return __all_sync(0xffffffffu, gemm_wait(bar, parity, abort));
}

// Zeros to the rows from `first` on, by one warp, which reports it to `bar`.
template <int DP>
__device__ __forceinline__ void zero_rows(unsigned tile, unsigned first, int lane, unsigned bar)
{
#pragma unroll
    for (int c = 0; c < DP / 64; ++c)
        for (unsigned r = first + (lane >> 3); r < kTile; r += 4)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" :: "r"(tile + c * kBoxTile + r * 128 + (lane & 7) * 16), "r"(0) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) arrive_bar(bar);
}

// Where four columns of a row of 2 DP float32 sums are kept: eight rows' pieces of one column lie in different banks.
template <int DP>
__device__ __forceinline__ unsigned sums_piece(unsigned base, unsigned row, unsigned piece) { return base + row * (2 * DP * 4) + ((piece ^ (row & 7)) << 4); }

// Columns col .. col + 31 of a row (null: zeros), and to 16 columns of tensor memory, as operand A; dim is a multiple of 8.
__device__ __forceinline__ void load_row32(const __nv_bfloat16 *row, unsigned col, unsigned dim, unsigned (&w)[16])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 x = row && col + 8 * j < dim ? __ldcg(reinterpret_cast<const uint4 *>(row + col + 8 * j)) : make_uint4(0u, 0u, 0u, 0u);
        w[4 * j] = x.x;
        w[4 * j + 1] = x.y;
        w[4 * j + 2] = x.z;
        w[4 * j + 3] = x.w;
    }
}

__device__ __forceinline__ void hold_row32(unsigned at, const __nv_bfloat16 *row, unsigned col, unsigned dim)
{
    unsigned w[16];
    load_row32(row, col, dim, w);
    tmem_st16(at, w);
}

// 32 columns of a row, times `by`, to bf16 columns col .. of an output row; dim is a multiple of 8.
__device__ __forceinline__ void store_row32(__nv_bfloat16 *row, unsigned col, unsigned dim, const unsigned (&r)[32], float by)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (col + 8 * j >= dim) return;
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack2(__uint_as_float(r[8 * j + 2 * i]) * by, __uint_as_float(r[8 * j + 2 * i + 1]) * by);
        *reinterpret_cast<uint4 *>(row + col + 8 * j) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// 2^x of two numbers on the multiply-add pipe: x = n + f with n the nearest integer (the sum with 1.5 2^23 rounds to it
// and holds it in its low bits), 2^f by a polynomial on [-1/2, 1/2], n into the exponent.  The coefficients are
// a minimax fit of the relative error with 2^0 = 1 held (a weighted least-squares iteration): 2.9e-6 in float32, far
// below the bf16 rounding that follows.  Below -127 the result is 0, near -126.5 it is off by less than 2^-126.
// A NaN ends as the largest float, since the last sum is one of integers: as a bf16 operand that is an infinity, and in ds
// the row's delta, which has weights of the other kind in it, is NaN.
__device__ __forceinline__ float2 exp2_poly(float2 x)
{
    constexpr float c[] = {1.0f, 0.6931241750717163f, 0.24024099111557007f, 0.055906426161527634f, 0.009582852944731712f}, kRound = 12582912.0f;
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-127.0f));               // a NaN goes on
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-127.0f));
    const float2 t = __fadd2_rn(x, make_float2(kRound, kRound)), n = __fadd2_rn(t, make_float2(-kRound, -kRound)),
                 f = __ffma2_rn(n, make_float2(-1.0f, -1.0f), x);
    float2 p = make_float2(c[4], c[4]);
#pragma unroll
    for (int i = 3; i >= 0; --i) p = __ffma2_rn(p, f, make_float2(c[i], c[i]));
    return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)), __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}

// 2^(x c + off) of two scores.
__device__ __forceinline__ float2 exp2_pair(unsigned x0, unsigned x1, float c, float2 off, bool poly = false)
{
    const float2 x = __ffma2_rn(make_float2(__uint_as_float(x0), __uint_as_float(x1)), make_float2(c, c), off);
    return poly ? exp2_poly(x) : make_float2(exp2_fast(x.x), exp2_fast(x.y));
}

// Maximum of three; a NaN among them is the result.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// p (dp - delta) of two, as bf16.
__device__ __forceinline__ unsigned ds_pair(float2 p, unsigned dp0, unsigned dp1, float2 minus_delta)
{
    const float2 d = __fmul2_rn(p, __fadd2_rn(make_float2(__uint_as_float(dp0), __uint_as_float(dp1)), minus_delta));
    return pack2(d.x, d.y);
}

// The tile of block-wide index `i`: most work first.  False: there is none.
__device__ __forceinline__ bool plan_item(const AttnArgs &a, unsigned i, PlanItem &item)
{
    if (!a.plan) {
        item = PlanItem{0u, a.tokens, a.tiles - 1 - i, 0u};
        return i < a.tiles;
    }
    if (i >= a.plan->count) return false;
    const uint4 w = __ldcg(reinterpret_cast<const uint4 *>(&a.plan->item[i]));
    item = PlanItem{w.x, w.y, w.z, 0u};
    return true;
}

// What all kernels begin and end with.
struct AttnShared {
    unsigned long long bars[31];
    int abort_flag;
    unsigned tmem_base;
};

template <int WARPS>
__device__ __forceinline__ unsigned attn_begin(AttnShared &sh, const AttnArgs &a, int warp)
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (threadIdx.x == 32 * WARPS)
        for (const CUtensorMap *m : {&a.q, &a.k, &a.v, a.delta ? &a.d_o : &a.q}) asm volatile("prefetch.tensormap [%0];" :: "l"(m) : "memory");
    if (warp == WARPS + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_addr(&sh.tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // only now: a launch behind this one would take the tensor memory and wait for this one's end
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    return __shfl_sync(0xffffffffu, sh.tmem_base, 0);
}

template <int WARPS>
__device__ __forceinline__ void attn_end(AttnShared &sh, const AttnArgs &a, int warp, unsigned tmem)
{
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == WARPS + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    if (threadIdx.x == 0 && sh.abort_flag && a.status) *a.status = DD_STATUS_WAIT_LIMIT;
}

// A launch has 168 registers for each of 384 threads (forward) or 96 for each of 640 (backward): 208 for two
// warpgroups and 88 for the third, or 104 for four and 64 for the fifth, are as many.
template <int WARPS>
__device__ __forceinline__ void more_registers()
{
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(WARPS == kFwdWarps ? 208 : 104));
}
template <int WARPS>
__device__ __forceinline__ void fewer_registers()
{
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(WARPS == kFwdWarps ? 88 : 64));
}

// Lane 0 of a warp reports that the warp is done with (or has written) its part of tensor memory.
__device__ __forceinline__ void warp_arrive(unsigned bar, int lane)
{
    tc_fence_before();
    __syncwarp();
    if (lane == 0) arrive_bar(bar);
}

// ---- turns -----------------------------------------------------------------------------------------

// Forward and in dq's kernel, a CTA that has issued the last copy of a block's work takes the place of a block that has not been
// launched yet (the hardware hands them out, most work first): the next operands arrive while the last rows are
// written, and a CTA's own beginning is paid once.

// The block that a launch would have started next, which then does not start; ~0: none.  Not to be asked again after that.
__device__ __forceinline__ unsigned take_block(unsigned reply, unsigned bar, unsigned parity, volatile int *abort)
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" :: "r"(reply), "r"(bar) : "memory");
    if (!mbar_wait_bounded(bar, parity)) {
        *abort = 1;
        return ~0u;
    }
    unsigned block = ~0u;
    asm volatile("{\n .reg .b128 r;\n .reg .pred p;\n .reg .b32 y, z, w;\n ld.shared.b128 r, [%1];\n"
                 " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n"
                 " @p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, y, z, w}, r;\n}" : "+r"(block) : "r"(reply) : "memory");
    return block;
}

// What comes after every other turn, as the copies' role found it; no length: nothing.
struct Turns {
    uint4 reply;
    PlanItem item[2];
};

// After turn k: the next block's item, its head in `pad`, for all roles; without length if there is none.
__device__ __forceinline__ PlanItem publish_next(Turns &turns, const AttnArgs &a, unsigned k, unsigned reply_full, unsigned next_full, volatile int *abort)
{
    const unsigned block = take_block(smem_addr(&turns.reply), reply_full, k & 1, abort);
    PlanItem item{0u, 0u, 0u, 0u};
    if (block != ~0u && plan_item(a, block / a.heads, item)) item.pad = block % a.heads;
    else item.len = 0;
    turns.item[k & 1] = item;
    arrive_bar(next_full + 8 * (k & 1));
    return item;
}

__device__ __forceinline__ bool read_next(const Turns &turns, unsigned k, unsigned next_full, PlanItem &item, volatile int *abort)
{
    if (!gemm_wait(next_full + 8 * (k & 1), k >> 1 & 1, abort)) return false;
    item = turns.item[k & 1];
    return true;
}

// The same by a whole warp, which reports that it has read: whether there is anything.
__device__ __forceinline__ bool warp_next(const Turns &turns, unsigned k, unsigned next_full, unsigned next_empty, PlanItem &item, int lane, volatile int *abort)
{
    if (!__all_sync(0xffffffffu, read_next(turns, k, next_full, item, abort))) return false;
    __syncwarp();
    if (lane == 0) arrive_bar(next_empty + 8 * (k & 1));
    return item.len != 0;
}

// ---- forward ---------------------------------------------------------------------------------------

// A CTA takes 256 query rows of a head: tile 0 and tile 1 of 128, warps 0-3 and 4-7.  They share every tile
// of keys and values, and while the weights of one are computed the products of the other run.
// For 128 columns a tile's two products and its exponentials both take 1024 cycles of their units, so the kernel is bound
// by both and by the steps between them: each is busy for 60 % of the time (8192 tokens, 8 heads of 128, causal).
// 16384 tokens: 420-430 us, 1290 TFLOP/s of products, on a cool GPU, 490 in a long run, where the power limit
// takes the clock to 1.5 GHz; 16 computing warps took 517, two issuing threads the same as one.
// Taking turns: 16384 tokens, 16 heads on 4 of 128, documents of 128 / 256 / 1024 / 4096 tokens: 84 -> 67, 83 -> 61, 112 -> 91, 253 -> 237 us.
// Every token of two documents of 4096 seeing all: 242 us, 264 in a long run.  168 registers at launch hold a thread's state but
// for 96 bytes in local memory (64 columns: 140).
__host__ __device__ constexpr int fwd_stages(int dp) { return dp == 128 ? 4 : 6; }
__host__ __device__ constexpr unsigned fwd_smem_bytes(int dp) { return 1024 + (2 + fwd_stages(dp)) * kTile * dp * 2; }

// 256 rows of a head and the tiles of keys that each half needs.
struct FwdWork {
    unsigned start, len, head, row0, n0, n1, n;
    bool cut;                                     // the last tile of values goes past the sequence's end
};

__device__ __forceinline__ FwdWork fwd_work(const AttnArgs &a, const PlanItem &item)
{
    FwdWork w;
    w.start = item.start;
    w.len = item.len;
    w.head = item.pad;
    w.row0 = item.tile * 2 * kTile;
    const unsigned all = (item.len + kTile - 1) / kTile, t0 = item.tile * 2;
    w.n0 = a.causal ? t0 + 1 : all;
    w.n1 = item.len - w.row0 <= kTile ? 0 : a.causal ? t0 + 2 : all;
    w.n = w.n0 > w.n1 ? w.n0 : w.n1;
    w.cut = item.len - (w.n - 1) * kTile < kTile;
    return w;
}

template <int DP>
__global__ void __launch_bounds__(32 * (kFwdWarps + 4), 1)
attention_forward_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr int kStages = fwd_stages(DP);
    constexpr unsigned kBytes = kTile * DP * 2;
    extern __shared__ unsigned char smem_raw[];
    __shared__ alignas(16) AttnShared sh;
    __shared__ alignas(16) Turns turns;
    const unsigned smem = (smem_addr(smem_raw) + 1023u) & ~1023u, ring = smem + 2 * kBytes;
    const unsigned bar = smem_addr(sh.bars), q_full = bar, full = bar + 8, empty = full + 8 * kStages, s_full = empty + 8 * kStages,
                   p_full = s_full + 16, o_full = p_full + 16, drain = o_full + 16, clean = drain + 8, tail = clean + 16,
                   q_empty = tail + 16, next_full = q_empty + 8, next_empty = next_full + 16, reply_full = next_empty + 16;
    static_assert(sizeof sh.bars >= 8 * (2 * kStages + 16), "barriers");
    volatile int *abort = &sh.abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        init_bar(q_full, 1);
        for (int s = 0; s < kStages; ++s) {
            init_bar(full + 8 * s, 1);
            init_bar(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            init_bar(s_full + 8 * s, 1);
            init_bar(p_full + 8 * s, 4);
            init_bar(o_full + 8 * s, 1);
            init_bar(clean + 8 * s, 1);
            init_bar(tail + 8 * s, 1);
            init_bar(next_full + 8 * s, 1);
            init_bar(next_empty + 8 * s, kFwdWarps + 2);
        }
        init_bar(drain, 1);
        init_bar(q_empty, 1);
        init_bar(reply_full, 1);
    }
    const unsigned tmem = attn_begin<kFwdWarps>(sh, a, warp);
    // all so far without waiting for the launch before
    asm volatile("griddepcontrol.wait;" ::: "memory");
    PlanItem item;
    if (!plan_item(a, blockIdx.x / a.heads, item)) {
        attn_end<kFwdWarps>(sh, a, warp, tmem);
        return;
    }
    item.pad = blockIdx.x % a.heads;
    const unsigned kS = tmem, kO = tmem + 2 * kTile;                         // scores of tile t at kS + 128 t, sums at kO + DP t
    if (warp >= kFwdWarps) {
        fewer_registers<kFwdWarps>();
        if (warp == kFwdWarps && elect_one()) {
            unsigned it = 0, k = 0, cuts = 0;                                // keys 0, values 0, keys 1, ...; turns; cut tiles
            for (;; ++k) {
                const FwdWork w = fwd_work(a, item);
                const int token = (int)(w.start + w.row0), hk = (int)(w.head / a.group);
                if (k && !gemm_wait(q_empty, (k - 1) & 1, abort)) break;
                mbar_arrive_expect_tx(q_full, (w.n1 ? 2 : 1) * kBytes + (a.expire && k == 0 ? 16u : 0u));
                load_tile<DP>(smem, &a.q, (int)w.head, token, q_full);
                if (w.n1) load_tile<DP>(smem + kBytes, &a.q, (int)w.head, token + kTile, q_full);
                unsigned i = 0;
                for (; i < 2 * w.n; ++i, ++it) {
                    const unsigned s = it % kStages;
                    if ((it >= kStages && !gemm_wait(empty + 8 * s, (it / kStages - 1) & 1, abort)) || *abort) break;
                    const bool cut = i == 2 * w.n - 1 && w.cut;
                    if (cut) arrive_bar(full + 8 * s);
                    // two such tiles at most are under way: the third one's queries wait for the first one's products
                    const unsigned to = cut ? tail + 8 * (cuts++ & 1) : full + 8 * s;
                    mbar_arrive_expect_tx(to, kBytes);
                    load_tile<DP>(ring + s * kBytes, i & 1 ? &a.v : &a.k, hk, (int)(w.start + (i >> 1) * kTile), to);
                }
                if (i < 2 * w.n || (k >= 2 && !gemm_wait(next_empty + 8 * (k & 1), (k >> 1) - 1 & 1, abort))) {
                    ++k;
                    break;
                }
                item = publish_next(turns, a, k, reply_full, next_full, abort);
                if (!item.len) {
                    ++k;
                    break;
                }
            }
            mbar_wait_bounded(q_full, (k - 1) & 1);
            for (unsigned j = it > kStages ? it - kStages : 0; j < it; ++j) mbar_wait_bounded(full + 8 * (j % kStages), (j / kStages) & 1);
            for (unsigned j = cuts > 2 ? cuts - 2 : 0; j < cuts; ++j) mbar_wait_bounded(tail + 8 * (j & 1), j >> 1 & 1);
        } else if (warp == kFwdWarps + 1 && elect_one()) {
            const auto tile_of = [&](unsigned it) { return ring + it % kStages * kBytes; };
            const auto ready = [&](unsigned it) { return gemm_wait(full + 8 * (it % kStages), (it / kStages) & 1, abort); };
            unsigned it = 0, cuts = 0, past0 = 0, past1 = 0;                 // tiles, cut ones, and those of each half, before this turn
            bool ok = true;
            for (unsigned k = 0; ok; ++k) {
                const FwdWork w = fwd_work(a, item);
                ok = gemm_wait(q_full, k & 1, abort) && ready(it);
                if (ok) {
                    tc_fence_after();
                    mma_rows<DP>(kS, smem, tile_of(it));
                    umma_commit(s_full);
                    if (w.n1) {
                        mma_rows<DP>(kS + kTile, smem + kBytes, tile_of(it));
                        umma_commit(s_full + 8);
                    }
                    umma_commit(empty + 8 * (it % kStages));
                    if (w.n == 1) umma_commit(q_empty);
                }
                for (unsigned j = 0; ok && j < w.n; ++j) {
                    const bool last = j + 1 == w.n;
                    ok = ready(it + 2 * j + 1) && (!last || !w.cut || gemm_wait(clean + 8 * (cuts & 1), cuts >> 1 & 1, abort)) && (last || ready(it + 2 * j + 2));
#pragma unroll 1
                    for (unsigned t = 0; ok && t < 2; ++t) {
                        const unsigned mine = t ? w.n1 : w.n0;
                        if (j >= mine) continue;
                        ok = gemm_wait(p_full + 8 * t, (t ? past1 : past0) + j & 1, abort);
                        if (!ok) break;
                        tc_fence_after();
                        mma_weights<DP, 16>(kO + t * DP, kS + t * kTile, tile_of(it + 2 * j + 1), j != 0);
                        if (j + 1 < mine) {
                            // behind the product that reads the weights, whose place the scores take
                            mma_rows<DP>(kS + t * kTile, smem + t * kBytes, tile_of(it + 2 * j + 2));
                            umma_commit(s_full + 8 * t);
                        } else {
                            umma_commit(o_full + 8 * t);
                        }
                    }
                    if (ok) {
                        umma_commit(empty + 8 * ((it + 2 * j + 1) % kStages));
                        if (!last) umma_commit(empty + 8 * ((it + 2 * j + 2) % kStages));
                        if (j + 2 == w.n) umma_commit(q_empty);
                    }
                }
                it += 2 * w.n;
                past0 += w.n0;
                past1 += w.n1;
                cuts += w.cut;
                ok = ok && read_next(turns, k, next_full, item, abort);
                if (!ok || !item.len) break;
                arrive_bar(next_empty + 8 * (k & 1));
            }
            umma_commit(drain);                                              // no product may be in flight when tensor memory is freed
            mbar_wait_bounded(drain, 0);
        } else if (warp == kFwdWarps + 2) {
            // the last tile of values reports here and not to the issuer
            unsigned it = 0, cuts = 0, k = 0;
            do {
                const FwdWork w = fwd_work(a, item);
                it += 2 * w.n;
                if (!w.cut) continue;
                if (!warp_wait(tail + 8 * (cuts & 1), cuts >> 1 & 1, abort)) break;
                zero_rows<DP>(ring + (it - 1) % kStages * kBytes, w.len - (w.n - 1) * kTile, lane, clean + 8 * (cuts & 1));
                ++cuts;
            } while (warp_next(turns, k++, next_full, next_empty, item, lane, abort));
        }
    } else {
        more_registers<kFwdWarps>();
        const int t = warp >> 2;
        const unsigned at = (unsigned)((warp & 3) * 32) << 16, s_at = kS + t * kTile + at, o_at = kO + t * DP + at;
        const float c = a.scale * kLog2e;
        unsigned past = 0, outs = 0, k = 0;                                  // tiles and turns with any before this turn
        bool ok = true;
        do {
            const FwdWork w = fwd_work(a, item);
            const unsigned mine = t ? w.n1 : w.n0, row = w.row0 + t * kTile + (warp & 3) * 32 + lane;
            float top = -INFINITY, base = 0.0f, sum = 0.0f;                  // base: top, as the exponents use it
            for (unsigned j = 0; j < mine; ++j) {
                ok = warp_wait(s_full + 8 * t, past + j & 1, abort);
                if (!ok) break;
                tc_fence_after();
                unsigned r[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_ld32(s_at + 32 * i, r[i]);
                tmem_ld_wait();
                const unsigned end = a.causal && row + 1 < w.len ? row + 1 : w.len, live = end > j * kTile ? end - j * kTile : 0;
                if (__any_sync(0xffffffffu, live < kTile)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (32 * i + k >= live) r[i][k] = 0xff800000u;        // -infinity
                }
                float m[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    m[i] = max3(__uint_as_float(r[i][0]), __uint_as_float(r[i][1]), i ? -INFINITY : top);
#pragma unroll
                    for (int k = 2; k < 32; k += 2) m[i] = max3(m[i], __uint_as_float(r[i][k]), __uint_as_float(r[i][k + 1]));
                }
                const float now = max3(m[0], m[1], max3(m[2], m[3], -INFINITY));
                // A row's sums are moved to a larger maximum only when it has grown by more than 2^8: until then the
                // weights stay below 2^8, exact in float32 and as far from the end of bf16's range.
                const bool grown = !((now - top) * c <= 8.0f);
                if (__any_sync(0xffffffffu, grown)) {
                    const float next = !grown ? base : now == -INFINITY ? 0.0f : now;
                    if (j) {
                        const float by = grown && top != -INFINITY ? exp2_fast((base - next) * c) : 1.0f;      // (sums of nothing are 0)
                        sum *= by;
#pragma unroll 1
                        for (int i = 0; i < DP / 16; ++i) {
                            unsigned o[16];
                            tmem_ld16(o_at + 16 * i, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * by);
                            tmem_st16(o_at + 16 * i, o);
                        }
                    }
                    top = grown ? now : top;
                    base = next;
                }
                const float off = -base * c;
                float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    unsigned u[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 p = exp2_pair(r[h][2 * k], r[h][2 * k + 1], c, make_float2(off, off));
                        part[k & 1] = __fadd2_rn(part[k & 1], p);
                        u[k] = pack2(p.x, p.y);
                    }
                    tmem_st16(s_at + 16 * h, u);
                }
                sum += (part[0].x + part[0].y) + (part[1].x + part[1].y);
                tmem_st_wait();
                warp_arrive(p_full + 8 * t, lane);
            }
            if (mine && ok) ok = warp_wait(o_full + 8 * t, outs++ & 1, abort);
            if (mine && ok) {
                tc_fence_after();
                const unsigned long long token = w.start + row;
                const float by = 1.0f / sum;
                __nv_bfloat16 *o = a.o.data + token * a.o.ld_token + w.head * a.o.ld_head;
#pragma unroll
                for (int i = 0; i < DP / 32; ++i) {
                    unsigned u[32];
                    tmem_ld32(o_at + 32 * i, u);
                    tmem_ld_wait();
                    if (row < w.len) store_row32(o, 32 * i, a.dim, u, by);
                }
                if (a.lse && row < w.len) a.lse[(unsigned long long)w.head * a.tokens + token] = fmaf(base, a.scale, logf(sum));
            }
            past += mine;
        } while (ok && warp_next(turns, k++, next_full, next_empty, item, lane, abort));
    }
    attn_end<kFwdWarps>(sh, a, warp, tmem);
}

// ---- backward --------------------------------------------------------------------------------------

// The pairs whose weights are polynomials, three of eight: all weights of a tile are wanted at one time, and the
// special function unit makes 16 a clock and SM (8192 tokens, 16 heads of 64: 636 -> 604 us, of 128 0.6 % less; in
// the forward pass, whose two tiles take turns, the same costs 3-7 %).
__host__ __device__ constexpr bool poly_pair(int k) { return 0x4a >> (k % 8) & 1; }

// What a backward CTA has in shared memory: seven tiles, and the rest.
struct BwdShared {
    AttnShared sh;
    alignas(16) float row[4][kTile];
    Turns turns;
};
constexpr unsigned bwd_smem_bytes(int dp) { return 7 * kTile * dp * 2 + sizeof(BwdShared); }
static_assert(bwd_smem_bytes(128) <= 227 * 1024, "shared memory of an SM");

// 128 rows of a head.
struct DqWork {
    unsigned start, len, head, row0, n;
    bool cut;                                     // the last tile of keys goes past the sequence's end
};

__device__ __forceinline__ DqWork dq_work(const AttnArgs &a, const PlanItem &item)
{
    const unsigned n = a.causal ? item.tile + 1 : (item.len + kTile - 1) / kTile;
    return {item.start, item.len, item.pad, item.tile * kTile, n, item.len - (n - 1) * kTile < kTile};
}

// dq of 128 query rows of a head.  Every four warps take 32 columns of the scores' rows.  Scores of the
// next tile of keys are made as soon as those of this one are in registers.
// Two launches (this and the next kernel) form the scores twice, which costs 7 products of a tile instead of 5,
// but no gradient is added to by several CTAs: no atomics, no float32 copy of dq in memory.
//
// delta_i = sum_j p_ij dp_ij is d_o_i . o_i, but o's rounding to bf16 is then in it, and where few keys share a row's
// weight dp - delta is a small difference.  So rows whose keys are all in one tile, the short sequences and the
// beginnings of long ones, take the sum itself and leave it for the next launch (two keys: gradients within
// 0.25 % instead of 0.75 %).
//
// Bound, like the next kernel, by the products (512 cycles each of a pair of tiles: 3 here, 4 there, 59-61 % of the
// time) and by the steps from one to the next.  8192 tokens, 8 heads of 128, causal: 190 and 240 us at 1.5 GHz; 16384
// tokens: 1455-1475 us with delta, 1310 TFLOP/s of executed products.  Taking turns, with the next turn's queries on
// their way: 16384 tokens, 16 heads on 4 of 128, documents of 128 / 1024 / 4096 tokens, the whole backward pass 285 -> 242,
// 405 -> 367, 877 -> 864 us; 8192 tokens, 8 heads on 2: 403 -> 393.
template <int DP>
__global__ void __launch_bounds__(32 * (kBwdWarps + 4), 1)
attention_dq_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr unsigned kBytes = kTile * DP * 2;
    constexpr bool kHeld = DP == 64;              // tensor memory has room for more operands

    extern __shared__ __align__(1024) unsigned char smem_tiles[];
    BwdShared &rest = *reinterpret_cast<BwdShared *>(smem_tiles + 7 * kBytes);
    AttnShared &sh = rest.sh;
    float (&shares)[4][kTile] = rest.row;         // of a row's delta
    const unsigned smem = smem_addr(smem_tiles), sdo = smem, sk = smem + kBytes, sv = smem + 4 * kBytes;
    const unsigned bar = smem_addr(sh.bars), k_full = bar, k_empty = bar + 24, v_full = bar + 48, v_empty = bar + 72, do_full = bar + 96,
                   s_full = bar + 104, dp_full = bar + 112, dq_full = bar + 120, drain = bar + 128, clean = bar + 136, tail = bar + 144,
                   q_full = bar + 152, s_read = bar + 160, ds_full = bar + 168, sum_full = bar + 176,
                   next_full = bar + 184, next_empty = bar + 200, reply_full = bar + 216, turned = bar + 224, clean2 = bar + 232, tail2 = bar + 240;
    const auto clean_of = [&](unsigned c) { return c & 1 ? clean2 : clean; };
    const auto tail_of = [&](unsigned c) { return c & 1 ? tail2 : tail; };
    volatile int *abort = &sh.abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        for (int i = 0; i < 19; ++i) init_bar(bar + 8 * i, 1);
        for (int i = 19; i < 23; ++i) init_bar(bar + 8 * i, kBwdWarps);
        for (int i = 23; i < 31; ++i) init_bar(bar + 8 * i, i == 25 || i == 26 ? kBwdWarps + 2 : 1);
    }
    const unsigned tmem = attn_begin<kBwdWarps>(sh, a, warp);
    // all so far without waiting for the launch before
    asm volatile("griddepcontrol.wait;" ::: "memory");
    PlanItem item;
    if (!plan_item(a, blockIdx.x / a.heads, item)) {
        attn_end<kBwdWarps>(sh, a, warp, tmem);
        return;
    }
    item.pad = blockIdx.x % a.heads;
    // the queries, and with 64 columns their gradients' operand d_o as well, are held in tensor memory
    const unsigned kS = tmem, kP = tmem + kTile, kDs = tmem + 2 * kTile, kDq = kDs + 64, kQ = tmem + 448, kDo = tmem + 384;

    if (warp >= kBwdWarps) {
        fewer_registers<kBwdWarps>();
        if (warp == kBwdWarps && elect_one()) {
            unsigned it = 0, k = 0, cuts = 0;                                // keys 0, values 0, keys 1, ...; turns; cut tiles
            for (;; ++k) {
                const DqWork w = dq_work(a, item);
                const int hk = (int)(w.head / a.group);
                // all products of the turn before but the last are issued
                if (k && !gemm_wait(turned, (k - 1) & 1, abort)) break;
                if (!kHeld) {
                    mbar_arrive_expect_tx(do_full, kBytes);
                    load_tile<DP>(sdo, &a.d_o, (int)w.head, (int)(w.start + w.row0), do_full);
                }
                unsigned i = 0;
                for (; i < 2 * w.n; ++i, ++it) {
                    const unsigned j = it >> 1, s = j % 3, full = (it & 1 ? v_full : k_full) + 8 * s, empty = (it & 1 ? v_empty : k_empty) + 8 * s;
                    if ((j >= 3 && !gemm_wait(empty, (j / 3 - 1) & 1, abort)) || *abort) break;
                    const bool cut = i == 2 * w.n - 2 && w.cut;
                    if (cut) arrive_bar(full);
                    // two such tiles at most are under way: the third one's turn waits for the first one's products
                    const unsigned to = cut ? tail_of(cuts++) : full;
                    mbar_arrive_expect_tx(to, kBytes + (a.expire && it == 0 ? 16u : 0u));
                    load_tile<DP>((it & 1 ? sv : sk) + s * kBytes, it & 1 ? &a.v : &a.k, hk, (int)(w.start + (i >> 1) * kTile), to);
                }
                if (i < 2 * w.n || (k >= 2 && !gemm_wait(next_empty + 8 * (k & 1), (k >> 1) - 1 & 1, abort))) {
                    ++k;
                    break;
                }
                item = publish_next(rest.turns, a, k, reply_full, next_full, abort);
                if (!item.len) {
                    ++k;
                    break;
                }
            }
            for (unsigned c = cuts > 2 ? cuts - 2 : 0; c < cuts; ++c) mbar_wait_bounded(tail_of(c), c >> 1 & 1);
            if (!kHeld) mbar_wait_bounded(do_full, (k - 1) & 1);
            for (unsigned i = it > 6 ? it - 6 : 0; i < it; ++i)
                mbar_wait_bounded((i & 1 ? v_full : k_full) + 8 * ((i >> 1) % 3), (i >> 1) / 3 & 1);
        } else if (warp == kBwdWarps + 1 && elect_one()) {
            unsigned past = 0, cuts = 0;                                     // tiles and cut ones before this turn
            DqWork w;
            const auto scores = [&](unsigned j) {
                const unsigned g = past + j;
                if (!gemm_wait(k_full + 8 * (g % 3), g / 3 & 1, abort)) return false;
                if (j + 1 == w.n && w.cut && !gemm_wait(clean_of(cuts), cuts >> 1 & 1, abort)) return false;
                tc_fence_after();
                mma_held<DP>(kS, kQ, sk + g % 3 * kBytes);
                umma_commit(s_full);
                return true;
            };
            const auto weights = [&](unsigned j) {                           // dp of tile j
                const unsigned g = past + j;
                if (!gemm_wait(v_full + 8 * (g % 3), g / 3 & 1, abort)) return false;
                tc_fence_after();
                if (kHeld) mma_held<DP>(kP, kDo, sv + g % 3 * kBytes);
                else mma_rows<DP>(kP, sdo, sv + g % 3 * kBytes);
                umma_commit(dp_full);
                umma_commit(v_empty + 8 * (g % 3));
                if (j + 1 == w.n) umma_commit(turned);
                return true;
            };
            bool ok = true;
            for (unsigned k = 0; ok; ++k) {
                w = dq_work(a, item);
                ok = gemm_wait(q_full, k & 1, abort) && (kHeld || gemm_wait(do_full, k & 1, abort));
                bool more = true;
                // each round makes the scores and dp of tile j and the product that tile j - 1 ends with
                for (unsigned j = 0; ok && more; ++j) {
                    const unsigned i = past + j - 1;
                    more = j < w.n;
                    if (j) ok = gemm_wait(s_read, i & 1, abort);
                    if (ok && more) ok = scores(j);
                    if (ok && j) ok = gemm_wait(ds_full, i & 1, abort);
                    if (ok && more) ok = weights(j);
                    if (!ok || !j) continue;
                    tc_fence_after();
                    mma_weights<DP, 16>(kDq, kDs, sk + i % 3 * kBytes, j != 1);
                    umma_commit(k_empty + 8 * (i % 3));
                    umma_commit(dq_full);
                }
                past += w.n;
                cuts += w.cut;
                ok = ok && read_next(rest.turns, k, next_full, item, abort);
                if (!ok || !item.len) break;
                arrive_bar(next_empty + 8 * (k & 1));
            }
            umma_commit(drain);
            mbar_wait_bounded(drain, 0);
        } else if (warp == kBwdWarps + 2) {
            // the last tile of keys, which dq sums over, reports here and not to the issuer
            unsigned past = 0, cuts = 0, k = 0;
            do {
                const DqWork w = dq_work(a, item);
                past += w.n;
                if (!w.cut) continue;
                if (!warp_wait(tail_of(cuts), cuts >> 1 & 1, abort)) break;
                zero_rows<DP>(sk + (past - 1) % 3 * kBytes, w.len - (w.n - 1) * kTile, lane, clean_of(cuts));
                ++cuts;
            } while (warp_next(rest.turns, k++, next_full, next_empty, item, lane, abort));
        }
    } else {
        more_registers<kBwdWarps>();
        const unsigned share = warp >> 2, at = (unsigned)((warp & 3) * 32) << 16;
        const float c = a.scale * kLog2e;
        unsigned past = 0, sums = 0, k = 0;                                  // tiles and turns of one tile before this turn
        unsigned held[16];                                                   // the next turn's queries
        float off, delta;
        // what a turn begins with, asked for before the last one ends (d_o's rows, where they are held too, would take
        // registers that spill: 64 columns, 4 documents of 4096 tokens 687 -> 694 us)
        const auto fetch = [&](const DqWork &w) {
            const unsigned row = w.row0 + (warp & 3) * 32 + lane;
            const unsigned long long token = w.start + row, stat = (unsigned long long)w.head * a.tokens + token;
            const bool here = row < w.len;
            off = here ? -a.lse[stat] * kLog2e : 0.0f;
            delta = here && w.n > 1 ? a.delta[stat] : 0.0f;
            if (32 * share >= DP) return;
            load_row32(here ? a.q_rows.data + token * a.q_rows.ld_token + w.head * a.q_rows.ld_head : nullptr, 32 * share, a.dim, held);
        };
        bool ok = true, more;
        fetch(dq_work(a, item));
        do {
            const DqWork w = dq_work(a, item);
            const unsigned row = w.row0 + (warp & 3) * 32 + lane;
            const unsigned long long token = w.start + row, stat = (unsigned long long)w.head * a.tokens + token;
            // columns below `end` count; a token that sees itself alone has ds = 0
            const unsigned end = row >= w.len ? 0 : a.causal ? row + 1 : w.len;
            if (32 * share < DP) {
                tmem_st16(kQ + at + 16 * share, held);
                if (kHeld)
                    hold_row32(kDo + at + 16 * share, row < w.len ? a.do_rows.data + token * a.do_rows.ld_token + w.head * a.do_rows.ld_head : nullptr,
                               32 * share, a.dim);
                tmem_st_wait();
            }
            warp_arrive(q_full, lane);
            for (unsigned j = 0; j < w.n; ++j) {
                ok = warp_wait(s_full, past + j & 1, abort);
                if (!ok) break;
                tc_fence_after();
                unsigned r[32], u[16];
                float2 p[16];
                tmem_ld32(kS + at + 32 * share, r);
                tmem_ld_wait();
                warp_arrive(s_read, lane);
#pragma unroll
                for (int k = 0; k < 16; ++k) p[k] = exp2_pair(r[2 * k], r[2 * k + 1], c, make_float2(off, off), poly_pair(k));
                ok = warp_wait(dp_full, past + j & 1, abort);
                if (!ok) break;
                tc_fence_after();
                tmem_ld32(kP + at + 32 * share, r);
                tmem_ld_wait();
                const unsigned first = j * kTile + 32 * share, live = end == 1 || end <= first ? 0 : end - first;
                if (w.n == 1) {
                    float sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (k < live) sum = fmaf(k & 1 ? p[k / 2].y : p[k / 2].x, __uint_as_float(r[k]), sum);
                    shares[share][row - w.row0] = sum;
                    __syncwarp();
                    if (lane == 0) arrive_bar(sum_full);
                    ok = warp_wait(sum_full, sums++ & 1, abort);
                    if (!ok) break;
                    delta = (shares[0][row - w.row0] + shares[1][row - w.row0]) + (shares[2][row - w.row0] + shares[3][row - w.row0]);
                    if (share == 0 && row < w.len) a.delta[stat] = delta;
                }
                if (__any_sync(0xffffffffu, live < 32)) {
                    // masked: a weight of 0, and a dp that may be NaN past the sequence's end counts as delta
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (k >= live) {
                            r[k] = __float_as_uint(delta);
                            (k & 1 ? p[k / 2].y : p[k / 2].x) = 0.0f;
                        }
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) u[k] = ds_pair(p[k], r[2 * k], r[2 * k + 1], make_float2(-delta, -delta));
                if (j) {                              // the product that reads the last tile's ds, long done by now
                    ok = warp_wait(dq_full, past + j - 1 & 1, abort);
                    if (!ok) break;
                    tc_fence_after();
                }
                tmem_st16(kDs + at + 16 * share, u);
                tmem_st_wait();
                warp_arrive(ds_full, lane);
            }
            more = ok && warp_next(rest.turns, k++, next_full, next_empty, item, lane, abort);
            if (more) fetch(dq_work(a, item));
            if (ok) ok = warp_wait(dq_full, past + w.n - 1 & 1, abort);
            if (ok && 32 * share < DP) {
                tc_fence_after();
                unsigned u[32];
                tmem_ld32(kDq + at + 32 * share, u);
                tmem_ld_wait();
                if (row < w.len) store_row32(a.dq.data + token * a.dq.ld_token + w.head * a.dq.ld_head, 32 * share, a.dim, u, a.scale);
            }
            past += w.n;
        } while (ok && more);
    }
    attn_end<kBwdWarps>(sh, a, warp, tmem);
}

// dk and dv of 128 rows of a head of keys, over the query heads that share it and their tiles of queries.
// Scores are made transposed (rows are keys), so that the weights are the A operand of both products as they lie.
// Products and weights alternate on the same places: dv of a tile, then the next tile's scores, run while ds
// is computed; dk and the next dp while the next weights are.
//
// The first keys of a long sequence are read by all its queries, in every query head of the group: where that is
// much beside what an SM has to do, the CTAs of a cluster take equal parts of those tiles and add their sums up through
// distributed shared memory, in rank order.
//
// 96 registers are few for a tile's statistics, scores and both weights: 52 bytes a thread are kept in local memory and 212 read
// back (64 columns: 44 and 192).
template <int DP>
__global__ void __launch_bounds__(32 * (kBwdWarps + 4), 1)
attention_dkv_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr unsigned kBytes = kTile * DP * 2;
    constexpr bool kHeld = DP == 64;              // tensor memory has room for more operands

    extern __shared__ __align__(1024) unsigned char smem_tiles[];
    BwdShared &rest = *reinterpret_cast<BwdShared *>(smem_tiles + 7 * kBytes);
    AttnShared &sh = rest.sh;
    float (*stats)[2][kTile] = reinterpret_cast<float (*)[2][kTile]>(rest.row);   // of every other tile: -lse log2(e) and -delta of its queries
    const unsigned smem = smem_addr(smem_tiles), sk = smem, sv = smem + kBytes, sq = smem + 2 * kBytes, sdo = smem + 5 * kBytes;
    const unsigned bar = smem_addr(sh.bars), q_full = bar, q_empty = bar + 24, do_full = bar + 48, do_empty = bar + 64, kv_full = bar + 80,
                   s_full = bar + 88, dp_full = bar + 96, done = bar + 104, drain = bar + 112, q_clean = bar + 120, do_clean = bar + 144,
                   q_tail = bar + 160, do_tail = bar + 184, p_full = bar + 200, ds_full = bar + 208, st_full = bar + 216;
    volatile int *abort = &sh.abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sh.abort_flag = 0;
        for (int i = 0; i < 25; ++i) init_bar(bar + 8 * i, 1);
        if (kHeld) init_bar(kv_full, kBwdWarps);
        init_bar(p_full, kBwdWarps);
        init_bar(ds_full, kBwdWarps);
        init_bar(st_full, 8);
        init_bar(st_full + 8, 8);
    }
    const unsigned tmem = attn_begin<kBwdWarps>(sh, a, warp);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned kv_heads = a.heads / a.group;
    PlanItem item;
    const unsigned rank = blockIdx.x % a.cluster, unit = blockIdx.x / a.cluster;
    if (!plan_item(a, unit / kv_heads, item)) {                              // (the cluster as a whole)
        attn_end<kBwdWarps>(sh, a, warp, tmem);
        return;
    }
    const unsigned hk = unit % kv_heads, all = (item.len + kTile - 1) / kTile;
    const unsigned tile = all - 1 - item.tile, row0 = tile * kTile;          // early keys are read by most queries
    // tiles of queries: `per` of each head that shares the keys, of which this CTA takes n from `start` on
    const unsigned i0 = a.causal ? tile : 0, per = all - i0, total = per * a.group;
    const unsigned start = (unsigned)((unsigned long long)total * rank / a.cluster), n = (unsigned)((unsigned long long)total * (rank + 1) / a.cluster) - start;
    const auto head_of = [&](unsigned j) { return hk * a.group + (start + j) / per; };
    const auto tile_of = [&](unsigned j) { return i0 + (start + j) % per; };
    const auto is_last = [&](unsigned j) { return tile_of(j) == all - 1; };
    const unsigned kS = tmem, kP = tmem + kTile, kDv = tmem + 2 * kTile, kDk = kDv + DP, kK = tmem + 384, kV = kK + 32;
    // tiles of queries whose rows past the sequence's end are zeroed: the last one of each head
    const unsigned last = item.len - (all - 1) * kTile;

    if (warp >= kBwdWarps) {
        fewer_registers<kBwdWarps>();
        if (warp == kBwdWarps && elect_one()) {
            if (!kHeld) {
                mbar_arrive_expect_tx(kv_full, 2 * kBytes);
                load_tile<DP>(sk, &a.k, (int)hk, (int)(item.start + row0), kv_full);
                load_tile<DP>(sv, &a.v, (int)hk, (int)(item.start + row0), kv_full);
            }
            unsigned it = 0, tails = 0, cuts = 0;
            for (; it < 2 * n; ++it) {                                       // queries 0, gradients 0, queries 1, ...
                const unsigned j = it >> 1, slots = it & 1 ? 2 : 3, s = j % slots, full = (it & 1 ? do_full : q_full) + 8 * s,
                               empty = (it & 1 ? do_empty : q_empty) + 8 * s;
                const int h = (int)head_of(j), token = (int)(item.start + tile_of(j) * kTile);
                if ((j >= slots && !gemm_wait(empty, (j / slots - 1) & 1, abort)) || *abort) break;
                const bool cut = last < kTile && is_last(j);
                const unsigned to = cut ? (it & 1 ? do_tail : q_tail) + 8 * s : full;
                if (cut) arrive_bar(full);
                mbar_arrive_expect_tx(to, kBytes + (a.expire && it == 0 ? 16u : 0u));
                load_tile<DP>((it & 1 ? sdo : sq) + s * kBytes, it & 1 ? &a.d_o : &a.q, h, token, to);
                if (cut) tails ^= 1u << (it & 1 ? 4 + s : s), cuts |= 1u << (it & 1 ? 4 + s : s);
            }
            for (unsigned s = 0; s < 6; ++s)                                 // the last tail of each slot
                if (cuts >> s & 1) mbar_wait_bounded(s < 4 ? q_tail + 8 * s : do_tail + 8 * (s - 4), ~tails >> s & 1);
            if (!kHeld) mbar_wait_bounded(kv_full, 0);
            for (unsigned i = it > 6 ? it - 6 : 0; i < it; ++i) {
                const unsigned j = i >> 1, slots = i & 1 ? 2 : 3;
                if (j + slots >= (it + 1 - (i & 1)) / 2) mbar_wait_bounded((i & 1 ? do_full : q_full) + 8 * (j % slots), (j / slots) & 1);
            }
        } else if (warp == kBwdWarps + 1 && elect_one()) {
            unsigned tails = 0;                                              // parities: of the queries' slots, from bit 4 on the gradients'

            // the product of the keys (values) with tile j of queries (their gradients)
            const auto product = [&](unsigned j, bool second) {
                const unsigned slots = second ? 2 : 3, s = j % slots, t = (second ? sdo : sq) + s * kBytes;
                if (!gemm_wait((second ? do_full : q_full) + 8 * s, j / slots & 1, abort)) return false;
                if (last < kTile && is_last(j)) {
                    const unsigned bit = second ? 4 + s : s;
                    if (!gemm_wait((second ? do_clean : q_clean) + 8 * s, tails >> bit & 1, abort)) return false;
                    tails ^= 1u << bit;
                }
                tc_fence_after();
                if (kHeld) mma_held<DP>(second ? kP : kS, second ? kV : kK, t);
                else mma_rows<DP>(second ? kP : kS, second ? sv : sk, t);
                umma_commit(second ? dp_full : s_full);
                return true;
            };
            bool ok = gemm_wait(kv_full, 0, abort), more = n > 0;
            // each round ends tile j - 1 and makes the scores and dp of tile j
            for (unsigned j = 0; ok && more; ++j) {
                const unsigned i = j - 1;
                more = j < n;
                if (j) {
                    ok = gemm_wait(p_full, i & 1, abort);
                    if (!ok) break;
                    tc_fence_after();
                    mma_weights<DP, 32>(kDv, kS, sdo + (i & 1) * kBytes, i != 0);
                    umma_commit(do_empty + 8 * (i & 1));
                }
                if (more) ok = product(j, false);
                if (ok && j) {
                    ok = gemm_wait(ds_full, i & 1, abort);
                    if (!ok) break;
                    tc_fence_after();
                    mma_weights<DP, 32>(kDk, kP, sq + i % 3 * kBytes, i != 0);
                    umma_commit(q_empty + 8 * (i % 3));
                }
                if (ok && more) ok = product(j, true);
            }
            if (ok) umma_commit(done);
            umma_commit(drain);
            mbar_wait_bounded(drain, 0);
        } else if (warp == kBwdWarps + 2 && last < kTile) {
            // the last tiles report here and not to the issuer
            unsigned tails = 0;
            for (unsigned j = all - 1 - tile_of(0); j < n; j += per) {
                const unsigned s = j % 3, d = j & 1;
                if (!warp_wait(q_tail + 8 * s, tails >> s & 1, abort)) break;
                zero_rows<DP>(sq + s * kBytes, last, lane, q_clean + 8 * s);
                if (!warp_wait(do_tail + 8 * d, tails >> (4 + d) & 1, abort)) break;
                zero_rows<DP>(sdo + d * kBytes, last, lane, do_clean + 8 * d);
                tails ^= 1u << s | 1u << (4 + d);
            }
        }
        if (a.cluster > 1) {                      // as the other warps do
            __syncwarp();
            cluster_sync();
            cluster_sync();
        }
    } else {
        more_registers<kBwdWarps>();
        const unsigned share = warp >> 2, at = (unsigned)((warp & 3) * 32) << 16, row = row0 + (warp & 3) * 32 + lane;
        const float c = a.scale * kLog2e;
        // the first 256 threads fetch the statistics: lse or delta of one query of tile j
        const auto stat = [&](unsigned j) {
            const unsigned i = tile_of(j) * kTile + (threadIdx.x & 127), h = head_of(j);
            if (share >= 2 || j >= n || i >= item.len) return 0.0f;
            const unsigned long long where = (unsigned long long)h * a.tokens + item.start + i;
            return share ? -a.delta[where] : -a.lse[where] * kLog2e;
        };
        float next = stat(0);
        if (kHeld) {
            if (32 * share < DP) {
                const unsigned long long token = item.start + row;
                const bool here = row < item.len;
                hold_row32(kK + at + 16 * share, here ? a.k_rows.data + token * a.k_rows.ld_token + hk * a.k_rows.ld_head : nullptr, 32 * share, a.dim);
                hold_row32(kV + at + 16 * share, here ? a.v_rows.data + token * a.v_rows.ld_token + hk * a.v_rows.ld_head : nullptr, 32 * share, a.dim);
                tmem_st_wait();
            }
            warp_arrive(kv_full, lane);
        }
        bool ok = true;
        for (unsigned j = 0; j < n; ++j) {
            if (share < 2) {
                stats[j & 1][share][threadIdx.x & 127] = next;
                __syncwarp();
                if (lane == 0) arrive_bar(st_full + 8 * (j & 1));
                if (j + 1 < n) next = stat(j + 1);
            }
            const unsigned q0 = tile_of(j) * kTile + 32 * share;          // the first of this warp's 32 queries
            // queries from `from` to `to` count
            const unsigned to = item.len > q0 ? item.len - q0 : 0, from = a.causal && row > q0 ? row - q0 : 0;
            const bool masked = __any_sync(0xffffffffu, to < 32 || from > 0) || (a.causal && q0 == 0);
            // (every other tile's statistics have a barrier of their own: with one, those of tile j + 1 could all be there
            // before a late warp has seen that those of tile j are, and it would wait for tile j + 2's)
            ok = gemm_wait(st_full + 8 * (j & 1), j >> 1 & 1, abort) && gemm_wait(s_full, j & 1, abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const float4 *offs = reinterpret_cast<const float4 *>(&stats[j & 1][0][32 * share]), *deltas = offs + kTile / 4;
            unsigned r[32], w[16];
            float2 p[16];
            tmem_ld32(kS + at + 32 * share, r);
            tmem_ld_wait();
            if (masked) {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (k < from || k >= to) r[k] = 0xff800000u;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 x = offs[k];
                p[2 * k] = exp2_pair(r[4 * k], r[4 * k + 1], c, make_float2(x.x, x.y), poly_pair(2 * k));
                p[2 * k + 1] = exp2_pair(r[4 * k + 2], r[4 * k + 3], c, make_float2(x.z, x.w), poly_pair(2 * k + 1));
                w[2 * k] = pack2(p[2 * k].x, p[2 * k].y);
                w[2 * k + 1] = pack2(p[2 * k + 1].x, p[2 * k + 1].y);
            }
            tmem_st16(kS + at + 32 * share, w);
            tmem_st_wait();
            warp_arrive(p_full, lane);
            ok = warp_wait(dp_full, j & 1, abort);
            if (!ok) break;
            tc_fence_after();
            tmem_ld32(kP + at + 32 * share, r);
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 x = deltas[k];
                w[2 * k] = ds_pair(p[2 * k], r[4 * k], r[4 * k + 1], make_float2(x.x, x.y));
                w[2 * k + 1] = ds_pair(p[2 * k + 1], r[4 * k + 2], r[4 * k + 3], make_float2(x.z, x.w));
            }
            if (masked) {
                // whatever dp was: past the sequence's end it may be NaN; a token that sees itself alone has ds = 0
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (k < from || k >= to || (k == 0 && (a.causal ? q0 == 0 : item.len == 1))) w[k / 2] &= k & 1 ? 0x0000ffffu : 0xffff0000u;
            }
            tmem_st16(kP + at + 32 * share, w);
            tmem_st_wait();
            warp_arrive(ds_full, lane);
        }
        if (ok) ok = warp_wait(done, 0, abort);
        if (ok) {
            tc_fence_after();
            const bool key = share >= 2;
            const HeadRows &out = key ? a.dk : a.dv;
            __nv_bfloat16 *o = out.data + (unsigned long long)(item.start + row) * out.ld_token + hk * out.ld_head;
#pragma unroll
            for (int i = 0; i < DP / 64; ++i) {
                unsigned w[32];
                const unsigned col = (share & 1) * (DP / 2) + 32 * i;
                tmem_ld32((key ? kDk : kDv) + at + col, w);
                tmem_ld_wait();
                if (a.cluster > 1) {              // to where the operands were
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        if (!n) w[k] = w[k + 1] = w[k + 2] = w[k + 3] = 0u;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(sums_piece<DP>(smem, row - row0, ((key ? DP : 0) + col + k) / 4)),
                                     "r"(w[k]), "r"(w[k + 1]), "r"(w[k + 2]), "r"(w[k + 3]) : "memory");
                    }
                } else if (row < item.len) {
                    store_row32(o, col, a.dim, w, key ? a.scale : 1.0f);
                }
            }
        }
        if (a.cluster > 1) {
            __syncwarp();
            cluster_sync();
            // this CTA's share of the rows, in pieces of four columns
            const unsigned rows = kTile / a.cluster, first = rank * rows;
#pragma unroll 2
            for (unsigned i = threadIdx.x; i < rows * (2 * DP / 4); i += 32 * kBwdWarps) {
                const unsigned r = first + i / (2 * DP / 4), piece = i % (2 * DP / 4), col = 4 * piece;
                float4 y[8];
#pragma unroll
                for (int other = 0; other < 8; ++other)
                    if (other < a.cluster) y[other] = ld_cluster4(sums_piece<DP>(smem, r, piece), other);
                float4 x = y[0];
#pragma unroll
                for (int other = 1; other < 8; ++other)
                    if (other < a.cluster) x.x += y[other].x, x.y += y[other].y, x.z += y[other].z, x.w += y[other].w;
                const bool key = col >= DP;
                const unsigned c4 = key ? col - DP : col;
                const HeadRows &out = key ? a.dk : a.dv;
                const float by = key ? a.scale : 1.0f;
                if (row0 + r < item.len && c4 < a.dim)
                    *reinterpret_cast<uint2 *>(out.data + (unsigned long long)(item.start + row0 + r) * out.ld_token + hk * out.ld_head + c4) =
                        make_uint2(pack2(x.x * by, x.y * by), pack2(x.z * by, x.w * by));
            }
            __syncwarp();
            cluster_sync();                           // nobody reads this CTA's sums any more
        }
    }
    attn_end<kBwdWarps>(sh, a, warp, tmem);
}

// ---- plan ------------------------------------------------------------------------------------------

constexpr unsigned kPlanKeys = 4096, kPlanThreads = 256;

// The tiles of `rows` tokens of all sequences, ordered by their place in the sequence, last first (by counting;
// the order among tiles of one place does not matter to any result).
struct PlanArgs {
    const int *offsets;
    unsigned sequences, tokens, rows;
    Plan *plan;                                   // null: none wanted
    int *status;
};

__device__ __forceinline__ void make_plan(const PlanArgs &a)
{
    __shared__ unsigned count[kPlanKeys], warp_sum[kPlanThreads / 32];
    const int *offsets = a.offsets;
    const unsigned sequences = a.sequences, tokens = a.tokens, rows = a.rows;
    Plan *plan = a.plan;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    bool good = offsets[0] >= 0;
    for (unsigned s = threadIdx.x; s < sequences; s += kPlanThreads)
        good = good && offsets[s] <= offsets[s + 1] && (unsigned)offsets[s + 1] <= tokens;
    for (unsigned i = threadIdx.x; i < kPlanKeys; i += kPlanThreads) count[i] = 0;
    if (!__syncthreads_and(good)) {
        if (threadIdx.x == 0) {
            plan->count = 0;
            if (a.status) *a.status = DD_STATUS_BAD_OFFSETS;
        }
        return;
    }
    unsigned shift = 0;
    while ((tokens / rows) >> shift >= kPlanKeys) ++shift;
    const auto key = [&](unsigned tile) { return kPlanKeys - 1 - (tile >> shift); };
    const auto each = [&](auto &&f) {
        for (unsigned s = warp; s < sequences; s += kPlanThreads / 32) {
            const unsigned start = (unsigned)offsets[s], len = (unsigned)offsets[s + 1] - start;
            for (unsigned t = lane; (unsigned long long)t * rows < len; t += 32) f(start, len, t);
        }
    };
    each([&](unsigned, unsigned, unsigned t) { atomicAdd(&count[key(t)], 1u); });
    __syncthreads();
    unsigned mine[kPlanKeys / kPlanThreads], sum = 0;
    for (unsigned i = 0; i < kPlanKeys / kPlanThreads; ++i) sum += mine[i] = count[threadIdx.x * (kPlanKeys / kPlanThreads) + i];
    unsigned before = sum;
    for (int d = 1; d < 32; d *= 2) {
        const unsigned x = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += x;
    }
    if (lane == 31) warp_sum[warp] = before;
    __syncthreads();
    unsigned base = 0;
    for (unsigned w = 0; w < warp; ++w) base += warp_sum[w];
    base += before - sum;
    if (threadIdx.x == kPlanThreads - 1) plan->count = base + sum;
    for (unsigned i = 0; i < kPlanKeys / kPlanThreads; ++i) {
        count[threadIdx.x * (kPlanKeys / kPlanThreads) + i] = base;
        base += mine[i];
    }
    __syncthreads();
    each([&](unsigned start, unsigned len, unsigned t) { plan->item[atomicAdd(&count[key(t)], 1u)] = PlanItem{start, len, t, 0u}; });
}

__global__ void __launch_bounds__(kPlanThreads)
attention_plan_kernel(const PlanArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    make_plan(a);
}

// ---- delta ---------------------------------------------------------------------------------------

// delta = d_o . o of every row of every head; LANES = lanes of a row, 8 elements each.  With offsets the first block
// makes the plan instead.
struct DeltaArgs {
    const __nv_bfloat16 *o, *d_o;
    unsigned long long o_token, o_head, d_token, d_head;
    float *delta;
    unsigned tokens, heads, dim;
};

template <int LANES>
__global__ void __launch_bounds__(kPlanThreads)
attention_delta_kernel(const DeltaArgs a, const PlanArgs plan)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const unsigned planning = plan.plan ? 1 : 0;
    if (blockIdx.x < planning) {
        make_plan(plan);
        return;
    }
    const unsigned long long i = ((unsigned long long)(blockIdx.x - planning) * 256 + threadIdx.x) / LANES, rows = (unsigned long long)a.tokens * a.heads;
    const unsigned col = threadIdx.x % LANES * 8;
    const unsigned long long t = i / a.heads;
    const unsigned h = (unsigned)(i - t * a.heads);
    float sum = 0.0f;
    if (i < rows && col < a.dim) {
        const uint4 x = *reinterpret_cast<const uint4 *>(a.o + t * a.o_token + h * a.o_head + col),
                    y = *reinterpret_cast<const uint4 *>(a.d_o + t * a.d_token + h * a.d_head + col);
        const unsigned u[4] = {x.x, x.y, x.z, x.w}, v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sum = fmaf(__uint_as_float(u[k] << 16), __uint_as_float(v[k] << 16), sum);
            sum = fmaf(__uint_as_float(u[k] & 0xffff0000u), __uint_as_float(v[k] & 0xffff0000u), sum);
        }
    }
#pragma unroll
    for (int s = LANES / 2; s; s /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (i < rows && col == 0) a.delta[(unsigned long long)h * a.tokens + t] = sum;
}

}  // namespace ddm
