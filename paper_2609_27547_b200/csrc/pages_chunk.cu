// Softmax attention of many query rows over paged keys and values (include/ebrl_pages.h), bf16, on tcgen05: out = softmax(scale q k^T) v.
//
//   Item = (sequence, piece of it, key/value head, 128 or 256 query rows), one CTA; rows are (token, member) pairs of the heads that share a key/value head.
//   Keys and values come in tiles of 128 tokens.  A CTA has one tile of 128 rows, and an SM two such CTAs, or two tiles that share every key and value; either
//   way the tensor core works on one tile while the other's softmax is taken.
//     softmax    four warps for each tile: one thread per row, so that statistics need no shuffles.  Scores come from tensor memory, weights go
//                back to it in place (they are the A operand of the second product; values are its B operand as they lie, tokens along the contraction)
//     copies     one warp: TMA boxes of up to 128 tokens of a page, keys and values in turn through one ring; pages that are not there lie outside the
//                tensor map, which reads zeros
//     products   one warp: S = Q K^T of a tile is issued behind the O += P V that reads its last weights, so that with two tiles the order is
//                PV_A(j) QK_A(j + 1) PV_B(j) QK_B(j + 1)
//   Weights are first taken against the reference as it stands, and a tile's maximum is looked for only where a row's weights would add up to more than 2^16 (or there
//   is no reference yet): bf16 keeps its 8 bits whatever their size.  Where they do so against the largest score, too (very many tokens), the reference goes 2^8 beyond
//   it, so that sums of weights times values never exceed 2^16 times the values.  Sums in tensor memory are then rescaled by the softmax threads themselves, which know from
//   S(j) being there that PV(j - 1) is done.
//   Tokens that no row may see are masked in S; their value rows are set to zero in shared memory before the product, so that what stands there (NaN in a
//   row nobody wrote) does not meet a weight of zero.
//   All waits are bounded: when one runs out the CTA notes it, marks its pieces, lets its copies land, frees tensor memory and returns.
//
//   What bounds it: 4 x 2000 - 2048 new tokens over 8 - 16 k x 16 heads of 128 take 755 us, 1.1 PFLOP/s.  The products alone (softmax skipped) take 630: a
//   128 x 128 x 128 product from shared memory reads 128 bytes a cycle, all there are, and the copies want a quarter of that, too.  The rest is
//   the softmax: its 128 exponentials a row keep the unit busy for 2064 of the 3500 cycles that two tiles take.
//   Tried and not kept (same case): weights handed over in halves of 64 tokens 757, products of 64 tokens with their own barriers 884, two threads per row
//   765, the scores read twice in short loops 830, a quarter / half of the exponentials by polynomial 870 / 980, registers split 208 / 88 795.
#include "pages_internal.h"
#include "f32x2.cuh"
#include "ptx_helpers.cuh"

#include <algorithm>
#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>

namespace ebrl {
namespace pg {

namespace {

using namespace ptx;

constexpr unsigned FULL = 0xffffffffu;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int ROWS = 128, KEYS = 128;

template <int HD, int TILES> struct Shape {
    static constexpr int THREADS = (4 * TILES + 2) * 32;
    static constexpr int PER_SM = 3 - TILES;                         // CTAs
    static constexpr int SWZ = HD >= 64 ? 128 : 64;                  // bytes of a swizzled row
    static constexpr int HALVES = HD * 2 / SWZ;                      // column blocks of a row
    static constexpr int HALF = 128 * SWZ;                           // bytes of 128 rows of one
    static constexpr int TILE = HALVES * HALF;
    static constexpr int STAGES = TILES == 2 ? 5 : (HD == 128 ? 2 : 4);
    static constexpr int BARS = 2 * STAGES + 4 * TILES;
    static constexpr int SMEM = (TILES + STAGES) * TILE + 8 * BARS + 16 + 1024;
    static constexpr int O_COL = TILES * KEYS;                       // tensor memory: the scores of each tile, then their sums
    static constexpr int COLS = TILES * 256;
};

__device__ int wait_status;       // EBRL_ERR_TIMEOUT once a wait ran out; one on each device

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, uint32_t nbytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(nbytes) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *tm, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// True in one lane of the warp, always the same one.
__device__ __forceinline__ bool elect()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)   // A from tensor memory
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
#define TMEM_REGS32 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31"
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {" TMEM_REGS32 "}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {" TMEM_REGS32 "};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                   "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
                   "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(a) : "memory");
}
#define TMEM_REGS16 "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15"
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {" TMEM_REGS16 "};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                   "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors.  Queries and keys: rows of SWZ bytes along the contracted index, groups of 8 rows one behind the other.
// Values: rows are tokens, the contracted index; a row's SWZ bytes run along the columns, further column blocks follow at LEAD bytes.
template <int HD, bool VALUES> __device__ __forceinline__ uint64_t smem_desc(uint32_t addr)
{
    uint64_t d = (uint64_t)((addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(VALUES ? Shape<HD, 1>::HALF >> 4 : 1) << 16;
    d |= (uint64_t)(8 * Shape<HD, 1>::SWZ >> 4) << 32;
    d |= (uint64_t)1 << 46;                                  // descriptor version of sm_100
    d |= (uint64_t)(Shape<HD, 1>::SWZ == 128 ? 2 : 4) << 61;    // 128- or 64-byte swizzle
    return d;
}
// kind::f16: fp32 accumulate, bf16 A and B, M = 128; B along the contracted index, or (VALUES) along its columns.
__host__ __device__ constexpr uint32_t instr_desc(int N, bool values)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((values ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
}

// An item and the tokens lo .. hi (lo a multiple of 128) that some row of it sees.
struct Item { int row, tab, part, m, len, R, r0, tiles, kh, piece, lo, hi, seen, n_kv; };   // (seen: no row sees a token below)

template <int TILES> __device__ __forceinline__ Item item_of(const AttendArgs &a, const AttendSeqs &sq, int x)
{
    constexpr int ITEM = TILES * ROWS;
    Item it;
    const AttendSeq seq = sq.s[find_seq(sq.n, x, [&](int i) { return sq.s[i].item; })];
    it.m = seq.m; it.len = seq.len; it.row = seq.row; it.part = seq.part; it.tab = seq.tab;
    it.R = it.m * a.G;
    const int RT = (it.R + ITEM - 1) / ITEM;
    int rest = x - seq.item;
    const int kh = rest % a.g.kvh; rest /= a.g.kvh;
    const int rt = RT - 1 - rest % RT;                        // the last rows see most
    it.kh = kh; it.piece = rest / RT;
    it.r0 = rt * ITEM;
    const int r1 = min(it.R, it.r0 + ITEM);
    it.tiles = r1 - it.r0 > ROWS ? 2 : 1;
    const Span span = seen_by(it.len, it.m, a.G, it.r0, r1, a.causal, a.window, a.split, it.piece);
    it.lo = span.lo / KEYS * KEYS; it.hi = span.hi; it.seen = span.lo;
    it.n_kv = it.hi > it.lo ? (it.hi - it.lo + KEYS - 1) / KEYS : 0;
    return it;
}

// A CTA's items: there and back through the list, which begins with the longest.
__device__ __forceinline__ int item_at(int k) { return k * (int)gridDim.x + (k & 1 ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x); }

// Mask words of an item's tokens, 32 of them (8 tiles) held by the lanes of a warp, the next 32 on their way.
struct Words {
    const int *tab;
    const AttendArgs *a;
    int seen, hi, base;
    unsigned now, next, full;        // full: which of the 32 words are all ones
    __device__ __forceinline__ unsigned fetch(int w) const
    {
        unsigned bits = 0;
        if (w * WORD < hi) {
            const int page = tab[(w * WORD) >> a->g.t_shift];
            if ((unsigned)page < (unsigned)a->p.n_pages) {
                bits = *reinterpret_cast<const unsigned *>(a->p.pool + (size_t)page * a->g.bytes + a->g.mask + ((w * WORD & (a->g.T - 1)) >> 3));
                if (w * WORD + WORD > hi) bits &= FULL >> (w * WORD + WORD - hi);
                if (w * WORD < seen) bits = w * WORD + WORD > seen ? bits & (FULL << (seen - w * WORD)) : 0;
            }
        }
        return bits;
    }
    __device__ __forceinline__ void start(const AttendArgs &args, const int *table, const Item &it, int lane)
    {
        a = &args; tab = table; seen = it.seen; hi = it.hi; base = it.lo / WORD;
        now = fetch(base + lane);
        next = fetch(base + 32 + lane);
        full = __ballot_sync(FULL, now == FULL);
    }
    // Moves on to tile j; called for j = 0, 1, 2, ... by all lanes.  Whether each of its tokens is seen by some row.
    __device__ __forceinline__ bool whole(int j, int lane)
    {
        if (j && (j & 7) == 0) {
            base += 32;
            now = next;
            full = __ballot_sync(FULL, now == FULL);
            next = fetch(base + 32 + lane);
        }
        return ((full >> ((j & 7) * 4)) & 15u) == 15u;
    }
    __device__ __forceinline__ unsigned word(int j, int i) const { return __shfl_sync(FULL, now, (j & 7) * 4 + i); }
};

// Where a wait ran out: the CTA's pieces (some may have been finished) are marked, so that the join leaves their rows alone.
template <int TILES> __device__ __noinline__ void mark_unfinished(const AttendArgs &a, const AttendSeqs &sq)
{
    for (int k = 0, x; (x = item_at(k)) < sq.items; ++k) {
        const Item it = item_of<TILES>(a, sq, x);
        for (int row = it.r0 + threadIdx.x; it.part >= 0 && row < min(it.R, it.r0 + TILES * ROWS); row += blockDim.x)
            a.part_ml[2 * (((size_t)it.part + (size_t)it.piece * it.m + row / a.G) * a.heads + it.kh * a.G + row % a.G)] = __int_as_float(0x7fffffff);
    }
}

template <int HD, int TILES>
__global__ void __launch_bounds__(Shape<HD, TILES>::THREADS, Shape<HD, TILES>::PER_SM)
chunk_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ AttendArgs a, const __grid_constant__ AttendSeqs sq)
{
    using C = Shape<HD, TILES>;
    constexpr uint32_t S_COL = 0, O_COL = C::O_COL;
    constexpr int COPY_WARP = 4 * TILES, MMA_WARP = COPY_WARP + 1;                     // the warps before take the softmax
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t q_at = smem_u32(smem), ring = q_at + TILES * C::TILE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + (TILES + C::STAGES) * C::TILE);
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (C::STAGES + s); };
    auto q_full = [&](int t) { return bar0 + 8u * (2 * C::STAGES + t); };
    auto s_full = [&](int t) { return bar0 + 8u * (2 * C::STAGES + TILES + t); };
    auto p_full = [&](int t) { return bar0 + 8u * (2 * C::STAGES + 2 * TILES + t); };
    auto o_full = [&](int t) { return bar0 + 8u * (2 * C::STAGES + 3 * TILES + t); };
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(bars + C::BARS);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(bars + C::BARS + 1);

    const int warp = __shfl_sync(FULL, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // (the same for all lanes, and known to be)
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int t = 0; t < TILES; ++t) { mbar_init(q_full(t), ROWS); mbar_init(s_full(t), 1); mbar_init(p_full(t), ROWS); mbar_init(o_full(t), 1); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm)) : "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void *)tmem_slot)), "r"((uint32_t)C::COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(FULL, *tmem_slot, 0);
    bool ok = true;
    pdl_launch_dependents();

    if (warp == COPY_WARP) {
        // ---- copies: the warp looks pages up, one lane issues
        constexpr int MAX_BOX = KEYS;
        const int box = a.g.T < MAX_BOX ? a.g.T : MAX_BOX, boxes = KEYS / box;
        int stage = 0;
        uint32_t phase = 0;
        for (int k = 0, x; (x = item_at(k)) < sq.items && ok && !a.test_drop_copies; ++k) {
            const Item it = item_of<TILES>(a, sq, x);
            const int *tab = a.p.table + it.tab * a.p.stride;
            const int first_page = it.lo >> a.g.t_shift, n_pages = it.hi > 0 ? (it.hi - 1) / a.g.T + 1 : 0;   // (of the sequence, those below n_pages hold tokens that are seen)
            auto fetch = [&](int p) {
                const int page = p < n_pages ? tab[p] : -1;
                return (unsigned)page < (unsigned)a.p.n_pages ? page : a.p.n_pages;      // (outside the pool: the copy engine writes zeros)
            };
            int base = first_page, now = fetch(base + lane), next = fetch(base + 32 + lane);
            const int row_k = (int)(a.g.at(a.layer, 0, it.kh) / (HD * 2)), row_v = (int)(a.g.at(a.layer, 1, it.kh) / (HD * 2));
            for (int j = 0; j < it.n_kv && ok; ++j) {
                const int tok = it.lo + j * KEYS;
                if ((tok >> a.g.t_shift) - base >= 32) { base += 32; now = next; next = fetch(base + 32 + lane); }
                int page[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) page[b] = __shfl_sync(FULL, now, ((tok + b * box) >> a.g.t_shift) - base);   // (pages of a tile are in one batch: 32 is a multiple of 4)
                if (lane == 0) {
                    for (int kv = 0; kv < 2 && ok; ++kv) {
                        if (!mbar_wait_relaxed(empty(stage), phase ^ 1u, a.limit_ns, abort_flag)) { ok = false; break; }
                        mbar_expect_tx(full(stage), C::TILE);
                        const uint32_t dst = ring + stage * C::TILE;
                        const int row = (kv ? row_v : row_k) + (tok & (a.g.T - 1));
#pragma unroll
                        for (int b = 0; b < 4; ++b)
                            if (b < boxes)
                                for (int h = 0; h < C::HALVES; ++h)
                                    tma_load_3d(dst + h * C::HALF + b * box * C::SWZ, &tm, full(stage), h * 64, row, page[b]);
                        if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
                    }
                }
                ok = __shfl_sync(FULL, ok ? 1 : 0, 0) != 0;
            }
        }
    } else if (warp == MMA_WARP) {
        // ---- products
        constexpr uint32_t id_qk = instr_desc(KEYS, false), id_pv = instr_desc(HD, true);
        constexpr int PER = C::SWZ / 32;                            // k-steps in a column block
        int stage = 0;
        uint32_t phase = 0, qph[2] = {0, 0}, pph[2] = {0, 0};
        auto advance = [&]() { if (++stage == C::STAGES) { stage = 0; phase ^= 1u; } };
        auto wait = [&](uint32_t bar, uint32_t parity) {            // by all lanes
            if (ok) ok = __all_sync(FULL, mbar_wait(bar, parity, a.limit_ns, abort_flag)) != 0;
            tc_fence_after();
        };
        // Operands are the same for all lanes, so that they stay in uniform registers: a product of 64 cycles leaves no time to bring them there
        // (computed by the issuing lane alone: 152 cycles each).
        const uint64_t q_desc = smem_desc<HD, false>(q_at), k_desc = smem_desc<HD, false>(ring), v_desc = smem_desc<HD, true>(ring);
        auto qk = [&](int t, int s) {
            const uint64_t ad = q_desc + (uint64_t)(t * (C::TILE >> 4)), bd = k_desc + (uint64_t)(s * (C::TILE >> 4));
            const uint32_t d = tmem + S_COL + t * KEYS;
            if (elect()) {
#pragma unroll
                for (int k = 0; k < HD / 16; ++k) {
                    const uint64_t off = (uint64_t)((k / PER * C::HALF + k % PER * 32) >> 4);
                    mma_ss(d, ad + off, bd + off, id_qk, k != 0);
                }
                tc_commit(s_full(t));
            }
        };
        auto pv = [&](int t, int s, bool first) {
            const uint64_t bd = v_desc + (uint64_t)(s * (C::TILE >> 4));
            const uint32_t d = tmem + O_COL + t * HD, w = tmem + S_COL + t * KEYS, more = first ? 0u : 1u;
            if (elect()) {
                mma_ts(d, w, bd, id_pv, more);
#pragma unroll
                for (int k = 1; k < KEYS / 16; ++k) mma_ts(d, w + k * 8, bd + (uint64_t)(k * 16 * C::SWZ >> 4), id_pv, 1u);
            }
        };
        auto commit = [&](uint32_t bar) { if (elect()) tc_commit(bar); };
        for (int k = 0, x; (x = item_at(k)) < sq.items && ok; ++k) {
            const Item it = item_of<TILES>(a, sq, x);
            if (it.n_kv == 0) continue;
            Words words;
            words.start(a, a.p.table + it.tab * a.p.stride, it, lane);
            // the first keys: S of both tiles
            wait(full(stage), phase);
            for (int t = 0; t < it.tiles && ok; ++t) {
                wait(q_full(t), qph[t]);
                qph[t] ^= 1u;
                if (ok) qk(t, stage);
            }
            if (!ok) break;
            commit(empty(stage));
            advance();
            for (int j = 0; j < it.n_kv && ok; ++j) {
                const int vs = stage;
                wait(full(vs), phase);
                if (!ok) break;
                advance();
                if (!words.whole(j, lane)) {                        // value rows that nobody sees become zeros
                    for (int i = 0; i < 4; ++i)
                        if (const int r = i * 32 + lane; !((words.word(j, i) >> lane) & 1))
#pragma unroll
                            for (int c = 0; c < HD * 2 / 16; ++c)
                                *reinterpret_cast<uint4 *>(smem + (TILES + vs) * C::TILE + (c / (C::SWZ / 16)) * C::HALF + r * C::SWZ + c % (C::SWZ / 16) * 16) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async();
                    __syncwarp();
                }
                const bool more = j + 1 < it.n_kv;
                const int ks = stage;
                for (int t = 0; t < it.tiles && ok; ++t) {
                    wait(p_full(t), pph[t]);
                    pph[t] ^= 1u;
                    if (!ok) break;
                    pv(t, vs, j == 0);
                    if (t == it.tiles - 1) commit(empty(vs));
                    if (more) {
                        if (t == 0) wait(full(ks), phase);
                        if (!ok) break;
                        qk(t, ks);
                        if (t == it.tiles - 1) commit(empty(ks));
                    } else {
                        commit(o_full(t));
                    }
                }
                if (more) advance();
            }
        }
    } else {
        // ---- softmax: one thread per row of a tile
        const int t = warp >> 2, tid = threadIdx.x & (ROWS - 1);
        const uint32_t lanes = tmem + ((uint32_t)(tid & ~31) << 16), s_at = lanes + S_COL + t * KEYS, o_at = lanes + O_COL + t * HD;
        const float sc = a.scale * LOG2E;
        // Scores of this size (in units of log 2) are 32 and more apart where they are not the same, so that a row's weights are 1 and next to nothing; the rounding of the
        // reference may be more than fp32 has exponents.  They are taken with a power of two for a scale (at most sc, at least half of it), whose products are exact.
        constexpr float FINE = 1073741824.f;
        const float sc_pow2 = __uint_as_float(__float_as_uint(sc) & 0x7f800000u);
        uint32_t sph = 0, oph = 0;
        for (int k = 0, x; (x = item_at(k)) < sq.items && ok; ++k) {
            const Item it = item_of<TILES>(a, sq, x);
            if (t >= it.tiles) continue;
            const int r0 = it.r0 + t * ROWS, row = min(r0 + tid, it.R - 1), tok_q = row / a.G, head = it.kh * a.G + row - tok_q * a.G, first = it.len - it.m;
            float R = -INFINITY, L = 0.f;                            // the reference, a score before the scale, and the sum of the weights
            if (it.n_kv) {
                // queries: every product that read the last item's is done (its results were waited for)
                constexpr int PIECES = HD / 8, PER_STEP = 32 / PIECES, PP = C::SWZ / 16;     // rows that a warp copies in a step: its own
                const unsigned long long mine = (unsigned long long)(a.q + (((long long)it.row + tok_q) * a.q_stride + (long long)head * HD) * 2);
                const int there = min(32, it.R - r0 - (tid & ~31));
#pragma unroll
                for (int i = 0; i < 32 / PER_STEP; ++i) {
                    const int k = i * PER_STEP + lane / PIECES, r = (tid & ~31) + k, p = lane % PIECES, sw = C::SWZ == 128 ? (r & 7) : ((r >> 1) & 3);
                    const char *src = (const char *)__shfl_sync(FULL, mine, k) + p * 16;
                    cp16(q_at + t * C::TILE + (p / PP) * C::HALF + r * C::SWZ + (((p % PP) ^ sw) << 4), src, k < there ? 16 : 0);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_proxy_async();
                mbar_arrive(q_full(t));
                Words words;
                words.start(a, a.p.table + it.tab * a.p.stride, it, lane);
                const int last = a.causal ? first + tok_q + 1 : 0x7fffffff, from = first_seen(first + tok_q, a.window);
                const int all_last = __reduce_min_sync(FULL, last), all_from = __reduce_max_sync(FULL, from);   // what every row of the warp sees
                const uint64_t sc2 = pk2(sc, sc);
                for (int j = 0; j < it.n_kv && ok; ++j) {
                    const int tok = it.lo + j * KEYS;
                    const bool whole = words.whole(j, lane) && tok + KEYS <= all_last && tok >= all_from;
                    // What the row does not see of columns i * 32 .. at -inf.
                    auto hide = [&](uint32_t *v, int i, unsigned w) {
                        const int b = tok + i * WORD;
                        if (last < b + WORD) w = last > b ? w & (FULL >> (b + WORD - last)) : 0;
                        if (from > b) w = from < b + WORD ? w & (FULL << (from - b)) : 0;
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!((w >> c) & 1)) v[c] = 0xff800000u;
                    };
                    // The weights of 32 columns, packed, and two times two sums of theirs.  They become bf16, because the values that they meet are (half a step is 2^-8 of a
                    // weight; the sums are not rounded): results are 2.0e-3 to 2.3e-3 off, of which their own rounding is 1.7e-3.  A second term would be half as many
                    // products again and four more instructions for each pair, which has five.
                    uint64_t sums[2];
                    auto weights = [&](const uint32_t *v, uint32_t *P, uint64_t sc2, uint64_t ref2) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float p0, p1;
                            upk2(fma2(pk2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), sc2, ref2), p0, p1);
                            p0 = ex2(p0);
                            p1 = ex2(p1);
                            sums[i & 1] = add2(sums[i & 1], pk2(p0, p1));
                            P[i] = pack_bf16(p0, p1);
                        }
                    };
                    auto total = [&]() {
                        float u, v;
                        upk2(add2(sums[0], sums[1]), u, v);
                        return u + v;
                    };
                    ok = __all_sync(FULL, mbar_wait(s_full(t), sph, a.limit_ns, abort_flag)) != 0;
                    sph ^= 1u;
                    if (!ok) break;
                    tc_fence_after();
                    // First with the reference as it is: a row's weights may grow to 2^16 in sum before anything needs to be done about it, so that
                    // the maximum of a tile is rarely asked for.
                    uint32_t P[64];
                    float sum = INFINITY;                                            // (an item's first tile: there is no reference yet)
                    const float M = __fmul_rn(R, sc);                                // (rounded: off by up to 2^5 below FINE, a factor that all of the row's weights share)
                    if (j) {
                        const uint64_t ref2 = pk2(-M, -M);
                        uint32_t A[32], B[32];
                        sums[0] = sums[1] = 0;
                        unsigned w[4];
                        if (!whole)
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] = words.word(j, i);
                        tmem_ld32(s_at, A);
                        tmem_wait_ld();
                        tmem_ld32(s_at + 32, B);
                        if (!whole) hide(A, 0, w[0]);
                        weights(A, P, sc2, ref2);
                        tmem_wait_ld();
                        tmem_ld32(s_at + 64, A);
                        if (!whole) hide(B, 1, w[1]);
                        weights(B, P + 16, sc2, ref2);
                        tmem_wait_ld();
                        tmem_ld32(s_at + 96, B);
                        if (!whole) hide(A, 2, w[2]);
                        weights(A, P + 32, sc2, ref2);
                        tmem_wait_ld();
                        if (!whole) hide(B, 3, w[3]);
                        weights(B, P + 48, sc2, ref2);
                        sum = total();
                    }
                    const bool redo = !(L + sum <= 65536.f) || !(fabsf(M) < FINE);  // (a NaN or no reference, too)
                    if (!__any_sync(FULL, redo)) {
                        tmem_st32(s_at, P);
                        tmem_st32(s_at + 32, P + 32);
                    } else {
                        // The scores once more: their maximum, the sums so far in its terms, the weights.
                        uint32_t A[32];
                        float part[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};   // (independent chains: each step waits for the one before it)
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            tmem_ld32(s_at + i * 32, A);
                            const unsigned w = words.word(j, i);
                            tmem_wait_ld();
                            if (!whole) hide(A, i, w);
#pragma unroll
                            for (int c = 0; c < 32; c += 8)
#pragma unroll
                                for (int k = 0; k < 4; ++k) part[k] = fmaxf(fmaxf(part[k], __uint_as_float(A[c + k])), __uint_as_float(A[c + 4 + k]));
                        }
                        const float top = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
                        float f = 1.f;
                        if (redo && top > R) { f = ex2((R - top) * sc); R = top; }   // (0 the first time)
                        if (redo && L * f > 32768.f) {                               // (this tile adds 128 at most)
                            const float up = fminf(R + a.up, 3.4028235e38f);
                            f *= ex2((R - up) * sc);
                            R = up;
                        }
                        L *= f;
                        if (j)
#pragma unroll 1
                            for (int i = 0; i < HD / 32; ++i) {
                                tmem_ld32(o_at + i * 32, A);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 32; ++c) A[c] = __float_as_uint(__uint_as_float(A[c]) * f);
                                tmem_st32(o_at + i * 32, A);
                            }
                        float scw = sc, ref = __fmul_rn(R, sc);
                        if (!(fabsf(ref) < FINE)) { scw = sc_pow2; ref = R * sc_pow2; }
                        if (R == -INFINITY) ref = 0.f;                               // (a row that has seen nothing yet)
                        sums[0] = sums[1] = 0;
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            tmem_ld32(s_at + i * 32, A);
                            const unsigned w = words.word(j, i);
                            tmem_wait_ld();
                            if (!whole) hide(A, i, w);
                            weights(A, P, pk2(scw, scw), pk2(-ref, -ref));
                            tmem_st16(s_at + i * 16, P);                             // (in place of scores that have been read)
                        }
                        sum = total();
                    }
                    L += sum;
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(p_full(t));
                }
                if (!ok) break;
                ok = __all_sync(FULL, mbar_wait(o_full(t), oph, a.limit_ns, abort_flag)) != 0;
                oph ^= 1u;
                if (!ok) break;
                tc_fence_after();
            }
            // the result: the output, or the piece's partial one
            const float M = R * sc;
            const bool mine = r0 + tid < it.R, cut = a.split && it.part >= 0;
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const size_t out_row = (size_t)it.row + tok_q;
            const size_t at = cut ? ((size_t)it.part + (size_t)it.piece * it.m + tok_q) * a.heads + head : 0;
            __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(a.out) + out_row * a.o_stride + (size_t)head * HD;
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) {
                uint32_t o[32];
                if (it.n_kv) { tmem_ld32(o_at + i * 32, o); tmem_wait_ld(); }
                else
#pragma unroll
                    for (int c = 0; c < 32; ++c) o[c] = 0;
                if (mine && cut) {
                    float4 *po = reinterpret_cast<float4 *>(a.part_o + at * HD + i * 32);
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        po[c] = make_float4(__uint_as_float(o[4 * c]), __uint_as_float(o[4 * c + 1]), __uint_as_float(o[4 * c + 2]), __uint_as_float(o[4 * c + 3]));
                } else if (mine) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = pack_bf16(__uint_as_float(o[8 * c + 2 * e]) * inv, __uint_as_float(o[8 * c + 2 * e + 1]) * inv);
                        *reinterpret_cast<uint4 *>(out + i * 32 + c * 8) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
                __syncwarp();
            }
            if (mine && cut) { a.part_ml[2 * at] = M; a.part_ml[2 * at + 1] = L; }
            if (mine && !cut && a.lse) a.lse[out_row * a.heads + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
            tc_fence_before();
        }
    }

    // ---- teardown
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) atomicExch(&wait_status, (int)EBRL_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && a.split) mark_unfinished<TILES>(a, sq);
    if (*abort_flag && threadIdx.x == 0) {
        // give copies that were still in flight time to land before shared memory is released
        const unsigned long long t0 = gtimer();
        while (gtimer() - t0 < 200000ull) { }
    }
    __syncthreads();
    if (warp == MMA_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::COLS) : "memory");
    }
    pdl_wait();      // (the end of this kernel is to be that of the ones beside it, too)
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static const EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

// The pool as (column, row of a page, page): boxes of a column block of up to 128 tokens; outside it reads zeros.
template <int HD> bool make_map(CUtensorMap *out, const Geometry &g, const Pages &p)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {HD, (cuuint64_t)g.layers * 2 * g.kvh * g.T, (cuuint64_t)p.n_pages};
    const cuuint64_t strides[2] = {HD * 2, g.bytes};
    const cuuint32_t box[3] = {Shape<HD, 1>::SWZ / 2, (cuuint32_t)(g.T < KEYS ? g.T : KEYS), 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p.pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              Shape<HD, 1>::SWZ == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, int TILES> cudaError_t go(const AttendArgs &a, const AttendSeqs &s, int quota, int sms, bool beside, cudaStream_t st)
{
    static std::atomic<bool> set[64];   // (calls may come from several threads; setting it twice is harmless)
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!set[dev]) {
        const cudaError_t err = cudaFuncSetAttribute(chunk_kernel<HD, TILES>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<HD, TILES>::SMEM);
        if (err != cudaSuccess) return err;
        set[dev] = true;
    }
    CUtensorMap tm;
    if (!make_map<HD>(&tm, a.g, a.p)) return cudaErrorInvalidValue;
    // Two tiles: one CTA per item, handed out by the hardware as the ones before end.  One tile, or under a quota: persistent CTAs, whose copies and products run on into
    // the next item (200 x 300 tokens x 64 rows 44 -> 38 us, 200 x 100 - 1500 tokens x 40 - 240 rows 88 -> 82; the most ragged batch tried 61 -> 63).
    const int grid = std::min(s.items, quota ? quota : (TILES == 1 ? sms * Shape<HD, TILES>::PER_SM : s.items));
    const Beside with(beside);
    return launch_kernel(chunk_kernel<HD, TILES>, grid, Shape<HD, TILES>::THREADS, Shape<HD, TILES>::SMEM, st, 1, tm, a, s);
}

}  // namespace

bool chunk_supported(const Geometry &g, int n_pages, float scale)
{
    return g.es == 2 && scale > 0.f && (long long)g.layers * 2 * g.kvh * g.T <= INT32_MAX && n_pages < INT32_MAX;
}

cudaError_t launch_chunk(const AttendArgs &a, const AttendSeqs &s, int rows, int quota, int sms, bool beside, cudaStream_t st)
{
    if (s.items == 0) return cudaSuccess;
    if (a.g.hd == 128) return rows == CHUNK_ROWS ? go<128, 2>(a, s, quota, sms, beside, st) : go<128, 1>(a, s, quota, sms, beside, st);
    return a.g.hd == 64 ? go<64, 1>(a, s, quota, sms, beside, st) : go<32, 1>(a, s, quota, sms, beside, st);
}

cudaError_t take_status(int *status)
{
    const int zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status, wait_status, sizeof(int));
    if (e == cudaSuccess && *status) e = cudaMemcpyToSymbol(wait_status, &zero, sizeof(int));
    return e;
}

}  // namespace pg
}  // namespace ebrl
