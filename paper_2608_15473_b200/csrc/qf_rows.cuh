// Attention of packed query rows over the paged cache on the tensor cores: whole prompts (causal) and prefixes that
// requests share.  The problem and its two forms are described in qf_rows_simple.cuh.
//
//   S = Q K^T / sqrt(d),  P = e^{S - m},  O = P V / sum P,   per 128 query rows, K and V in tiles of 128 positions.
//
// Both products are tcgen05.mma (bf16 in, fp32 in tensor memory), 64 positions at a time: S 128 x 64 x 128, O 128 x 128
// x 64.  A row tile holds the G query heads of 128 / G tokens of one KV head, so one K and V tile serves all of them,
// whatever G is (rows past G * (128 / G) are unused).  A CTA owns TWO row tiles ("wide") that share every K and V tile
// it streams: with one, shared memory (A and B operands are both read from it) would bound the products.  Every group
// of 128 softmax threads (one per row, no shuffles) has two slots of scores, so that the tensor cores work on one while
// the threads turn the other into P; P goes back to tensor memory over S and is the A operand of the second product
// from there.  Tensor memory is then full: 2 groups x (2 x 64 columns of scores + 128 of O).
// A block with no more rows than one tile ("narrow": a few decode tokens, a small group of requests) has the two
// softmax groups take the two halves of every position tile for the same rows instead, each with an accumulator of its
// own, merged at the block's end: a lone tile's chain product -> softmax -> product would leave the K/V stream waiting.
// (Whole tiles in turn held four of the five tiles of the ring at a time: 2,600 cycles per tile against 1,600.)
//
// Roles (384 threads, one CTA per SM): warps 0-3 and 4-7 softmax of the two tiles (and their epilogues), warps 8 and 9
// issue the products of one group each, warp 10 loads (TMA, 5 tiles of 32 KB in flight or in use), warp 11 walks the
// schedule.
//
// Schedule: all row blocks lie on one axis (KV heads, then sequences, then blocks) with the cost that a block and its
// tiles were measured to have, and every CTA takes an equal slice of it, found in its prologue from the lengths alone
// (no plan kernel, no host copy of the lengths).  A slice end that falls close to a block's border moves there;
// otherwise the block is cut along its positions and the pieces, (m, sum, unnormalised O) in fp32, are merged by a
// second small kernel in slice order.  Long contexts with few rows are split over all SMs by the same rule.  Heads are
// outermost so that CTAs that run together share a prefix's or a long prompt's pages in L2 (8 packed prompts: 159 us
// against 204 with sequences outermost).  No atomics: the order of every sum follows from the lengths.
//
// Numbers: scores, maxima, sums and accumulators are fp32.  The reference that the exponents subtract moves only when a
// row's maximum has grown by more than 2^8; until then it is the same factor in O and in the sum, and cancels.  So O is
// rescaled rarely.  Prompt form: P is rounded to bf16 (at most 2^-8 of each weight; the output itself is bf16).  Prefix
// form, whose states are fp32: P = hi + lo, two bf16 terms, 16 bits, and twice the second product, which the stream of
// K and V hides up to about 200 rows.  How accumulators drift, and what is done about it: kChainUnits.  A row with a score
// that is NaN or +infinity is NaN; a row whose every score is -infinity is empty.
//
// Measured (32 query heads on 8 KV heads; a copy reaches 6.54 TB/s, a library product 1.67 PFLOP/s, 1.40 for seconds on
// end).  One prompt of 16,384 tokens: 1.82 ms, 1.21 PFLOP/s; 2.1 ms and 1.04 among other work, when the card is at its
// power limit and the clock near 1.4 GHz.  64 positions of two row tiles take about 1,600 cycles, of which the products
// alone would take 1,140: a row's thread needs 1,450 from its scores' arrival to its weights' (tensor memory, maximum,
// 64 exponentials, rounding, tensor memory) and waits 150-300 for the next.  Narrow blocks stream at 5.9 TB/s.
// Outside the loops latency rules: about 9,000 cycles until a CTA's first product (lengths -> cuts -> block -> table ->
// copies, chains of dependent scalar steps; running that code once beforehand on made-up lengths, to have it fetched,
// changed nothing) and 5,800 per wide block.  Every role has ONE copy of its code, in rolled loops: with 131 KB of
// unrolled code a block cost 7,500 (8 packed prompts 169 us against 155).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdio>
#include <mutex>

#include "qf_common.cuh"
#include "qf_page_math.cuh"
#include "qf_proj.cuh"
#include "qf_rows_simple.cuh"

namespace qf {

constexpr int kRowTile = 128;                    // query rows of a tile, and cached positions of a tile
constexpr int kTilePages = kRowTile / kPageSize;
constexpr int kUnit = 64;                        // positions of one product S = Q K^T and of one softmax pass
constexpr int kRowsThreads = 12 * 32;
constexpr int kRowsRing = 5;                     // K and V tiles in flight or in use
constexpr int kTileBytes = kRowTile * kHeadDim * 2;
constexpr int kHalfPageBytes = kPageBytes / 2;    // 16 rows x 64 channels
constexpr int kInfoRing = 4;
constexpr int kRowsMaxCtas = 160;                // one per SM
// What things cost, in units of about 400 cycles, fitted to the cycles of some 7,000 slices of random batches: a position
// tile of two row tiles 3,100 cycles and of one 2,100 to 2,600 (it reads as much K and V: HBM is what it waits for), and
// what a block costs beside its tiles 5,800 and 3,700.  (7,500 and 5,000 when the units were chosen; 8, 5, 14 and 9, which
// would fit better now, balance no better.)  A cut is not charged the second prologue and end that it causes.
constexpr int kWideTileCost = 8, kNarrowTileCost = 6, kWideBlockCost = 18, kNarrowBlockCost = 12;
constexpr int kMinSlice = 12;                    // less per CTA is not worth a merge
constexpr int kWideSnap = 18, kNarrowSnap = 6;   // a cut this close to a block's border moves there
constexpr float kRescaleLog2 = 8.f;
// Units after which a group's accumulator is set aside and begun anew.  The tensor cores cut off what does not fit when
// they add a product to an accumulator, so a long chain drifts towards zero: 1.6e-8 of the value per 16-position step
// (measured: -1.4e-5 after 55 tiles of a prefix).  Prefix states are fp32, and an addition every 32 units (2,048
// positions, 4,096 when two groups share them), in fp32 and rounded, keeps the drift at 4e-6 for 5 % of the time;
// prompts' bf16 results want it only after 1,024 units.
template <bool PREFIX> constexpr int kChainUnits = PREFIX ? 32 : 1024;
// Of every 8 pairs of scores, how many take their exponentials from the multiply-add units.  Slowest CTA, in thousand
// cycles, with 1, 2, 3, 4 of 8: a prompt of 16,384 tokens 3,186, 3,046, 2,990, 3,346; 256 requests behind 32,768 tokens
// (whose polynomial is one degree longer and whose weights are split in two) 265, 267, 294, 307.
template <bool PREFIX> constexpr int kPolyPairs = PREFIX ? 1 : 3;

// One block's stretch of positions, as the schedule hands it to the other warps.
struct __align__(16) RowsBlock {
    int seq;        // -1: no more work
    int head;       // KV head
    int row0;       // first row of the block
    int i0;         // its index within the sequence
    int rows;       // tokens (prompt) or requests (prefix) in the block
    int off, len;   // SeqRows of the sequence
    int t_lo, t_hi; // position tiles
    int slot;       // >= 0: a piece, its state goes to this slot; -1: the whole block
    int narrow;
    int pad;
};
// What a CTA leaves for the merge kernel: the block it began but did not finish, and whether its first piece ended one.
struct __align__(16) RowsRecord { RowsBlock tail; int has_tail, head_state; int pad[2]; };   // head_state: 0 none, 1 goes on, 2 ends
static_assert(sizeof(RowsRecord) == 64 && sizeof(RowsBlock) == 48, "the merge kernel reads records as four 16-byte words");
struct RowsLayout { size_t record_off, aside_off, slot_off, total; };
constexpr size_t kRowsAsideFloats = (size_t)2 * kRowTile * kHeadDim;         // per CTA: both groups' accumulators set aside
constexpr size_t kRowsSlotFloats = (size_t)2 * kRowTile * (kHeadDim + 4);   // O, then m (log2 units), sum, true maximum
inline RowsLayout rows_layout()
{
    RowsLayout L;
    L.record_off = 256;
    L.aside_off = (L.record_off + kRowsMaxCtas * sizeof(RowsRecord) + 255) & ~(size_t)255;
    L.slot_off = L.aside_off + kRowsMaxCtas * kRowsAsideFloats * sizeof(float);
    L.total = (L.slot_off + 2 * kRowsMaxCtas * kRowsSlotFloats * sizeof(float) + 255) & ~(size_t)255;
    return L;
}

// ------------------------------------------------------------------ schedule arithmetic (host and device)
// One axis of units: KV heads in order, for each the sequences in order, for each its row blocks in order.
struct SeqPlan { int n, off, len; };     // rows, positions before row 0, positions in all
struct RowShape { int causal, tile_rows, group; };   // tile_rows: tokens of a row tile
__host__ __device__ inline int min_int(int a, int b) { return a < b ? a : b; }
__host__ __device__ inline int seq_blocks(SeqPlan q, RowShape f)
{
    return q.n > 0 && q.len > 0 ? (int)(((unsigned)q.n + 2u * f.tile_rows - 1) / (2u * f.tile_rows)) : 0;
}
__host__ __device__ inline int block_rows(SeqPlan q, RowShape f, int j) { return min_int(q.n - j * 2 * f.tile_rows, 2 * f.tile_rows); }
__host__ __device__ inline int block_tiles(SeqPlan q, RowShape f, int j)
{
    unsigned lim = (unsigned)q.len;
    if (f.causal) {
        const unsigned last = (unsigned)q.off + (unsigned)(j * 2 * f.tile_rows + block_rows(q, f, j));
        if (last < lim) lim = last;
    }
    return (int)((lim + kRowTile - 1) / kRowTile);
}
__host__ __device__ inline bool block_is_wide(SeqPlan q, RowShape f, int j) { return block_rows(q, f, j) > f.tile_rows; }
__host__ __device__ inline int block_cost(SeqPlan q, RowShape f, int j)
{
    const int nt = block_tiles(q, f, j);
    return block_is_wide(q, f, j) ? kWideTileCost * nt + kWideBlockCost : kNarrowTileCost * nt + kNarrowBlockCost;
}
__host__ __device__ inline long long seq_cost(SeqPlan q, RowShape f)
{
    long long c = 0;
    const int n = seq_blocks(q, f);
#pragma unroll 1
    for (int j = 0; j < n; ++j) c += block_cost(q, f, j);
    return c;
}
// How many slices the work is worth, and where cut c of them lies.
__host__ __device__ inline int slices_of(long long total, int n_ctas)
{
    return total >= (long long)kMinSlice * n_ctas ? n_ctas : total < kMinSlice ? 1 : (int)((unsigned)total / kMinSlice);
}
__host__ __device__ inline long long cut_at(long long total, int n, int c) { return (long long)((double)total / n * c); }
// Position x of the axis: its KV head, and the rest within the head.
__host__ __device__ inline int head_of(long long x, long long per_head, long long &rest)
{
    int h = (int)((double)x / (double)per_head);
    rest = x - h * per_head;
    if (rest < 0) { --h; rest += per_head; }
    if (rest >= per_head) { ++h; rest -= per_head; }
    return h;
}
struct SlicePos { int seq, head, block, tile; };   // a cut: this block's tiles below `tile` lie before it
// Where offset r of block j falls: the tile that a cut there precedes.
__host__ __device__ inline int place_in_block(SeqPlan q, RowShape f, int j, int r)
{
    const bool wide = block_is_wide(q, f, j);
    const int snap = wide ? kWideSnap : kNarrowSnap, each = wide ? kWideTileCost : kNarrowTileCost;
    const int fixed = wide ? kWideBlockCost : kNarrowBlockCost;
    const int nt = block_tiles(q, f, j);
    if (r < snap) return 0;
    if (each * nt + fixed - r < snap) return nt;
    const int t = (r - fixed + each - 1) / each;
    return t < 0 ? 0 : t > nt ? nt : t;
}
// Offset r of sequence seq.  On the device the lanes of a warp add up 32 blocks at a time.
__host__ __device__ inline SlicePos locate_in_seq(SeqPlan q, RowShape f, int seq, int head, long long r)
{
    SlicePos p{seq, head, 0, 0};
    const int n = seq_blocks(q, f);
#ifdef __CUDA_ARCH__
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int j0 = 0; j0 < n; j0 += 32) {
        const long long c = j0 + lane < n ? block_cost(q, f, j0 + lane) : 0;
        long long x = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, x > r);
        if (past) {
            const int l = __ffs((int)past) - 1;
            p.block = j0 + l;
            p.tile = place_in_block(q, f, p.block, (int)(r - __shfl_sync(0xffffffffu, x - c, l)));
            return p;
        }
        r -= __shfl_sync(0xffffffffu, x, 31);
    }
#else
    for (int j = 0; j < n; ++j) {
        const int c = block_cost(q, f, j);
        if (r < c) {
            p.block = j;
            p.tile = place_in_block(q, f, j, (int)r);
            return p;
        }
        r -= c;
    }
#endif
    p.block = n - 1;      // not reached: r lies within the sequence
    p.tile = block_tiles(q, f, n - 1);
    return p;
}
// The blocks between two cuts, in order.  `plan(s)` gives sequence s's SeqPlan, `first(s)` its first row.
template <class Plan, class First>
struct SliceWalk {
    Plan plan;
    First first;
    SlicePos at, end;
    int n_seq, heads, cta, n_blocks, row0;
    RowShape f;
    SeqPlan q;
    __host__ __device__ SliceWalk(Plan p, First fi, RowShape f_, SlicePos a, SlicePos z, int n_seq_, int heads_, int cta_)
        : plan(p), first(fi), at(a), end(z), n_seq(n_seq_), heads(heads_), cta(cta_), f(f_)
    {
        q = plan(at.seq);
        row0 = first(at.seq);
        n_blocks = seq_blocks(q, f);
    }
    // false: no block is left.  nt: the whole block's tiles.
    __host__ __device__ bool next(RowsBlock &b, int &nt)
    {
        while (at.head < heads) {
            const int j = at.block;
            const bool last = at.head == end.head && at.seq == end.seq && j == end.block;
            nt = block_tiles(q, f, j);
            const int lo = at.tile, hi = last ? end.tile : nt;
            const bool some = lo < hi;
            if (some) {
                b.seq = at.seq; b.head = at.head; b.i0 = j * 2 * f.tile_rows; b.row0 = row0 + b.i0;
                b.rows = block_rows(q, f, j); b.off = q.off; b.len = q.len; b.t_lo = lo; b.t_hi = hi;
                b.narrow = b.rows <= f.tile_rows ? 1 : 0; b.pad = 0;
                b.slot = (lo == 0 && hi == nt) ? -1 : lo > 0 ? 2 * cta : 2 * cta + 1;
            }
            if (last) at.head = heads;
            else {
                at.tile = 0;
                if (++at.block == n_blocks) {
                    at.block = 0;
                    if (n_seq > 1) {      // the next sequence with work, in the next head after the last
                        do {
                            if (++at.seq == n_seq) { at.seq = 0; ++at.head; }
                            q = plan(at.seq);
                            n_blocks = seq_blocks(q, f);
                        } while (n_blocks == 0 && at.head < heads);
                        row0 = first(at.seq);
                    } else {
                        ++at.head;
                    }
                }
            }
            if (some) return true;
        }
        return false;
    }
};

#define QF_COLD __noinline__      // rare paths: as functions they leave the instruction cache to the loops

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// Issuing a product costs its thread more than the product costs the tensor cores unless the operands are ready in
// uniform registers: the descriptors' upper words are constants, the lower ones a warp-uniform base plus a constant.
constexpr uint32_t kDescHi = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);   // stride 1,024 B, version 1, 128B swizzle
__device__ __forceinline__ uint32_t desc_lo_k(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | (1u << 16); }
// A V page as the B operand (16 positions x 128 channels, channels contiguous): [2 channel halves][16 rows][128 B],
// 128B swizzle.  Leading offset: the next 64 channels, 2,048 B; stride offset: the next 8 positions, 1,024 B.
__device__ __forceinline__ uint32_t desc_lo_v(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | ((uint32_t)(2048 >> 4) << 16); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// D[tmem] (+)= A[smem] . B[smem]^T
template <bool ACC>
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "n"(kDescHi), "r"(idesc), "n"(ACC ? 1 : 0) : "memory");
}
// D[tmem] (+)= A[tmem] . B[smem]
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 b, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "n"(kDescHi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, float *v)
{
    float (&r)[32] = *reinterpret_cast<float (*)[32]>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
          "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
          "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Ties 32 loaded registers to this point of the program: nothing that uses them moves above the wait before it.
__device__ __forceinline__ void pin32(float *v)
{
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7]));
}
// A bounded wait of a whole warp: every lane leaves with the same answer.  The loop is a function of its own.
__device__ QF_COLD bool warp_wait_loop(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
// The same for one thread.
__device__ QF_COLD bool wait_loop(uint32_t bar, uint32_t parity, volatile int *abort_flag) { return mbar_wait(bar, parity, abort_flag); }
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return warp_wait_loop(bar, parity, abort_flag);
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

// ------------------------------------------------------------------ the kernel
// Pairs of fp32 in one 64-bit register: add, multiply and multiply-add issue once for both.
__device__ __forceinline__ unsigned long long pack2(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(unsigned long long v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 2^x for a pair, on the multiply-add units (the special-function unit makes 16 exponentials per SM and cycle, which
// is what bounds a softmax): x = n + f with n the nearest integer (added into the low mantissa bits of 1.5 * 2^23),
// 2^f on [-1/2, 1/2] by a polynomial whose largest relative error is least among those with p(0) = 1 (linear program
// over Chebyshev points: 2.9e-6 in degree 4, 1.7e-7 in degree 5, in fp32), n added to its exponent.  Below -127 the result
// is exactly 0: p(0) = 1 and the exponent field becomes 0.  x <= 127; a NaN does not come through.
template <int DEGREE>
__device__ __forceinline__ void exp2_pair(unsigned long long x, float &p0, float &p1)
{
    float a, b;
    unpack2(x, a, b);
    x = pack2(fmaxf(a, -127.f), fmaxf(b, -127.f));
    const unsigned long long magic = pack2(12582912.f, 12582912.f), n_magic = pack2(-12582912.f, -12582912.f);
    const unsigned long long n = add2(x, magic), minus = pack2(-1.f, -1.f);
    const unsigned long long f = fma2(add2(n, n_magic), minus, x);
    unsigned long long p;
    if (DEGREE == 4) {
        p = fma2(pack2(0.009581047110259533f, 0.009581047110259533f), f, pack2(0.05590597167611122f, 0.05590597167611122f));
        p = fma2(p, f, pack2(0.24024145305156708f, 0.24024145305156708f));
        p = fma2(p, f, pack2(0.6931243538856506f, 0.6931243538856506f));
    } else {
        p = fma2(pack2(0.00132546026725322f, 0.00132546026725322f), f, pack2(0.009671999141573906f, 0.009671999141573906f));
        p = fma2(p, f, pack2(0.05550779402256012f, 0.05550779402256012f));
        p = fma2(p, f, pack2(0.24022231996059418f, 0.24022231996059418f));
        p = fma2(p, f, pack2(0.6931469440460205f, 0.6931469440460205f));
    }
    p = fma2(p, f, pack2(1.f, 1.f));
    float n0, n1;
    unpack2(n, n0, n1);
    unpack2(p, p0, p1);
    p0 = __int_as_float(__float_as_int(p0) + (__float_as_int(n0) << 23));
    p1 = __int_as_float(__float_as_int(p1) + (__float_as_int(n1) << 23));
}
__device__ __forceinline__ void st_global_32b(void *p, const uint32_t (&r)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// Units of 64 positions that row group w of a block takes: [2 t_lo, this).
template <bool PREFIX>
__device__ __forceinline__ int unit_end(const RowsBlock &b, int w, int tile_rows)
{
    const int last = b.narrow || w ? b.rows : min(b.rows, tile_rows);
    const int lim = PREFIX ? b.len : min(b.off + b.i0 + last, b.len);
    return min(2 * b.t_hi, (lim + kUnit - 1) / kUnit);
}
struct RowsSmem {
    alignas(1024) uint8_t q[2][kTileBytes];            // [row tile][channel half][128 rows][128 B]
    alignas(1024) uint8_t kv[kRowsRing][kTileBytes];   // K: [half][128 positions][128 B]; V: [page][half][16][128 B]
    alignas(16) RowsBlock info[kInfoRing];
    alignas(8) unsigned long long kv_full[kRowsRing], kv_empty[kRowsRing], q_full, q_empty, s_full[2][2], p_full[2][2], o_full[2], o_last[2],
        info_full[kInfoRing], info_empty[kInfoRing], pair[2], drain[2];
    float2 ml[2][kRowTile];          // narrow blocks: each group's (maximum, sum) per row
    unsigned bad_pages[8];           // per position tile (by its running number): pages without a valid table entry
    int dirty[kInfoRing];            // a value the mask hides from some row of the block is not finite
    SlicePos cut[2];
    long long scan[kRowsThreads / 32];
    long long cut_rest[2];
    int cut_seq[2];
    uint32_t tmem_base;
    int abort_flag;
};
static_assert(sizeof(RowsSmem) <= 227 * 1024, "one CTA per SM");

// A thread's row of an accumulator plus f times the part set aside (if any), into memory or back into tensor memory.
// All 32 lanes call it together.
__device__ QF_COLD void exchange_aside(uint32_t t_o, float *aside, bool has_aside, bool to_memory, float f)
{
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
        float4 *at = reinterpret_cast<float4 *>(aside + (size_t)c * 8 * kRowTile * 4);      // [channels / 4][row]
        float4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = has_aside ? __ldcg(at + i * kRowTile) : make_float4(0.f, 0.f, 0.f, 0.f);
        float o[32];
        tmem_ld32_nowait(t_o + c * 32, o);
        tmem_wait_ld();
        pin32(o);
        if (has_aside) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[4 * i] = fmaf(x[i].x, f, o[4 * i]); o[4 * i + 1] = fmaf(x[i].y, f, o[4 * i + 1]);
                o[4 * i + 2] = fmaf(x[i].z, f, o[4 * i + 2]); o[4 * i + 3] = fmaf(x[i].w, f, o[4 * i + 3]);
            }
        }
        if (to_memory) {
#pragma unroll
            for (int i = 0; i < 8; ++i) __stcg(at + i * kRowTile, make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[16 * h + i]);
                tmem_st16(t_o + c * 32 + 16 * h, w);
            }
        }
    }
}

// The rare end of a block whose last tiles hold non-finite values (see clean_values): this thread's row, already
// written, gets those it sees.  A weight is positive, so an infinity stays one and two of opposite signs make a NaN.
__device__ QF_COLD void add_hidden(const RowsArgs &A, const DevParams &P, const RowsBlock &b, int lim, int c0, int c1,
                                   float *slot_base, int slot_row, size_t out_row)
{
    const int common = min(b.off + b.i0 + 1, b.len);
#pragma unroll 1
    for (int pos = max(b.t_lo * kRowTile, common / kPageSize * kPageSize); pos < min(lim, b.t_hi * kRowTile); ++pos) {
        const long long at = (long long)b.seq * A.table_width + (pos >> 4);
        const long long phys = A.table ? (long long)A.table[at] : at;
        if (phys < 0 || phys >= P.num_pages) continue;
        const uint16_t *v = A.v_cache + kv_row_offset(P, phys, b.head, pos & 15);
#pragma unroll 1
        for (int d = c0 * 32; d < c1 * 32; ++d) {
            if ((v[d] & 0x7f80u) != 0x7f80u) continue;
            const float x = __uint_as_float((uint32_t)v[d] << 16);
            if (b.slot >= 0) {
                float *o = slot_base + ((size_t)(d >> 2) * (2 * kRowTile) + slot_row) * 4 + (d & 3);
                __stcg(o, __ldcg(o) + x);
            } else {
                uint16_t *o = A.out + out_row * kHeadDim + d;
                *o = (uint16_t)(pack_bf16(__uint_as_float((uint32_t)*reinterpret_cast<volatile uint16_t *>(o) << 16) + x, 0.f) & 0xffffu);
            }
        }
    }
}

// The rare end of a prefix block whose values are not all finite.  Weights are positive, but the second term of a weight may
// be 0 or negative, and an infinity times that, or an accumulator's infinity times a factor that underflows, is NaN.  So the
// warp searches the values of the stretch, and every row that is not NaN or empty itself gets what it sees, over what it
// has written: NaN, or both infinities, make NaN, infinities of one sign make that infinity.
__device__ QF_COLD void mend_infinite(const RowsArgs &A, const DevParams &P, const RowsBlock &b, bool mine, int c0, int c1,
                                      float *slot_base, int slot_row, size_t out_row)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int c = c0; c < c1; ++c) {
        unsigned nan = 0, pos = 0, neg = 0;      // bit i: channel 32 c + i
#pragma unroll 1
        for (int i = b.t_lo * kRowTile + lane; i < min(b.len, b.t_hi * kRowTile); i += 32) {
            const long long at = (long long)b.seq * A.table_width + (i >> 4);
            const long long phys = A.table ? (long long)A.table[at] : at;
            if (phys < 0 || phys >= P.num_pages) continue;
            const uint4 *v = reinterpret_cast<const uint4 *>(A.v_cache + kv_row_offset(P, phys, b.head, i & 15) + c * 32);
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                const uint4 x = v[k];
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t u = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu, bit = 1u << (8 * k + e);
                    if ((u & 0x7f80u) != 0x7f80u) continue;
                    if (u & 0x7fu) nan |= bit;
                    else if (u >> 15) neg |= bit;
                    else pos |= bit;
                }
            }
        }
        nan = __reduce_or_sync(0xffffffffu, nan);
        pos = __reduce_or_sync(0xffffffffu, pos);
        neg = __reduce_or_sync(0xffffffffu, neg);
        nan |= pos & neg;
        if (!mine) continue;
        for (unsigned left = nan | pos | neg; left; left &= left - 1) {
            const int i = __ffs((int)left) - 1, d = c * 32 + i;
            const float x = __uint_as_float((nan >> i) & 1 ? 0x7fc00000u : (pos >> i) & 1 ? 0x7f800000u : 0xff800000u);
            if (b.slot >= 0) __stcg(slot_base + ((size_t)(d >> 2) * (2 * kRowTile) + slot_row) * 4 + (d & 3), x);
            else A.o_part[out_row * kHeadDim + d] = x;
        }
    }
}

// A tile of values in shared memory, by one warp: rows from `exist` on, as far as their page goes, become 0, and so do
// non-finite values among rows seen_by_all .. used - 1 (from the page's start), which `dirty` then reports.
__device__ QF_COLD void clean_tile(uint8_t *v, int exist, int seen_by_all, int used, volatile int *dirty)
{
    const int lane = threadIdx.x & 31;
    if (exist & 15) {
        uint8_t *page = v + (exist >> 4) * kPageBytes;
        const int r0 = exist & 15, n16 = (16 - r0) * 8;    // 16-byte words per half
#pragma unroll 1
        for (int i = lane; i < 2 * n16; i += 32) {
            const int half = i >= n16, x = i - half * n16;
            *reinterpret_cast<uint4 *>(page + half * kHalfPageBytes + r0 * 128 + x * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
    }
    const int from = seen_by_all / kPageSize * (kPageBytes / 16), to = (used + kPageSize - 1) / kPageSize * (kPageBytes / 16);
    if (seen_by_all < used) {
        // a product with 0 keeps only what is not finite: one instruction for two values
        uint32_t bad[4] = {0u, 0u, 0u, 0u};
#pragma unroll 1
        for (int i = from + lane; i < to; i += 256)          // a page is 256 words
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint4 x = *reinterpret_cast<const uint4 *>(v + (i + 32 * e) * 16);
                asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(bad[0]) : "r"(x.x), "r"(0u));
                asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(bad[1]) : "r"(x.y), "r"(0u));
                asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(bad[2]) : "r"(x.z), "r"(0u));
                asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(bad[3]) : "r"(x.w), "r"(0u));
            }
        if (__any_sync(0xffffffffu, ((bad[0] | bad[1] | bad[2] | bad[3]) & 0x7fff7fffu) != 0)) {
            if (lane == 0) *dirty = 1;
            __threadfence_block();      // said before the first value is gone: the other warp may find none left
            __syncwarp();
#pragma unroll 1
            for (int i = from * 8 + lane; i < to * 8; i += 32) {
                uint16_t *x = reinterpret_cast<uint16_t *>(v) + i;
                if ((*x & 0x7f80u) == 0x7f80u) *x = 0;
            }
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the products read what is there now
    __syncwarp();
}

struct RowsMaps { CUtensorMap q, k, v; };

template <bool PREFIX>
__global__ void __launch_bounds__(kRowsThreads, 1)
rows_kernel(const __grid_constant__ RowsMaps maps, const __grid_constant__ RowsArgs A, const __grid_constant__ DevParams P,
            RowsRecord *__restrict__ records, float *__restrict__ asides, float *__restrict__ slots)
{
    extern __shared__ __align__(1024) uint8_t rows_smem[];
    RowsSmem &sm = *reinterpret_cast<RowsSmem *>(rows_smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int Hq = P.num_q_heads, Hkv = P.num_kv_heads, G = P.group;
    const int tile_rows = kRowTile / G;               // tokens per row tile
    volatile int *abort_flag = &sm.abort_flag;

    if (tid == 0) {
        for (int i = 0; i < kRowsRing; ++i) { mbar_init(smem_u32(&sm.kv_full[i]), 1); mbar_init(smem_u32(&sm.kv_empty[i]), 2); }
        mbar_init(smem_u32(&sm.q_full), 1);
        mbar_init(smem_u32(&sm.q_empty), 2);         // one per product warp
        for (int w = 0; w < 2; ++w) {
            for (int i = 0; i < 2; ++i) {
                mbar_init(smem_u32(&sm.s_full[w][i]), 1);
                mbar_init(smem_u32(&sm.p_full[w][i]), 4);    // one arrival per softmax warp
            }
            mbar_init(smem_u32(&sm.o_last[w]), 1);
            mbar_init(smem_u32(&sm.o_full[w]), 1);
            mbar_init(smem_u32(&sm.pair[w]), 8);
        }
        for (int i = 0; i < kInfoRing; ++i) { mbar_init(smem_u32(&sm.info_full[i]), 1); mbar_init(smem_u32(&sm.info_empty[i]), 11); }
        mbar_init(smem_u32(&sm.drain[0]), 1);
        mbar_init(smem_u32(&sm.drain[1]), 1);
        sm.abort_flag = 0;
        sm.cut_seq[0] = sm.cut_seq[1] = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(smem_u32(&sm.tmem_base), 512);
    if (tid == 0) {
        prefetch_map(&maps.q);
        prefetch_map(&maps.k);
        prefetch_map(&maps.v);
    }
    grid_dependency_wait();
    grid_launch_dependents();

    const RowShape shape{PREFIX ? 0 : 1, tile_rows, G};
    auto seq_plan = [&](int s) -> SeqPlan {
        const SeqRows r = seq_rows<PREFIX>(A, s);
        return SeqPlan{r.n, r.off, r.len};
    };
    auto give_up = [&]() {      // a bounded wait ran out (or another warp's did)
        sm.abort_flag = 1;
        rows_status_or(A.status, kStatusTimeout);
    };

    if (PREFIX) {
        // empty states: requests of groups with an empty prefix, and of no group
        auto empties = [&](int lo, int hi) {
            const long long n4 = (long long)max(hi - lo, 0) * Hq * (kHeadDim / 4);
#pragma unroll 1
            for (long long i = tid; i < n4; i += kRowsThreads) {
                const long long row = lo + i / (Hq * (kHeadDim / 4));
                const int rest = (int)(i % (Hq * (kHeadDim / 4)));
                const size_t o = ((size_t)row * A.out_shards + A.slot) * Hq;
                reinterpret_cast<float4 *>(A.o_part + o * kHeadDim)[rest] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (rest < Hq) { A.m_part[o + rest] = neg_inf(); A.lse_part[o + rest] = neg_inf(); }
            }
        };
        for (int s = (int)blockIdx.x; s < A.n_seq + 2; s += (int)gridDim.x) {
            if (s == A.n_seq) empties(0, min(max(A.cu[0], 0), A.total_rows));
            else if (s == A.n_seq + 1) empties(min(max(A.cu[A.n_seq], 0), A.total_rows), A.total_rows);
            else {
                const SeqRows r = seq_rows<PREFIX>(A, s);
                if (r.len == 0) empties(r.first, r.first + r.n);
            }
        }
    }

    if (P.check_bounds)
        for (int s = (int)blockIdx.x * kRowsThreads + tid; s < A.n_seq; s += (int)gridDim.x * kRowsThreads)
            if (seq_overruns<PREFIX>(A, s)) rows_status_or(A.status, kStatusBadPage);

    // ---- this CTA's slice.  A thread adds up a sequence's blocks, or a warp does while there are no more sequences
    // than warps.
    const int n_ctas = (int)gridDim.x;
    constexpr int kWarps = kRowsThreads / 32;
    if (A.n_seq <= kWarps) {
        if (warp < A.n_seq) {
            const SeqPlan q = seq_plan(warp);
            const int n = seq_blocks(q, shape);
            long long c = 0;
#pragma unroll 1
            for (int j = lane; j < n; j += 32) c += block_cost(q, shape, j);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
            if (lane == 0) sm.scan[warp] = c;
        }
        __syncthreads();
    }
    long long running = 0;       // units of the sequences so far
    // (units before sequence base + tid, its own units); adds the round's total to `running`
    auto scan_round = [&](int base, long long &before, long long &cost) {
        cost = base + tid < A.n_seq ? seq_cost(seq_plan(base + tid), shape) : 0;
        long long x = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) sm.scan[warp] = x;
        __syncthreads();
        before = running + x - cost;
#pragma unroll 1
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sm.scan[w];
            running += sm.scan[w];
        }
        __syncthreads();
    };
    const int me = (int)blockIdx.x;
    bool working = false;
    long long ra = -1, rb = -1;          // where this CTA's cuts fall within their heads ha and hb
    int ha = 0, hb = 0;
    // the first pass finds the total, the second, for more sequences than threads, the cuts' sequences
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        long long before = 0, cost = 0;
        auto offer = [&](int s) {
            if (ra >= before && ra < before + cost) { sm.cut_seq[0] = s; sm.cut_rest[0] = ra - before; }
            if (rb >= before && rb < before + cost) { sm.cut_seq[1] = s; sm.cut_rest[1] = rb - before; }
        };
        running = 0;
        if (A.n_seq <= kWarps) {
#pragma unroll 1
            for (int s = 0; s < A.n_seq; ++s) {
                if (s == tid) { before = running; cost = sm.scan[s]; }
                running += sm.scan[s];
            }
        } else {
#pragma unroll 1
            for (int base = 0; base < A.n_seq; base += kRowsThreads) {
                scan_round(base, before, cost);
                if (pass) offer(base + tid);
            }
        }
        if (pass) break;
        const long long total = running * Hkv;
        const int n_eff = slices_of(total, n_ctas);
        working = total > 0 && me < n_eff;
        if (!working) break;
        ha = head_of(cut_at(total, n_eff, me), running, ra);
        hb = Hkv;
        if (me + 1 < n_eff) hb = head_of(cut_at(total, n_eff, me + 1), running, rb);
        if (A.n_seq <= kRowsThreads) {
            offer(tid);
            break;
        }
    }
    if (working) {
        __syncthreads();
        if (warp < 2) {
            SlicePos at{0, Hkv, 0, 0};                      // the end of everything
            if (sm.cut_seq[warp] >= 0)
                at = locate_in_seq(seq_plan(sm.cut_seq[warp]), shape, sm.cut_seq[warp], warp ? hb : ha, sm.cut_rest[warp]);
            if (lane == 0) sm.cut[warp] = at;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(&sm.tmem_base);
    const uint32_t t_s0 = tmem, t_o0 = tmem + 256;      // S (and P over it) of the two groups, then their O

    if (!working) {
        if (tid == 0) { records[me].has_tail = 0; records[me].head_state = 0; }
    } else if (warp == 11) {
        // ============================ schedule ============================
        if (lane == 0) {
            const SlicePos a = sm.cut[0], z = sm.cut[1];
            RowsBlock tail = {};
            int has_tail = 0, head_state = 0, idx = 0;
            bool ok = true;
            auto publish = [&](const RowsBlock &b) {
                const int slot = idx % kInfoRing;
                if (!wait_loop(smem_u32(&sm.info_empty[slot]), (uint32_t)(((idx / kInfoRing) & 1) ^ 1), abort_flag)) { ok = false; return; }
                sm.info[slot] = b;
                sm.dirty[slot] = 0;
                mbar_arrive(smem_u32(&sm.info_full[slot]));
                ++idx;
            };
            auto first = [&](int s) { return seq_rows<PREFIX>(A, s).first; };
            SliceWalk<decltype(seq_plan), decltype(first)> walk(seq_plan, first, shape, a, z, A.n_seq, Hkv, me);
            RowsBlock b;
            int nt = 0;
            while (ok && walk.next(b, nt)) {
                if (b.t_lo > 0) head_state = b.t_hi == nt ? 2 : 1;
                else if (b.t_hi < nt) { has_tail = 1; tail = b; }
                publish(b);
            }
            RowsBlock end = {};
            end.seq = -1;
            if (ok) publish(end);
            if (!ok) give_up();
            RowsRecord &rec = records[me];
            rec.tail = tail;
            rec.has_tail = ok ? has_tail : 0;
            rec.head_state = head_state;
        }
    } else if (warp == 10) {
        // ============================ loads ============================
        int stage = 0, idx = 0, issued = 0, tile_no = 0;
        uint32_t phase = 0;
        int q_fill = -1;
        bool ok = true;
        const int none_c2 = (int)(P.kv_nhd ? P.num_pages * kPageSize : P.num_pages * Hkv);   // out of range: zeros
        const uint32_t q_box = (uint32_t)(64 * 2) * G * tile_rows;
        if (A.table) {      // the first block's table entries, while the schedule names it
            const int at = sm.cut[0].tile * kTilePages + lane;
            if (at < A.table_width) asm volatile("prefetch.global.L1 [%0];" ::"l"(A.table + (size_t)sm.cut[0].seq * A.table_width + at));
        }
        for (; ok; ++idx) {
            const int slot = idx % kInfoRing;
            if (!warp_wait(smem_u32(&sm.info_full[slot]), (uint32_t)((idx / kInfoRing) & 1), abort_flag)) { ok = false; break; }
            const RowsBlock b = sm.info[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.info_empty[slot]));
            if (b.seq < 0) break;
            const int last_page = (b.len - 1) >> 4, c1 = P.kv_nhd ? b.head : 0;
            const long long row_base = (long long)b.seq * A.table_width;
            auto entry = [&](int lp) -> int {
                return lp <= last_page ? (A.table ? A.table[row_base + lp] : (int)(row_base + lp)) : -1;
            };
            // 64 table entries in registers; the second half is on its way while the first is used.  Values come last
            // through a page, keys at most two tiles before them, so the window moves when values leave its first half.
            int win = b.t_lo * kTilePages;
            int tbl0 = entry(win + lane), tbl1 = entry(win + 32 + lane);
            auto pages_of = [&](int page0, bool is_v) -> int {      // lane i: physical page page0 + i % 8, or -1
                if (is_v && page0 - win >= 32) {
                    win += 32;
                    tbl0 = tbl1;
                    tbl1 = entry(win + 32 + lane);
                }
                const int at = page0 - win;
                return __shfl_sync(0xffffffffu, at < 32 ? tbl0 : tbl1, (at & 31) + (lane & 7));
            };
            // a tile's pages, K or V, into the ring's next slot
            auto load_tile = [&](int t, bool is_v) {
                const int page0 = t * kTilePages;
                int phys = pages_of(page0, is_v);
                const bool in = page0 + (lane & 7) <= last_page;
                const bool bad = in && (phys < 0 || (long long)phys >= P.num_pages);
                const unsigned bad_mask = __ballot_sync(0xffffffffu, bad) & 0xffu;
                if (!warp_wait(smem_u32(&sm.kv_empty[stage]), phase ^ 1, abort_flag)) { ok = false; return; }
                // One thread issues every copy, with operands that are the same for the warp: a lane per page made each copy
                // a turn of a loop over lanes, 1,500 cycles per tile and the bound of the whole kernel.
                const int c2 = !in || bad ? none_c2 : P.kv_nhd ? phys * kPageSize : phys * Hkv + b.head;
                int at[kTilePages];
#pragma unroll
                for (int i = 0; i < kTilePages; ++i) at[i] = __shfl_sync(0xffffffffu, c2, i);
                if (elect_one()) {
                    const uint32_t full = smem_u32(&sm.kv_full[stage]), dst = smem_u32(sm.kv[stage]);
                    // before the arrival, which releases it to whoever works on this tile
                    if (!is_v) sm.bad_pages[tile_no & 7] = bad_mask;
                    mbar_arrive_expect_tx(full, kTileBytes);
                    if (is_v) {
#pragma unroll
                        for (int i = 0; i < kTilePages; ++i) tma_load_4d(dst + i * kPageBytes, &maps.v, 0, c1, at[i], 0, full);
                    } else {
                        if (bad_mask && P.check_bounds) rows_status_or(A.status, kStatusBadPage);
#pragma unroll
                        for (int i = 0; i < 2 * kTilePages; ++i)
                            tma_load_4d(dst + i * kHalfPageBytes, &maps.k, 0, c1, at[i & 7], i >> 3, full);
                    }
                }
                __syncwarp();
                if (!is_v) ++tile_no;
                ++issued;
                if (++stage == kRowsRing) { stage = 0; phase ^= 1; }
            };
            // The order the products consume them in: K is one tile (wide) or two (narrow) ahead of V.  Q after the first.
            const int ahead = b.narrow ? 2 : 1;
            int k_next = b.t_lo, v_next = b.t_lo;
#pragma unroll 1
            while (v_next < b.t_hi) {
                const bool is_v = k_next == b.t_hi || k_next - v_next >= ahead;
                load_tile(is_v ? v_next++ : k_next++, is_v);
                if (!ok) break;
                if (is_v || k_next != b.t_lo + 1) continue;
                if (!warp_wait(smem_u32(&sm.q_empty), (uint32_t)((idx & 1) ^ 1), abort_flag)) { ok = false; break; }
                if (lane == 0) {
                    const uint32_t full = smem_u32(&sm.q_full);
                    const int n_tiles = b.narrow ? 1 : 2;
                    mbar_arrive_expect_tx(full, q_box * 2u * n_tiles);
#pragma unroll 1
                    for (int i = 0; i < 2 * n_tiles; ++i) {
                        const int w = i >> 1, half = i & 1;
                        tma_load_3d(smem_u32(sm.q[w]) + half * (kTileBytes / 2), &maps.q, half * 64, b.head * G, b.row0 + w * tile_rows, full);
                    }
                }
                __syncwarp();
                q_fill = idx;
            }
        }
        if (!ok) {
            // flag it, then wait (bounded) for the copies still in flight
            if (lane == 0) give_up();
            __syncwarp();
            int s2 = stage;
            uint32_t ph2 = phase;
            for (int k = 0; k < min(issued, kRowsRing); ++k) {
                if (--s2 < 0) { s2 = kRowsRing - 1; ph2 ^= 1; }
                for (unsigned it = 0; it < (1u << 20); ++it)
                    if (mbar_try_wait(smem_u32(&sm.kv_full[s2]), ph2)) break;
            }
            if (q_fill >= 0)
                for (unsigned it = 0; it < (1u << 20); ++it)
                    if (mbar_try_wait(smem_u32(&sm.q_full), (uint32_t)(q_fill & 1))) break;
        }
    } else if (warp >= 8) {
        // ============================ products ============================
        // One warp per softmax group, so that neither group waits for the other's turn and the few dozen instructions
        // between two products of a group overlap the other group's.
        const int w = warp - 8;
        constexpr uint32_t idesc_qk = umma_idesc_bf16(kUnit);
        constexpr uint32_t idesc_pv = umma_idesc_bf16(kHeadDim) | (1u << 16);     // B (values) is channel-major
        const uint32_t q_lo = desc_lo_k(smem_u32(sm.q[0])), k_lo = desc_lo_k(smem_u32(sm.kv[0])), v_lo = desc_lo_v(smem_u32(sm.kv[0]));
        const uint32_t t_s = t_s0 + w * 128, t_o = t_o0 + w * 128;
        const uint32_t bar_full = smem_u32(sm.kv_full), bar_empty = smem_u32(sm.kv_empty), bar_s = smem_u32(sm.s_full[w]),
                       bar_p = smem_u32(sm.p_full[w]), bar_o = smem_u32(&sm.o_full[w]), bar_last = smem_u32(&sm.o_last[w]);
        int stage = 0, idx = 0;
        uint32_t phase = 0, p_phase = 0;       // p_phase: bit h is p_full[w][h]'s
        bool ok = true;
        for (; ok; ++idx) {
            const int slot = idx % kInfoRing;
            if (!warp_wait(smem_u32(&sm.info_full[slot]), (uint32_t)((idx / kInfoRing) & 1), abort_flag)) { ok = false; break; }
            const RowsBlock b = sm.info[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.info_empty[slot]));
            if (b.seq < 0) break;
            // positions every row of the block sees; tiles that reach beyond hold values hidden from some row
            const int common = PREFIX ? b.len : min(b.off + b.i0 + 1, b.len);
            const int end = unit_end<PREFIX>(b, w, tile_rows);
            const uint32_t q_at = q_lo + (b.narrow ? 0 : w) * (kTileBytes >> 4);
            auto take = [&](int at, uint32_t ph) -> bool {      // a tile of the ring has landed
                if (!warp_wait(bar_full + at * 8, ph, abort_flag)) { ok = false; return false; }
                tc_fence_after();
                return true;
            };
            // This warp is done with the ring's next tile when its products so far are.
            auto release = [&]() {
                if (elect_one()) umma_commit(bar_empty + stage * 8);
                if (++stage == kRowsRing) { stage = 0; phase ^= 1; }
            };
            // A unit's slot: its half of the tile, or, narrow, where a group has one half of every tile, the tile's parity.
            // S[slot] = Q (K half h)^T
            auto qk = [&](int h, int sl, int at) {
                const uint32_t k = k_lo + at * (kTileBytes >> 4) + h * (kUnit * 128 >> 4), d = t_s + sl * kUnit;
                if (elect_one()) {
                    umma_ss<false>(d, q_at, k, idesc_qk);
#pragma unroll
                    for (int kk = 1; kk < 8; ++kk) {
                        const uint32_t o = ((kk >> 2) * (kTileBytes / 2) + (kk & 3) * 32) >> 4;
                        umma_ss<true>(d, q_at + o, k + o, idesc_qk);
                    }
                    umma_commit(bar_s + sl * 8);
                }
            };
            // O += P[slot] (V half h)
            auto pv = [&](int h, int sl, int at, bool first, bool last) {
                if (!warp_wait(bar_p + sl * 8, (p_phase >> sl) & 1, abort_flag)) { ok = false; return; }
                p_phase ^= 1u << sl;
                tc_fence_after();
                const uint32_t v = v_lo + at * (kTileBytes >> 4) + h * ((kUnit / kPageSize) * kPageBytes >> 4), pa = t_s + sl * kUnit;
                const uint32_t acc = first ? 0u : 1u;
                if (elect_one()) {
#pragma unroll
                    for (int part = 0; part < (PREFIX ? 2 : 1); ++part)
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            umma_ts(t_o, pa + part * 32 + kk * 8, v + kk * (kPageBytes >> 4), idesc_pv, part == 0 && kk == 0 ? acc : 1u);
                    umma_commit(bar_o);
                    if (last) umma_commit(bar_last);
                }
            };
            // Values that no row, or not every row, may see.  Weights there are exactly 0, but 0 times a NaN or an
            // infinity is not: rows of the last page beyond the context (never written) become 0, and so do non-finite
            // values of a tile that is hidden from some row, which the epilogue then adds where they are seen.  Both
            // product warps do it, each before its own products: what the second one writes is what is there.
            auto clean_values = [&](int t, int at) {
                const int exist = min(b.len - t * kRowTile, kRowTile);          // positions of the tile that exist
                const int seen_by_all = PREFIX ? exist : max(common - t * kRowTile, 0);
                const int used = min(end * kUnit - t * kRowTile, exist);        // this group's products use these (and their pages' rest)
                clean_tile(sm.kv[at], exist, seen_by_all, used, &sm.dirty[slot]);
            };
            auto needs_clean = [&](int t) {
                return (!PREFIX && (t + 1) * kRowTile > common) || ((t + 1) * kRowTile > b.len && (b.len & 15));
            };
            if (!warp_wait(smem_u32(&sm.q_full), (uint32_t)(idx & 1), abort_flag)) { ok = false; break; }
            auto q_done = [&]() { if (elect_one()) umma_commit(smem_u32(&sm.q_empty)); };
            // The order: S of a tile's two units, then for every unit P V of this tile and, into the slot that P V has
            // just freed (a thread's products run in the order of issue), S of the tile this group takes next.
            const int ahead = b.narrow ? 2 : 1;      // tiles between the values in use and the keys
            const int step = ahead, first = b.narrow ? w : 0;      // this group's units of a tile: first, first + step
            for (int t = b.t_lo; t < b.t_hi && t < b.t_lo + ahead; ++t) {
                if (!take(stage, phase)) break;
#pragma unroll 1
                for (int i = 0; i < 2 / step; ++i)
                    if (2 * t + first + i < end) qk(first + i, b.narrow ? t & 1 : i, stage);
                release();
            }
            if (ok && b.t_hi - b.t_lo <= ahead) q_done();
            // The tiles with nothing special about them (every unit there, nothing to clean, keys to come): one thread, no
            // votes, constants where the operands allow it.
            int t_plain = min(b.t_hi - ahead, b.narrow ? (end - w - 3) >> 1 : (end - 2) >> 1);
            if (!PREFIX) t_plain = min(t_plain, common / kRowTile);
            else if (b.len & 15) t_plain = min(t_plain, b.len / kRowTile);
            t_plain = max(t_plain, b.t_lo);
            if (ok && t_plain > b.t_lo) {
                bool fine = true;
                if (elect_one()) {
                    int at = stage;
                    uint32_t ph = phase, pp = p_phase;
                    auto wait = [&](uint32_t bar, uint32_t parity) {
                        if (!mbar_try_wait(bar, parity) && !wait_loop(bar, parity, abort_flag)) fine = false;
                    };
#pragma unroll 1
                    for (int t = b.t_lo; t < t_plain; ++t) {
                        const int v_at = at;
                        const uint32_t v_ph = ph;
                        if (++at == kRowsRing) { at = 0; ph ^= 1; }
                        wait(bar_full + v_at * 8, v_ph);
                        wait(bar_full + at * 8, ph);
                        if (!fine) break;
                        tc_fence_after();
                        const uint32_t v = v_lo + v_at * (kTileBytes >> 4), k = k_lo + at * (kTileBytes >> 4);
                        // a group's first unit, and every kChainUnits-th, begins its accumulator anew
                        const uint32_t acc = ((t - b.t_lo) * (b.narrow ? 1 : 2) & (kChainUnits<PREFIX> - 1)) ? 1u : 0u;
                        auto unit = [&](int h, int sl, uint32_t first_acc) {
                            wait(bar_p + sl * 8, (pp >> sl) & 1);
                            if (!fine) return;
                            tc_fence_after();
                            const uint32_t v_h = v + h * (4 * kPageBytes >> 4), k_h = k + h * (kUnit * 128 >> 4), slot_at = t_s + sl * kUnit;
#pragma unroll
                            for (int part = 0; part < (PREFIX ? 2 : 1); ++part)
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk)
                                    umma_ts(t_o, slot_at + part * 32 + kk * 8, v_h + kk * (kPageBytes >> 4), idesc_pv, part == 0 && kk == 0 ? first_acc : 1u);
                            umma_commit(bar_o);
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk) {
                                const uint32_t o = ((kk >> 2) * (kTileBytes / 2) + (kk & 3) * 32) >> 4;
                                if (kk == 0) umma_ss<false>(slot_at, q_at + o, k_h + o, idesc_qk);
                                else umma_ss<true>(slot_at, q_at + o, k_h + o, idesc_qk);
                            }
                            umma_commit(bar_s + sl * 8);
                            pp ^= 1u << sl;
                        };
                        if (b.narrow) {
                            unit(w, t & 1, acc);
                        } else {
                            unit(0, 0, acc);
                            if (fine) unit(1, 1, 1u);
                        }
                        if (!fine) break;
                        umma_commit(bar_empty + v_at * 8);
                        umma_commit(bar_empty + at * 8);
                        if (++at == kRowsRing) { at = 0; ph ^= 1; }
                    }
                }
                if (!__all_sync(0xffffffffu, fine)) { ok = false; break; }
                // where that thread has got to
                const int n = t_plain - b.t_lo;
                if (!b.narrow) {
                    if (n & 1) p_phase ^= 3;
                } else {
                    if (((n + 1) >> 1) & 1) p_phase ^= 1u << (b.t_lo & 1);
                    if ((n >> 1) & 1) p_phase ^= 2u >> (b.t_lo & 1);
                }
                const int moved = stage + 2 * n;
                phase ^= (uint32_t)((moved / kRowsRing) & 1);
                stage = moved % kRowsRing;
            }
            if (ok && t_plain > b.t_lo && t_plain + ahead == b.t_hi) q_done();
            for (int t = t_plain; ok && t < b.t_hi; ++t) {
                const bool more = t + ahead < b.t_hi;
                const int v_at = stage, k_at = stage + 1 == kRowsRing ? 0 : stage + 1;
                const uint32_t v_phase = phase, k_phase = k_at ? phase : phase ^ 1;
                if (!take(v_at, v_phase)) break;
                if (needs_clean(t)) clean_values(t, v_at);
                if (more && !take(k_at, k_phase)) break;
#pragma unroll 1
                for (int i = 0; ok && i < 2 / step; ++i) {
                    const int h = first + i, u = 2 * t + h, sl = b.narrow ? t & 1 : i;
                    if (u < end) pv(h, sl, v_at, i == 0 && !((t - b.t_lo) * (2 / step) & (kChainUnits<PREFIX> - 1)), u + step >= end);
                    if (ok && more && u + 2 * ahead < end) qk(h, sl, k_at);
                }
                if (!ok) break;
                release();
                if (more) {
                    release();
                    if (t + ahead + 1 == b.t_hi) q_done();
                }
            }
        }
        if (!ok) {
            if (lane == 0) give_up();
            __syncwarp();
            if (elect_one()) {
                umma_commit(smem_u32(&sm.drain[w]));      // products in flight still write tensor memory: wait (bounded)
                for (unsigned it = 0; it < (1u << 20); ++it)
                    if (mbar_try_wait(smem_u32(&sm.drain[w]), 0)) break;
            }
            __syncwarp();
        }
    } else {
        // ============================ softmax ============================
        const int wg = warp >> 2, r = tid & 127;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = t_s0 + wg * 128 + lane_base, t_o = t_o0 + wg * 128 + lane_base;
        const float scale2 = P.sm_scale * 1.4426950408889634f;      // scores are kept in units of log 2
        const float kLn2 = 0.6931471805599453f;
        const int my_tok = r / G, my_g = r - my_tok * G;
        uint32_t s_phase = 0, o_count = 0, last_phase = 0, pair_phase0 = 0, pair_phase1 = 0;   // s_phase: bit i is s_full[wg][i]'s
        int tile_no = 0;
        bool ok = true;
        for (int idx = 0; ok; ++idx) {
            const int slot = idx % kInfoRing;
            if (!warp_wait(smem_u32(&sm.info_full[slot]), (uint32_t)((idx / kInfoRing) & 1), abort_flag)) { ok = false; break; }
            const RowsBlock b = sm.info[slot];
            if (b.seq < 0) break;
            const int tok = (b.narrow ? 0 : wg * tile_rows) + my_tok;
            const bool live = r < G * tile_rows && tok < b.rows;
            const int lim = PREFIX ? b.len : min(b.off + b.i0 + tok + 1, b.len);
            // positions that every row of this warp sees: units below need no mask
            const int warp_lim = __shfl_sync(0xffffffffu, lim, 0);
            const int u_end = unit_end<PREFIX>(b, wg, tile_rows);
            float m_ref = neg_inf(), m_true = neg_inf(), l = 0.f;
            bool started = false;
            // accumulators set aside: their own reference, and how many units the present one holds
            float *aside = asides + ((size_t)me * 2 + wg) * kRowTile * kHeadDim + r * 4;      // [channels / 4][row]
            float m_aside = neg_inf();
            bool has_aside = false;
            auto aside_weight = [&]() { return m_aside == neg_inf() ? 0.f : fast_exp2((m_aside - m_ref) * scale2); };
            int u = 2 * b.t_lo + (b.narrow ? wg : 0);
            const int step = b.narrow ? 2 : 1;
            for (;;) {
                const int chain_end = min(u_end, u + kChainUnits<PREFIX> * step);
                for (; u < chain_end; u += step) {
                    const int h = u & 1, sl = b.narrow ? (u >> 1) & 1 : h;      // half of the tile, slot of the scores
                    const uint32_t t_u = t_s + sl * kUnit;
                    if (!warp_wait(smem_u32(&sm.s_full[wg][sl]), (s_phase >> sl) & 1, abort_flag)) { ok = false; break; }
                    s_phase ^= 1u << sl;
                    tc_fence_after();
                    float s[kUnit];
                    tmem_ld32_nowait(t_u, s);
                    tmem_ld32_nowait(t_u + 32, s + 32);
                    const unsigned bad = (sm.bad_pages[(tile_no + (u >> 1) - b.t_lo) & 7] >> (4 * h)) & 15u;
                    tmem_wait_ld();
                    pin32(s);
                    pin32(s + 32);
                    if ((u + 1) * kUnit > warp_lim || bad) {
#pragma unroll
                        for (int g = 0; g < kUnit / kPageSize; ++g) {
                            const int n = ((bad >> g) & 1) ? 0 : lim - u * kUnit - g * kPageSize;
#pragma unroll
                            for (int i = 0; i < kPageSize; ++i)
                                if (i >= n) s[g * kPageSize + i] = neg_inf();
                        }
                    }
                    // NaN wins every maximum here: a NaN score must make its row NaN, and the polynomial would lose it
                    float mx0 = max_nan(s[0], s[1]), mx1 = max_nan(s[2], s[3]), mx2 = max_nan(s[4], s[5]), mx3 = max_nan(s[6], s[7]);
#pragma unroll
                    for (int i = 8; i < kUnit; i += 8) {
                        mx0 = max3_nan(mx0, s[i], s[i + 1]);
                        mx1 = max3_nan(mx1, s[i + 2], s[i + 3]);
                        mx2 = max3_nan(mx2, s[i + 4], s[i + 5]);
                        mx3 = max3_nan(mx3, s[i + 6], s[i + 7]);
                    }
                    const float mx = max_nan(max_nan(mx0, mx1), max_nan(mx2, mx3));
                    m_true = max_nan(m_true, mx);
                    if (!started) {
                        m_ref = mx;
                        started = true;
                    } else {
                        const bool grow = mx > m_ref && (m_ref == neg_inf() || (mx - m_ref) * scale2 > kRescaleLog2);
                        if (__any_sync(0xffffffffu, grow)) {
                            // O of the units so far, once their products are done (all but the last are: S came after them)
                            if (!warp_wait(smem_u32(&sm.o_full[wg]), (o_count + 1) & 1, abort_flag)) { ok = false; break; }
                            tc_fence_after();
                            const float f = grow ? fast_exp2((m_ref - mx) * scale2) : 1.f;
                            if (grow) { l *= f; m_ref = mx; }
#pragma unroll 1
                            for (int c = 0; c < 8; ++c) {
                                float o[16];
                                tmem_ld16(t_o + c * 16, o);
                                uint32_t w[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * f);
                                tmem_st16(t_o + c * 16, w);
                            }
                        }
                    }
                    const float m2 = m_ref == neg_inf() ? 0.f : m_ref * scale2;
                    const unsigned long long scale22 = pack2(scale2, scale2), m22 = pack2(-m2, -m2);
                    unsigned long long la = pack2(0.f, 0.f), lb = la;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t hi[16], lo[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const unsigned long long x = fma2(pack2(s[c * 32 + 2 * i], s[c * 32 + 2 * i + 1]), scale22, m22);
                            float p0, p1;
                            if ((i & 7) >= 8 - kPolyPairs<PREFIX>) {
                                exp2_pair<PREFIX ? 5 : 4>(x, p0, p1);
                            } else {
                                unpack2(x, p0, p1);
                                p0 = fast_exp2(p0);
                                p1 = fast_exp2(p1);
                            }
                            if (i & 1) la = add2(la, pack2(p0, p1)); else lb = add2(lb, pack2(p0, p1));
                            hi[i] = pack_bf16(p0, p1);
                            if (PREFIX) lo[i] = pack_bf16(p0 - bf16lo_to_f32(hi[i]), p1 - bf16hi_to_f32(hi[i]));
                        }
                        tmem_st16(t_u + c * 16, hi);
                        if (PREFIX) tmem_st16(t_u + 32 + c * 16, lo);
                    }
                    float l0, l1;
                    unpack2(add2(la, lb), l0, l1);
                    l += l0 + l1;
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sm.p_full[wg][sl]));
                    ++o_count;       // one product of this group's O per unit
                }
                if (!ok || u >= u_end) break;
                // a chain is full: its products are waited for and set aside
                const int sl = b.narrow ? (u >> 1) & 1 : u & 1;      // the next scores came after all products but the last
                if (!warp_wait(smem_u32(&sm.s_full[wg][sl]), (s_phase >> sl) & 1, abort_flag) ||
                    !warp_wait(smem_u32(&sm.o_full[wg]), (o_count + 1) & 1, abort_flag)) { ok = false; break; }
                tc_fence_after();
                exchange_aside(t_o, aside, has_aside, true, aside_weight());
                has_aside = true;
                m_aside = m_ref;
            }
            if (!ok) break;
            tile_no += b.t_hi - b.t_lo;

            // ---- the block's (or piece's) result
            if (started) {
                if (!warp_wait(smem_u32(&sm.o_last[wg]), last_phase, abort_flag)) { ok = false; break; }
                last_phase ^= 1;
                tc_fence_after();
                if (has_aside) {
                    exchange_aside(t_o, aside, true, false, aside_weight());
                    tmem_wait_st();
                }
            }
            // A score was NaN or +infinity: the row is NaN, and not empty, whatever its reference was when the score came.
            if (!(m_true < __int_as_float(0x7f800000))) l = m_ref = __int_as_float(0x7fc00000);
            float w_own = 1.f, w_other = 0.f;     // weights of this group's accumulator and, narrow, the other's
            int c0 = 0, c1 = 4;                   // column chunks of 32 that this thread finishes
            uint32_t t_x = t_o;                   // the other group's accumulator
            if (b.narrow) {
                sm.ml[wg][r] = make_float2(m_ref, l);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.pair[0]));
                if (!warp_wait(smem_u32(&sm.pair[0]), pair_phase0, abort_flag)) { ok = false; break; }
                pair_phase0 ^= 1;
                tc_fence_after();
                const float2 other = sm.ml[wg ^ 1][r];
                const float M = max_nan(m_ref, other.x);
                if (M != neg_inf()) {
                    w_own = m_ref == neg_inf() ? 0.f : fast_exp2((m_ref - M) * scale2);
                    w_other = other.x == neg_inf() ? 0.f : fast_exp2((other.x - M) * scale2);
                }
                l = l * w_own + other.y * w_other;
                m_ref = M;
                c0 = wg * 2;
                c1 = c0 + 2;
                t_x = t_o0 + (wg ^ 1) * 128 + lane_base;
            }
            // Nothing visible, or weights that are all 0: the result is 0, whatever the values (and the accumulator) hold.
            const bool empty = m_ref == neg_inf();
            if (empty) w_own = w_other = 0.f;
            const bool any_empty = __any_sync(0xffffffffu, empty);
            const float inv = b.slot >= 0 ? 1.f : empty ? 0.f : 1.f / l;
            const int row = b.row0 + tok, h = b.head * G + my_g;
            const size_t out_row = PREFIX ? ((size_t)row * A.out_shards + A.slot) * Hq + h : (size_t)row * Hq + h;
            float *slot_base = b.slot >= 0 ? slots + (size_t)b.slot * kRowsSlotFloats : nullptr;
            const int slot_row = (b.narrow ? 0 : wg * kRowTile) + r;
            const bool dirty = !PREFIX && *reinterpret_cast<volatile int *>(&sm.dirty[slot]) != 0;
            float odd = 0.f;      // prefix: NaN once a result is not finite
            auto finish = [&](int c, const float (&o)[32]) {
                if (!live) return;
                if (PREFIX) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) odd = fmaf(o[i], 0.f, odd);
                }
                if (b.slot >= 0) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        __stcg(reinterpret_cast<float4 *>(slot_base) + (size_t)(c * 8 + i / 4) * (2 * kRowTile) + slot_row,
                               make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
                } else {
                    // whole 32-byte sectors: each thread's row is its own, so nothing else is coalesced
                    constexpr int kPer = PREFIX ? 8 : 16;
#pragma unroll
                    for (int i = 0; i < 32; i += kPer) {
                        uint32_t w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            w[e] = PREFIX ? __float_as_uint(o[i + e] * inv) : pack_bf16(o[i + 2 * e % kPer] * inv, o[i + (2 * e + 1) % kPer] * inv);
                        if (PREFIX) st_global_32b(A.o_part + out_row * kHeadDim + c * 32 + i, w);
                        else st_global_32b(A.out + out_row * kHeadDim + c * 32 + i, w);
                    }
                }
            };
            // one chunk at a time, in one rolled loop for both kinds of block: this code runs once per block, between loops
            // that it would push out of the instruction cache
#pragma unroll 1
            for (int c = c0; c < c1; ++c) {
                float o[32];
                tmem_ld32_nowait(t_o + c * 32, o);
                tmem_wait_ld();
                pin32(o);
                if (b.narrow || any_empty) {
                    float x[32];
                    tmem_ld32_nowait(t_x + c * 32, x);
                    tmem_wait_ld();
                    pin32(x);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        o[i] = w_own == 0.f ? 0.f : o[i] * w_own;
                        o[i] = w_other == 0.f ? o[i] : fmaf(x[i], w_other, o[i]);
                    }
                }
                finish(c, o);
            }
            if (dirty && live && !empty) add_hidden(A, P, b, lim, c0, c1, slot_base, slot_row, out_row);
            if (PREFIX) {
                const bool mine = live && !empty && l == l;
                if (__any_sync(0xffffffffu, mine && odd != odd)) mend_infinite(A, P, sm.info[slot], mine, c0, c1, slot_base, slot_row, out_row);
            }
            if (b.narrow) {
                // nobody may touch either accumulator, or ml, before both groups have read them
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.pair[1]));
                if (!warp_wait(smem_u32(&sm.pair[1]), pair_phase1, abort_flag)) { ok = false; break; }
                pair_phase1 ^= 1;
                if (PREFIX) {
                    // the second group's true maximum, to the first, in a word that only the first overwrites later
                    if (wg == 1) sm.ml[0][r].y = m_true;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sm.pair[0]));
                    if (!warp_wait(smem_u32(&sm.pair[0]), pair_phase0, abort_flag)) { ok = false; break; }
                    pair_phase0 ^= 1;
                    if (wg == 0) m_true = max_nan(m_true, sm.ml[0][r].y);
                }
            }
            if (live && (!b.narrow || wg == 0)) {
                if (b.slot >= 0) {
                    float *ml = slot_base + (size_t)2 * kRowTile * kHeadDim;
                    __stcg(ml + slot_row, empty ? neg_inf() : m_ref * scale2);
                    __stcg(ml + 2 * kRowTile + slot_row, l);
                    if (PREFIX) __stcg(ml + 4 * kRowTile + slot_row, m_true);
                } else {
                    const float lse = empty ? neg_inf() : fmaf(m_ref, P.sm_scale, log2f(l) * kLn2);
                    if (PREFIX) { A.m_part[out_row] = m_true * P.sm_scale; A.lse_part[out_row] = lse; }
                    else A.lse[out_row] = lse;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.info_empty[slot]));
        }
        if (!ok && lane == 0) give_up();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------ pieces of cut blocks
// CTA (c, part): the block that slice c began and did not finish, channels [32 part, 32 part + 32); thread = row.
// Bound by the latency of dependent loads, so whatever does not depend on another load is requested with it: the
// record and every slice's state first, then all maxima, then sums and channels of two pieces at a time.
constexpr int kRowsMergeParts = 4, kRowsMergeBatch = 2;
template <bool PREFIX>
__global__ void __launch_bounds__(2 * kRowTile, 2)
rows_merge_kernel(const __grid_constant__ RowsArgs A, const __grid_constant__ DevParams P, const RowsRecord *__restrict__ records,
                  const float *__restrict__ slots, int n_slices)
{
    __shared__ int slot_of[kRowsMaxCtas];      // the pieces' slots, in slice order
    __shared__ int n_pieces;
    grid_dependency_wait();
    grid_launch_dependents();
    const int me = (int)blockIdx.x, r = threadIdx.x;
    const int state = r > me && r < n_slices ? __ldcg(&records[r].head_state) : 0;
    const int4 *rec = reinterpret_cast<const int4 *>(records + me);
    const int4 r0 = __ldcg(rec), r1 = __ldcg(rec + 1), r2 = __ldcg(rec + 2), r3 = __ldcg(rec + 3);
    if (!r3.x) return;                          // has_tail; the same for every thread
    // the owner's tail, then every later slice's first piece up to the one that ends the block
    const int row0 = r0.z, rows = r1.x, narrow = r2.z, head = r0.y;
    __shared__ unsigned some[kRowsMaxCtas / 32], ends[kRowsMaxCtas / 32];
    if (r < kRowsMaxCtas) {
        const unsigned x = __ballot_sync(0xffffffffu, state != 0), y = __ballot_sync(0xffffffffu, state == 2);
        if ((r & 31) == 0) { some[r >> 5] = x; ends[r >> 5] = y; }
    }
    __syncthreads();
    if (r < 32) {
        // lane w holds word w; `past`: the block has ended in an earlier word
        unsigned x = r < kRowsMaxCtas / 32 ? some[r] : 0, y = r < kRowsMaxCtas / 32 ? ends[r] : 0;
        const unsigned has_end = __ballot_sync(0xffffffffu, y != 0);
        const int end_word = has_end ? __ffs((int)has_end) - 1 : 31;
        if (r > end_word) x = 0;
        else if (r == end_word && y) x &= (2u << (__ffs((int)y) - 1)) - 1u;
        int before = __popc(x), mine = before;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, before, o);
            if (r >= o) before += v;
        }
        if (r == 31) n_pieces = before + 1;
        int at = before - mine + 1;
        for (; x; x &= x - 1) slot_of[at++] = 2 * (r * 32 + __ffs((int)x) - 1);
        if (r == 0) slot_of[0] = 2 * me + 1;
    }
    __syncthreads();
    const int n = n_pieces;
    const int wg = r >> 7, G = P.group, Hq = P.num_q_heads, tile_rows = kRowTile / G;
    if (narrow && wg) return;
    const int rr = r & 127, tok = wg * tile_rows + rr / G, g = rr - rr / G * G;
    if (rr >= G * tile_rows || tok >= rows) return;
    const int part = (int)blockIdx.y;
    auto piece = [&](int i) { return slots + (size_t)slot_of[i] * kRowsSlotFloats; };
    constexpr size_t kMl = (size_t)2 * kRowTile * kHeadDim;
    float M = neg_inf(), top = neg_inf();
    for (int i0 = 0; i0 < n; i0 += 2 * kRowsMergeBatch) {
        float m[2 * kRowsMergeBatch], x[2 * kRowsMergeBatch];
#pragma unroll
        for (int i = 0; i < 2 * kRowsMergeBatch; ++i) {
            m[i] = i0 + i < n ? __ldcg(piece(i0 + i) + kMl + r) : neg_inf();
            x[i] = PREFIX && i0 + i < n ? __ldcg(piece(i0 + i) + kMl + 4 * kRowTile + r) : neg_inf();
        }
#pragma unroll
        for (int i = 0; i < 2 * kRowsMergeBatch; ++i) { M = fmaxf(M, m[i]); top = max_nan(top, x[i]); }
    }
    float z = 0.f;
    float4 acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n; i0 += kRowsMergeBatch) {
        float m[kRowsMergeBatch], l[kRowsMergeBatch];
        float4 x[kRowsMergeBatch][8];
#pragma unroll
        for (int i = 0; i < kRowsMergeBatch; ++i) {
            if (i0 + i < n) {
                const float *p = piece(i0 + i);
                m[i] = __ldcg(p + kMl + r);
                l[i] = __ldcg(p + kMl + 2 * kRowTile + r);
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    x[i][c] = __ldcg(reinterpret_cast<const float4 *>(p) + (size_t)(part * 8 + c) * (2 * kRowTile) + r);
            }
        }
#pragma unroll
        for (int i = 0; i < kRowsMergeBatch; ++i) {
            if (i0 + i >= n || m[i] == neg_inf()) continue;      // nothing visible in this piece
            const float w = fast_exp2(m[i] - M);
            z = fmaf(l[i], w, z);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                acc[c].x = fmaf(x[i][c].x, w, acc[c].x); acc[c].y = fmaf(x[i][c].y, w, acc[c].y);
                acc[c].z = fmaf(x[i][c].z, w, acc[c].z); acc[c].w = fmaf(x[i][c].w, w, acc[c].w);
            }
        }
    }
    const bool empty = M == neg_inf() && z == 0.f;      // not so if a piece's reference is NaN: its weight is NaN too
    const float inv = empty ? 0.f : 1.f / z;
    const float kLn2 = 0.6931471805599453f;
    const float lse = empty ? neg_inf() : (M + log2f(z)) * kLn2;
    const int row = row0 + tok, h = head * G + g;
    if (PREFIX) {
        const size_t o = ((size_t)row * A.out_shards + A.slot) * Hq + h;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            *reinterpret_cast<float4 *>(A.o_part + o * kHeadDim + part * 32 + i * 4) =
                make_float4(acc[i].x * inv, acc[i].y * inv, acc[i].z * inv, acc[i].w * inv);
        if (part == 0) { A.m_part[o] = top * P.sm_scale; A.lse_part[o] = lse; }
    } else {
        const size_t o = (size_t)row * Hq + h;
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            *reinterpret_cast<uint4 *>(A.out + o * kHeadDim + part * 32 + i * 4) =
                make_uint4(pack_bf16(acc[i].x * inv, acc[i].y * inv), pack_bf16(acc[i].z * inv, acc[i].w * inv),
                           pack_bf16(acc[i + 1].x * inv, acc[i + 1].y * inv), pack_bf16(acc[i + 1].z * inv, acc[i + 1].w * inv));
        if (part == 0) A.lse[o] = lse;
    }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled_fn()
{
    static std::mutex mu;
    static EncodeTiledFn fn = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)p;
    }
    return fn;
}
// Descriptors of one call (encoded every call: under a microsecond each).  q: [rows, Hq, 128] in boxes of 64 channels
// x G heads x 128 / G rows; K pages in boxes of one channel half (so that a tile is two K-major operands of 128
// positions), V pages whole (a page is one step of the second product).
inline int make_rows_maps(RowsMaps *m, const RowsArgs &A, const DevParams &P, char *msg, size_t msg_len)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) { snprintf(msg, msg_len, "cuTensorMapEncodeTiled entry point not available"); return -1; }
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    auto make = [&](CUtensorMap *out, const void *base, int dims, const cuuint64_t *size, const cuuint64_t *stride, const cuuint32_t *box) {
        return encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dims, const_cast<void *>(base), size, stride, box, ones,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    const cuuint64_t q_size[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)P.num_q_heads, (cuuint64_t)A.total_rows};
    const cuuint64_t q_stride[2] = {(cuuint64_t)kHeadDim * 2, (cuuint64_t)A.q_stride * 2};
    const cuuint32_t q_box[3] = {64, (cuuint32_t)P.group, (cuuint32_t)(kRowTile / P.group)};
    CUresult r = make(&m->q, A.q, 3, q_size, q_stride, q_box);
    const cuuint64_t hkv = (cuuint64_t)P.num_kv_heads, rows = (cuuint64_t)P.num_pages * kPageSize;
    // both layouts as [half][.][.][64 channels]: a page of a head is 16 rows of one plane, or one head of 16 planes
    const cuuint64_t hnd[4] = {64, kPageSize, (cuuint64_t)P.num_pages * hkv, 2}, hnd_stride[3] = {(cuuint64_t)kHeadDim * 2, kPageBytes, 128};
    const cuuint64_t nhd[4] = {64, hkv, rows, 2}, nhd_stride[3] = {(cuuint64_t)kHeadDim * 2, hkv * kHeadDim * 2, 128};
    const cuuint32_t hnd_box[4] = {64, kPageSize, 1, 1}, nhd_box[4] = {64, 1, kPageSize, 1};
    cuuint32_t box[4];
    std::copy(P.kv_nhd ? nhd_box : hnd_box, (P.kv_nhd ? nhd_box : hnd_box) + 4, box);
    const cuuint64_t *size = P.kv_nhd ? nhd : hnd, *stride = P.kv_nhd ? nhd_stride : hnd_stride;
    if (r == CUDA_SUCCESS) r = make(&m->k, A.k_cache, 4, size, stride, box);
    box[3] = 2;
    if (r == CUDA_SUCCESS) r = make(&m->v, A.v_cache, 4, size, stride, box);
    if (r != CUDA_SUCCESS) { snprintf(msg, msg_len, "cuTensorMapEncodeTiled failed with CUresult %d", (int)r); return -1; }
    return 0;
}

template <bool PREFIX>
cudaError_t launch_rows_kernels(const RowsMaps &maps, const RowsArgs &A, const DevParams &P, char *ws, int sms, cudaStream_t st)
{
    {   // per-device kernel attribute, set once under a lock
        static std::mutex mu;
        static bool done[64];
        int dev = 0;
        cudaGetDevice(&dev);
        std::lock_guard<std::mutex> lock(mu);
        if (!done[dev & 63]) {
            const cudaError_t e = cudaFuncSetAttribute(rows_kernel<PREFIX>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(RowsSmem));
            if (e != cudaSuccess) return e;
            done[dev & 63] = true;
        }
    }
    const RowsLayout L = rows_layout();
    RowsRecord *records = reinterpret_cast<RowsRecord *>(ws + L.record_off);
    float *asides = reinterpret_cast<float *>(ws + L.aside_off), *slots = reinterpret_cast<float *>(ws + L.slot_off);
    const int n = sms < kRowsMaxCtas ? sms : kRowsMaxCtas;
    cudaError_t e = launch_pdl(rows_kernel<PREFIX>, dim3(n), dim3(kRowsThreads), sizeof(RowsSmem), st, maps, A, P, records, asides, slots);
    if (e != cudaSuccess) return e;
    return launch_pdl(rows_merge_kernel<PREFIX>, dim3(n, kRowsMergeParts), dim3(2 * kRowTile), 0, st, A, P,
                      (const RowsRecord *)records, (const float *)slots, n);
}

}  // namespace qf
