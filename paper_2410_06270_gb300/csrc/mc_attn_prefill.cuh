// mc_attn_prefill.cuh -- attention of many new tokens per sequence over the paged cache, on
// the 5th-generation tensor cores.
//
// An item is 256 consecutive (token, head of the group) rows of one sequence and key head,
// as two tiles of 128 rows, and the keys that any of them sees, in units of 128.  Packing a
// group's heads into the rows lets them share a unit's keys and values, and keeps the
// diagonal short (256 rows are 256 / group tokens).  For each unit and tile
//   S = Q K^T            tcgen05.mma, both operands in shared memory, S in tensor memory
//   P = 2^(c S - m)      one row per thread: maximum, exponentials, sum, no exchange
//   O (+)= P V           tcgen05.mma with P (rounded to the cache's type) in tensor memory
//                        over S's columns, V as stored, key-major
// The two tiles alternate: the tensor pipe works for one while the other's softmax runs.
// The reference m moves only when a row's scores pass the maximum that it was taken from by 2^8 (the
// weights stay below 2^15), so O is rescaled in the first few units of a row and hardly after.
//
// Units of the whole batch, in order, are dealt to the CTAs (one per SM) as equal
// contiguous runs, found on the device from the lengths; a run that ends inside an item
// leaves (m, l, O) in fp32 and prefill_join_kernel adds an item's pieces in their order.
// This splits a long cache over the SMs when there are few rows, and balances short causal
// triangles, by the same rule.  Batches with many items deal them whole, largest first, from a
// common count (which CTA takes an item does not change its result).
//
// What bounds it: a unit's 32 MMAs are 2048 cycles of the tensor pipe; it takes 2830, as QK^T with
// both operands in shared memory runs at 78 cycles an MMA (8 KB each, all that shared memory
// gives in 64), PV with P in tensor memory at 65, and the change of tiles costs the rest; the
// softmax's 575 instructions a warp (1160 cycles) run beside it.  A prompt of 8192 tokens, 32 heads
// on 8 of 128: 357 us, 1.54 PFLOP/s of the visible pairs, 0.81 of cuBLAS's burst rate and 0.90 of its
// sustained one (at the power cap).  Capped scores take 1.7 times the time (a polynomial each: 175 us at
// 4096 tokens, 104 without), rows with scores beyond 3/4 of the cap 2.8 times (293).
//
// Warps: 0-3 and 4-7 the softmax of tile 0 and 1 (also the epilogue), 8 and 9 issue a tile's MMAs,
// 10 copies keys and values (TMA, a box per page and 64 columns), 11 the queries (TMA where a
// tile is whole tokens of the group's heads, else cp.async).
// Tensor memory: S (and P) of tile t at column 128 t, O at 256 + 128 t.
//
// Q4, the cache in 4 bits: warps 12-15 read the codes and write a tile as exact numbers of the type, in 310 instructions
// a warp a tile of 128 keys, two tiles a unit; 240 tokens over 30000 keys take 2260 cycles a tile all in all, more than the
// products where those are back to back (1400).  Beside the 16-bit cache: 64 tokens over 30000 keys 51 / 48 us, 16 x 16 over 4000 71 / 60, 1000 tokens 33 / 29, 240
// over 30000 134 / 96, 4096 tokens 155 / 104: the last have their keys unpacked before (mc_kv.cu) and come here as a 16-bit
// cache.  It hangs on registers: with 212 bytes spilled to a local memory that has no L1 left 64 tokens over 30000
// keys took 76 us.  None are spilled without a cap, but 8 bytes by fp16 heads of 128; 50 to 58 with one (the 16-bit kernel 66 to 114).
#pragma once
#include <math.h>

#include <algorithm>
#include <atomic>

#include <cuda.h>

#include "mc_attn_row.cuh"
#include "mc_host.h"
#include "mc_profile.h"
#include "mc_umma.cuh"

namespace mc {

constexpr int kPfRows = 256, kPfTile = 128, kPfKeys = 128;
constexpr int kPfMma = 8, kPfKv = 10, kPfUnpack = 12;  // MMA: two warps; after kPfKv the queries
constexpr int pf_threads(bool q4) { return q4 ? 512 : 384; }
constexpr int kPfMaxStages = 8;
constexpr int kPfAhead = 8;   // items that a block's roles may be apart (the copies lead the softmax by 4 at most)
constexpr int kPfCount = 32;  // the queue's count: a word of the 256 bytes behind the status word
// Items come from a queue where there are at least kPfQueueItems a block, none costs more than a
// block's mean, and the last ones given out (a sequence's first row tile) at most 1 / kPfQueueFirst of it.
constexpr int kPfQueueItems = 2, kPfQueueFirst = 4;

struct PfSeq {
    int first, n, len, prefix;  // first token row, new tokens, length, prefix
};

// Keys [base, end) that an item's rows see, base rounded down to a unit; at least one unit (of
// zeros, all masked), so that rows without keys take the same way.
struct PfKeys {
    int base, end, units, first;  // first: the first key that is seen
};

// Row tile mt of key head h of sequence b; of its units, n from u on.
struct PfItem {
    int b, h, mt, u, n;
    PfSeq s;
    PfKeys k;
};

struct PfShared {
    uint64_t kfull[kPfMaxStages], kempty[kPfMaxStages];  // ring of keys / values
    uint64_t qfull[2], qempty[2], sfull[2], pfull[2], ofull[2];  // per tile
    uint64_t drain, vpatch;
    uint32_t tmem_base;
    volatile int abort;
    int odd;                                             // a finished row came out infinite or NaN
    int b[2], h[2], mt[2], u[2];                         // where this CTA's run starts and ends
    int off;                                             // the end's cost offset in its item
    int run;                                             // cost of a run
    int64_t total;                                       // cost of the batch
    int queued;                                          // items come from the common queue, not as a run
    uint64_t ifull[kPfAhead], iempty[kPfAhead];
    union {
        int sums[2][32];                                 // before the roles part
        PfItem item[kPfAhead];                           // the block's items, in turn; n = 0: no more
    };
};

template <int D>
struct PfShape {
    static constexpr int kHalf = kPfKeys * 128;               // 64 columns of a tile: SW128 atoms
    static constexpr int kTileBytes = kHalf * (D / 64);
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kHdr = 1024;
    static constexpr int kRing = kHdr + 2 * kTileBytes;       // after the two query tiles
    static constexpr int kSmem = kRing + kStages * kTileBytes;
};
static_assert(sizeof(PfShared) <= PfShape<128>::kHdr, "prefill header");
static_assert(PfShape<128>::kSmem <= 232448, "prefill shared memory");

struct PfOpen;

struct PfParams {
    AttnParams a;
    PfOpen *open;
    int32_t *odd;  // of each CTA: whether a row that it finished came out infinite or NaN
    float *part;
    uint64_t timeout_ns;
    int debug;
    int q_boxes;   // a tile's queries are boxes of whole groups of heads (the group divides 128)
    int out32;     // rows of the output start at multiples of 32 bytes
    int box_rows;  // rows of a copied box: the largest power of two that divides a page, at most a unit
};

// Header of a CTA's open item: its pieces are this CTA's tail partial and the head
// partials of the next pieces - 1 CTAs; 0: none.
struct PfOpen {
    int32_t pieces, b, h, mt;
};

// A partial: O [D / 4][256 rows] float4 (a warp's rows are consecutive), then (m, l).
__host__ __device__ constexpr size_t pf_part_floats(int D) { return (size_t)kPfRows * (D + 2); }

__device__ __forceinline__ bool g_wait(uint64_t *bar, uint32_t parity, const PfParams &p, PfShared *sh)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    while (true) {
        if (mbar_try_wait_sleep(bar, parity, kWaitHintNs)) return true;
        if (sh->abort) return false;
        if (globaltimer_ns() - t0 > p.timeout_ns) {
            set_status(p.a.status, MC_ERR_TIMEOUT);
            sh->abort = 1;
            return false;
        }
    }
}

// One answer for the warp (what follows is executed by all of its lanes together).
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, const PfParams &p, PfShared *sh)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    return __all_sync(0xffffffffu, g_wait(bar, parity, p, sh));
}

// ------------------------------------------------------------------ items --

__device__ __forceinline__ PfSeq pf_seq(const AttnParams &p, int b, int32_t *status)
{
    PfSeq s;
    s.n = seq_rows(p.b, b, s.first, status);
    s.len = seq_len(p.b, p.c, b, status);
    s.prefix = p.prefix ? __ldg(p.prefix + b) : 0;
    return s;
}

__device__ __forceinline__ PfKeys pf_keys(const AttnParams &p, const PfSeq &s, int mt)
{
    PfKeys k;
    const int last = min((mt + 1) * kPfRows, s.n * p.group) - 1;
    const int p_lo = s.len - s.n + p.by_group.div(mt * kPfRows);
    const int p_hi = s.len - s.n + p.by_group.div(last);
    k.end = p_hi < 0 ? 0 : min(s.len, max(p_hi + 1, s.prefix));
    k.first = p.window ? max(0, p_lo - p.window + 1) : 0;
    k.base = k.first & ~(kPfKeys - 1);
    k.units = max(1, (k.end - k.base + kPfKeys - 1) / kPfKeys);
    return k;
}

__device__ __forceinline__ int pf_tiles(const AttnParams &p, const PfSeq &s)
{
    return (s.n * p.group + kPfRows - 1) / kPfRows;
}

// The next item of a block's run, which ends before unit `u` of item (b, h, mt).
struct PfRun {
    int b, h, mt, u;
};
__device__ __forceinline__ int pf_units(const PfRun &r, const PfItem &at)  // 0: the run is over
{
    return (at.b == r.b && at.h == r.h && at.mt == r.mt ? r.u : at.k.units) - at.u;
}
__device__ __forceinline__ void pf_next(const AttnParams &p, const PfRun &run, PfItem &at)
{
    const bool over = at.u + at.n < at.k.units;
    at.u = at.n = 0;
    if (over) return;
    if (++at.mt >= pf_tiles(p, at.s)) {
        at.mt = 0;
        if (++at.h >= p.c.kv_heads) {
            at.h = 0;
            do {
                if (++at.b >= p.b.seqs) return;
                at.s = pf_seq(p, at.b, nullptr);
            } while (at.s.n == 0);
        }
    }
    at.k = pf_keys(p, at.s, at.mt);
    at.n = pf_units(run, at);
}

// The block's turn-th item.  The role that copies keys finds the items, one ahead; the others read
// them, where they need a field (held in registers through a unit's softmax, they would be spilled).
__device__ __forceinline__ const volatile PfItem *pf_item(const PfParams &pp, PfShared *sh, int turn)
{
    const volatile PfItem *it = &sh->item[turn % kPfAhead];
    return warp_wait(&sh->ifull[turn % kPfAhead], (turn / kPfAhead) & 1, pp, sh) && it->n > 0 ? it : nullptr;
}
__device__ __forceinline__ int pf_rows(const AttnParams &p, const volatile PfItem *it) { return it->s.n * p.group - it->mt * kPfRows; }

// What an item costs on top of its units, in units: the change of queries, the first
// unit's softmax with no other work beside it, the epilogue.  Runs are equal in cost
// (equal in units alone, a CTA with the 29 short items at a causal prompt's start took a
// third longer than the mean: 8192 tokens 489 us against 364).
constexpr int kPfItemCost = 2;

// The order in which a run takes an item's units.  Runs of one key head start at different
// places of a long cache; if each went straight on, a unit would be read for one row tile now
// and for the next ones a large part of the call later, when L2 has lost it.  An item longer
// than a run's cost R is started at the unit that is `spent` modulo R, spent the cost since the
// run's start, and taken round: all runs are then at the same units modulo R at the same time.
// 509 tokens over 30000 keys of 8 heads, 8 row tiles a head: 190 -> 167 us, 1024 over 60000 758 ->
// 653.  Where the sequence's cache stays in L2 it goes straight on: 300 tokens over 120000 keys of
// one head (61 MB) 190 us, taken round 200.
constexpr int64_t kPfL2 = 64 << 20;
struct PfOrder {
    int first, n, shift;
    __device__ __forceinline__ PfOrder(const AttnParams &p, int key_bytes, const volatile PfItem &at, int run, int spent)
        : first(at.u), n(at.n), shift(0)
    {
        if (at.k.units <= run || (int64_t)at.s.len * p.c.kv_heads * key_bytes <= kPfL2) return;
        const int ahead = (spent - at.u) % run, to = ahead < 0 ? ahead + run : ahead;
        if (to < n) shift = to;
    }
    __device__ __forceinline__ int unit(int i) const { return first + (i + shift < n ? i + shift : i + shift - n); }
};

// Costs of 32 sequences from b0 on (per key head) into sums, by one warp: the
// sequences' items are laid end to end and taken 32 at a time.  Returns their total, and in mix
// (if it is not NULL) what the choice of schedule asks for, of the lane's sequence.
struct PfMix {
    int items, most, first;  // items of a key head, cost of the largest and of the first one
};
__device__ __forceinline__ int64_t pf_sums(const AttnParams &p, int *sums, int b0, int lane, int32_t *status, PfMix *mix)
{
    PfSeq s = {0, 0, 0, 0};
    if (b0 + lane < p.b.seqs) s = pf_seq(p, b0 + lane, status);
    const int tiles = pf_tiles(p, s);
    if (mix && tiles) {
        const int first = pf_keys(p, s, 0).units + kPfItemCost, last = pf_keys(p, s, tiles - 1).units + kPfItemCost;
        *mix = {tiles, max(first, last), first};
    }
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    const int all = __shfl_sync(0xffffffffu, upto, 31);
    __syncwarp();
    sums[lane] = 0;
    __syncwarp();
    for (int i0 = 0; i0 < all; i0 += 32) {
        const int i = i0 + lane;
        int own = 0;  // the sequence that holds item i: the lanes whose upto <= i come before it
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1)
            if (__shfl_sync(0xffffffffu, upto, own + d - 1) <= i) own += d;
        own = min(own, 31);
        PfSeq t;
        t.first = 0;
        t.n = __shfl_sync(0xffffffffu, s.n, own);
        t.len = __shfl_sync(0xffffffffu, s.len, own);
        t.prefix = __shfl_sync(0xffffffffu, s.prefix, own);
        const int before = __shfl_sync(0xffffffffu, upto - tiles, own);
        if (i < all) atomicAdd(&sums[own], pf_keys(p, t, i - before).units + kPfItemCost);
    }
    __syncwarp();
    int64_t sum = sums[lane];
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum;
}

// ------------------------------------------------------------ device pieces --

#define PF_R8(a, i) \
    "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3]), "=r"(a[i + 4]), "=r"(a[i + 5]), "=r"(a[i + 6]), "=r"(a[i + 7])
#define PF_P8(a, i) \
    "+r"(a[i]), "+r"(a[i + 1]), "+r"(a[i + 2]), "+r"(a[i + 3]), "+r"(a[i + 4]), "+r"(a[i + 5]), "+r"(a[i + 6]), "+r"(a[i + 7])
#define PF_I8(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3]), "r"(a[i + 4]), "r"(a[i + 5]), "r"(a[i + 6]), "r"(a[i + 7])

// 32 columns of the warp's 32 lanes; the values may be used after pf_ld_wait of them.
__device__ __forceinline__ void pf_ld32(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : PF_R8(r, 0), PF_R8(r, 8), PF_R8(r, 16), PF_R8(r, 24)
        : "r"(taddr)
        : "memory");
}

// Waits for every load of the warp; the operands tie the registers' uses to it.
__device__ __forceinline__ void pf_ld_wait(uint32_t *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : PF_P8(r, 0), PF_P8(r, 8), PF_P8(r, 16), PF_P8(r, 24) : : "memory");
}

__device__ __forceinline__ void pf_tie(uint32_t *r)
{
    asm volatile("" : PF_P8(r, 0), PF_P8(r, 8), PF_P8(r, 16), PF_P8(r, 24) : : "memory");
}

__device__ __forceinline__ void pf_st16(uint32_t taddr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 PF_I8(r, 0), PF_I8(r, 8)
                 : "memory");
}

// 16 columns, waited for.
__device__ __forceinline__ void pf_ld16(uint32_t taddr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : PF_R8(r, 0), PF_R8(r, 8)
        : "r"(taddr)
        : "memory");
}

// Instruction descriptor: fp16 or bf16 operands, fp32 accumulator, M = 128; b_mn: the B
// operand's N dimension is the contiguous one (values: [key][d]).
__host__ __device__ constexpr uint32_t pf_idesc(bool bf16, int N, bool b_mn)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24);
}

// Shared-memory descriptors, 128-byte swizzle: the upper word is the same for all operands
// here (1024 bytes from one group of 8 rows, or keys, to the next), so a descriptor is its
// lower word, and the steps along a tile are additions to it.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
// Rows of 64 columns, K contiguous.
__device__ __forceinline__ uint32_t pf_desc_k(uint32_t addr) { return ((addr >> 4) & 0x3FFFu) | (1u << 16); }
// A value tile as B operand, N (d) contiguous: atoms of 64 d x 8 keys, a half-tile from one
// 64-column block to the next.
__device__ __forceinline__ uint32_t pf_desc_mn(uint32_t addr, uint32_t half) { return ((addr >> 4) & 0x3FFFu) | ((half >> 4) << 16); }

__device__ __forceinline__ void pf_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "n"(kDescHi)
        : "memory");
}

__device__ __forceinline__ void pf_mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),
        "r"(a_tmem), "r"(b), "r"(idesc), "r"((uint32_t)accumulate), "n"(kDescHi)
        : "memory");
}

// One box of a page: 64 columns from c on, rows from r on, of a head.
__device__ __forceinline__ void pf_tma(uint32_t dst, const CUtensorMap *map, int c, int r, int head, int page, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                 "l"(map), "r"(smem_u32(bar)), "r"(c), "r"(r), "r"(head), "r"(page)
                 : "memory");
}

__device__ __forceinline__ void pf_tma3(uint32_t dst, const CUtensorMap *map, int c, int head, int token, uint64_t *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                 "l"(map), "r"(smem_u32(bar)), "r"(c), "r"(head), "r"(token)
                 : "memory");
}

// 16 bytes, or 16 zeros where !real (the address is then not read).
__device__ __forceinline__ void pf_copy16z(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}

// Registers: the softmax threads hold a row of 128 scores, the others little.  The shares
// (2 warpgroups of kSoft and the others of kRest) are within what the block has at
// launch, kAll a thread (checked before the launch: a larger share would wait for ever).
// Q4 has a warpgroup more.
template <bool Q4>
struct PfRegs {
    static constexpr int kAll = Q4 ? 128 : 168, kSoft = Q4 ? 192 : 208, kRest = Q4 ? 48 : 80, kUnpack = 80;
    static_assert(2 * kSoft + kRest + (Q4 ? kUnpack : 0) <= (Q4 ? 4 : 3) * kAll, "register shares");
    static __device__ __forceinline__ void take() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoft)); }
    static __device__ __forceinline__ void give() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRest)); }
    static __device__ __forceinline__ void give_unpack() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kUnpack)); }
};

// ---------------------------------------------------------------- softmax --

// What the scores go through before the softmax.
enum { kPfPlain = 0, kPfBias = 1, kPfCap = 2 };  // kPfCap: and the bias, if there is one

// The low n bits, n any number.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// One row's 128 scores of a unit.  c: the factor to units of log 2; at0: the first key's
// distance (key - query); slope in units of log 2; [lo, hi): the keys of the unit that the
// row sees, where `masked`.
template <bool BF16, int MODE>
__device__ __forceinline__ void pf_softmax(uint32_t (&s)[128], uint32_t s_tmem, uint32_t o_tmem, int D, bool masked, int lo,
                                           int hi, float c, float cap, bool biased, float slope, float at0, bool fresh, float &m, float &l)
{
    if (MODE == kPfCap) {
        float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 128; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = fmaxf(t[k], fmaxf(fabsf(__uint_as_float(s[i + k])), fabsf(__uint_as_float(s[i + k + 4]))));
        const float most = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) * c;
        auto cap_all = [&](auto form) {
#pragma unroll
            for (int i = 0; i < 128; i += 2) {
                float a, b;
                unpair2(form(mul2(pair2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), pair2(c, c)), cap), a, b);
                s[i] = __float_as_uint(a);
                s[i + 1] = __float_as_uint(b);
            }
        };
        // (rows of scores below 3/4 of the cap, the common ones, without the clamps and the reciprocal)
        if (most <= kTanhNear) cap_all([](uint64_t y, float top) { return capped2_near(y, top); });
        else cap_all([](uint64_t y, float top) { return capped2(y, top); });
        __syncwarp();
        c = 1.f;
    }
    if (MODE == kPfBias || (MODE == kPfCap && biased)) {
        // the bias is slope * (at0 + i): the distance counts up exactly, two keys at a time;
        // without a cap it is brought to the scores' units, so that c applies to both
        uint64_t at = pair2(at0, at0 + 1.f);
        const uint64_t two = pair2(2.f, 2.f);
        const float sl = MODE == kPfBias ? slope / c : slope;
        const uint64_t sl2 = pair2(sl, sl);
#pragma unroll
        for (int i = 0; i < 128; i += 2) {
            float a, b;
            unpair2(fma2(sl2, at, pair2(__uint_as_float(s[i]), __uint_as_float(s[i + 1]))), a, b);
            at = add2(at, two);
            s[i] = __float_as_uint(a);
            s[i + 1] = __float_as_uint(b);
        }
    }
    if (masked) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t see = low_bits(hi - 32 * q) & ~low_bits(lo - 32 * q);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (!((see >> i) & 1u)) s[32 * q + i] = 0xff800000u;
        }
    }
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = __uint_as_float(s[i]);
#pragma unroll
    for (int i = 4; i < 128; i += 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = i + k + 4 < 128 ? fmaxf(t[k], fmaxf(__uint_as_float(s[i + k]), __uint_as_float(s[i + k + 4])))
                                                           : fmaxf(t[k], __uint_as_float(s[i + k]));
    }
    float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
    top *= c;
    if (__any_sync(0xffffffffu, top > m + kLazy)) {
        const float next = top > m + kLazy ? top - kBelow : m;
        const float keep = next == m ? 1.f : ex2(m - next);
        m = next;
        l *= keep;
        if (!fresh) {
            for (int d = 0; d < D; d += 16) {
                uint32_t o[16];
                pf_ld16(o_tmem + d, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
                pf_st16(o_tmem + d, o);
            }
        }
    }
    const float ref = m == -INFINITY ? 0.f : -m;
    const uint64_t c2 = pair2(c, c), r2 = pair2(ref, ref);
    uint64_t sum[2] = {pair2(0.f, 0.f), pair2(0.f, 0.f)};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint64_t x = pair2(__uint_as_float(s[32 * q + 2 * i]), __uint_as_float(s[32 * q + 2 * i + 1]));
            const uint64_t y = fma2(x, c2, r2);
            float a, b;
            unpair2(y, a, b);
            a = ex2(a);
            b = ex2(b);
            sum[i & 1] = add2(sum[i & 1], pair2(a, b));
            w[i] = pack2<BF16>(a, b);  // rounded to the cache's type for the product with V; l keeps fp32
        }
        pf_st16(s_tmem + 16 * q, w);
    }
    float a, b;
    unpair2(add2(sum[0], sum[1]), a, b);
    l += a + b;
}

// ------------------------------------------------------------------ kernel --

// Where a warp's 32 keys of a unit lie in either side of the 4-bit cache: two runs of 16, each in one page.  Byte offsets of
// the lane's first chunk of codes in each run (negative: no such page, zeros), and of the words of the lane's own key
// (negative: zeros, as for keys that no row sees).
struct PfPlace {
    int64_t codes[2], words;
};

// A lane's part of them: 16-byte chunks of codes, as they lie, kPer of them, 32 / kPer keys apart, and its key's words; and
// into a tile, as exact numbers of the type, to where a copy would have put them (a group's 64 columns in 8 chunks of 16
// bytes, swizzled).
template <int D>
struct PfRaw {
    static constexpr int kPer = D / 32, kChunks = D / 32, kStep = 32 / kPer;
    uint4 w[kPer];
    uint32_t words;

    __device__ __forceinline__ void load(const uint16_t *side, const PfPlace &at)
    {
        const uint8_t *base = reinterpret_cast<const uint8_t *>(side);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int run = i / (kPer / 2), k = i % (kPer / 2);
            w[i] = at.codes[run] < 0 ? make_uint4(0, 0, 0, 0)
                                     : __ldg(reinterpret_cast<const uint4 *>(base + at.codes[run] + k * kStep * kv4_code_bytes(D)));
        }
        words = at.words < 0 ? 0u
                : D == 128   ? __ldg(reinterpret_cast<const uint32_t *>(base + at.words))
                             : __ldg(reinterpret_cast<const uint16_t *>(base + at.words));
    }

    // tile: of the warp's first key
    template <bool BF16>
    __device__ __forceinline__ void store(uint8_t *tile, int half, int lane) const
    {
        using P = Kv4Pairs<BF16>;
        constexpr int kGroups = D / kKv4Group;
        const int ch = lane % kChunks;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int key = lane / kChunks + kStep * i;
            const uint32_t word = __shfl_sync(0xffffffffu, words, key);
            uint32_t z[kGroups], sc[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                z[g] = P::zeros(word >> (16 * g));
                sc[g] = P::scales(word >> (16 * g));
            }
            const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
            uint32_t y[4][4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[x][j] = P::magic(v[x], j);
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[x][j] = P::mul(P::sub(y[x][j], z[x % kGroups]), sc[x % kGroups]);
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *reinterpret_cast<uint4 *>(tile + (x % kGroups) * half + key * 128 + ((((4 * ch + x) / kGroups) ^ (key & 7)) << 4)) =
                    make_uint4(y[x][0], y[x][1], y[x][2], y[x][3]);
        }
    }
};

// QUEUE: the batch may have the items for a queue (the host's bound), so the kernel looks at them.
template <int D, bool BF16, int MODE, bool QUEUE, bool Q4>
__global__ void __launch_bounds__(pf_threads(Q4), 1) prefill_kernel(const PfParams pp, const __grid_constant__ CUtensorMap kmap,
                                                                   const __grid_constant__ CUtensorMap vmap,
                                                                   const __grid_constant__ CUtensorMap qmap)
{
    using Sh = PfShape<D>;
    using Regs = PfRegs<Q4>;
    constexpr int kKeyBytes = Q4 ? 2 * kv4_row_bytes(D) : 4 * D;
    extern __shared__ __align__(1024) uint8_t smem[];
    PfShared *sh = reinterpret_cast<PfShared *>(smem);
    const AttnParams &p = pp.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < Sh::kStages; ++i) {
            mbar_init(&sh->kfull[i], Q4 ? 4 : 1);
            mbar_init(&sh->kempty[i], 2);
        }
        mbar_init(&sh->vpatch, 1);
        for (int i = 0; i < kPfAhead; ++i) {
            mbar_init(&sh->ifull[i], 1);
            mbar_init(&sh->iempty[i], 8);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&sh->qfull[t], pp.q_boxes ? 1 : 32);
            mbar_init(&sh->qempty[t], 1);
            mbar_init(&sh->sfull[t], 1);
            mbar_init(&sh->pfull[t], 4);
            mbar_init(&sh->ofull[t], 1);
        }
        mbar_init(&sh->drain, 2);
        sh->abort = sh->odd = 0;
        fence_mbar_init();
    }
    if (warp == kPfMma) tmem_alloc(&sh->tmem_base, 512);
    pdl_wait();
    if (warp < 2) {
        // where the run starts (warp 0) and ends (warp 1)
        int *sums = sh->sums[warp];
        int64_t total = 0;
        PfMix mix = {0, 0, 0};
        for (int b0 = 0; b0 < p.b.seqs; b0 += 32) total += pf_sums(p, sums, b0, lane, p.status, QUEUE ? &mix : nullptr);
        total *= p.c.kv_heads;
        const int64_t ctas = total < (int64_t)gridDim.x ? total : gridDim.x;
        // Long prompts have items enough to be dealt one by one, largest first: no pieces to join, and
        // SMs that are slower than others (units of the same work take up to a tenth longer on some) get
        // fewer.  Runs / queue: 3000 tokens, 2.5 items a block, 84 / 73 us, 4096 124 / 105, 8192 378 / 358, four
        // prompts of 2000 142 / 122, six ragged ones on top of a cache 247 / 237.
        bool queued = false;
        if (QUEUE) {
            const int64_t items = (int64_t)__reduce_add_sync(0xffffffffu, mix.items) * p.c.kv_heads;
            const int most = __reduce_max_sync(0xffffffffu, mix.most), first = __reduce_max_sync(0xffffffffu, mix.first);
            queued = items >= kPfQueueItems * ctas && most * ctas <= total && kPfQueueFirst * first * ctas <= total;
        }
        int fb = -1, fh = 0, fmt = 0, fu = 0, off = 0;
        if (!queued && (int64_t)blockIdx.x < ctas) {
            int64_t r = muldiv64(total, blockIdx.x + warp, (int)ctas);  // cost before the place
            if (r == total) fb = p.b.seqs;
            for (int b0 = 0; b0 < p.b.seqs && fb < 0; b0 += 32) {
                if (p.b.seqs > 32) pf_sums(p, sums, b0, lane, nullptr, nullptr);
                const int64_t own = (int64_t)sums[lane] * p.c.kv_heads;
                int64_t upto = own;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int64_t o = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += o;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, upto > r);
                if (!hit) {
                    r -= __shfl_sync(0xffffffffu, upto, 31);
                    continue;
                }
                const int who = __ffs(hit) - 1;
                r -= __shfl_sync(0xffffffffu, upto - own, who);
                const int per = __shfl_sync(0xffffffffu, sums[lane], who);
                fb = b0 + who;
                fh = (int)div64(r, per);
                off = (int)(r - (int64_t)fh * per);
                const PfSeq s = pf_seq(p, fb, nullptr);
                const int tiles = pf_tiles(p, s);
                for (int t0 = 0; t0 < tiles; t0 += 32) {
                    const int n = t0 + lane < tiles ? pf_keys(p, s, t0 + lane).units + kPfItemCost : 0;
                    int sum = n;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) {
                        const int o = __shfl_up_sync(0xffffffffu, sum, d);
                        if (lane >= d) sum += o;
                    }
                    const unsigned in = __ballot_sync(0xffffffffu, sum > off);
                    if (in) {
                        const int w = __ffs(in) - 1;
                        fmt = t0 + w;
                        off -= __shfl_sync(0xffffffffu, sum - n, w);
                        fu = max(0, off - kPfItemCost);
                        break;
                    }
                    off -= __shfl_sync(0xffffffffu, sum, 31);
                }
            }
        }
        if (lane == 0) {
            sh->b[warp] = fb;
            sh->h[warp] = fh;
            sh->mt[warp] = fmt;
            sh->u[warp] = fu;
            if (warp) {
                sh->queued = queued;
                sh->total = total;
                sh->off = off;
                sh->run = max(1, (int)div64(total, max(ctas, (int64_t)1)));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // All 512 columns are this block's, so they start at column 0: constant addresses below
    if (sh->tmem_base != 0) {
        if (tid == 0) set_status(p.status, MC_ERR_CUDA);
        sh->abort = 1;
    }
    if (warp >= kPfMma) {
        if (Q4 && warp >= kPfUnpack) {
            Regs::give_unpack();
            // ------------------------------------------------- keys and values in 4 bits --
            // A warp 32 keys of a tile: loaded a tile ahead, while the tile before is written out.
            const int first_key = 32 * (warp - kPfUnpack);
            int it = 0;
            bool ok = !(pp.debug & kDebugNoProducer);
            const volatile PfItem *item = ok ? pf_item(pp, sh, 0) : nullptr;
            int b = 0, h = 0, from = 0, to = 0, spent = 0;  // keys that the item's rows see, from its first unit's first on
            int base = 0, next[2], next_row[2];
            const int block_bytes = p.c.page_size * kv4_row_bytes(D);
            PfPlace at;
            // the pages of the warp's two runs of unit u, as the table has them
            auto look = [&](int u) {
#pragma unroll
                for (int run = 0; run < 2; ++run) {
                    const int j = u * kPfKeys + first_key + 16 * run;
                    next[run] = -1;
                    next_row[run] = 0;
                    if (j < to && j + 16 > from)
                        next[run] = __ldg(p.b.table + (int64_t)b * p.b.table_width + p.c.page.div(base + j, next_row[run]));
                }
            };
            auto turn_to = [&](int u) {  // what look found
                const int j0 = u * kPfKeys + first_key;
#pragma unroll
                for (int run = 0; run < 2; ++run) {
                    const int j = j0 + 16 * run;
                    at.codes[run] = -1;
                    if ((unsigned)next[run] >= (unsigned)p.c.num_pages) {
                        if (j < to && j + 16 > from) set_status(p.status, MC_ERR_RANGE);
                    } else {
                        at.codes[run] = next[run] * p.c.page_stride + (int64_t)h * block_bytes +
                                        ((next_row[run] + lane / PfRaw<D>::kChunks) * kv4_code_bytes(D) + 16 * (lane % PfRaw<D>::kChunks));
                    }
                }
                const int run = lane >> 4, page = run ? next[1] : next[0], row = run ? next_row[1] : next_row[0];
                at.words = (unsigned)page < (unsigned)p.c.num_pages && j0 + lane >= from && j0 + lane < to
                               ? page * p.c.page_stride + (int64_t)h * block_bytes +
                                     (p.c.page_size * kv4_code_bytes(D) + (row + (lane & 15)) * kv4_word_bytes(D))
                               : -1;
            };
            auto enter = [&]() {
                b = item->b;
                h = item->h;
                base = item->k.base;
                from = item->k.first - base;
                to = min(item->k.end, item->s.len) - base;
            };
            // tile number `it`, when its slot is free
            auto put = [&](const PfRaw<D> &x) {
                const int slot = it % Sh::kStages;
                if (it >= Sh::kStages && !(ok = warp_wait(&sh->kempty[slot], (it / Sh::kStages + 1) & 1, pp, sh))) return;
                x.template store<BF16>(smem + Sh::kRing + slot * Sh::kTileBytes + first_key * 128, Sh::kHalf, lane);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->kfull[slot]);
                ++it;
            };
            PfRaw<D> k, v;
            int n = 0, u = 0;
            PfOrder order(p, kKeyBytes, sh->item[0], sh->run, 0);
            if (item) {
                enter();
                n = item->n;
                u = order.unit(0);
                look(u);
                turn_to(u);
                k.load(p.c.k, at);
            }
            for (int turn = 0; ok && n > 0;) {
                for (int i = 0; ok && i < n; ++i) {
                    v.load(p.c.v, at);
                    if (i + 1 < n) {
                        u = order.unit(i + 1);
                        look(u);
                    }
                    put(k);
                    if (!ok) break;
                    if (i + 1 == n) {
                        spent += n + kPfItemCost;
                        item = pf_item(pp, sh, ++turn);
                        n = 0;
                        if (item) {
                            enter();
                            order = PfOrder(p, kKeyBytes, *item, sh->run, spent);
                            n = item->n;
                            u = order.unit(0);
                            look(u);
                        }
                        i = -2;  // (the item is done)
                    }
                    if (n) {
                        turn_to(u);
                        k.load(p.c.k, at);
                    }
                    put(v);
                    if (i < 0) break;
                }
            }
        } else if (Regs::give(), warp >= kPfKv) {  // one instruction for the warpgroup
            // -------------------------------------------------------------- copies --
            const uint32_t smem0 = smem_u32(smem);
            if (warp == kPfKv) {
                // keys and values: lane i copies the i-th box (of a page) of a tile.  A page that is
                // not there, and boxes before the first key or past the last, are read beyond the map:
                // zeros.
                const int boxes = kPfKeys / pp.box_rows;
                int it = 0, patches = 0;
                bool ok = !(pp.debug & kDebugNoProducer);
                // The block's items.  Where they come from the queue: by falling row tile, then sequence and
                // key head; the first is that of the block's number, the next ones those that a common
                // count (zero between calls) gives it.
                const bool queued = QUEUE && sh->queued;
                const PfRun run = {sh->b[1], sh->h[1], sh->mt[1], sh->u[1]};
                int level = 0, above = 0, tiles = 0;  // row tile at hand, items of higher ones; lane: its sequence's
                auto queue_item = [&](int which, PfItem &x) {
                    unsigned have;
                    while ((have = __ballot_sync(0xffffffffu, tiles > level)), which - above >= __popc(have) * p.c.kv_heads && level >= 0) {
                        above += __popc(have) * p.c.kv_heads;
                        --level;
                    }
                    x.u = x.n = 0;
                    if (level < 0 || which < 0) return;  // (below 0: the workspace was not zeroed)
                    x.h = which - above;
                    for (; x.h >= p.c.kv_heads; x.h -= p.c.kv_heads) have &= have - 1;
                    const int b = __ffs(have) - 1;
                    x.mt = level;
                    if (b != x.b) x.s = pf_seq(p, b, nullptr);
                    x.b = b;
                    x.k = pf_keys(p, x.s, x.mt);
                    x.n = x.k.units;
                };
                // The place is free once the softmax warps are done with the item before it; the roles
                // between are ahead of them, or behind the copies by less than the places there are.
                auto give = [&](const PfItem &x, int turn) {
                    const int e = turn % kPfAhead;
                    if (turn >= kPfAhead && !warp_wait(&sh->iempty[e], (turn / kPfAhead + 1) & 1, pp, sh)) return false;
                    if (lane == 0) {
                        sh->item[e] = x;
                        mbar_arrive(&sh->ifull[e]);
                    }
                    __syncwarp();
                    return true;
                };
                PfItem at = {};
                auto pages = [&](int u) {
                    const int j = at.k.base + u * kPfKeys + lane * pp.box_rows;
                    if (Q4 || lane >= boxes || j >= at.k.end || j + pp.box_rows <= at.k.first) return -1;
                    return __ldg(p.b.table + (int64_t)at.b * p.b.table_width + p.c.page.div(j));
                };
                at.b = -1;
                if (queued) {
                    if (lane < p.b.seqs) tiles = pf_tiles(p, pf_seq(p, lane, nullptr));
                    level = __reduce_max_sync(0xffffffffu, tiles) - 1;
                    queue_item(blockIdx.x, at);
                } else {
                    at.b = sh->b[0];
                    at.h = sh->h[0];
                    at.mt = sh->mt[0];
                    at.u = sh->u[0];
                    at.n = 0;
                    if (at.b >= 0) {
                        at.s = pf_seq(p, at.b, nullptr);
                        at.k = pf_keys(p, at.s, at.mt);
                        at.n = pf_units(run, at);
                    }
                }
                give(at, 0);
                int spent = 0;
                for (int turn = 0; ok && at.n > 0; ++turn) {
                    const int n = at.n;
                    const PfOrder order(p, kKeyBytes, at, sh->run, spent);
                    int page = pages(order.unit(0)), count = 0;
                    PfItem next_item = at;
                    if (queued && lane == 0) count = atomicAdd(p.status + kPfCount, 1);
                    for (int i = 0; ok && i < n; ++i) {
                        const int u = order.unit(i), next = i + 1 < n ? pages(order.unit(i + 1)) : -1;  // used a unit later
                        const int j0 = at.k.base + u * kPfKeys, j = j0 + lane * pp.box_rows;
                        int row;
                        p.c.page.div(j, row);
                        if (!Q4 && (unsigned)page >= (unsigned)p.c.num_pages) {
                            if (lane < boxes && j < at.k.end && j + pp.box_rows > at.k.first) set_status(p.status, MC_ERR_RANGE);
                            page = p.c.num_pages;
                        }
                        for (int kv = 0; kv < 2; ++kv, ++it) {
                            const int slot = it % Sh::kStages;
                            if (it >= Sh::kStages && !(ok = warp_wait(&sh->kempty[slot], (it / Sh::kStages + 1) & 1, pp, sh))) break;
                            if (Q4) continue;  // (others fill it; this role keeps to their pace)
                            // values past the sequence's end may be NaN, and a weight of 0 would not
                            // hide that (nor would a capped key's neighbour): their rows are zeroed
                            // before the tile is given on
                            const bool patch = (kv || MODE == kPfCap) && j0 + kPfKeys > at.s.len;
                            uint64_t *bar = patch ? &sh->vpatch : &sh->kfull[slot];
                            if (lane == 0) mbar_arrive_expect_tx(bar, Sh::kTileBytes);
                            __syncwarp();
                            if (lane < boxes) {
                                const uint32_t dst = smem0 + Sh::kRing + slot * Sh::kTileBytes + lane * pp.box_rows * 128;
#pragma unroll
                                for (int h = 0; h < D / 64; ++h)
                                    pf_tma(dst + h * Sh::kHalf, kv ? &vmap : &kmap, 64 * h, row, at.h, page, bar);
                            }
                            if (patch) {
                                if (!(ok = warp_wait(&sh->vpatch, patches++ & 1, pp, sh))) break;
                                const int from = max(0, at.s.len - j0);
                                for (int i = from * 8 + lane; i < kPfKeys * 8; i += 32)
#pragma unroll
                                    for (int h = 0; h < D / 64; ++h)
                                        *reinterpret_cast<uint4 *>(smem + Sh::kRing + slot * Sh::kTileBytes + h * Sh::kHalf + i * 16) =
                                            make_uint4(0, 0, 0, 0);
                                fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0) mbar_arrive(&sh->kfull[slot]);
                            }
                        }
                        page = next;
                        if (i == 0) {  // early enough for the others, late enough not to hold the copies up
                            if (queued) queue_item((int)gridDim.x + __shfl_sync(0xffffffffu, count, 0), next_item);
                            else pf_next(p, run, next_item);
                            ok = give(next_item, turn + 1) && ok;
                        }
                    }
                    spent += n + kPfItemCost;
                    at = next_item;
                }
                // the last copies land before the block's shared memory is given back, on an abort too
                const uint64_t t0 = globaltimer_ns();
                for (int i = Q4 ? it : max(0, it - Sh::kStages); i < it; ++i)
                    while (!__all_sync(0xffffffffu, mbar_try_wait(&sh->kfull[i % Sh::kStages], (i / Sh::kStages) & 1)))
                        if (__any_sync(0xffffffffu, globaltimer_ns() - t0 > pp.timeout_ns)) break;
                pdl_trigger();
            } else {
                // queries, a tile as soon as the last item's has been read
                constexpr int kChunks = D / 8, kPer = 32 / kChunks, kQStep = kPer;
                const int lc = lane % kChunks, lr = lane / kChunks;
                const uint32_t col = (uint32_t)(lc >> 3) * Sh::kHalf + ((lc & 7) << 4);  // 16-byte chunk, unswizzled
                const int step_hg = kQStep % p.group;
                const int64_t q_step = kQStep / p.group * p.q_stride + step_hg * D, q_wrap = p.q_stride - p.group * D;
                int uses[2] = {0, 0};
                bool ok = !(pp.debug & kDebugNoProducer);
                const volatile PfItem *it;
                for (int turn = 0; ok && (it = pf_item(pp, sh, turn)); ++turn) {
                    const int first = it->s.first, head0 = it->h * p.group, rows0 = it->mt * kPfRows, rows = min(kPfRows, pf_rows(p, it));
                    for (int t = 0; t < 2 && t * kPfTile < rows; ++t) {
                        if (uses[t] && !(ok = warp_wait(&sh->qempty[t], (uses[t] + 1) & 1, pp, sh))) break;
                        ++uses[t];
                        const uint32_t tile = smem0 + Sh::kHdr + t * Sh::kTileBytes;
                        if (pp.q_boxes) {
                            // rows past the sequence's last are other tokens', or zeros: not stored
                            if (lane == 0) {
                                mbar_arrive_expect_tx(&sh->qfull[t], Sh::kTileBytes);
#pragma unroll
                                for (int h = 0; h < D / 64; ++h)
                                    pf_tma3(tile + h * Sh::kHalf, &qmap, 64 * h, head0,
                                            first + p.by_group.div(rows0 + t * kPfTile), &sh->qfull[t]);
                            }
                            continue;
                        }
                        // one row per kChunks lanes, zeros past the last
                        int r = t * kPfTile + lr;
                        int hg;
                        const int tok = p.by_group.div(rows0 + r, hg);
                        const uint16_t *src = p.q + (first + tok) * p.q_stride + (head0 + hg) * D + lc * 8;
                        for (; r < (t + 1) * kPfTile; r += kQStep) {
                            const bool real = r < rows;
                            pf_copy16z((tile + col + (r & 127) * 128) ^ ((r & 7) << 4), real ? src : p.q, real);
                            src += q_step;
                            if ((hg += step_hg) >= p.group) {
                                hg -= p.group;
                                src += q_wrap;
                            }
                        }
                        asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
                        fence_proxy_async_smem();
                        mbar_arrive(&sh->qfull[t]);
                    }
                    if (!ok) break;
                }
                if (pp.q_boxes) {  // the last copies land before the block's shared memory is given back
                    const uint64_t t0 = globaltimer_ns();
                    for (int t = 0; t < 2; ++t)
                        while (uses[t] && !__all_sync(0xffffffffu, mbar_try_wait(&sh->qfull[t], (uses[t] + 1) & 1)))
                            if (__any_sync(0xffffffffu, globaltimer_ns() - t0 > pp.timeout_ns)) break;
                }
            }
        } else {
            // ---------------------------------------------------------------- MMAs --
            const volatile PfItem *at = pf_item(pp, sh, 0);
            constexpr uint32_t kIdS = pf_idesc(BF16, kPfKeys, false), kIdO = pf_idesc(BF16, D, true);
            const uint32_t q0 = pf_desc_k(smem_u32(smem + Sh::kHdr)), k0 = pf_desc_k(smem_u32(smem + Sh::kRing));
            const uint32_t v0 = pf_desc_mn(smem_u32(smem + Sh::kRing), Sh::kHalf);
            constexpr uint32_t kStep = Sh::kTileBytes >> 4;
            int uses = 0, quses = 0;
            bool ok = true;
            auto qk = [&](int t, int slot) {  // S_t = Q_t K^T
                const uint32_t a = q0 + t * kStep, b = k0 + slot * kStep;
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    const uint32_t o = (s >> 2) * (Sh::kHalf >> 4) + (s & 3) * 2;
                    pf_mma_ss(128 * t, a + o, b + o, kIdS, s > 0);
                }
            };
            auto pv = [&](int t, int slot, bool first) {  // O_t (+)= P_t V
                const uint32_t b = v0 + slot * kStep;
#pragma unroll
                for (int s = 0; s < kPfKeys / 16; ++s) pf_mma_ts(256 + 128 * t, 128 * t + 8 * s, b + s * (2048 >> 4), kIdO, !first || s > 0);
            };
            struct Slot {
                int i;
                uint32_t phase;
                __device__ Slot next() const { return i + 1 == Sh::kStages ? Slot{0, phase ^ 1u} : Slot{i + 1, phase}; }
            };
            auto full = [&](const Slot &x) { return warp_wait(&sh->kfull[x.i], x.phase, pp, sh); };
            auto tiles_of = [&](const volatile PfItem *a) { return !a ? 0 : pf_rows(p, a) > kPfTile ? 2 : 1; };
            // Unit j's PV of the tile is followed by unit j + 1's QK of it, the next item's first one
            // after the last: the next queries and the other tile's softmax hide the change of item.
            // A warp for each tile: their waits do not add up, and either's MMAs fill the pipe.
            const int t = warp - kPfMma;
            Slot k = {0, 0};  // of the last keys that QK was issued for
            int n = at ? at->n : 0, tiles = tiles_of(at), turn = 0;
            // a ring slot that this warp has no MMA for (the item has one tile) is given back at once
            auto pass = [&](const Slot &x) {
                if (lane == 0) mbar_arrive(&sh->kempty[x.i]);
            };
            auto first_qk = [&](const Slot &x, bool last_unit) {
                if (!warp_wait(&sh->qfull[t], quses++ & 1, pp, sh)) return false;
                tc_fence_after();
                if (elect_one()) {
                    qk(t, x.i);
                    umma_commit(&sh->sfull[t]);
                    umma_commit(&sh->kempty[x.i]);
                    if (last_unit) umma_commit(&sh->qempty[t]);
                }
                __syncwarp();
                return true;
            };
            if (n > 0 && (ok = full(k))) {
                if (t < tiles) ok = first_qk(k, n == 1);
                else pass(k);
            }
            while (ok && n > 0) {
                const volatile PfItem *next = pf_item(pp, sh, ++turn);
                const int next_n = next ? next->n : 0, next_tiles = tiles_of(next);
                // inside the item: unit j's PV and unit j + 1's QK are issued together
                for (int j = 0; ok && j + 1 < n; ++j) {
                    const Slot v = k.next(), k2 = v.next();
                    if (!(ok = full(v) && full(k2))) break;
                    if (t < tiles) {
                        if (!(ok = warp_wait(&sh->pfull[t], uses++ & 1, pp, sh))) break;
                        tc_fence_after();
                        if (elect_one()) {
                            pv(t, v.i, j == 0);
                            umma_commit(&sh->kempty[v.i]);
                            qk(t, k2.i);
                            umma_commit(&sh->sfull[t]);
                            umma_commit(&sh->kempty[k2.i]);
                            if (j + 2 == n) umma_commit(&sh->qempty[t]);
                        }
                        __syncwarp();
                    } else {
                        pass(v);
                        pass(k2);
                    }
                    k = k2;
                }
                if (!ok) break;
                // its last unit's PV, and the next item's first QK
                const Slot v = k.next();
                if (!(ok = full(v))) break;
                k = v.next();
                if (t < tiles) {
                    if (!(ok = warp_wait(&sh->pfull[t], uses++ & 1, pp, sh))) break;
                    tc_fence_after();
                    if (elect_one()) {
                        pv(t, v.i, n == 1);
                        umma_commit(&sh->kempty[v.i]);
                        umma_commit(&sh->ofull[t]);
                    }
                    __syncwarp();
                } else {
                    pass(v);
                }
                if (next_n > 0) {
                    if (!(ok = full(k))) break;
                    if (t < next_tiles) ok = first_qk(k, next_n == 1);
                    else pass(k);
                }
                n = next_n;
                tiles = next_tiles;
            }
            // the tensor pipe is idle before shared and tensor memory are given back
            if (elect_one()) umma_commit(&sh->drain);
            __syncwarp();
            const uint64_t t0 = globaltimer_ns();
            while (!__all_sync(0xffffffffu, mbar_try_wait(&sh->drain, 0)))
                if (__any_sync(0xffffffffu, globaltimer_ns() - t0 > pp.timeout_ns)) break;
        }
    } else {
        // -------------------------------------------------- softmax and epilogue --
        Regs::take();
        const int t = warp >> 2, wt = warp & 3, row = wt * 32 + lane;
        const uint32_t lanes = (uint32_t)(wt * 32) << 16;
        const uint32_t s_tmem = lanes + 128 * t, o_tmem = lanes + 256 + 128 * t;
        int su = 0, ou = 0, spent = 0;
        bool ok = true, tail = false;
        const volatile PfItem *it;
        for (int turn = 0; ok && (it = pf_item(pp, sh, turn)); ++turn) {
            const int n = it->n, rows = min(kPfTile, pf_rows(p, it) - t * kPfTile);
            auto place = [&](int &tok, int &head) {  // of this thread's row (the last one where it has none)
                int hg;
                tok = p.by_group.div(it->mt * kPfRows + t * kPfTile + min(row, rows - 1), hg);
                head = it->h * p.group + hg;
            };
            if (rows > 0) {
                int tok, head;
                place(tok, head);
                const int len = it->s.len, off = len - it->s.n, pos = off + tok, prefix = it->s.prefix;
                const int lo = p.window ? max(0, pos - p.window + 1) : 0;
                const int hi = pos < 0 ? 0 : min(len, max(pos + 1, prefix));
                // what the tile's first and last rows see decides whether a unit needs the mask
                const int rows0 = it->mt * kPfRows + t * kPfTile, base = it->k.base;
                const int p_first = off + p.by_group.div(rows0), p_last = off + p.by_group.div(rows0 + rows - 1);
                const int all_hi = p_first < 0 ? 0 : min(len, max(p_first + 1, prefix));
                const int all_lo = p.window ? p_last - p.window + 1 : 0;
                const float slope = MODE != kPfPlain && p.slopes ? __ldg(p.slopes + head) * kLog2e : 0.f;
                float m = -INFINITY, l = 0.f;
                const PfOrder order(p, kKeyBytes, *it, sh->run, spent);
                for (int i = 0; i < n; ++i) {
                    if (!(ok = warp_wait(&sh->sfull[t], su & 1, pp, sh))) break;
                    ++su;
                    tc_fence_after();
                    if (wt * 32 < rows) {
                        const int j0 = base + order.unit(i) * kPfKeys;
                        uint32_t s[128];
#pragma unroll
                        for (int q = 0; q < 4; ++q) pf_ld32(s_tmem + 32 * q, s + 32 * q);
                        pf_ld_wait(s);
#pragma unroll
                        for (int q = 1; q < 4; ++q) pf_tie(s + 32 * q);
                        pf_softmax<BF16, MODE>(s, s_tmem, o_tmem, D, j0 < all_lo || j0 + kPfKeys > all_hi, lo - j0, hi - j0, p.scale,
                                                p.cap, p.slopes != nullptr, slope, (float)(j0 - pos), i == 0, m, l);
                        tmem_st_wait();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh->pfull[t]);
                }
                place(tok, head);
                const bool live = row < rows, from_first = it->u == 0, whole = from_first && n == it->k.units;
                const int first = it->s.first;
                if (!ok || !(ok = warp_wait(&sh->ofull[t], ou & 1, pp, sh))) break;
                ++ou;
                tc_fence_after();
                const float inv = 1.f / l;
                uint16_t *out = p.out + (first + tok) * p.out_stride + head * D;
                float *mine = pp.part + (2 * blockIdx.x + (from_first ? 1 : 0)) * pf_part_floats(D);
                if (wt * 32 < rows) {
                    float odd = 0.f;  // NaN once an element of the row is infinite or NaN
#pragma unroll
                    for (int d = 0; d < D; d += 32) {
                        uint32_t o[32];
                        pf_ld32(o_tmem + d, o);
                        pf_ld_wait(o);
                        if (live && whole) {
                            uint32_t v[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                v[i] = l == 0.f ? 0u : pack2<BF16>(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
#pragma unroll
                            for (int i = 0; i < 32; ++i) odd = fmaf(__uint_as_float(o[i]), 0.f, odd);
                            // a lane's row is 2 D bytes from its neighbour's: whole 32-byte sectors
#pragma unroll
                            for (int i = 0; i < 16; i += 8) {
                                if (pp.out32) {
                                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + d + 2 * i),
                                                 PF_I8(v, i) : "memory");
                                } else {
                                    *reinterpret_cast<uint4 *>(out + d + 2 * i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                                    *reinterpret_cast<uint4 *>(out + d + 2 * i + 8) = make_uint4(v[i + 4], v[i + 5], v[i + 6], v[i + 7]);
                                }
                            }
                        } else if (live) {
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                reinterpret_cast<uint4 *>(mine)[(size_t)((d + i) / 4) * kPfRows + t * kPfTile + row] =
                                    make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                        }
                        __syncwarp();
                    }
                    if (live && whole && p.lse)
                        p.lse[(int64_t)(first + tok) * p.q_heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
                    if (live && !whole)
                        reinterpret_cast<float2 *>(mine + kPfRows * D)[t * kPfTile + row] = make_float2(m, l);
                    // (redone by the join launch: here the other roles would wait for a row's keys, one by
                    // one, for longer than their waits last)
                    if (odd != odd) sh->odd = 1;
                }
                tc_fence_before();
            }
            if (it->u == 0 && n < it->k.units) {
                tail = true;
                if (tid == 0) {
                    // the pieces lie in the CTAs whose runs start before the item's end
                    const int64_t total = sh->total, ctas = total < (int64_t)gridDim.x ? total : gridDim.x;
                    const int64_t end = muldiv64(total, blockIdx.x + 1, (int)ctas) - sh->off + kPfItemCost + it->k.units;
                    pp.open[blockIdx.x] = {(int32_t)(div64(end * ctas + total - 1, total) - blockIdx.x), it->b, it->h, it->mt};
                }
            }
            spent += n + kPfItemCost;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->iempty[turn % kPfAhead]);
        }
        if (!tail && tid == 0) pp.open[blockIdx.x].pieces = 0;
    }

    tc_fence_before();
    __syncthreads();
    if (tid == 0) pp.odd[blockIdx.x] = sh->odd;
    if (warp == kPfMma) {
        tc_fence_after();
        tmem_dealloc(sh->tmem_base, 512);
    }
}

// Whether a key that was copied for an item, and that one of its tokens t0 .. t1 hides, is infinite or
// NaN: by `warps` warps, the answer the warp's.
template <int D, bool BF16, bool Q4>
__device__ __forceinline__ bool pf_hides_odd(const PfParams &pp, int b, int h, int mt, const PfSeq &s, int t0, int t1, int warp, int warps,
                                             int lane)
{
    const AttnParams &p = pp.a;
    const PfKeys k = pf_keys(p, s, mt);
    const int from = k.first & -pp.box_rows, to = min(s.len, (k.end + pp.box_rows - 1) & -pp.box_rows);  // whole boxes
    const int p0 = s.len - s.n + t0, p1 = s.len - s.n + t1;
    const int lo = p.window ? max(0, p1 - p.window + 1) : 0, hi = p0 < 0 ? 0 : max(p0 + 1, s.prefix);
    return odd_keys<D, BF16, Q4>(p, b, h, from, min(lo, to), warp, warps, lane) ||
           odd_keys<D, BF16, Q4>(p, b, h, max(hi, from), to, warp, warps, lane);
}

constexpr int kPfJoinRows = 16;  // rows of an open item that a block of the join launch adds

// A row that came out infinite or NaN, redone if it hides a key that is.
template <int D, bool BF16, bool Q4>
__device__ __noinline__ void pf_redo_row(const PfParams &pp, int b, int mt, int tok, int head, int lane)
{
    const PfSeq s = pf_seq(pp.a, b, nullptr);
    if (pf_hides_odd<D, BF16, Q4>(pp, b, pp.a.by_group.div(head), mt, s, tok, tok, 0, 1, lane))
        exact_row<D, BF16, Q4>(pp.a, b, s.len - s.n + tok, s.len, s.prefix, s.first + tok, head, lane);
}

// 16 rows of a CTA's open item: adds its pieces in their order, the loads of four pieces
// in flight at once.
template <int D, bool BF16, bool Q4>
__device__ __forceinline__ void pf_join(const PfParams &pp, const PfOpen &it)
{
    constexpr int kQuads = D / 4 / 16;  // column quads of a thread: threadIdx.x / 16, + 16, ...
    __shared__ float2 ml[kAttnMaxSms][kPfJoinRows];
    __shared__ int odd[kPfJoinRows];
    const AttnParams &p = pp.a;
    const int r = threadIdx.x % kPfJoinRows, c0 = threadIdx.x / kPfJoinRows, row = blockIdx.y * kPfJoinRows + r;
    auto piece = [&](int i) { return pp.part + (2 * ((size_t)blockIdx.x + i) + (i == 0 ? 1 : 0)) * pf_part_floats(D); };
    for (int i = c0; i < it.pieces; i += 16) ml[i][r] = reinterpret_cast<const float2 *>(piece(i) + kPfRows * D)[row];
    const PfSeq s = pf_seq(p, it.b, nullptr);
    const int f = it.mt * kPfRows + row;
    __syncthreads();
    int hg;
    const int tok = p.by_group.div(f, hg), head = it.h * p.group + hg;
    float strange = 0.f;
    if (f < s.n * p.group) {
        float top = -INFINITY;
        for (int i = 0; i < it.pieces; ++i) top = fmaxf(top, ml[i][r].x);
        float4 acc[kQuads];
#pragma unroll
        for (int k = 0; k < kQuads; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
#pragma unroll 4
        for (int i = 0; i < it.pieces; ++i) {
            const float *q = piece(i);
            const float w = ml[i][r].x == -INFINITY ? 0.f : ex2(ml[i][r].x - top);
            sum = fmaf(w, ml[i][r].y, sum);
#pragma unroll
            for (int k = 0; k < kQuads; ++k) {
                const float4 v = reinterpret_cast<const float4 *>(q)[(size_t)(c0 + 16 * k) * kPfRows + row];
                acc[k] = make_float4(fmaf(w, v.x, acc[k].x), fmaf(w, v.y, acc[k].y), fmaf(w, v.z, acc[k].z), fmaf(w, v.w, acc[k].w));
            }
        }
        const float inv = 1.f / sum;
        uint16_t *out = p.out + (s.first + tok) * p.out_stride + head * D;
#pragma unroll
        for (int k = 0; k < kQuads; ++k) {
            *reinterpret_cast<uint2 *>(out + 4 * (c0 + 16 * k)) =
                sum == 0.f ? make_uint2(0, 0)
                           : make_uint2(pack2<BF16>(acc[k].x * inv, acc[k].y * inv), pack2<BF16>(acc[k].z * inv, acc[k].w * inv));
            strange = fmaf(acc[k].x, 0.f, fmaf(acc[k].y, 0.f, fmaf(acc[k].z, 0.f, fmaf(acc[k].w, 0.f, strange))));
        }
        if (p.lse && c0 == 0)
            p.lse[(int64_t)(s.first + tok) * p.q_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
    if (!__syncthreads_or(strange != strange)) return;
    if (threadIdx.x < kPfJoinRows) odd[threadIdx.x] = 0;
    __syncthreads();
    if (strange != strange) odd[r] = 1;
    __syncthreads();
    for (int x = threadIdx.x >> 5; x < kPfJoinRows; x += 8) {
        if (!odd[x]) continue;
        int g2;
        const int t2 = p.by_group.div(it.mt * kPfRows + blockIdx.y * kPfJoinRows + x, g2);
        pf_redo_row<D, BF16, Q4>(pp, it.b, it.mt, t2, it.h * p.group + g2, threadIdx.x & 31);
    }
}

// Rows of whole items that came out infinite or NaN and hide a key that is, redone by the definition: the
// launch's blocks take the items' rows, kPfRedoRows at a time, in turn.  An open item's rows are its join's.
// A prompt of 4096 tokens, every row of which sees a NaN, takes 135 us instead of 112 (115 ms with every row redone).
constexpr int kPfRedoRows = 32;
template <int D, bool BF16, bool Q4>
__device__ __noinline__ void pf_redo(const PfParams &pp)
{
    const AttnParams &p = pp.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int grid = gridDim.x * gridDim.y;
    int turn = blockIdx.y * gridDim.x + blockIdx.x;  // this block's next slice, counted from the sequence's first
    for (int b = 0; b < p.b.seqs; ++b) {
        const PfSeq s = pf_seq(p, b, nullptr);
        const int tiles = pf_tiles(p, s), slices = tiles * p.c.kv_heads * (kPfRows / kPfRedoRows);
        for (; turn < slices; turn += grid) {
            const int item = turn / (kPfRows / kPfRedoRows), h = item / tiles, mt = item - h * tiles;
            const int r0 = mt * kPfRows + turn % (kPfRows / kPfRedoRows) * kPfRedoRows, rows = min(kPfRedoRows, s.n * p.group - r0);
            const PfOpen o = threadIdx.x < gridDim.x ? pp.open[threadIdx.x] : PfOpen{0, 0, 0, 0};
            if (__syncthreads_or(o.pieces && o.b == b && o.h == h && o.mt == mt) || rows <= 0) continue;
            if (!__syncthreads_or(pf_hides_odd<D, BF16, Q4>(pp, b, h, mt, s, p.by_group.div(r0), p.by_group.div(r0 + rows - 1), warp, 8, lane)))
                continue;
            for (int r = warp; r < rows; r += 8) {
                int hg;
                const int tok = p.by_group.div(r0 + r, hg), head = h * p.group + hg;
                const uint16_t *out = p.out + (s.first + tok) * p.out_stride + head * D;
                float odd = 0.f;
#pragma unroll
                for (int d = 2 * lane; d < D; d += 64) {
                    const float2 v = unpack2<BF16>(*reinterpret_cast<const uint32_t *>(out + d));
                    odd = fmaf(v.x, 0.f, fmaf(v.y, 0.f, odd));
                }
                if (__any_sync(0xffffffffu, odd != odd))
                    exact_row<D, BF16, Q4>(p, b, s.len - s.n + tok, s.len, s.prefix, s.first + tok, head, lane);
            }
        }
        turn -= slices;
    }
}

// (most blocks have nothing to add: with the 62 registers that heads of 64 take unbounded, four
// blocks an SM, the launch is 0.6 us longer)
template <int D, bool BF16, bool Q4>
__global__ void __launch_bounds__(256, D == 64 ? 5 : 4) prefill_join_kernel(const PfParams pp)
{
    pdl_trigger();
    pdl_wait();
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) pp.a.status[kPfCount] = 0;
    const PfOpen it = pp.open[blockIdx.x];
    const bool odd = __builtin_expect(__syncthreads_or(threadIdx.x < gridDim.x && pp.odd[threadIdx.x]), 0);
    if (it.pieces) pf_join<D, BF16, Q4>(pp, it);
    if (odd) pf_redo<D, BF16, Q4>(pp);
}
static_assert(kAttnMaxSms <= 256, "a thread per CTA of the first launch");

// A tensor map of 16-bit elements in boxes of 64 columns, with the 128-byte swizzle.
static bool pf_map(CUtensorMap *m, const void *base, bool bf16, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                   const cuuint32_t *box)
{
    using Encode = decltype(&cuTensorMapEncodeTiled);
    static std::atomic<Encode> known{nullptr};
    Encode encode = known.load(std::memory_order_relaxed);
    if (!encode) {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &r) != cudaSuccess || !f) return false;
        encode = (Encode)f;
        known.store(encode, std::memory_order_relaxed);
    }
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return encode(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void *>(base), dims,
                  strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool BF16, int MODE, bool QUEUE, bool Q4>
static cudaError_t launch_prefill_t(const PfParams &p, int ctas, cudaStream_t st)
{
    const KvView &c = p.a.c;
    CUtensorMap kmap = {}, vmap = {}, qmap;
    const cuuint64_t dims[4] = {D, (cuuint64_t)c.page_size, (cuuint64_t)c.kv_heads, (cuuint64_t)c.num_pages};
    const cuuint64_t strides[3] = {D * 2, (cuuint64_t)c.page_size * D * 2, (cuuint64_t)c.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)p.box_rows, 1, 1};
    if (!Q4 && (!pf_map(&kmap, c.k, BF16, 4, dims, strides, box) || !pf_map(&vmap, c.v, BF16, 4, dims, strides, box))) return cudaErrorInvalidValue;
    if (p.q_boxes) {
        const cuuint64_t qdims[3] = {D, (cuuint64_t)p.a.q_heads, (cuuint64_t)p.a.b.tokens};
        const cuuint64_t qstrides[2] = {D * 2, (cuuint64_t)p.a.q_stride * 2};
        const cuuint32_t qbox[3] = {64, (cuuint32_t)p.a.group, (cuuint32_t)(kPfTile / p.a.group)};
        if (!pf_map(&qmap, p.a.q, BF16, 3, qdims, qstrides, qbox)) return cudaErrorInvalidValue;
    } else {
        qmap = kmap;  // not used
    }
    using Sh = PfShape<D>;
    auto k = prefill_kernel<D, BF16, MODE, QUEUE, Q4>;
    static std::atomic<bool> known{false};  // (the same build on every device)
    cudaError_t e = cudaSuccess;
    if (!known.load(std::memory_order_relaxed)) {
        cudaFuncAttributes at;
        e = cudaFuncGetAttributes(&at, k);
        if (e != cudaSuccess) return e;
        if (at.numRegs < PfRegs<Q4>::kAll) return cudaErrorInvalidConfiguration;
        known.store(true, std::memory_order_relaxed);
    }
    static SmemAttr attr;
    e = attr.set((const void *)k, Sh::kSmem);
    if (e != cudaSuccess) return e;
    profile_begin(kKAttnPrefill, st);
    e = launch_k(k, dim3(ctas), dim3(pf_threads(Q4)), Sh::kSmem, st, p, kmap, vmap, qmap);
    profile_end(kKAttnPrefill, st);
    if (e != cudaSuccess) return e;
    profile_begin(kKAttnJoin, st);
    e = launch_k(prefill_join_kernel<D, BF16, Q4>, dim3(ctas, kPfRows / kPfJoinRows), dim3(256), 0, st, p);
    profile_end(kKAttnJoin, st);
    return e;
}

template <int D, bool BF16, int MODE, bool Q4>
static cudaError_t launch_prefill_q(const PfParams &p, int ctas, cudaStream_t st)
{
    // What the lengths decide is the kernel's; where there cannot be items enough, or sequences are
    // more than the queue takes, one without the queue's code does (9 ragged prompts 32.7 -> 32.2 us).
    const int64_t items = ((int64_t)p.a.b.tokens * p.a.group / kPfRows + p.a.b.seqs) * p.a.c.kv_heads;  // at most
    return p.a.b.seqs <= 32 && items >= kPfQueueItems * ctas && items < 1 << 30 ? launch_prefill_t<D, BF16, MODE, true, Q4>(p, ctas, st)
                                                                                : launch_prefill_t<D, BF16, MODE, false, Q4>(p, ctas, st);
}

template <int D, bool BF16, bool Q4>
static cudaError_t launch_prefill_m(const PfParams &p, int mode, int ctas, cudaStream_t st)
{
    return mode == kPfCap    ? launch_prefill_q<D, BF16, kPfCap, Q4>(p, ctas, st)
           : mode == kPfBias ? launch_prefill_q<D, BF16, kPfBias, Q4>(p, ctas, st)
                             : launch_prefill_q<D, BF16, kPfPlain, Q4>(p, ctas, st);
}

template <bool Q4>
cudaError_t launch_prefill_d(const PfParams &p, int head_dim, bool bf16, int mode, int ctas, cudaStream_t st)
{
    return head_dim == 64 ? (bf16 ? launch_prefill_m<64, true, Q4>(p, mode, ctas, st) : launch_prefill_m<64, false, Q4>(p, mode, ctas, st))
                          : (bf16 ? launch_prefill_m<128, true, Q4>(p, mode, ctas, st) : launch_prefill_m<128, false, Q4>(p, mode, ctas, st));
}

}  // namespace mc
