// mc_attn_decode.cu -- attention of one new token per sequence over the paged cache.
//
// o = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m), one pass over the keys with a running
// reference m (the maximum, less a constant) and sum l (scores carried in units of log 2).  Every
// key and value is read once for a group of query heads, 4 head_dim bytes for 4 head_dim group
// flops: bound by HBM, so the design is about keeping loads in flight on every SM whatever the
// lengths are.
//
// Work is cut into units of 64 (heads of 64: 128) keys of one (sequence, key head); the units of
// the whole batch, in order, are dealt to the CTAs as contiguous runs of equal cost, which each
// CTA finds from the lengths by itself (no host knowledge of them, so a captured graph serves
// any).  A run that ends inside an item leaves a partial result (m, l, o in fp32); join_kernel
// adds the pieces of an item in their order.  At most two partials per CTA, whatever the batch.
// Each warp streams its own 16 or 32 keys of a unit through a ring of its own (three stages of 8
// KB, two CTAs an SM: 128 KB in flight), so the main loop has no block barrier.
//
// More rows than a group's heads (a few new tokens per sequence, with causal, window and prefix
// masks row by row) are further columns of the same products, up to 32.
//
// Measured: 64 sequences of 8192 keys, 32 heads on 8 of 128, 310 to 318 us by the box, 6.8 to 6.9 TB/s
// of keys and values (1.00 to 1.02 of the measured copy rate); one of 131071 keys 83 us, 6.5 TB/s; DRAM
// bytes 537.1 MB for 536.9 (ncu, 16 x 8192).  Short ones are bound by latency: 777 keys 7.4 us, of which
// the schedule 1, the first keys 1.5, the join and its launch 3; so are caps over more than 8 rows (33
// sequences of a window of 1024 keys, 12 heads a key head: 17 us, special functions 4 % active).
#include <math.h>

#include "mc_attn.h"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

constexpr int kDecWarps = 4, kDecThreads = 32 * kDecWarps;
// Keys of a unit that one warp takes, in tiles of 16: heads of 64 take two tiles in one step,
// whose chains of products and exponentials overlap (a step of 16 keys takes about as long
// whatever the head, and 16 keys of 64 are half the bytes).
constexpr int dec_tiles(int D) { return D == 64 ? 2 : 1; }
constexpr int dec_unit(int D) { return 16 * dec_tiles(D) * kDecWarps; }
constexpr int kDecCtasPerSm = 2;
constexpr int kDecMaxTiles = 4;                // n-tiles of the largest slice
constexpr int kDecItemCost = 2;  // what an item costs on top of its units, in units (up to 128 sequences; 64 of up
                                // to 500 keys 23.8 us at 0, 18.4 at 1, 18.1 at 2, 18.4 at 3)

template <bool BF16>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        mma16816(d, a[0], a[1], a[2], a[3], b0, b1);
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ uint32_t transposed8x8(uint32_t a)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
    return r;
}

// 16 bytes to shared memory, or 16 zeros where !real (the address is then not read).  The
// cache is read once a step and leaves L2 first: lengths, tables and what other kernels keep
// there stay.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool real, uint64_t policy)
{
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0),
                 "l"(policy)
                 : "memory");
}

// A sequence's new tokens and the keys [start, len) that any of them sees, as units of
// keys from `base` on (start rounded down to 16, so that 16 keys lie in one page).  Its rows
// are (token, head of the group), token-major, in slices.
struct Keys {
    int first, n;  // token rows
    int start, len, base, units;
};

template <int D>
__device__ __forceinline__ Keys keys_of(const AttnParams &p, int b, int32_t *status)
{
    Keys k;
    k.n = seq_rows(p.b, b, k.first, status);
    k.len = seq_len(p.b, p.c, b, status);
    const int p0 = k.len - k.n;
    k.start = p.window ? max(0, p0 - p.window + 1) : 0;
    k.base = k.start & ~15;
    k.units = k.n > 0 ? (k.len - k.base + dec_unit(D) - 1) / dec_unit(D) : 0;
    return k;
}

// Slices of 8 NT rows of a key head, and a sequence's units of all.
template <int NT>
__device__ __forceinline__ int slices_of(const AttnParams &p, const Keys &k)
{
    return (k.n * p.group + 8 * NT - 1) / (8 * NT);
}
template <int NT>
__device__ __forceinline__ int64_t units_of(const AttnParams &p, const Keys &k)
{
    return k.units ? (int64_t)k.units * (slices_of<NT>(p, k) * p.c.kv_heads) : 0;
}

// A place in the run of units: sequence, key head, slice of its rows, unit of its keys.
struct Place {
    int b, h, sl, slices, u;  // slices: of a key head
    Keys k;
};

template <int D, int NT>
__device__ __forceinline__ void step(const AttnParams &p, Place &at)
{
    if (++at.u < at.k.units) return;
    at.u = 0;
    if (++at.sl < at.slices) return;
    at.sl = 0;
    if (++at.h < p.c.kv_heads) return;
    at.h = 0;
    while (++at.b < p.b.seqs) {
        at.k = keys_of<D>(p, at.b, nullptr);
        if (at.k.units) {
            at.slices = slices_of<NT>(p, at.k);
            return;
        }
    }
}

// Header of a CTA's open item, for the join: the pieces of (sequence b, head h, slice sl) are this
// CTA's tail partial and the head partials of the next pieces - 1 CTAs; 0: none.
struct OpenItem {
    int32_t pieces, b, h, sl;
};

// What a row of a slice sees: keys [lo, hi); its bias is slope * (key - pos).
struct Row {
    int lo, hi, pos;
    float slope;
};

// Token tok of sequence b's, head `head`: a row that came out infinite or NaN, redone if a key of the
// sequence's units that it hides is.
template <int D, bool BF16>
__device__ __noinline__ void redo_row(const AttnParams &p, int b, int tok, int head, int lane)
{
    const Keys k = keys_of<D>(p, b, nullptr);
    const int h = p.by_group.div(head), pos = k.len - k.n + tok, prefix = p.prefix ? __ldg(p.prefix + b) : 0;
    const int lo = p.window ? max(0, pos - p.window + 1) : 0, hi = pos < 0 ? 0 : max(pos + 1, prefix);
    if (odd_keys<D, BF16>(p, b, h, k.start, min(lo, k.len), 0, 1, lane) || odd_keys<D, BF16>(p, b, h, max(hi, k.start), k.len, 0, 1, lane))
        exact_row<D, BF16>(p, b, pos, k.len, prefix, k.first + tok, head, lane);
}

__host__ __device__ constexpr size_t dec_part_floats(int D, int nt) { return (size_t)8 * nt * (D + 2); }

// Four elements of a finished row, and its lse with the first; a row without keys is zero.
template <bool BF16>
__device__ __forceinline__ void store_row(const AttnParams &p, int token, int head, int D, int d, float4 acc, float top, float sum)
{
    const float inv = 1.f / sum;
    *reinterpret_cast<uint2 *>(p.out + token * p.out_stride + head * D + d) =
        sum == 0.f ? make_uint2(0, 0) : make_uint2(pack2<BF16>(acc.x * inv, acc.y * inv), pack2<BF16>(acc.z * inv, acc.w * inv));
    if (p.lse && d == 0) p.lse[(int64_t)token * p.q_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

__device__ __forceinline__ bool finite4(const float4 &a)
{
    const float z = fmaf(a.x, 0.f, fmaf(a.y, 0.f, fmaf(a.z, 0.f, a.w * 0.f)));
    return z == z;
}

template <int D, int NT>
struct DecShape {
    static constexpr int kRow = D * 2;                       // bytes of a key
    static constexpr int kTiles = dec_tiles(D), kKeys = 16 * kTiles;
    static constexpr int kSlot = 2 * kKeys * kRow;           // a warp's keys and values of a unit
    static constexpr int kStages = 3;
    static constexpr int kRing = kSlot * kStages * kDecWarps;
    static constexpr int kPitch = D + 4;                     // floats of a row in the join: O, m, l
    static constexpr int kJoin = kDecWarps * 8 * kPitch * 4; // a piece's rows and queries lie over it
    static constexpr bool kQShared = NT > 2;                 // the queries' fragments: shared memory or registers
    static constexpr int kRows0 = kQShared ? NT * (D / 16) * 256 : 0;
    static constexpr int kSmem = kRing + kJoin;
    static_assert(kRows0 + 8 * NT * (int)sizeof(Row) <= kJoin, "rows of a slice");
};

// NT: n-tiles of 8 rows of a slice, 1 to 4.  The products are formed transposed, S^T = K Q^T and
// O^T += V^T P^T: the 16 keys of a warp fill the rows of the m16n8k16 instruction and the
// slice's rows its 8 columns, half the instructions and accumulators of the other way.
template <int D, bool BF16, int NT>
__global__ void __launch_bounds__(kDecThreads, kDecCtasPerSm) decode_kernel(const AttnParams p, FastDiv by_grid, OpenItem *open,
                                                                             float *part)
{
    using Sh = DecShape<D, NT>;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
    float *jo = reinterpret_cast<float *>(smem + Sh::kRing);
    uint2 *qs = reinterpret_cast<uint2 *>(smem + Sh::kRing);  // [n-tile][k-step][lane]
    Row *rows = reinterpret_cast<Row *>(smem + Sh::kRing + Sh::kRows0);
    int *marks = reinterpret_cast<int *>(smem + Sh::kRing);
    const uint32_t ring = smem_u32(smem) + warp * Sh::kSlot * Sh::kStages;
    pdl_trigger();
    pdl_wait();

    // the batch's cost, and where this CTA's run of it starts and ends
    int64_t total = 0, own = 0;
    int ctas, left = 0;
    int64_t u0 = 0, u1 = 0;
    Place at;  // compute side
    at.b = -1;
    const bool few = p.b.seqs <= 128;
    const int each = p.b.seqs <= 32 ? 1 : 4;  // sequences a lane
    int cost[4] = {0, 0, 0, 0}, units[4] = {0, 0, 0, 0}, cost4 = 0, units4 = 0;
    bool small = true;
    if (few) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= each) break;
            const int b = each * lane + i;
            if (b >= p.b.seqs) break;
            const Keys k = keys_of<D>(p, b, p.status);
            const int64_t n = units_of<NT>(p, k);
            small &= n < 1 << 22;
            units[i] = (int)n;
            cost[i] = n ? units[i] + kDecItemCost * slices_of<NT>(p, k) * p.c.kv_heads : 0;
            units4 += units[i];
            cost4 += cost[i];
        }
    }
    if (few && __all_sync(0xffffffffu, small)) {
        // 32 bits hold it all, and the divisions are by fixed numbers but one
        int upto = cost4, units_upto = units4;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, d), v = __shfl_up_sync(0xffffffffu, units_upto, d);
            if (lane >= d) upto += o, units_upto += v;
        }
        const int all = __shfl_sync(0xffffffffu, upto, 31);
        total = all;
        ctas = min(all, (int)gridDim.x);
        // place of a cost in the batch; returns the units before it
        auto find = [&](int pos, Place &x) {
            const int l = __ffs(__ballot_sync(0xffffffffu, upto > pos)) - 1;
            int r = pos - __shfl_sync(0xffffffffu, upto - cost4, l), before = __shfl_sync(0xffffffffu, units_upto - units4, l);
            x.b = each * l;
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                if (i + 1 >= each) break;
                const int n = __shfl_sync(0xffffffffu, cost[i], l), v = __shfl_sync(0xffffffffu, units[i], l);
                if (x.b == each * l + i && r >= n) {
                    r -= n;
                    before += v;
                    ++x.b;
                }
            }
            x.k = keys_of<D>(p, x.b, nullptr);
            x.slices = slices_of<NT>(p, x.k);
            const int per = x.k.units + kDecItemCost, item = (int)((unsigned)r / (unsigned)per);
            x.u = max(0, r - item * per - kDecItemCost);
            x.h = x.slices == 1 ? item : (int)((unsigned)item / (unsigned)x.slices);
            x.sl = item - x.h * x.slices;
            return before + item * x.k.units + x.u;
        };
        if ((int)blockIdx.x < ctas) {
            int rest = 0, q = 1;
            if (ctas == (int)gridDim.x) q = by_grid.div(all, rest);
            const int c = blockIdx.x, first = q * c + by_grid.div(rest * c), end = q * (c + 1) + by_grid.div(rest * (c + 1));
            u1 = end;
            Place past;
            const int until = end < all ? find(end, past) : __shfl_sync(0xffffffffu, units_upto, 31);
            left = until - find(first, at);
        }
    } else {
        for (int b0 = 0; b0 < p.b.seqs; b0 += 32) {
            own = b0 + lane < p.b.seqs ? units_of<NT>(p, keys_of<D>(p, b0 + lane, p.status)) : 0;
            int64_t n = own;
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
            total += n;
        }
        ctas = total < (int64_t)gridDim.x ? (int)total : gridDim.x;
        const bool any = (int)blockIdx.x < ctas;
        u0 = any ? muldiv64(total, blockIdx.x, ctas) : 0;
        u1 = any ? muldiv64(total, blockIdx.x + 1, ctas) : 0;
        int64_t skipped = 0;
        for (int b0 = 0; any && at.b < 0 && b0 < p.b.seqs; b0 += 32) {
            own = b0 + lane < p.b.seqs ? units_of<NT>(p, keys_of<D>(p, b0 + lane, nullptr)) : 0;
            int64_t sum = own;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int64_t o = __shfl_up_sync(0xffffffffu, sum, d);
                if (lane >= d) sum += o;
            }
            sum += skipped;
            const unsigned hit = __ballot_sync(0xffffffffu, sum > u0);
            if (!hit) {
                skipped = __shfl_sync(0xffffffffu, sum, 31);
                continue;
            }
            const int l = __ffs(hit) - 1;
            at.b = b0 + l;
            at.k = keys_of<D>(p, at.b, nullptr);
            at.slices = slices_of<NT>(p, at.k);
            const int64_t r = u0 - __shfl_sync(0xffffffffu, sum - own, l), item = div64(r, at.k.units);
            at.u = (int)(r - item * at.k.units);
            at.h = (int)div64(item, at.slices);
            at.sl = (int)(item - (int64_t)at.h * at.slices);
            left = (int)(u1 - u0);
        }
    }
    // ---- loads: this warp's 16 keys and values of a unit into ring slot i % kStages
    constexpr int kChunks = D / 8, kPer = 32 / kChunks;  // 16-byte chunks of a row; rows per warp copy
    const int lc = lane % kChunks, lr = lane / kChunks;
    const uint64_t policy = policy_evict_first();
    Place ld = at;
    int ld_left = left, page[Sh::kTiles];
    auto fetch_page = [&]() {
#pragma unroll
        for (int kt = 0; kt < Sh::kTiles; ++kt) {
            const int j = ld.k.base + ld.u * dec_unit(D) + warp * Sh::kKeys + 16 * kt;
            page[kt] = ld_left > 0 && j < ld.k.len ? seq_page(p.b, p.c, ld.b, p.c.page.div(j), p.status) : -1;
        }
    };
    auto issue = [&](int slot) {
        if (ld_left > 0) {
#pragma unroll
            for (int kt = 0; kt < Sh::kTiles; ++kt) {
                const int j = ld.k.base + ld.u * dec_unit(D) + warp * Sh::kKeys + 16 * kt;
                int row;
                p.c.page.div(j, row);
                const int64_t off = (page[kt] < 0 ? 0 : page[kt] * p.c.page_stride) +
                                    ((int64_t)ld.h * p.c.page_size + row + lr) * D + lc * 8;
                const uint32_t dst = ring + slot * Sh::kSlot + 16 * kt * Sh::kRow;
#pragma unroll
                for (int i = 0; i < 16 / kPer; ++i) {
                    const int r = lr + i * kPer;
                    const bool real = page[kt] >= 0 && j + r >= ld.k.start && j + r < ld.k.len;
                    const uint32_t d = dst + r * Sh::kRow + ((lc ^ (r & 7)) << 4);
                    copy16(d, p.c.k + (real ? off + i * kPer * D : 0), real, policy);
                    copy16(d + Sh::kKeys * Sh::kRow, p.c.v + (real ? off + i * kPer * D : 0), real, policy);
                }
            }
            --ld_left;
            step<D, NT>(p, ld);
            fetch_page();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch_page();
#pragma unroll
    for (int s = 0; s < Sh::kStages - 1; ++s) issue(s);

    int slot = 0;
    bool open_tail = false;
    while (left > 0) {
        // ---- one piece: units [at.u, at.u + n) of one item
        const int n = min(left, at.k.units - at.u);
        const bool from_first = at.u == 0, to_last = at.u + n == at.k.units;
        const int h0 = at.h * p.group, r0 = at.sl * 8 * NT, nrows = min(8 * NT, at.k.n * p.group - r0);  // rows of the slice
        const Keys keys = at.k;
        const int p0 = keys.len - keys.n, prefix = p.prefix ? __ldg(p.prefix + at.b) : 0;
        auto row_of = [&](int r) {  // r < nrows
            Row w;
            int hg;
            w.pos = p0 + p.by_group.div(r0 + r, hg);
            w.lo = p.window ? max(0, w.pos - p.window + 1) : 0;
            w.hi = w.pos < 0 ? 0 : min(keys.len, max(w.pos + 1, prefix));
            w.slope = p.slopes ? __ldg(p.slopes + h0 + hg) * kLog2e : 0.f;
            return w;
        };
        auto query = [&](int r) {
            int hg;
            const int tok = p.by_group.div(r0 + min(r, nrows - 1), hg);
            return p.q + (keys.first + tok) * p.q_stride + (h0 + hg) * D;
        };
        auto pair = [&](const uint16_t *q, int d, int r) { return r < nrows ? *reinterpret_cast<const uint32_t *>(q + d) : 0u; };
        uint32_t qf[Sh::kQShared ? 1 : NT][D / 16][2];
        if (Sh::kQShared) {
            for (int i = tid; i < NT * (D / 16) * 32; i += kDecThreads) {
                const int l = i & 31, ks = (i >> 5) % (D / 16), nt = (i >> 5) / (D / 16);
                const int r = 8 * nt + (l >> 2), d = 16 * ks + 2 * (l & 3);
                const uint16_t *q = query(r);
                qs[i] = make_uint2(pair(q, d, r), pair(q, d + 8, r));
            }
        } else {
#pragma unroll
            for (int nt = 0; nt < (Sh::kQShared ? 1 : NT); ++nt) {
                const uint16_t *q = query(8 * nt + g) + 2 * t4;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    qf[nt][ks][0] = pair(q, 16 * ks, 8 * nt + g);
                    qf[nt][ks][1] = pair(q, 16 * ks + 8, 8 * nt + g);
                }
            }
        }
        if (tid < 8 * NT) rows[tid] = row_of(min(tid, nrows - 1));
        // keys that every row of the slice sees: below the first row's end, from the last's start on
        const int all_hi = row_of(0).hi, all_lo = row_of(nrows - 1).lo;
        __syncthreads();
        float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[nt][mt][c] = 0.f;
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
        }
        for (int u = at.u; u < at.u + n; ++u) {
            asm volatile("cp.async.wait_group %0;" ::"n"(Sh::kStages - 2) : "memory");
            __syncwarp();  // every lane is done with the slot of the round before, which is filled next
            issue(slot == 0 ? Sh::kStages - 1 : slot - 1);
            const uint32_t kk = ring + slot * Sh::kSlot, vv = kk + Sh::kKeys * Sh::kRow;
            const int j0 = keys.base + u * dec_unit(D) + warp * Sh::kKeys;
            if (j0 < keys.len) {
                // S^T: rows are keys g, g + 8; columns the slice's rows 2 t4, 2 t4 + 1; few
                // tiles take two accumulators each, so that the chain is half as long
                constexpr int kChains = NT * Sh::kTiles > 2 ? 1 : 2;
                float s[Sh::kTiles][NT][kChains][4];
#pragma unroll
                for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c) s[kt][nt][0][c] = s[kt][nt][kChains - 1][c] = 0.f;
                const int kr = lane & 15;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    uint32_t a[Sh::kTiles][4];
#pragma unroll
                    for (int kt = 0; kt < Sh::kTiles; ++kt)
                        ldsm4(a[kt], kk + (16 * kt + kr) * Sh::kRow + (((2 * ks + (lane >> 4)) ^ (kr & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        uint2 q;
                        if (Sh::kQShared) q = qs[(nt * (D / 16) + ks) * 32 + lane];
                        else q = make_uint2(qf[Sh::kQShared ? 0 : nt][ks][0], qf[Sh::kQShared ? 0 : nt][ks][1]);
#pragma unroll
                        for (int kt = 0; kt < Sh::kTiles; ++kt) mma16<BF16>(s[kt][nt][ks % kChains], a[kt], q.x, q.y);
                    }
                }
                const bool masked = j0 < all_lo || j0 + Sh::kKeys > all_hi;
                bool over = false;
                float x[Sh::kTiles][NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            x[kt][nt][c] = (kChains == 2 ? s[kt][nt][0][c] + s[kt][nt][kChains - 1][c] : s[kt][nt][0][c]) * p.scale;
                    if (p.cap > 0.f) {
#pragma unroll
                        for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                            for (int c = 0; c < 2; ++c)  // two keys of a row share a reciprocal
                                unpair2(capped2(pair2(x[kt][nt][c], x[kt][nt][c + 2]), p.cap), x[kt][nt][c], x[kt][nt][c + 2]);
                    }
                    if (p.slopes) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const Row w = rows[8 * nt + 2 * t4 + c];
                            const float first = (float)(j0 + g - w.pos);
#pragma unroll
                            for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                                for (int e = c; e < 4; e += 2)
                                    x[kt][nt][e] = fmaf(w.slope, first + (float)(16 * kt + (e >> 1) * 8), x[kt][nt][e]);
                        }
                    }
                    if (masked) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const Row w = rows[8 * nt + 2 * t4 + c];
#pragma unroll
                            for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                                for (int e = c; e < 4; e += 2) {
                                    const int j = j0 + 16 * kt + g + (e >> 1) * 8;
                                    if (j < w.lo || j >= w.hi) x[kt][nt][e] = -INFINITY;
                                }
                        }
                    }
#pragma unroll
                    for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                        for (int c = 0; c < 4; ++c) over |= x[kt][nt][c] > m[nt][c & 1] + kLazy;
                }
                if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float top = -INFINITY;
#pragma unroll
                            for (int kt = 0; kt < Sh::kTiles; ++kt) top = fmaxf(top, fmaxf(x[kt][nt][c], x[kt][nt][c + 2]));
#pragma unroll
                            for (int d = 4; d <= 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            top = fmaxf(m[nt][c], top - kBelow);
                            const float keep = top == m[nt][c] ? 1.f : ex2(m[nt][c] - top);
                            m[nt][c] = top;
                            l[nt][c] *= keep;
#pragma unroll
                            for (int mt = 0; mt < D / 16; ++mt) {
                                o[nt][mt][c] *= keep;
                                o[nt][mt][c + 2] *= keep;
                            }
                        }
                }
                uint32_t pf[Sh::kTiles][NT][2];
#pragma unroll
                for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float pr[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float ref = m[nt][c & 1];
                            pr[c] = ex2(x[kt][nt][c] - (ref == -INFINITY ? 0.f : ref));
                            l[nt][c & 1] += pr[c];
                        }
                        // rounded to the cache's type for the second product; l keeps fp32
                        pf[kt][nt][0] = transposed8x8(pack2<BF16>(pr[0], pr[1]));
                        pf[kt][nt][1] = transposed8x8(pack2<BF16>(pr[2], pr[3]));
                    }
                const int vr = (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int kt = 0; kt < Sh::kTiles; ++kt)
#pragma unroll
                    for (int mt = 0; mt < D / 16; ++mt) {
                        uint32_t a[4];
                        ldsm4t(a, vv + (16 * kt + vr) * Sh::kRow + (((2 * mt + ((lane >> 3) & 1)) ^ (vr & 7)) << 4));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16<BF16>(o[nt][mt], a, pf[kt][nt][0], pf[kt][nt][1]);
                    }
            }
            if (++slot == Sh::kStages) slot = 0;
        }

        // ---- the four warps' parts, an n-tile at a time
        const bool whole = from_first && to_last;
        unsigned odd = 0;  // rows that came out infinite or NaN
        float *mine = part + (2 * blockIdx.x + (from_first ? 1 : 0)) * dec_part_floats(D, NT);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (8 * nt >= nrows) break;
            __syncthreads();  // the queries, the n-tile before
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
                if (g == 0)
                    *reinterpret_cast<float2 *>(jo + (warp * 8 + 2 * t4 + c) * Sh::kPitch + D) = make_float2(m[nt][c], l[nt][c]);
            }
#pragma unroll
            for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    jo[(warp * 8 + 2 * t4 + (c & 1)) * Sh::kPitch + 16 * mt + g + (c >> 1) * 8] = o[nt][mt][c];
            __syncthreads();
            for (int i = tid; i < 8 * (D / 4); i += kDecThreads) {
                const int h = i / (D / 4), d = (i % (D / 4)) * 4, r = 8 * nt + h;
                if (r >= nrows) continue;
                float2 ml[kDecWarps];
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kDecWarps; ++w) {
                    ml[w] = *reinterpret_cast<const float2 *>(jo + (w * 8 + h) * Sh::kPitch + D);
                    top = fmaxf(top, ml[w].x);
                }
                float sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kDecWarps; ++w) {
                    const float k = ml[w].x == -INFINITY ? 0.f : ex2(ml[w].x - top);
                    const float4 v = *reinterpret_cast<const float4 *>(jo + (w * 8 + h) * Sh::kPitch + d);
                    sum = fmaf(k, ml[w].y, sum);
                    acc = make_float4(fmaf(k, v.x, acc.x), fmaf(k, v.y, acc.y), fmaf(k, v.z, acc.z), fmaf(k, v.w, acc.w));
                }
                if (whole) {
                    int hg;
                    const int tok = p.by_group.div(r0 + r, hg);
                    store_row<BF16>(p, keys.first + tok, h0 + hg, D, d, acc, top, sum);
                    // (one token's row hides no key of its units: what it sums is what it sees)
                    if (keys.n > 1 && !finite4(acc)) odd |= 1u << r;
                } else {
                    *reinterpret_cast<float4 *>(mine + r * D + d) = acc;
                    if (d == 0) *reinterpret_cast<float2 *>(mine + 8 * NT * D + 2 * r) = make_float2(top, sum);
                }
            }
        }
        if (__syncthreads_or(odd)) {  // the join buffers are free again
            if (tid < 8 * NT) marks[tid] = 0;
            __syncthreads();
            for (unsigned x = odd; x; x &= x - 1) marks[__ffs(x) - 1] = 1;
            __syncthreads();
            for (int r = warp; r < nrows; r += kDecWarps) {
                if (!marks[r]) continue;
                int hg;
                const int tok = p.by_group.div(r0 + r, hg);
                redo_row<D, BF16>(p, at.b, tok, h0 + hg, lane);
            }
            __syncthreads();
        }
        if (from_first && !to_last) {
            open_tail = true;
            if (tid == 0) {
                const int64_t end = u1 - n + at.k.units;  // the item's end: the run ends n units into it
                const int64_t last = div64(end * ctas + total - 1, total);  // one past the CTA that holds it
                open[blockIdx.x] = {(int32_t)(last - blockIdx.x), at.b, at.h, at.sl};
            }
        }
        left -= n;
        at.u += n - 1;
        step<D, NT>(p, at);
    }
    if (!open_tail && tid == 0) open[blockIdx.x].pieces = 0;

    // sequences without keys
    for (int b = blockIdx.x; b < p.b.seqs; b += gridDim.x) {
        const Keys k = keys_of<D>(p, b, nullptr);
        if (k.len > 0) continue;
        for (int t = k.first; t < k.first + k.n; ++t) {
            for (int i = tid; i < p.q_heads * D / 8; i += kDecThreads)
                *reinterpret_cast<uint4 *>(p.out + t * p.out_stride + 8 * i) = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = tid; i < p.q_heads; i += kDecThreads) p.lse[(int64_t)t * p.q_heads + i] = -INFINITY;
        }
    }
}

// One CTA per (CTA of the pass before, row of a slice): adds the pieces of that CTA's open
// item in their order.
template <int D, bool BF16>
__global__ void __launch_bounds__(128, 12) join_kernel(const AttnParams p, const OpenItem *open, const float *part, int nt)
{
    constexpr int kCols = D / 4, kGroups = 128 / kCols;
    __shared__ float red[4], sums[kGroups];
    __shared__ float4 acc_s[128];
    pdl_trigger();
    pdl_wait();
    const OpenItem it = open[blockIdx.x];
    if (it.pieces == 0) return;
    const int r = blockIdx.y, tid = threadIdx.x;
    int first, hg;
    const int n = seq_rows(p.b, it.b, first, nullptr), f = it.sl * 8 * nt + r;
    if (f >= n * p.group) return;
    const int tok = p.by_group.div(f, hg);
    const size_t stride = dec_part_floats(D, nt);
    auto piece = [&](int i) { return part + (2 * ((size_t)blockIdx.x + i) + (i == 0 ? 1 : 0)) * stride; };
    float top = -INFINITY;
    for (int i = tid; i < it.pieces; i += 128) top = fmaxf(top, piece(i)[8 * nt * D + 2 * r]);
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if ((tid & 31) == 0) red[tid >> 5] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int col = tid % kCols, grp = tid / kCols;
#pragma unroll 4
    for (int i = grp; i < it.pieces; i += kGroups) {
        const float *q = piece(i);
        const float2 ml = *reinterpret_cast<const float2 *>(q + 8 * nt * D + 2 * r);
        const float4 v = *reinterpret_cast<const float4 *>(q + r * D + 4 * col);
        const float k = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
        sum = fmaf(k, ml.y, sum);
        acc = make_float4(fmaf(k, v.x, acc.x), fmaf(k, v.y, acc.y), fmaf(k, v.z, acc.z), fmaf(k, v.w, acc.w));
    }
    acc_s[tid] = acc;
    if (col == 0) sums[grp] = sum;
    __syncthreads();
    bool odd = false;
    if (grp == 0) {
        sum = 0.f;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const float4 v = acc_s[i * kCols + col];
            sum += sums[i];
            acc = make_float4(acc.x + v.x, acc.y + v.y, acc.z + v.z, acc.w + v.w);
        }
        store_row<BF16>(p, first + tok, it.h * p.group + hg, D, 4 * col, acc, top, sum);
        odd = n > 1 && !finite4(acc);
    }
    if (__syncthreads_or(odd) && tid < 32) redo_row<D, BF16>(p, it.b, tok, it.h * p.group + hg, tid);
}

constexpr int kDecMaxCtas = kDecCtasPerSm * kAttnMaxSms;

size_t decode_part_bytes(int head_dim)
{
    return kDecMaxCtas * (sizeof(OpenItem) + 2 * 4 * dec_part_floats(head_dim, kDecMaxTiles));
}

template <int D, bool BF16, int NT>
static cudaError_t launch_decode_t(const AttnParams &p, int ctas, cudaStream_t st)
{
    using Sh = DecShape<D, NT>;
    OpenItem *open = reinterpret_cast<OpenItem *>(p.part);
    float *part = reinterpret_cast<float *>(p.part + kDecMaxCtas * sizeof(OpenItem));
    auto k = decode_kernel<D, BF16, NT>;
    static SmemAttr attr;
    cudaError_t e = attr.set((const void *)k, Sh::kSmem);
    if (e != cudaSuccess) return e;
    profile_begin(kKAttnDecode, st);
    e = launch_k(k, dim3(ctas), dim3(kDecThreads), Sh::kSmem, st, p, FastDiv(ctas), open, part);
    profile_end(kKAttnDecode, st);
    // A sequence that the table holds in one unit is never split.  (Adding the pieces of the
    // others within the launch, by the CTA that finishes an item's last one, saves its launch but
    // not time: an atomic and two dependent reads by one CTA against a CTA per row: 777 keys 7.8 us
    // with the second launch, 9.9 without, 16 ragged sequences 26.9 and 29.5, 8000 keys of one key
    // head 12.5 and 32.1.)
    if (e != cudaSuccess || (int64_t)p.b.table_width * p.c.page_size <= dec_unit(D)) return e;
    profile_begin(kKAttnJoin, st);
    e = launch_k(join_kernel<D, BF16>, dim3(ctas, 8 * NT), dim3(128), 0, st, p, (const OpenItem *)open, (const float *)part, NT);
    profile_end(kKAttnJoin, st);
    return e;
}

template <int D, bool BF16>
static cudaError_t launch_decode_n(const AttnParams &p, int rows, int ctas, cudaStream_t st)
{
    return rows <= 8    ? launch_decode_t<D, BF16, 1>(p, ctas, st)
           : rows <= 16 ? launch_decode_t<D, BF16, 2>(p, ctas, st)
           : rows <= 24 ? launch_decode_t<D, BF16, 3>(p, ctas, st)
                        : launch_decode_t<D, BF16, kDecMaxTiles>(p, ctas, st);
}

// rows: what most sequences have, (token, head of the group) each; the smallest slice that
// holds them is taken, and sequences with more take several.
int launch_decode(const AttnParams &p, int head_dim, bool bf16, int rows, cudaStream_t st)
{
    int nsm = 0;
    cudaError_t e = sm_count(&nsm);
    if (e == cudaSuccess) {
        const int ctas = kDecCtasPerSm * (nsm < kAttnMaxSms ? nsm : kAttnMaxSms);
        e = head_dim == 64 ? (bf16 ? launch_decode_n<64, true>(p, rows, ctas, st) : launch_decode_n<64, false>(p, rows, ctas, st))
                           : (bf16 ? launch_decode_n<128, true>(p, rows, ctas, st) : launch_decode_n<128, false>(p, rows, ctas, st));
    }
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "decode launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
