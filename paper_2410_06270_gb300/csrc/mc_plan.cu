// mc_plan.cu -- mc_kv_plan: pages, positions and slots of a step's new tokens, from the lengths.
//
// Per sequence three running sums decide everything (pages that come back, pages asked for, rows), so a block
// goes over the sequences, 1024 or 4096 at a time; the tokens, of which there may be hundreds of
// thousands, then find their sequence in the boundaries and write 12 bytes each.  A step of few tokens is
// one launch of one block, with the sums still in shared memory.  Others are two: the first has several blocks, which
// all make the sums and each copy a part of the returned pages (its results go to the workspace, since lens and the
// counts may be overwritten by the call), the second as many as the tokens fill.
// Bound by latency: 250 sequences of one token, 23 of them finished with 2000 pages, 8.1 us, of which the launch, three
// round trips to memory (lengths; pages returned and taken; slots) and the sums; 1000 sequences, 40 of them with
// prompts of 82000 tokens, 90 finished with 17000 pages, 13.0 us.  The host knows no lengths: with finished ones a table that
// has room for more than kPlanEntries pages is two launches, whatever comes back (250 sequences 9.1 us where 8.3).
#include "mc_attn.h"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

constexpr int kPlanThreads = 1024;
constexpr int kPlanFew = 4096;      // tokens that one block does by itself
constexpr int kPlanEntries = 1 << 16;  // and table entries that it may have to give back pages of
constexpr int kPlanBlocks = 32;     // of the first of two launches
constexpr int kPlanPer = 4;         // tokens a thread of the second launch
constexpr int kPlanStaged = 4096;   // sequences whose boundaries it takes to shared memory

struct PlanParams {
    int32_t *ring;
    const int64_t *state;
    int num_pages, page_size, table_width, seqs, tokens;
    FastDiv page;
    const int32_t *lens, *add;
    const uint8_t *done;
    int32_t *table, *lens_out, *cu_q, *positions;
    int64_t *slots, *state_out;
    int32_t *status;
    // workspace of two launches: where a sequence's new pages stand in the ring, its new length, the counts
    int32_t *base, *length;
    int64_t *counts;
    int alone;  // one launch
    int preview;  // not committed: the table's rows of finished sequences stay as they are, for the next call to read
};

// What the tokens of a sequence need.
struct PlanSeq {
    int first, length, held, base, last;  // row of its first new token, tokens before, their pages, place in the ring, last page
    // (base: the complement of the place where the table's row is to stay as it is)
};

__device__ __forceinline__ int ring_at(int64_t i, int pages) { return (int)((uint64_t)i % (uint32_t)pages); }

// The k-th place after `base` (both below the ring's size where the counts are sound).
__device__ __forceinline__ int ring_next(const PlanParams &p, int base, int k)
{
    const int64_t i = (int64_t)base + k;
    if (i < p.num_pages) return (int)i;
    return i < 2 * (int64_t)p.num_pages ? (int)(i - p.num_pages) : ring_at(i, p.num_pages);
}

// Row t of sequence b: position, page and slot.  Tokens before the first new page lie in the last one held, which
// they fill; the first row of a page enters it into the table (a finished sequence's row names the pages that it gives
// back: only the call that commits writes over it).
__device__ __forceinline__ void plan_token(const PlanParams &p, int t, int b, const PlanSeq &s)
{
    const int pos = s.length + (t - s.first);
    int row;
    const int i = p.page.div(pos, row);
    int page = s.last;
    if (i >= s.held) {
        const bool stays = s.base < 0;
        page = p.ring[ring_next(p, stays ? ~s.base : s.base, i - s.held)];
        if (row == 0 && !stays) p.table[(int64_t)b * p.table_width + i] = page;
    }
    if (p.positions) p.positions[t] = pos;
    const bool in = (unsigned)page < (unsigned)p.num_pages;
    if (!in) set_status(p.status, MC_ERR_RANGE);
    if (p.slots) p.slots[t] = in ? (int64_t)page * p.page_size + row : -1;
}

__device__ __forceinline__ void plan_padding(const PlanParams &p, int t)
{
    if (p.positions) p.positions[t] = -1;
    if (p.slots) p.slots[t] = -1;
}

__device__ __forceinline__ int pages_of(const PlanParams &p, int tokens)
{
    int rest;
    const int n = p.page.div(tokens, rest);
    return n + (rest > 0);
}

// Sums of numbers that are not negative stop at 2^31 - 1, which is beyond every limit they are held against.
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }

// Sums over the block's threads: of those before (before) and of all (total).
template <int N>
__device__ __forceinline__ void block_sums(const uint32_t (&own)[N], uint32_t (&before)[N], uint32_t (&total)[N], uint32_t (*part)[32])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto[N];
#pragma unroll
    for (int k = 0; k < N; ++k) upto[k] = own[k];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto[k], d);
            if (lane >= d) upto[k] = plus(upto[k], o);
        }
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < N; ++k) part[k][warp] = upto[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        uint32_t sum = part[k][lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum = plus(sum, o);
        }
        total[k] = __shfl_sync(0xffffffffu, sum, 31);
        const uint32_t warps = __shfl_sync(0xffffffffu, sum, warp ? warp - 1 : 0), lanes = __shfl_up_sync(0xffffffffu, upto[k], 1);
        before[k] = plus(warp ? warps : 0, lane ? lanes : 0);
    }
}

// ITEMS: sequences a thread (one launch: 1).
template <int ITEMS>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p)
{
    constexpr int kAtOnce = kPlanThreads * ITEMS;
    __shared__ uint32_t part[4][32];
    __shared__ PlanSeq seq[ITEMS == 1 ? kPlanThreads : 1];
    __shared__ uint32_t given[kAtOnce];  // pages returned by the sequences before (of these)
    const int tid = threadIdx.x, lane = tid & 31;
    pdl_trigger();
    pdl_wait();
    const int64_t taken = p.state[0], returned = p.state[1];
    const uint32_t free = (uint32_t)max((int64_t)0, min(returned - taken, (int64_t)kMaxLen));
    const int64_t room = (int64_t)p.table_width * p.page_size, most = room < kMaxLen ? room : kMaxLen;
    uint32_t back0 = 0, need0 = 0, want0 = 0, took = 0;  // sums of the sequences before
    int rows0 = 0;
    const bool writes = blockIdx.x == 0;
    for (int b0 = 0; b0 < p.seqs; b0 += kAtOnce) {
        const int b = b0 + tid * ITEMS;
        int old[ITEMS], n[ITEMS], last = -1;
        bool over[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool real = b + i < p.seqs;
            old[i] = real ? max(p.lens[b + i], 0) : 0;
            n[i] = real ? p.add[b + i] : 0;
            over[i] = real && p.done && p.done[b + i];
        }
        int length[ITEMS], held[ITEMS];
        bool fits[ITEMS];
        uint32_t back[ITEMS], need[ITEMS], upto[3] = {0, 0, 0}, total[3];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            back[i] = over[i] ? min(pages_of(p, old[i]), p.table_width) : 0;
            length[i] = over[i] ? 0 : old[i];
            held[i] = pages_of(p, length[i]);
            fits[i] = n[i] >= 0 && (int64_t)length[i] + n[i] <= most;
            need[i] = fits[i] ? pages_of(p, length[i] + n[i]) - held[i] : 0;
            upto[0] = plus(upto[0], back[i]);
            upto[1] = plus(upto[1], need[i]);
            upto[2] = plus(upto[2], fits[i] ? n[i] : 0);
        }
        if (ITEMS == 1 && fits[0] && n[0] && held[0] && held[0] * (int64_t)p.page_size != length[0])
            last = p.table[(int64_t)b * p.table_width + held[0] - 1];
        uint32_t before[3];  // of the threads before, and then of the sequences before
        block_sums<3>(upto, before, total, part);
        uint32_t got[ITEMS], rows[1] = {0}, rows_before[1], all[1];
        int base[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const bool real = b + i < p.seqs;
            if (real) given[tid * ITEMS + i] = before[0];
            const uint32_t asked = plus(plus(need0, before[1]), need[i]);
            before[0] = plus(before[0], back[i]);
            before[1] = plus(before[1], need[i]);
            before[2] = plus(before[2], fits[i] ? n[i] : 0);
            const bool served = fits[i] && (need[i] == 0 || asked <= free) && (n[i] == 0 || plus(want0, before[2]) <= (uint32_t)p.tokens);
            got[i] = served ? n[i] : 0;
            rows[0] += got[i];
            const int64_t at = taken + (asked - need[i]);
            base[i] = at >= 0 && at < p.num_pages ? (int)at : ring_at(at, p.num_pages);
            if (p.preview && over[i]) base[i] = ~base[i];
            if (served && need[i]) took = asked;
            if (real && !served && writes) set_status(p.status, MC_ERR_RANGE);
        }
        block_sums<1>(rows, rows_before, all, part + 3);
        int first = rows0 + (int)rows_before[0];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (b + i < p.seqs) {
                if (ITEMS == 1) seq[tid] = {first, length[i], held[i], base[i], last};
                if (writes) {
                    p.cu_q[b + i + 1] = first + (int)got[i];
                    if (b + i == 0) p.cu_q[0] = 0;
                    (p.alone ? p.lens_out : p.length)[b + i] = length[i] + (int)got[i];
                    if (!p.alone) p.base[b + i] = base[i];
                }
            }
            first += (int)got[i];
        }
        if (total[0]) {
            // finished sequences' pages, end to end; none overwrites a page that is still to be given out
            __syncthreads();
            const int count = min(kAtOnce, p.seqs - b0);
            const int ring0 = ring_at(returned + back0, p.num_pages);
            for (int64_t f = (int64_t)blockIdx.x * kPlanThreads + tid; f < total[0]; f += (int64_t)gridDim.x * kPlanThreads) {
                int lo = 0, hi = count;  // the last sequence whose pages start at f or before it
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (given[mid] <= f) lo = mid;
                    else hi = mid;
                }
                const int page = p.table[(int64_t)(b0 + lo) * p.table_width + (f - given[lo])];
                if (returned + back0 + f - taken < p.num_pages) p.ring[ring_next(p, ring0, (int)f)] = page;
                else set_status(p.status, MC_ERR_RANGE);
                if ((unsigned)page >= (unsigned)p.num_pages) set_status(p.status, MC_ERR_RANGE);
            }
        }
        back0 = plus(back0, total[0]);
        need0 = plus(need0, total[1]);
        want0 = plus(want0, total[2]);
        rows0 += (int)all[0];
        if (b0 + kAtOnce < p.seqs) __syncthreads();  // (the sums and places have been read)
    }
    if (!writes) return;
    // the last sequence that took pages has the largest sum
    took = __reduce_max_sync(0xffffffffu, took);
    __syncthreads();
    if (lane == 0) part[0][tid >> 5] = took;
    __syncthreads();
    if (tid < 32) {
        took = __reduce_max_sync(0xffffffffu, part[0][lane]);
        if (lane == 0) {
            const int64_t end = taken + p.num_pages, to = returned + back0;
            int64_t *out = p.alone ? p.state_out : p.counts;
            out[0] = taken + took;
            out[1] = to <= end ? to : max(returned, end);
        }
    }
    if constexpr (ITEMS == 1) {
        if (!p.alone) return;
        for (int t = tid; t < p.tokens; t += kPlanThreads) {
            if (t >= rows0) {
                plan_padding(p, t);
                continue;
            }
            int lo = 0, hi = p.seqs;  // the last sequence that starts at t or before it
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (seq[mid].first <= t) lo = mid;
                else hi = mid;
            }
            plan_token(p, t, lo, seq[lo]);
        }
    }
}

// The tokens of a step, kPlanPer a thread in turn; and what the launch before left in the workspace, to its place.
__global__ void __launch_bounds__(256) plan_tokens_kernel(const PlanParams p)
{
    __shared__ int staged[kPlanStaged + 1];
    pdl_trigger();
    pdl_wait();
    for (int b = blockIdx.x * 256 + threadIdx.x; b < p.seqs; b += gridDim.x * 256) p.lens_out[b] = p.length[b];
    if (blockIdx.x == 0 && threadIdx.x < 2) p.state_out[threadIdx.x] = p.counts[threadIdx.x];
    const bool all = p.seqs <= kPlanStaged;
    if (all) {
        for (int b = threadIdx.x; b <= p.seqs; b += 256) staged[b] = __ldg(p.cu_q + b);
        __syncthreads();
    }
    auto start = [&](int b) { return all ? staged[b] : __ldg(p.cu_q + b); };
    const int rows = start(p.seqs), t0 = blockIdx.x * (256 * kPlanPer) + threadIdx.x;
    int lo = 0;
#pragma unroll
    for (int k = 0; k < kPlanPer; ++k) {
        const int t = t0 + 256 * k;
        if (t >= p.tokens) return;
        if (t >= rows) {
            plan_padding(p, t);
            continue;
        }
        int hi = p.seqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start(mid) <= t) lo = mid;
            else hi = mid;
        }
        const int first = start(lo), length = __ldg(p.length + lo) - (start(lo + 1) - first), held = pages_of(p, length);
        int last = -1;
        if (p.page.div(length + (t - first)) < held) last = p.table[(int64_t)lo * p.table_width + held - 1];
        plan_token(p, t, lo, {first, length, held, __ldg(p.base + lo), last});
    }
}

}  // namespace mc

using namespace mc;

extern "C" {

size_t mc_kv_plan_workspace_size(int seqs)
{
    clear_error();
    if (seqs < 0 || seqs > kMaxLen) {
        set_error(MC_ERR_INVALID_ARG, "%d sequences", seqs);
        return 0;
    }
    return 256 + 16 + (size_t)seqs * 8;
}

int mc_kv_plan(const mc_kv_pool *pool, const int32_t *lens, const int32_t *add, const uint8_t *done, int seqs, int tokens,
               int32_t *table, int table_width, int32_t *lens_out, int32_t *cu_q, int32_t *positions, int64_t *slots,
               int64_t *state_out, void *workspace, size_t ws_bytes, void *stream)
{
    clear_error();
    if (!pool) return set_error(MC_ERR_INVALID_ARG, "NULL pool");
    if (pool->num_pages < 1 || pool->page_size < 1 || pool->page_size > 32768)
        return set_error(MC_ERR_INVALID_ARG, "%d pages of %d", pool->num_pages, pool->page_size);
    if (seqs < 0 || tokens < 0) return set_error(MC_ERR_INVALID_ARG, "seqs %d, tokens %d", seqs, tokens);
    if (seqs > kMaxLen || tokens > kMaxLen || pool->num_pages > kMaxLen) return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d sequences in one call, %d pages", tokens, seqs, pool->num_pages);
    if (seqs == 0 && tokens > 0) return set_error(MC_ERR_INVALID_ARG, "%d tokens of no sequence", tokens);
    if (seqs == 0) return MC_OK;
    if (table_width < 1) return set_error(MC_ERR_INVALID_ARG, "table_width %d", table_width);
    if (!pool->ring || !pool->state || !lens || !add || !table || !lens_out || !cu_q || !state_out)
        return set_error(MC_ERR_INVALID_ARG, "NULL pointer argument");
    if (!aligned(pool->ring, 4) || !aligned(pool->state, 8) || !aligned(lens, 4) || !aligned(add, 4) || !aligned(table, 4) ||
        !aligned(lens_out, 4) || !aligned(cu_q, 4) || !aligned(positions, 4) || !aligned(slots, 8) || !aligned(state_out, 8))
        return set_error(MC_ERR_INVALID_ARG, "misaligned pointer argument");
    if (!workspace || !aligned(workspace, 256)) return set_error(MC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const size_t need = mc_kv_plan_workspace_size(seqs);
    if (ws_bytes < need) return set_error(MC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", ws_bytes, need);
    PlanParams p = {};
    p.ring = pool->ring;
    p.state = pool->state;
    p.num_pages = pool->num_pages;
    p.page_size = pool->page_size;
    p.table_width = table_width;
    p.seqs = seqs;
    p.tokens = tokens;
    p.page = FastDiv(pool->page_size);
    p.lens = lens;
    p.add = add;
    p.done = done;
    p.table = table;
    p.lens_out = lens_out;
    p.cu_q = cu_q;
    p.positions = positions;
    p.slots = slots;
    p.state_out = state_out;
    p.preview = done && state_out != pool->state && lens_out != lens;
    p.status = (int32_t *)workspace;
    // (nothing but the status word in the first 256 bytes: the attentions keep a count there)
    p.counts = (int64_t *)((uint8_t *)workspace + 256);
    p.base = (int32_t *)(p.counts + 2);
    p.length = p.base + seqs;
    p.alone = seqs <= kPlanThreads && tokens <= kPlanFew && (!done || (int64_t)seqs * table_width <= kPlanEntries);
    cudaStream_t st = (cudaStream_t)stream;
    profile_begin(kKPlan, st);
    auto k = seqs <= kPlanThreads ? plan_kernel<1> : plan_kernel<4>;
    cudaError_t e = launch_k(k, dim3(p.alone || !done ? 1 : kPlanBlocks), dim3(kPlanThreads), 0, st, p);
    if (e == cudaSuccess && !p.alone) {
        const int64_t per = 256 * kPlanPer, blocks = (tokens + per - 1) / per;
        e = launch_k(plan_tokens_kernel, dim3((unsigned)(blocks ? blocks : 1)), dim3(256), 0, st, p);
    }
    profile_end(kKPlan, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "plan launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // extern "C"
