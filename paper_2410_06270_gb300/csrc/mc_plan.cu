// mc_plan.cu -- mc_kv_plan: pages, positions and slots of a step's new tokens, from the lengths.
//
// Per sequence three running sums decide everything (pages that come back, pages asked for, rows), so one
// block goes over the sequences, a thread each, 1024 at a time; the tokens, of which there may be hundreds of
// thousands, then find their sequence in the boundaries and write 12 bytes each.  A step of few tokens is
// one launch: the block that made the sums does the tokens too, with the sums still in shared memory.  More are a
// second launch of as many blocks as they fill.
#include "mc_attn.h"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

constexpr int kPlanThreads = 1024;
constexpr int kPlanFew = 4096;      // tokens that the first block does itself
constexpr int kPlanPer = 4;         // tokens a thread of the second launch

struct PlanParams {
    int32_t *ring;
    const int64_t *state;
    int num_pages, page_size, table_width, seqs, tokens;
    FastDiv page;
    const int32_t *lens, *add;
    const uint8_t *done;
    int32_t *table, *lens_out, *cu_q, *positions;
    int64_t *slots, *state_out;
    int32_t *status, *base;  // base: where a sequence's new pages stand in the ring (workspace)
    int alone;               // the tokens are the first block's too
};

// What the tokens of a sequence need.
struct PlanSeq {
    int first, length, held, base;  // row of its first new token, tokens before, their pages, place in the ring
};

__device__ __forceinline__ int64_t ring_at(int64_t i, int pages)
{
    return (int64_t)((uint64_t)i % (uint32_t)pages);
}

// Token t, the i-th of a sequence's new ones: its page, slot and position; the first row of a page also
// enters the page into the table (new pages begin with a new token, since the last held one is filled first).
__device__ __forceinline__ void plan_token(const PlanParams &p, int t, int b, const PlanSeq &s)
{
    const int pos = s.length + (t - s.first);
    int row;
    const int i = p.page.div(pos, row);
    int32_t *at = p.table + (int64_t)b * p.table_width + i;
    int page;
    if (i >= s.held) {
        int64_t k = (int64_t)s.base + (i - s.held);
        if (k >= p.num_pages) k = ring_at(k, p.num_pages);
        page = p.ring[k];
        if (row == 0) *at = page;
    } else {
        page = *at;
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

// Inclusive sums over the block; `upto` comes back with them, the total is returned.
template <int N>
__device__ __forceinline__ void block_sums(int64_t (&upto)[N], int64_t (&total)[N], int64_t (*part)[32])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t o = __shfl_up_sync(0xffffffffu, upto[k], d);
            if (lane >= d) upto[k] += o;
        }
    __syncthreads();  // (the sums before these have been read)
    if (lane == 31)
#pragma unroll
        for (int k = 0; k < N; ++k) part[k][warp] = upto[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t mine = part[k][lane];
        int64_t sum = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += o;
        }
        total[k] = __shfl_sync(0xffffffffu, sum, 31);
        upto[k] += __shfl_sync(0xffffffffu, sum - mine, warp);
    }
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p)
{
    __shared__ int64_t part[3][32];
    __shared__ PlanSeq seq[kPlanThreads + 1];
    const int tid = threadIdx.x, lane = tid & 31;
    pdl_trigger();
    pdl_wait();
    const int64_t taken = p.state[0], returned = p.state[1], free = returned - taken;
    const int64_t room = (int64_t)p.table_width * p.page_size, most = room < kMaxLen ? room : kMaxLen;
    int64_t back0 = 0, need0 = 0, want0 = 0, took = 0;  // sums of the sequences before
    int rows0 = 0;
    for (int b0 = 0; b0 < p.seqs; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const bool real = b < p.seqs;
        int old = 0, n = 0;
        bool over = false;
        if (real) {
            old = max(p.lens[b], 0);
            n = p.add[b];
            over = p.done && p.done[b];
        }
        const int back = over ? min(pages_of(p, old), p.table_width) : 0;
        const int length = over ? 0 : old, held = pages_of(p, length);
        const bool fits = n >= 0 && (int64_t)length + n <= most;
        const int need = fits ? pages_of(p, length + n) - held : 0;
        int64_t upto[3] = {back, need, fits ? n : 0}, total[3];
        block_sums<3>(upto, total, part);
        const int64_t before = back0 + upto[0] - back, asked = need0 + upto[1];
        const bool served = fits && (need == 0 || asked <= free) && (n == 0 || want0 + upto[2] <= p.tokens);
        if (real && !served) set_status(p.status, MC_ERR_RANGE);
        const int got = served ? n : 0;
        int64_t rows[1] = {got}, all[1];
        block_sums<1>(rows, all, part);
        const PlanSeq s = {rows0 + (int)rows[0] - got, length, held, (int)ring_at(taken + asked - need, p.num_pages)};
        if (real) {
            p.lens_out[b] = length + got;
            p.cu_q[b + 1] = s.first + got;
            if (b == 0) p.cu_q[0] = 0;
            if (p.alone) seq[tid] = s;
            else p.base[b] = s.base;
            if (served && need > 0) took = asked;
        }
        // a finished sequence's pages, by the warp; none overwrites a page that is still to be given out
        unsigned gone = __ballot_sync(0xffffffffu, back > 0);
        while (gone) {
            const int l = __ffs(gone) - 1;
            gone &= gone - 1;
            const int count = __shfl_sync(0xffffffffu, back, l);
            const int64_t first = returned + __shfl_sync(0xffffffffu, before, l);
            const int32_t *row = p.table + (int64_t)__shfl_sync(0xffffffffu, b, l) * p.table_width;
            for (int k = lane; k < count; k += 128) {
                int32_t page[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) page[i] = k + 32 * i < count ? row[k + 32 * i] : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (k + 32 * i >= count) break;
                    if (first + k + 32 * i - taken < p.num_pages) p.ring[ring_at(first + k + 32 * i, p.num_pages)] = page[i];
                    else set_status(p.status, MC_ERR_RANGE);
                    if ((unsigned)page[i] >= (unsigned)p.num_pages) set_status(p.status, MC_ERR_RANGE);
                }
            }
        }
        back0 += total[0];
        need0 += total[1];
        want0 += total[2];
        rows0 += (int)all[0];
    }
    // the last sequence that took pages has the largest sum
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) took = max(took, __shfl_xor_sync(0xffffffffu, took, d));
    __syncthreads();
    if (lane == 0) part[0][tid >> 5] = took;
    __syncthreads();
    if (tid == 0) {
        for (int i = 1; i < kPlanThreads / 32; ++i) took = max(took, part[0][i]);
        const int64_t end = taken + p.num_pages, to = returned + back0;
        p.state_out[0] = taken + took;
        p.state_out[1] = to <= end ? to : max(returned, end);
    }
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

// The tokens of a step, kPlanPer a thread in turn.
__global__ void __launch_bounds__(256) plan_tokens_kernel(const PlanParams p)
{
    pdl_trigger();
    pdl_wait();
    const int rows = __ldg(p.cu_q + p.seqs);
    const int t0 = blockIdx.x * (256 * kPlanPer) + threadIdx.x;
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
            if (__ldg(p.cu_q + mid) <= t) lo = mid;
            else hi = mid;
        }
        const int first = __ldg(p.cu_q + lo), length = __ldg(p.lens_out + lo) - (__ldg(p.cu_q + lo + 1) - first);
        plan_token(p, t, lo, {first, length, pages_of(p, length), __ldg(p.base + lo)});
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
    return 256 + (size_t)seqs * 4;
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
    if (seqs > kMaxLen || tokens > kMaxLen) return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d sequences in one call", tokens, seqs);
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
    p.status = (int32_t *)workspace;
    p.base = (int32_t *)((uint8_t *)workspace + 256);
    p.alone = seqs <= kPlanThreads && tokens <= kPlanFew;
    cudaStream_t st = (cudaStream_t)stream;
    profile_begin(kKPlan, st);
    cudaError_t e = launch_k(plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    if (e == cudaSuccess && !p.alone && tokens)
        e = launch_k(plan_tokens_kernel, dim3((unsigned)((tokens + 256 * kPlanPer - 1) / (256 * kPlanPer))), dim3(256), 0, st, p);
    profile_end(kKPlan, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "plan launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // extern "C"
