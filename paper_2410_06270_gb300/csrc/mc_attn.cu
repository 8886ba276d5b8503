// mc_attn.cu -- the entry points of the paged cache and its attention: argument checks,
// workspace and dispatch.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "mc_attn.h"
#include "mc_host.h"
#include "mc_kv4.cuh"
#include "mc_profile.h"

namespace mc {

cudaError_t sm_count(int *out)
{
    static std::atomic<int> known[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    int n = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
    if (!n) {
        e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return cudaSuccess;
}

// q4: the cache is the 4-bit one (page_stride in bytes)
static int check_cache(const mc_kv_cache *c, int q_heads, bool q4)
{
    if (!c) return set_error(MC_ERR_INVALID_ARG, "NULL cache");
    if (c->dtype != MC_BF16 && c->dtype != MC_FP16) return set_error(MC_ERR_UNSUPPORTED, "cache dtype %d", c->dtype);
    if (c->head_dim != 64 && c->head_dim != 128)
        return set_error(MC_ERR_UNSUPPORTED, "head_dim %d (64 or 128)", c->head_dim);
    if (c->kv_heads < 1 || c->kv_heads > 1024 || q_heads < c->kv_heads || q_heads > 4096 || q_heads % c->kv_heads)
        return set_error(MC_ERR_INVALID_ARG, "%d query heads on %d key heads", q_heads, c->kv_heads);
    if (c->page_size < 16 || c->page_size > 32768 || c->page_size % 16)
        return set_error(MC_ERR_INVALID_ARG, "page_size %d (a multiple of 16, at most 32768)", c->page_size);
    if (c->num_pages < 1) return set_error(MC_ERR_INVALID_ARG, "num_pages %d", c->num_pages);
    const int64_t page = (int64_t)c->kv_heads * c->page_size * (q4 ? kv4_row_bytes(c->head_dim) : c->head_dim);
    if (c->page_stride % (q4 ? 16 : 8) || c->page_stride < page || c->page_stride >= (int64_t)1 << 38)
        return set_error(MC_ERR_INVALID_ARG, "page_stride %lld", (long long)c->page_stride);
    return MC_OK;
}

static int check_batch(const mc_kv_cache *c, const mc_kv_batch *b)
{
    if (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16))
        return set_error(MC_ERR_INVALID_ARG, "cache pointers must be 16-byte aligned");
    if (!b->lens || !b->table) return set_error(MC_ERR_INVALID_ARG, "NULL pointer argument");
    if (!aligned(b->lens, 4) || !aligned(b->table, 4) || !aligned(b->cu_q, 4))
        return set_error(MC_ERR_INVALID_ARG, "misaligned batch pointer");
    if (b->table_width < 1) return set_error(MC_ERR_INVALID_ARG, "table_width %d", b->table_width);
    if (!b->cu_q && b->tokens != b->seqs)
        return set_error(MC_ERR_INVALID_ARG, "%d tokens of %d sequences need cu_q", b->tokens, b->seqs);
    return MC_OK;
}

// A batch's token count: 0 and no error for an empty one.
static int check_counts(const mc_kv_batch *b)
{
    if (!b) return set_error(MC_ERR_INVALID_ARG, "NULL batch");
    if (b->seqs < 0 || b->tokens < 0) return set_error(MC_ERR_INVALID_ARG, "seqs %d, tokens %d", b->seqs, b->tokens);
    if (b->tokens > kMaxLen || b->seqs > kMaxLen)
        return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d sequences in one call", b->tokens, b->seqs);
    return MC_OK;
}

static int check_rows(const char *what, const void *p, int64_t stride, int heads, int D)
{
    if (!p || !aligned(p, 16)) return set_error(MC_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
    if (stride % 8 || stride < (int64_t)heads * D)
        return set_error(MC_ERR_INVALID_ARG, "%s: token stride %lld", what, (long long)stride);
    return MC_OK;
}

static KvView view(const mc_kv_cache *c)
{
    return {(uint16_t *)c->k, (uint16_t *)c->v, c->page_stride, c->num_pages, c->page_size, c->kv_heads,
            FastDiv(c->page_size)};
}

static BatchView view(const mc_kv_batch *b)
{
    return {b->lens, b->table, b->cu_q, b->seqs, b->tokens, b->table_width};
}

// The schedules count a sequence's work in 32 bits, and a CTA's share of the batch's; what it could
// be at most, every sequence as long as its table row, must fit (8192 tokens of a group of 8 over
// 2^20 keys are 2^21 of the 2^31).
static bool countable(const mc_kv_cache *c, const mc_kv_batch *b, int group)
{
    const int64_t room = (int64_t)b->table_width * c->page_size, most = room < kMaxLen ? room : kMaxLen;
    const double rows = (double)b->tokens * group;
    return (rows / 256 + 1) * (most / 128 + 3) < 0x7fffffff && (rows / 8 + b->seqs) * c->kv_heads * (most / 64 + 3) < 0x1p38;
}

constexpr int64_t kUnpackBytes = (int64_t)256 << 20;  // of a workspace for the 4-bit cache: keys and values in 16 bits
constexpr int kUnpackRows = 1024;  // (token, head of the group) of a sequence in the mean
constexpr int kUnpackUnits = 4096;  // of 256 rows and 128 keys, as far as the tables reach

static size_t workspace_size(int head_dim) { return (256 + std::max(decode_part_bytes(head_dim), prefill_part_bytes(head_dim)) + 255) & ~(size_t)255; }

constexpr int kFewRows = 16, kFewRowsCap = 32;

static int attention(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, int q_heads,
                     const mc_attn_opts *o, void *out, int64_t out_stride, float *lse, void *workspace, size_t ws_bytes,
                     bool decode, bool q4, void *stream)
{
    clear_error();
    int rc = check_cache(cache, q_heads, q4);
    if (rc || (rc = check_counts(batch))) return rc;
    if (!o) return set_error(MC_ERR_INVALID_ARG, "NULL options");
    // (the scale, its product with log2 e and its quotient by the cap stay in fp32's range)
    if (!(o->scale >= 1e-18f) || !(o->scale <= 1e18f) || !(o->softcap == 0.f || (o->softcap >= 1e-18f && o->softcap <= 1e18f)) ||
        o->window < 0)
        return set_error(MC_ERR_INVALID_ARG, "scale %g, softcap %g, window %d", o->scale, o->softcap, o->window);
    if (decode && batch->cu_q) return set_error(MC_ERR_INVALID_ARG, "one token per sequence: cu_q must be NULL");
    if (decode && o->prefix) return set_error(MC_ERR_INVALID_ARG, "a prefix is mc_attn_prefill's");
    if (batch->tokens == 0 || batch->seqs == 0) return MC_OK;
    if ((rc = check_batch(cache, batch))) return rc;
    if ((rc = check_rows("q", q, q_stride, q_heads, cache->head_dim))) return rc;
    if ((rc = check_rows("out", out, out_stride, q_heads, cache->head_dim))) return rc;
    if (!aligned(lse, 4) || !aligned(o->slopes, 4) || !aligned(o->prefix, 4))
        return set_error(MC_ERR_INVALID_ARG, "misaligned lse, slopes or prefix");
    if (!workspace || !aligned(workspace, 256)) return set_error(MC_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const size_t need = workspace_size(cache->head_dim);
    if (ws_bytes < need) return set_error(MC_ERR_INVALID_ARG, "workspace has %zu bytes, needs %zu", ws_bytes, need);
    if (!countable(cache, batch, q_heads / cache->kv_heads))
        return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d sequences, tables of %d pages of %d keys, in one call", batch->tokens,
                         batch->seqs, batch->table_width, cache->page_size);
    AttnParams p = {};
    p.c = view(cache);
    p.b = view(batch);
    p.q = (const uint16_t *)q;
    p.q_stride = q_stride;
    p.q_heads = q_heads;
    p.group = q_heads / cache->kv_heads;
    p.by_group = FastDiv(p.group);
    p.cap = o->softcap * kLog2e;
    p.scale = o->softcap > 0.f ? o->scale / o->softcap : o->scale * kLog2e;
    p.window = o->window >= kMaxLen ? 0 : o->window;  // no length passes kMaxLen
    p.slopes = o->slopes;
    p.prefix = o->prefix;
    p.out = (uint16_t *)out;
    p.out_stride = out_stride;
    p.lse = lse;
    p.status = (int32_t *)workspace;
    p.part = (uint8_t *)workspace + 256;
    // Few rows (tokens x heads of a group) a sequence take the decode kernel, whose time grows
    // with them, more the tensor-memory one, whose rows come 128 at a time; the counts are the
    // device's, so the mean decides.  8 sequences of 4000 keys, decode / tensor-memory kernel:
    // 16 rows 30 / 36 us, 20 rows 37 / 36, 32 rows 42 / 36; with a cap, whose cost follows the rows,
    // 36 / 51 at 20 and 44 / 51 at 32; one sequence of 2000 keys, 16 rows, 12 / 14.
    // Over the 4-bit cache up to 32 rows, with a cap or without: 64 sequences of 4000 keys, 20 rows, 131 / 280 us; 16 of
    // them, 24 rows 44 / 73, 32 rows 62 / 74, 48 rows 103 / 77; one of 2000 keys, 32 rows, 20 / 17.
    const int64_t rows = ((int64_t)batch->tokens + batch->seqs - 1) / batch->seqs * p.group;
    const bool bf16 = cache->dtype == MC_BF16;
    if (rows <= (q4 || p.cap > 0.f ? kFewRowsCap : kFewRows)) return launch_decode(p, cache->head_dim, bf16, q4, (int)rows, (cudaStream_t)stream);
    if (q4) {
        // Prompts of many rows, and enough of them: their keys are unpacked once, where the workspace holds what the
        // batch's tables reach, not for every 256 rows.  Unpacked / in the kernel, us: 3000 tokens of a group of 4 on 8 heads
        // (9000 units) 74 / 102, 509 over 30000 keys (15000) 194 / 250, 256 over 30000 (7500) 126 / 134, 8 x 300 over 4000
        // (10200) 172 / 188, 2048 (4100) 67 / 67; 1024 (1000) 39 / 34, 8 x 256 over 1000 (2000) 71 / 61, 300 over 8000 (2500)
        // 67 / 58; and 128 rows short of that, 128 over 30000 keys (3800) 106 / 84.  All with tables as wide as the texts: the
        // host knows no lengths.  What wider ones cost: 8192 tokens, whose tables reach 8192 to 65500 keys 340 to 346, from
        // 65536 on 544; 256 tokens over 300 keys in a table of 65000 25 where the kernel takes 19.
        const double reach = (double)batch->seqs * batch->table_width * cache->kv_heads * cache->page_size * cache->head_dim * 4;
        const bool few = reach < (double)kUnpackBytes && batch->seqs <= 65535;  // (the sizes below are small numbers)
        const int64_t pages = few ? (int64_t)batch->seqs * batch->table_width : 0;
        const int64_t side = pages * cache->kv_heads * cache->page_size * cache->head_dim * 2, table = (pages * 4 + 255) & ~(int64_t)255;
        const double units = (double)batch->tokens * p.group / 256 * cache->kv_heads * ((double)batch->table_width * cache->page_size / 128);
        if (few && rows >= kUnpackRows && units >= kUnpackUnits && (int64_t)need + 2 * side + table <= (int64_t)ws_bytes) {
            uint8_t *to = (uint8_t *)workspace + need;
            Unpack4Params u = {p.c, p.b, p.window, (uint16_t *)(to + table), (uint16_t *)(to + table + side), (int32_t *)to, p.status};
            if ((rc = launch_unpack4(u, cache->head_dim, bf16, (cudaStream_t)stream))) return rc;
            p.c.k = u.k;
            p.c.v = u.v;
            p.c.page_stride = (int64_t)cache->kv_heads * cache->page_size * cache->head_dim;
            p.c.num_pages = (int)pages;
            p.b.table = u.table;
            q4 = false;
        }
    }
    return launch_prefill(p, cache->head_dim, bf16, q4, (cudaStream_t)stream);
}

static int append(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, const void *k,
                  int64_t k_stride, const void *v, int64_t v_stride, int q_heads, const void *q_norm, const void *k_norm,
                  float eps, const float *rope, int rope_rows, int rot_dim, int interleaved, void *q_out, void *workspace,
                  bool q4, void *stream)
{
    clear_error();
    int rc = check_cache(cache, q_heads, q4);
    if (rc || (rc = check_counts(batch))) return rc;
    const int D = cache->head_dim;
    if (rot_dim < 0 || rot_dim > D || rot_dim % 16)
        return set_error(MC_ERR_INVALID_ARG, "rot_dim %d (a multiple of 16 up to head_dim %d)", rot_dim, D);
    if (rot_dim && (!rope || !aligned(rope, 16) || rope_rows < 1))
        return set_error(MC_ERR_INVALID_ARG, "rope must be 16-byte aligned and have rows");
    if (!(eps >= 0.f) || !isfinite(eps)) return set_error(MC_ERR_INVALID_ARG, "eps %g", eps);
    if (batch->tokens == 0 || batch->seqs == 0) return MC_OK;
    if ((rc = check_batch(cache, batch))) return rc;
    if ((rc = check_rows("q", q, q_stride, q_heads, D)) || (rc = check_rows("k", k, k_stride, cache->kv_heads, D)) ||
        (rc = check_rows("v", v, v_stride, cache->kv_heads, D)) ||
        (rc = check_rows("q_out", q_out, (int64_t)q_heads * D, q_heads, D)))
        return rc;
    if (!aligned(q_norm, 8) || !aligned(k_norm, 8) || !aligned(workspace, 4))
        return set_error(MC_ERR_INVALID_ARG, "misaligned norm or workspace");
    AppendParams p = {};
    p.c = view(cache);
    p.b = view(batch);
    p.q = (const uint16_t *)q;
    p.k = (const uint16_t *)k;
    p.v = (const uint16_t *)v;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_heads = q_heads;
    p.q_norm = (const uint16_t *)q_norm;
    p.k_norm = (const uint16_t *)k_norm;
    p.eps = eps;
    p.rope = rope;
    p.rope_rows = rope_rows;
    p.rot = rot_dim;
    p.interleaved = interleaved != 0;
    p.q_out = (uint16_t *)q_out;
    p.status = (int32_t *)workspace;
    return launch_append(p, D, cache->dtype == MC_BF16, q4, (cudaStream_t)stream);
}

}  // namespace mc

using namespace mc;

extern "C" {

size_t mc_attn_workspace_size(const mc_kv_cache *cache, int q_heads)
{
    clear_error();
    return check_cache(cache, q_heads, false) ? 0 : workspace_size(cache->head_dim);
}

size_t mc_attn4_workspace_size(const mc_kv_cache *cache, int q_heads, int prompts)
{
    clear_error();
    return check_cache(cache, q_heads, true) ? 0 : workspace_size(cache->head_dim) + (prompts ? kUnpackBytes : 0);
}

size_t mc_kv4_block_size(int page_size, int head_dim)
{
    clear_error();
    const mc_kv_cache c = {nullptr, nullptr, (int64_t)1 << 37, 1, page_size, 1, head_dim, MC_BF16};
    return check_cache(&c, 1, true) ? 0 : (size_t)page_size * kv4_row_bytes(head_dim);
}

int mc_kv_append(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, const void *k,
                 int64_t k_stride, const void *v, int64_t v_stride, int q_heads, const void *q_norm,
                 const void *k_norm, float eps, const float *rope, int rope_rows, int rot_dim, int interleaved,
                 void *q_out, void *workspace, void *stream)
{
    return append(cache, batch, q, q_stride, k, k_stride, v, v_stride, q_heads, q_norm, k_norm, eps, rope, rope_rows, rot_dim,
                  interleaved, q_out, workspace, false, stream);
}

int mc_kv4_append(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, const void *k,
                  int64_t k_stride, const void *v, int64_t v_stride, int q_heads, const void *q_norm,
                  const void *k_norm, float eps, const float *rope, int rope_rows, int rot_dim, int interleaved,
                  void *q_out, void *workspace, void *stream)
{
    return append(cache, batch, q, q_stride, k, k_stride, v, v_stride, q_heads, q_norm, k_norm, eps, rope, rope_rows, rot_dim,
                  interleaved, q_out, workspace, true, stream);
}

int mc_kv4_read(const mc_kv_cache *cache, const mc_kv_batch *batch, void *k, void *v, void *workspace, void *stream)
{
    clear_error();
    int rc = check_cache(cache, cache ? cache->kv_heads : 1, true);
    if (rc || (rc = check_counts(batch))) return rc;
    if (batch->tokens == 0 || batch->seqs == 0 || (!k && !v)) return MC_OK;
    if ((rc = check_batch(cache, batch))) return rc;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(workspace, 4))
        return set_error(MC_ERR_INVALID_ARG, "k and v must be 16-byte aligned, the workspace 4");
    ReadParams p = {view(cache), view(batch), (uint16_t *)k, (uint16_t *)v, (int32_t *)workspace};
    return launch_read4(p, cache->head_dim, cache->dtype == MC_BF16, (cudaStream_t)stream);
}

int mc_attn_decode(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, int q_heads,
                   const mc_attn_opts *opts, void *out, int64_t out_stride, float *lse, void *workspace,
                   size_t ws_bytes, void *stream)
{
    return attention(cache, batch, q, q_stride, q_heads, opts, out, out_stride, lse, workspace, ws_bytes, true, false, stream);
}

int mc_attn_prefill(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, int q_heads,
                    const mc_attn_opts *opts, void *out, int64_t out_stride, float *lse, void *workspace,
                    size_t ws_bytes, void *stream)
{
    return attention(cache, batch, q, q_stride, q_heads, opts, out, out_stride, lse, workspace, ws_bytes, false, false, stream);
}

int mc_attn4_decode(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, int q_heads,
                   const mc_attn_opts *opts, void *out, int64_t out_stride, float *lse, void *workspace,
                   size_t ws_bytes, void *stream)
{
    return attention(cache, batch, q, q_stride, q_heads, opts, out, out_stride, lse, workspace, ws_bytes, true, true, stream);
}

int mc_attn4_prefill(const mc_kv_cache *cache, const mc_kv_batch *batch, const void *q, int64_t q_stride, int q_heads,
                    const mc_attn_opts *opts, void *out, int64_t out_stride, float *lse, void *workspace,
                    size_t ws_bytes, void *stream)
{
    return attention(cache, batch, q, q_stride, q_heads, opts, out, out_stride, lse, workspace, ws_bytes, false, true, stream);
}

}  // extern "C"
