// mc_kv.cu -- mc_kv_append and mc_kv4_append: new tokens into the paged key-value cache, in 16 or in 4 bits,
// with the per-head norms and the position rotation on the way; mc_kv4_read: the 4-bit cache's rows as they stand.
#include <math.h>

#include "mc_attn.h"
#include "mc_host.h"
#include "mc_kv4.cuh"
#include "mc_profile.h"

namespace mc {

constexpr int kAppendPasses = 4;  // rows a half or quarter warp takes, loads first
constexpr int kAppendThreads = 128;

// Warps that a token's heads of one kind take.
__host__ __device__ constexpr int append_warps(int heads, int D)
{
    return (heads * D / 256 + kAppendPasses - 1 + (heads * D % 256 != 0)) / kAppendPasses;
}

__device__ __forceinline__ uint64_t swapped(uint64_t v)
{
    float a, b;
    unpair2(v, a, b);
    return pair2(b, a);
}

// A head's row of D elements is shared by D / 8 lanes; a warp takes 256 / D rows at a time,
// kAppendPasses times, heads of one token and one kind (queries, keys or values), so its place,
// its rotation and the norm's weights are found once for them and values are only copied.  A lane
// holds two runs of four elements, chosen so that both members of every pair that the rotation
// turns lie in it (runs 4i and rot/2 + 4i, or 8i and 8i + 4 for interleaved pairs): no exchange
// between lanes but the norm's sum.  With the weights g folded in, the two elements of a pair are
//   a' = (a (g_a c) - b (g_b s)) / rms,  b' = (b (g_b c) + a (g_a s)) / rms
// two at a time (f32x2).  Issue-bound before that (850 instructions a warp, rows of all kinds
// alike): 8192 tokens of 48 heads of 128, norms and rotation, 48 us; now 37 us, 5.6 TB/s (issue
// 77 % active, ALU 61 %).  Eight passes a warp (84 registers) took 48 us where four took 41.
//
// Q4: a key's or value's row, rounded to the type, is brought into its own order where the rotation's runs are
// not (through shared memory, a row of D elements by its D / 8 lanes), so that the 8 lanes of a group hold its 64
// elements, 8 each; they find its ends by exchanging pairs and each writes a word of codes.  8192 tokens as above 47 us
// (issue 68 % active, ALU 56 %: 120 instructions more for two rows of 128).
template <int D, bool BF16, bool Q4>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendParams p)
{
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    __shared__ __align__(16) uint16_t rows_s[Q4 ? kAppendThreads / 32 : 1][Q4 ? 256 : 8];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, li = lane % kLanes;
    const int wq = append_warps(p.q_heads, D), wk = append_warps(p.c.kv_heads, D);
    const int64_t warp = (int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
    int w;  // of the token's warps
    const int t = p.per_token.div((int)warp, w);
    if (t >= p.b.tokens) {
        // the warp after the last token's looks over cu_q, of which a token meets one sequence's part
        if (p.b.cu_q && t == p.b.tokens && w == 0)
            for (int i = lane; i < p.b.seqs; i += 32) {
                int first;
                seq_rows(p.b, i, first, p.status);
            }
        return;
    }
    const bool is_q = w < wq, is_v = w >= wq + wk;
    const int heads = is_q ? p.q_heads : p.c.kv_heads;
    const int h0 = (is_q ? w : is_v ? w - wq - wk : w - wq) * kRows * kAppendPasses + lane / kLanes;
    const uint16_t *src = is_q ? p.q + t * p.q_stride : is_v ? p.v + t * p.v_stride : p.k + t * p.k_stride;
    const uint16_t *gain = is_q ? p.q_norm : is_v ? nullptr : p.k_norm;
    const int rot = is_v ? 0 : p.rot;

    const bool turn = p.interleaved ? 8 * li < rot : 4 * li < rot / 2;
    int ea = 8 * li, eb = ea + 4;
    if (turn && !p.interleaved) ea = 4 * li, eb = rot / 2 + ea;  // (the runs that are not turned stay in place)

    uint2 a[kAppendPasses], b[kAppendPasses];
#pragma unroll
    for (int i = 0; i < kAppendPasses; ++i) {
        const int h = h0 + i * kRows;
        a[i] = b[i] = make_uint2(0, 0);
        if (h < heads) {
            a[i] = *reinterpret_cast<const uint2 *>(src + h * D + ea);
            b[i] = *reinterpret_cast<const uint2 *>(src + h * D + eb);
        }
    }
    uint2 ga = make_uint2(0, 0), gb = ga;
    if (gain) {
        ga = *reinterpret_cast<const uint2 *>(gain + ea);
        gb = *reinterpret_cast<const uint2 *>(gain + eb);
    }

    const TokenPlace place = token_place(p.b, p.c, t, lane, p.status);
    if (place.seq < 0) return;  // padding
    int pos = place.pos;
    int64_t at = -1;  // the row's element offset in the cache (Q4: of its page, in bytes)
    int at_row = 0;
    float4 cs = make_float4(1.f, 1.f, 1.f, 1.f), sn = make_float4(0.f, 0.f, 0.f, 0.f);
    if (p.rot && pos >= p.rope_rows) {
        set_status(p.status, MC_ERR_RANGE);
        pos = -1;
    }
    if (pos >= 0) {
        if (turn) {
            const float *r = p.rope + (int64_t)pos * rot + 4 * li;
            cs = *reinterpret_cast<const float4 *>(r);
            sn = *reinterpret_cast<const float4 *>(r + rot / 2);
        }
        if (!is_q) {
            int row;
            const int i = p.c.page.div(pos, row), page = seq_page(p.b, p.c, place.seq, i, p.status);
            if (page >= 0) at = page * p.c.page_stride + (Q4 ? 0 : (int64_t)row * D);
            at_row = row;
        }
    }
    if (!is_q && at < 0) return;
    uint16_t *dst = is_q ? p.q_out + (int64_t)t * p.q_heads * D : Q4 ? nullptr : (is_v ? p.c.v : p.c.k) + at;
    const int64_t head_stride = is_q ? D : (int64_t)p.c.page_size * D;
    constexpr int kGroups = D / kKv4Group;
    const int block_bytes = p.c.page_size * kv4_row_bytes(D);
    uint8_t *const block = Q4 && !is_q ? reinterpret_cast<uint8_t *>(is_v ? p.c.v : p.c.k) + at + (int64_t)h0 * block_bytes : nullptr;
    uint8_t *const codes_at = block + at_row * kv4_code_bytes(D) + 4 * (li % 8 * kGroups + li / 8);
    uint8_t *const words_at = block + p.c.page_size * kv4_code_bytes(D) + at_row * kv4_word_bytes(D) + 2 * (li / 8);
    const bool grids = Q4 && !is_q;
    // a row of a key or value on its grids; the whole warp, with rows of heads past the last among them
    auto store4 = [&](int i, const uint32_t (&v)[4]) {
        uint32_t x[4] = {v[0], v[1], v[2], v[3]}, word;
        if (rot && !p.interleaved) {
            uint16_t *own = rows_s[threadIdx.x >> 5] + lane / kLanes * D;
            *reinterpret_cast<uint2 *>(own + ea) = make_uint2(v[0], v[1]);
            *reinterpret_cast<uint2 *>(own + eb) = make_uint2(v[2], v[3]);
            __syncwarp();
            const uint4 y = *reinterpret_cast<const uint4 *>(own + 8 * li);
            x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
            __syncwarp();
        }
        const uint32_t codes = kv4_quantise<BF16>(x, word);
        if (h0 + i * kRows >= heads) return;
        const int64_t off = (int64_t)i * kRows * block_bytes;
        *reinterpret_cast<uint32_t *>(codes_at + off) = codes;
        if (li % 8 == 0) *reinterpret_cast<uint16_t *>(words_at + off) = (uint16_t)word;
    };
    if ((!gain && !rot) || pos < 0) {  // copied, or zero
#pragma unroll
        for (int i = 0; i < kAppendPasses; ++i) {
            const int h = h0 + i * kRows;
            if (grids) {
                if (h - lane / kLanes < heads) store4(i, {a[i].x, a[i].y, b[i].x, b[i].y});  // (for all lanes)
            } else if (h < heads) {
                *reinterpret_cast<uint2 *>(dst + h * head_stride + ea) = pos < 0 ? make_uint2(0, 0) : a[i];
                *reinterpret_cast<uint2 *>(dst + h * head_stride + eb) = pos < 0 ? make_uint2(0, 0) : b[i];
            }
        }
        return;
    }

    // factors of the pair members: own (u) and partner's (v) of runs a and b
    uint64_t ua[2], va[2], ub[2], vb[2];
    {
        float f[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (gain) {
            *reinterpret_cast<float2 *>(f) = unpack2<BF16>(ga.x);
            *reinterpret_cast<float2 *>(f + 2) = unpack2<BF16>(ga.y);
            *reinterpret_cast<float2 *>(f + 4) = unpack2<BF16>(gb.x);
            *reinterpret_cast<float2 *>(f + 6) = unpack2<BF16>(gb.y);
        }
        if (p.interleaved) {  // pairs (0, 1), (2, 3) of each run: the partner is the other half
            ua[0] = pair2(f[0] * cs.x, f[1] * cs.x), ua[1] = pair2(f[2] * cs.y, f[3] * cs.y);
            ub[0] = pair2(f[4] * cs.z, f[5] * cs.z), ub[1] = pair2(f[6] * cs.w, f[7] * cs.w);
            va[0] = pair2(-f[1] * sn.x, f[0] * sn.x), va[1] = pair2(-f[3] * sn.y, f[2] * sn.y);
            vb[0] = pair2(-f[5] * sn.z, f[4] * sn.z), vb[1] = pair2(-f[7] * sn.w, f[6] * sn.w);
        } else {  // element e of run a with element e of run b
            ua[0] = pair2(f[0] * cs.x, f[1] * cs.y), ua[1] = pair2(f[2] * cs.z, f[3] * cs.w);
            ub[0] = pair2(f[4] * cs.x, f[5] * cs.y), ub[1] = pair2(f[6] * cs.z, f[7] * cs.w);
            va[0] = pair2(-f[4] * sn.x, -f[5] * sn.y), va[1] = pair2(-f[6] * sn.z, -f[7] * sn.w);
            vb[0] = pair2(f[0] * sn.x, f[1] * sn.y), vb[1] = pair2(f[2] * sn.z, f[3] * sn.w);
        }
    }
#pragma unroll
    for (int i = 0; i < kAppendPasses; ++i) {
        const int h = h0 + i * kRows;
        if (h - lane / kLanes >= heads) break;  // (for all lanes)
        const uint32_t words[4] = {a[i].x, a[i].y, b[i].x, b[i].y};
        uint64_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = unpack2<BF16>(words[e]);
            x[e] = pair2(f.x, f.y);
        }
        float inv = 1.f;
        if (gain) {
            float lo, hi;
            unpair2(fma2(x[3], x[3], fma2(x[2], x[2], fma2(x[1], x[1], mul2(x[0], x[0])))), lo, hi);
            float ss = lo + hi;
#pragma unroll
            for (int m = kLanes / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
            inv = rsqrtf(ss * (1.f / D) + p.eps);
        }
        uint64_t y[4] = {0, 0, 0, 0};  // partners; none (not a product with an infinity) where nothing turns
        if (turn) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = p.interleaved ? swapped(x[e]) : x[e ^ 2];
        }
        const uint64_t i2 = pair2(inv, inv);
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint64_t z = fma2(x[e], e < 2 ? ua[e] : ub[e - 2], mul2(y[e], e < 2 ? va[e] : vb[e - 2]));
            if (gain) z = mul2(z, i2);
            float lo, hi;
            unpair2(z, lo, hi);
            out[e] = pack2<BF16>(lo, hi);
        }
        if (grids) {
            store4(i, out);
        } else if (h < heads) {
            *reinterpret_cast<uint2 *>(dst + h * head_stride + ea) = make_uint2(out[0], out[1]);
            *reinterpret_cast<uint2 *>(dst + h * head_stride + eb) = make_uint2(out[2], out[3]);
        }
    }
}

// Rows of the batch's new tokens as they are stored: a warp takes a token's heads of one side (keys or values),
// 256 elements at a time, a word of codes a lane.  Bound by the writes: 8192 tokens of 8 heads of 128, 42 MB in all, 9 us.
template <int D, bool BF16>
__global__ void __launch_bounds__(kAppendThreads) read4_kernel(const ReadParams p)
{
    constexpr int kLanes = D / 8, kRows = 32 / kLanes, kGroups = D / kKv4Group;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, li = lane % kLanes, g = li / 8, i = li % 8;
    const int64_t warp = (int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
    const int t = (int)(warp >> 1);
    if (t >= p.b.tokens) return;
    uint16_t *out = warp & 1 ? p.v : p.k;
    if (!out) return;
    const TokenPlace place = token_place(p.b, p.c, t, lane, p.status);
    if (place.seq < 0) return;  // padding
    int row = 0, page = -1;
    if (place.pos >= 0) {
        const int n = p.c.page.div(place.pos, row);
        page = seq_page(p.b, p.c, place.seq, n, p.status);
    }
    out += (int64_t)t * p.c.kv_heads * D;
#pragma unroll 4
    for (int h = lane / kLanes; h < p.c.kv_heads; h += kRows) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (page >= 0) {
            const uint8_t *block = kv4_block<D>(p.c, warp & 1 ? p.c.v : p.c.k, page, h);
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(block + row * kv4_code_bytes(D) + 4 * (i * kGroups + g));
            const uint32_t word = *reinterpret_cast<const uint16_t *>(block + p.c.page_size * kv4_code_bytes(D) + row * kv4_word_bytes(D) + 2 * g);
            using P = Kv4Pairs<BF16>;
            const uint32_t z = P::zeros(word), s = P::scales(word);
            x = make_uint4(P::mul(P::sub(P::magic(codes, 0), z), s), P::mul(P::sub(P::magic(codes, 1), z), s),
                           P::mul(P::sub(P::magic(codes, 2), z), s), P::mul(P::sub(P::magic(codes, 3), z), s));
        }
        *reinterpret_cast<uint4 *>(out + h * D + 8 * li) = x;
    }
}

int launch_read4(const ReadParams &p, int head_dim, bool bf16, cudaStream_t st)
{
    const int64_t ctas = ((int64_t)p.b.tokens * 2 + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    auto k = head_dim == 64 ? (bf16 ? read4_kernel<64, true> : read4_kernel<64, false>)
                            : (bf16 ? read4_kernel<128, true> : read4_kernel<128, false>);
    profile_begin(kKRead, st);
    cudaError_t e = launch_k(k, dim3((unsigned)ctas), dim3(kAppendThreads), 0, st, p);
    profile_end(kKRead, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "read launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

// The keys that a batch's new tokens see, as 16-bit pages of sequence after sequence (page i of sequence b at
// b * table_width + i, which is also what the table written here says): what attention of prompts reads, so that a key
// is unpacked once and not for every 256 rows that see it.  A block takes 64 keys of four heads, a thread
// a 16-byte chunk of codes of a key and of a value of each.  Bound by the writes, 4 D bytes a key (they stay in L2 for the
// attention as far as they fit): 8192 keys of 8 heads of 128, 33 MB, 9 us.
constexpr int kUnpackKeys = 64, kUnpackHeads = 4;  // heads of a block
template <int D, bool BF16>
__global__ void __launch_bounds__(kUnpackKeys * D / 32) unpack4_kernel(const Unpack4Params p)
{
    constexpr int kChunks = D / 32, kGroups = D / kKv4Group;  // 16-byte chunks of a row's codes
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.z, h0 = blockIdx.y * kUnpackHeads, row = threadIdx.x / kChunks, ch = threadIdx.x % kChunks;
    const int j = blockIdx.x * kUnpackKeys + row;
    if (h0 == 0)
        for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.b.table_width; i += gridDim.x * blockDim.x)
            p.table[(int64_t)b * p.b.table_width + i] = b * p.b.table_width + i;
    int first;
    const int n = seq_rows(p.b, b, first, p.status), len = seq_len(p.b, p.c, b, p.status);
    const int seen = p.window ? max(0, len - n - p.window + 1) : 0;
    if (n == 0 || j >= len || j < (seen & ~127)) return;
    int r;
    const int i = p.c.page.div(j, r), page = j < seen ? -1 : seq_page(p.b, p.c, b, i, p.status);
    const int64_t plane = (int64_t)p.c.page_size * D;
    const int64_t to = (((int64_t)b * p.b.table_width + i) * p.c.kv_heads + h0) * plane + (int64_t)r * D;
    const int block_bytes = p.c.page_size * kv4_row_bytes(D);
    using P = Kv4Pairs<BF16>;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const uint8_t *block = kv4_block<D>(p.c, side ? p.c.v : p.c.k, max(page, 0), h0);
        uint4 codes[kUnpackHeads];
        uint32_t words[kUnpackHeads];
#pragma unroll
        for (int h = 0; h < kUnpackHeads; ++h) {  // all loads before the first use
            codes[h] = make_uint4(0, 0, 0, 0);
            words[h] = 0;  // (no such page, or behind the window: zeros)
            if (page < 0 || h0 + h >= p.c.kv_heads) continue;
            codes[h] = __ldg(reinterpret_cast<const uint4 *>(block + h * block_bytes + r * kv4_code_bytes(D)) + ch);
            const uint8_t *w = block + h * block_bytes + p.c.page_size * kv4_code_bytes(D) + r * kv4_word_bytes(D);
            words[h] = D == 128 ? __ldg(reinterpret_cast<const uint32_t *>(w)) : __ldg(reinterpret_cast<const uint16_t *>(w));
        }
#pragma unroll
        for (int h = 0; h < kUnpackHeads; ++h) {
            if (h0 + h >= p.c.kv_heads) break;
            uint16_t *out = (side ? p.v : p.k) + to + h * plane;
            const uint32_t w[4] = {codes[h].x, codes[h].y, codes[h].z, codes[h].w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int at = 4 * ch + x, g = at % kGroups;  // word at / kGroups of group g
                const uint32_t z = P::zeros(words[h] >> (16 * g)), sc = P::scales(words[h] >> (16 * g));
                *reinterpret_cast<uint4 *>(out + 64 * g + 8 * (at / kGroups)) =
                    make_uint4(P::mul(P::sub(P::magic(w[x], 0), z), sc), P::mul(P::sub(P::magic(w[x], 1), z), sc),
                               P::mul(P::sub(P::magic(w[x], 2), z), sc), P::mul(P::sub(P::magic(w[x], 3), z), sc));
            }
        }
    }
}

int launch_unpack4(const Unpack4Params &p, int head_dim, bool bf16, cudaStream_t st)
{
    const int64_t room = (int64_t)p.b.table_width * p.c.page_size;
    const dim3 grid((unsigned)((room + kUnpackKeys - 1) / kUnpackKeys), (p.c.kv_heads + kUnpackHeads - 1) / kUnpackHeads, p.b.seqs);
    auto k = head_dim == 64 ? (bf16 ? unpack4_kernel<64, true> : unpack4_kernel<64, false>)
                            : (bf16 ? unpack4_kernel<128, true> : unpack4_kernel<128, false>);
    profile_begin(kKUnpack, st);
    cudaError_t e = launch_k(k, grid, dim3(kUnpackKeys * head_dim / 32), 0, st, p);
    profile_end(kKUnpack, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "unpack launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

template <bool Q4>
static auto append_of(int head_dim, bool bf16)
{
    return head_dim == 64 ? (bf16 ? append_kernel<64, true, Q4> : append_kernel<64, false, Q4>)
                          : (bf16 ? append_kernel<128, true, Q4> : append_kernel<128, false, Q4>);
}

int launch_append(AppendParams p, int head_dim, bool bf16, bool q4, cudaStream_t st)
{
    const int per = append_warps(p.q_heads, head_dim) + 2 * append_warps(p.c.kv_heads, head_dim);
    const int64_t ctas = ((int64_t)p.b.tokens * per + (p.b.cu_q ? 1 : 0) + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (ctas > 0x7fffffff / (kAppendThreads / 32))
        return set_error(MC_ERR_UNSUPPORTED, "%d tokens of %d heads in one call", p.b.tokens, p.q_heads + 2 * p.c.kv_heads);
    p.per_token = FastDiv(per);
    auto k = q4 ? append_of<true>(head_dim, bf16) : append_of<false>(head_dim, bf16);
    profile_begin(kKAppend, st);
    cudaError_t e = launch_k(k, dim3((unsigned)ctas), dim3(kAppendThreads), 0, st, p);
    profile_end(kKAppend, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "append launch: %s", cudaGetErrorString(e));
    return MC_OK;
}

}  // namespace mc
