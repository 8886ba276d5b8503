// mc_residual.cu -- mc_residual_norm: the norm behind a block, its gate and scale, the residual sum and
// the norm before the next block, a token's row at a time.
//
//   u = y r(y) post,  h' = a h + b gate u,  x = h' r(h') pre,   r(v) = 1 / sqrt(mean(v^2) + eps)
//
// Bound by HBM: y, h (and a whole gate) read once, h' and x written once, 8 to 10 bytes an element for a dozen
// flops.  A row stays in registers between the passes, all of its loads issued before the first use.  8192 rows of 4096 in
// bf16, both norms and a whole gate: 51.5 us, 6.5 TB/s (0.96 of the measured copy rate); 16 rows 3.1 us, latency.
// The sums take mc_rmsnorm's order (thread i of 256 over the 8-element chunks i, i + 256, ...; lanes by halves;
// warps in turn), so x is bit for bit mc_rmsnorm of h_out, and short rows share a block, warps of 256 columns
// each, with the same sums.
#include <math.h>

#include "mc_attn.h"
#include "mc_host.h"
#include "mc_profile.h"

namespace mc {

struct ResidualParams {
    int T, H, rows, warps;  // rows a block, warps a row
    const uint16_t *y, *h, *post, *pre, *gate;
    int64_t y_stride, h_stride, gate_row, out_stride, x_stride;
    int gate_col;
    float scale, residual_scale, eps;
    uint16_t *out, *x;
    int narrow;  // operands whose rows do not start at 16 bytes: bits y, h, post, pre, gate, out, x
};
enum { kY = 1, kH = 2, kPost = 4, kPre = 8, kGate = 16, kOut = 32, kX = 64 };

template <bool BF16>
__device__ __forceinline__ float load1(const uint16_t *p)
{
    return BF16 ? __uint_as_float((uint32_t)*p << 16) : __half2float(*reinterpret_cast<const __half *>(p));
}
template <bool BF16>
__device__ __forceinline__ uint16_t store1(float v)
{
    return (uint16_t)pack2<BF16>(v, 0.f);
}

// Eight columns, by one access or (where the operand's rows are not aligned) one by one.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load8(const ResidualParams &p, int which, const uint16_t *src)
{
    if (ALIGNED || !(p.narrow & which)) return *reinterpret_cast<const uint4 *>(src);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = src[2 * k] | (uint32_t)src[2 * k + 1] << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool ALIGNED>
__device__ __forceinline__ void store8(const ResidualParams &p, int which, uint16_t *dst, const uint32_t (&w)[4])
{
    if (ALIGNED || !(p.narrow & which)) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        dst[2 * k] = (uint16_t)w[k];
        dst[2 * k + 1] = (uint16_t)(w[k] >> 16);
    }
}

// 1 / sqrt of a row's mean square, from each of its threads' part.
__device__ __forceinline__ float row_rms(const ResidualParams &p, float ss, float *red, int w0)
{
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    if (p.warps == 1) return rsqrtf(ss / p.H + p.eps);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = ss;
    __syncthreads();
    float tot = 0.f;
    for (int w = 0; w < p.warps; ++w) tot += red[w0 + w];
    return rsqrtf(tot / p.H + p.eps);
}

__device__ __forceinline__ float value(const ResidualParams &p, float y, float h, float gate) { return fmaf(p.residual_scale, h, p.scale * (gate * y)); }

// Rows of whole chunks of 8 columns, PER of them a thread.
template <int PER, bool BF16, bool ALIGNED>
__global__ void __launch_bounds__(256) residual_kernel(const ResidualParams p)
{
    __shared__ float red[2][16];  // (warps of no row read past the eighth)
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5, sub = p.warps == 8 ? 0 : warp / p.warps, w0 = sub * p.warps;
    const int first = threadIdx.x - 32 * w0, step = 32 * p.warps, n8 = p.H >> 3;
    const int64_t t = (int64_t)blockIdx.x * p.rows + sub;
    const bool real = sub < p.rows && t < p.T;
    const bool gated = p.gate && p.gate_col;
    uint4 y[PER], h[PER], gate[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = first + step * i;
        const bool in = real && c < n8;
        gate[i] = gated && in ? load8<ALIGNED>(p, kGate, p.gate + t * p.gate_row + 8 * c) : make_uint4(0, 0, 0, 0);
        y[i] = in ? load8<ALIGNED>(p, kY, p.y + t * p.y_stride + 8 * c) : make_uint4(0, 0, 0, 0);
        h[i] = in ? load8<ALIGNED>(p, kH, p.h + t * p.h_stride + 8 * c) : make_uint4(0, 0, 0, 0);
    }
    const float whole = p.gate && !p.gate_col && real ? load1<BF16>(p.gate + t * p.gate_row) : 1.f;
    float inv = 1.f;
    if (p.post) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t w[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = unpack2<BF16>(w[k]);
                ss = fmaf(f.x, f.x, ss);
                ss = fmaf(f.y, f.y, ss);
            }
        }
        inv = row_rms(p, ss, red[0], w0);
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = first + step * i;
        if (!real || c >= n8) continue;
        const uint4 post = p.post ? load8<ALIGNED>(p, kPost, p.post + 8 * c) : make_uint4(0, 0, 0, 0);
        const uint32_t w[4] = {y[i].x, y[i].y, y[i].z, y[i].w}, r[4] = {h[i].x, h[i].y, h[i].z, h[i].w};
        const uint32_t pw[4] = {post.x, post.y, post.z, post.w}, g[4] = {gate[i].x, gate[i].y, gate[i].z, gate[i].w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float2 u = unpack2<BF16>(w[k]);
            if (p.post) {
                const float2 a = unpack2<BF16>(pw[k]);
                u = make_float2(u.x * inv * a.x, u.y * inv * a.y);
            }
            const float2 b = gated ? unpack2<BF16>(g[k]) : make_float2(whole, whole);
            const float2 res = unpack2<BF16>(r[k]);
            o[k] = pack2<BF16>(value(p, u.x, res.x, b.x), value(p, u.y, res.y, b.y));
            const float2 f = unpack2<BF16>(o[k]);
            ss = fmaf(f.x, f.x, ss);
            ss = fmaf(f.y, f.y, ss);
        }
        h[i] = make_uint4(o[0], o[1], o[2], o[3]);
        store8<ALIGNED>(p, kOut, p.out + t * p.out_stride + 8 * c, o);
    }
    if (!p.pre) return;
    inv = row_rms(p, ss, red[1], w0);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = first + step * i;
        if (!real || c >= n8) continue;
        const uint4 pre = load8<ALIGNED>(p, kPre, p.pre + 8 * c);
        const uint32_t w[4] = {h[i].x, h[i].y, h[i].z, h[i].w}, a[4] = {pre.x, pre.y, pre.z, pre.w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = unpack2<BF16>(w[k]), g = unpack2<BF16>(a[k]);
            o[k] = pack2<BF16>(f.x * inv * g.x, f.y * inv * g.y);
        }
        store8<ALIGNED>(p, kX, p.x + t * p.x_stride + 8 * c, o);
    }
}

// A thread's k-th column, as mc_rmsnorm has them: its 8-element chunks in turn where the width is a multiple of 8, else
// every 256th.
template <bool CHUNKS>
__device__ __forceinline__ int narrow_col(int first, int k)
{
    return CHUNKS ? 8 * (first + 256 * (k >> 3)) + (k & 7) : first + 256 * k;
}

// Rows that are not whole chunks, element by element, up to 256 PER columns; rows of up to 256 share a block, a warp for
// each 32 columns.  Bound by the accesses of 2 bytes: 8000 rows of 999 32 us (of 1000 15).
template <int PER, bool BF16>
__global__ void __launch_bounds__(256) residual_narrow_kernel(const ResidualParams p)
{
    __shared__ float red[2][16];
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5, sub = p.warps == 8 ? 0 : warp / p.warps, w0 = sub * p.warps, first = threadIdx.x - 32 * w0;
    const int64_t t = (int64_t)blockIdx.x * p.rows + sub;
    const int end = sub < p.rows && t < p.T ? p.H : 0;
    const uint16_t *yr = p.y + t * p.y_stride, *hr = p.h + t * p.h_stride;
    uint16_t y[PER], h[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = first + 256 * k;
        y[k] = h[k] = 0;
        if (c < end) y[k] = yr[c], h[k] = hr[c];
    }
    float inv = 1.f, ss = 0.f;
    if (p.post) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const float v = load1<BF16>(y + k);
            ss = fmaf(v, v, ss);
        }
        inv = row_rms(p, ss, red[0], w0);
    }
    uint16_t *out = p.out + t * p.out_stride, *x = p.x + t * p.x_stride;
    ss = 0.f;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = first + 256 * k;
        if (c >= end) continue;
        float u = load1<BF16>(y + k);
        if (p.post) u = u * inv * load1<BF16>(p.post + c);
        const float g = p.gate ? load1<BF16>(p.gate + t * p.gate_row + (p.gate_col ? c : 0)) : 1.f;
        h[k] = store1<BF16>(value(p, u, load1<BF16>(h + k), g));
        out[c] = h[k];
        const float v = load1<BF16>(h + k);
        ss = fmaf(v, v, ss);
    }
    if (!p.pre) return;
    inv = row_rms(p, ss, red[1], w0);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = first + 256 * k;
        if (c < end) x[c] = store1<BF16>(load1<BF16>(h + k) * inv * load1<BF16>(p.pre + c));
    }
}

// Wider rows, a block a row; h' is read back by the thread that wrote it.
template <bool CHUNKS, bool BF16>
__global__ void __launch_bounds__(256) residual_any_kernel(const ResidualParams p)
{
    __shared__ float red[2][16];
    pdl_trigger();
    pdl_wait();
    const int64_t t = blockIdx.x;
    const uint16_t *y = p.y + t * p.y_stride, *h = p.h + t * p.h_stride;
    uint16_t *out = p.out + t * p.out_stride, *x = p.x + t * p.x_stride;
    const int tid = threadIdx.x, count = CHUNKS ? (p.H / 8 - tid + 255) / 256 * 8 : (p.H - tid + 255) / 256;
    float inv = 1.f;
    if (p.post) {
        float ss = 0.f;
#pragma unroll 8
        for (int k = 0; k < count; ++k) {
            const float v = load1<BF16>(y + narrow_col<CHUNKS>(tid, k));
            ss = fmaf(v, v, ss);
        }
        inv = row_rms(p, ss, red[0], 0);
    }
    float ss = 0.f;
#pragma unroll 8
    for (int k = 0; k < count; ++k) {
        const int c = narrow_col<CHUNKS>(tid, k);
        float u = load1<BF16>(y + c);
        if (p.post) u = u * inv * load1<BF16>(p.post + c);
        const float g = p.gate ? load1<BF16>(p.gate + t * p.gate_row + (p.gate_col ? c : 0)) : 1.f;
        const uint16_t o = store1<BF16>(value(p, u, load1<BF16>(h + c), g));
        out[c] = o;
        const float v = load1<BF16>(&o);
        ss = fmaf(v, v, ss);
    }
    if (!p.pre) return;
    inv = row_rms(p, ss, red[1], 0);
#pragma unroll 8
    for (int k = 0; k < count; ++k) {
        const int c = narrow_col<CHUNKS>(tid, k);
        x[c] = store1<BF16>(load1<BF16>(out + c) * inv * load1<BF16>(p.pre + c));
    }
}

template <bool BF16, bool ALIGNED>
static cudaError_t launch_chunks(ResidualParams p, cudaStream_t st)
{
    if (p.H < 2048) {
        p.warps = (p.H + 255) / 256;
        p.rows = 8 / p.warps;
    }
    auto k = p.H <= 2048 ? residual_kernel<1, BF16, ALIGNED> : p.H <= 4096 ? residual_kernel<2, BF16, ALIGNED>
             : p.H <= 8192 ? residual_kernel<4, BF16, ALIGNED> : residual_kernel<8, BF16, ALIGNED>;
    return launch_k(k, dim3((unsigned)((p.T + p.rows - 1) / p.rows)), dim3(256), 0, st, p);
}

template <bool BF16>
static cudaError_t launch_residual(ResidualParams p, cudaStream_t st)
{
    p.rows = 1;
    p.warps = 8;
    if (p.H % 8 == 0) {
        if (p.H > 16384) return launch_k(residual_any_kernel<true, BF16>, dim3(p.T), dim3(256), 0, st, p);
        return p.narrow ? launch_chunks<BF16, false>(p, st) : launch_chunks<BF16, true>(p, st);
    }
    if (p.H <= 256) {
        p.warps = (p.H + 31) / 32;
        p.rows = 8 / p.warps;
    }
    // Wider rows stay in registers only where they are few: 4096 rows of 4099 columns 95 us, read again 68; 16 of them 9.6 and 12.8.
    auto k = p.H <= 256 ? residual_narrow_kernel<1, BF16> : p.H <= 2048 ? residual_narrow_kernel<8, BF16>
             : p.H <= 8192 && p.T <= 304 ? residual_narrow_kernel<32, BF16> : residual_any_kernel<false, BF16>;
    return launch_k(k, dim3((unsigned)((p.T + p.rows - 1) / p.rows)), dim3(256), 0, st, p);
}

}  // namespace mc

using namespace mc;

extern "C" int mc_residual_norm(const mc_residual_norm_args *a, void *stream)
{
    clear_error();
    if (!a) return set_error(MC_ERR_INVALID_ARG, "NULL arguments");
    if (a->dtype != MC_BF16 && a->dtype != MC_FP16) return set_error(MC_ERR_UNSUPPORTED, "dtype %d", a->dtype);
    if (a->T < 0 || a->H < 1 || !(a->eps >= 0.f) || !isfinite(a->eps)) return set_error(MC_ERR_INVALID_ARG, "T %d, H %d, eps %g", a->T, a->H, a->eps);
    if (a->H > 65536) return set_error(MC_ERR_UNSUPPORTED, "H %d (at most 65536)", a->H);
    if (!isfinite(a->scale) || !isfinite(a->residual_scale))
        return set_error(MC_ERR_INVALID_ARG, "scale %g, residual_scale %g", a->scale, a->residual_scale);
    if (a->T == 0) return MC_OK;
    if (!a->y || !a->h || !a->h_out || (a->pre_norm && !a->x)) return set_error(MC_ERR_INVALID_ARG, "NULL pointer argument");
    const void *ptrs[7] = {a->y, a->h, a->post_norm, a->pre_norm, a->gate, a->h_out, a->pre_norm ? a->x : nullptr};
    int narrow = 0;
    for (int i = 0; i < 7; ++i) {
        if (!aligned(ptrs[i], 2)) return set_error(MC_ERR_INVALID_ARG, "misaligned pointer argument");
        if (!aligned(ptrs[i], 16)) narrow |= 1 << i;
    }
    const struct {
        int which;
        int64_t stride;
    } rows[4] = {{kY, a->y_stride}, {kH, a->h_stride}, {kOut, a->h_out_stride}, {kX, a->pre_norm ? a->x_stride : a->H}};
    for (const auto &r : rows) {
        if (r.stride < a->H && a->T > 1) return set_error(MC_ERR_INVALID_ARG, "row stride %lld of %d columns", (long long)r.stride, a->H);
        if (r.stride % 8 && a->T > 1) narrow |= r.which;
    }
    if (a->gate) {
        if (a->gate_col != 0 && a->gate_col != 1) return set_error(MC_ERR_INVALID_ARG, "gate_col %d (0 or 1)", a->gate_col);
        if (a->gate_row < 0) return set_error(MC_ERR_INVALID_ARG, "gate_row %lld", (long long)a->gate_row);
        if (a->gate_row % 8 && a->T > 1) narrow |= kGate;
    }
    if (!a->gate || a->gate_col == 0) narrow &= ~kGate;  // (a gate of one value a row is read as such)
    if (a->x && a->pre_norm && a->x == a->h_out) return set_error(MC_ERR_INVALID_ARG, "x must not be h_out");
    if (a->x && a->pre_norm && a->x == a->h) return set_error(MC_ERR_INVALID_ARG, "x must not be h");
    // (in place, a row's block writes what it alone has read)
    const struct {
        const char *what;
        const void *to, *from;
        int64_t to_stride, from_stride;
    } over[3] = {{"h_out over h", a->h_out, a->h, a->h_out_stride, a->h_stride}, {"h_out over y", a->h_out, a->y, a->h_out_stride, a->y_stride},
                 {"x over y", a->pre_norm ? a->x : nullptr, a->y, a->x_stride, a->y_stride}};
    for (const auto &o : over)
        if (a->T > 1 && o.to == o.from && o.to_stride != o.from_stride)
            return set_error(MC_ERR_INVALID_ARG, "%s with row strides %lld and %lld", o.what, (long long)o.to_stride, (long long)o.from_stride);
    ResidualParams p = {};
    p.T = a->T;
    p.H = a->H;
    p.y = (const uint16_t *)a->y;
    p.h = (const uint16_t *)a->h;
    p.post = (const uint16_t *)a->post_norm;
    p.pre = (const uint16_t *)a->pre_norm;
    p.gate = (const uint16_t *)a->gate;
    p.y_stride = a->y_stride;
    p.h_stride = a->h_stride;
    p.gate_row = a->gate_row;
    p.gate_col = a->gate_col;
    p.out_stride = a->h_out_stride;
    p.x_stride = a->x_stride;
    p.scale = a->scale;
    p.residual_scale = a->residual_scale;
    p.eps = a->eps;
    p.out = (uint16_t *)a->h_out;
    p.x = (uint16_t *)a->x;
    p.narrow = narrow;
    cudaStream_t st = (cudaStream_t)stream;
    profile_begin(kKResidual, st);
    const cudaError_t e = a->dtype == MC_BF16 ? launch_residual<true>(p, st) : launch_residual<false>(p, st);
    profile_end(kKResidual, st);
    if (e != cudaSuccess) return set_error(MC_ERR_CUDA, "residual launch: %s", cudaGetErrorString(e));
    return MC_OK;
}
