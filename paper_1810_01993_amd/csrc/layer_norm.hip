// Layer norm over the channels of each pixel, and its backward pass, alone or behind a residual add with dropout.
//   forward:   s = residual + dropout(x)  (or x itself);  m = sum_c s / C;  v = sum_c (s - m)^2 / C;  r = 1 / sqrt(v + eps)
//              y = (s - m) r gamma + beta
//   backward:  h = (s - m) r;  g = dy gamma;  a = sum_c g / C;  b = sum_c g h / C
//              ds = r (g - a - h b)  (+ the gradient that reaches s by another way);  dx = dropout's mask and scale on ds
//              dgamma = sum_pixels dy h;  dbeta = sum_pixels dy
// The norm is that of s as stored (rounded), so that the backward pass, which has nothing else, sees the same numbers.
#include <algorithm>

#include "rows.h"

namespace dlk {

constexpr int LN_THREADS = 256;

__device__ __forceinline__ float block_sum(float v, float *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();                                    // red may still be read from the sum before
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// One row per workgroup, each thread the elements c = thread, thread + 256, ...: any number of channels.
template <class T, bool JOINED>
__global__ __launch_bounds__(LN_THREADS) void layer_norm_fwd_kernel(const LayerNormArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    __shared__ float red[4];
    const Philox rng(p.drop);
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x) {
        const int64_t base = row * p.C;
        const elem *x = static_cast<const elem *>(p.x) + base;
        const elem *s = x;
        float sum = 0.f;
        if constexpr (JOINED) {
            const elem *res = p.residual ? static_cast<const elem *>(p.residual) + base : nullptr;
            elem *out = static_cast<elem *>(p.s) + base;
            for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
                float v = R::get(x[c]);
                if (p.drop.t) {
                    const uint64_t i = (uint64_t)(base + c);
                    v = philox_field(rng(i >> 3), (int)(i & 7)) >= p.drop.t ? v : 0.f;
                    v = res ? fmaf(v, p.drop.scale, R::get(res[c])) : v * p.drop.scale;
                } else if (res) v += R::get(res[c]);
                out[c] = R::put(v);
                sum += R::get(R::put(v));
            }
            s = out;
        } else {
            for (int c = threadIdx.x; c < p.C; c += LN_THREADS) sum += R::get(x[c]);
        }
        const float mean = block_sum(sum, red) / (float)p.C;
        float sq = 0.f;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const float d = R::get(s[c]) - mean;
            sq = fmaf(d, d, sq);
        }
        const float rstd = 1.f / sqrtf(block_sum(sq, red) / (float)p.C + p.eps);
        elem *y = static_cast<elem *>(p.y) + base;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const float h = (R::get(s[c]) - mean) * rstd;
            y[c] = R::put(p.gamma ? fmaf(h, p.gamma[c], p.beta[c]) : h);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <class T, bool JOINED>
__global__ __launch_bounds__(LN_THREADS) void layer_norm_bwd_kernel(const LayerNormArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    __shared__ float red[4];
    const Philox rng(p.drop);
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x) {
        const int64_t base = row * p.C;
        const elem *dy = static_cast<const elem *>(p.dy) + base, *s = static_cast<const elem *>(p.x) + base;
        const float mean = p.mean[row], rstd = p.rstd[row];
        float a = 0.f, b = 0.f;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const float g = R::get(dy[c]) * (p.gamma ? p.gamma[c] : 1.f);
            a += g;
            b = fmaf(g, (R::get(s[c]) - mean) * rstd, b);
        }
        a = block_sum(a, red) / (float)p.C;
        b = block_sum(b, red) / (float)p.C;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const float g = R::get(dy[c]) * (p.gamma ? p.gamma[c] : 1.f);
            float d = rstd * (g - a - (R::get(s[c]) - mean) * rstd * b);
            if constexpr (JOINED) {
                if (p.ds) d += R::get(static_cast<const elem *>(p.ds)[base + c]);
                if (p.dres) static_cast<elem *>(p.dres)[base + c] = R::put(d);
                if (p.drop.t) {
                    const uint64_t i = (uint64_t)(base + c);
                    d = philox_field(rng(i >> 3), (int)(i & 7)) >= p.drop.t ? d * p.drop.scale : 0.f;
                }
                if (p.dx) static_cast<elem *>(p.dx)[base + c] = R::put(d);
            } else {
                static_cast<elem *>(p.dx)[base + c] = R::put(d);
            }
        }
    }
}

// Sums over the pixels of a slab: partial[slab][0][c] of dy h, [1][c] of dy.  A workgroup has 64 channels and four rows.
template <class T>
__global__ __launch_bounds__(LN_THREADS) void layer_norm_param_kernel(const LayerNormArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    __shared__ float red[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.y * 64 + lane;
    const int64_t begin = (int64_t)blockIdx.x * p.chunk, end = min(p.n, begin + p.chunk);
    float dg = 0.f, db = 0.f;
    if (c < p.C)
        for (int64_t row = begin + wave; row < end; row += 4) {
            const float g = R::get(static_cast<const elem *>(p.dy)[row * p.C + c]);
            const float h = (R::get(static_cast<const elem *>(p.x)[row * p.C + c]) - p.mean[row]) * p.rstd[row];
            dg = fmaf(g, h, dg);
            db += g;
        }
    red[0][wave][lane] = dg;
    red[1][wave][lane] = db;
    __syncthreads();
    if (wave < 2 && c < p.C)
        p.partial[((size_t)blockIdx.x * 2 + wave) * p.C + c] =
            (red[wave][0][lane] + red[wave][1][lane]) + (red[wave][2][lane] + red[wave][3][lane]);
}

// dgamma and dbeta from the slabs' sums, in ascending order of the slabs.
__global__ __launch_bounds__(LN_THREADS) void layer_norm_param_sum_kernel(const float *partial, int slabs, int C, float *dgamma,
                                                                          float *dbeta)
{
    const int64_t i = (int64_t)blockIdx.x * LN_THREADS + threadIdx.x;
    if (i >= 2 * (int64_t)C) return;
    float sum = 0.f;
    for (int z = 0; z < slabs; ++z) sum += partial[(size_t)z * 2 * C + i];
    if (i < C) dgamma[i] = sum;
    else dbeta[i - C] = sum;
}

int layer_norm_slabs(int64_t n, int C)
{
    (void)C;
    const int64_t b = (n + 63) / 64;
    return (int)(b < 1 ? 1 : b > 512 ? 512 : b);
}

template <class T>
static hipError_t launch_ln_fwd(const LayerNormArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20)), block(LN_THREADS);
    if (a.joined) DLK_LAUNCH("layer_norm_fwd_kernel", (layer_norm_fwd_kernel<T, true>), grid, block, 0, stream, a);
    else DLK_LAUNCH("layer_norm_fwd_kernel", (layer_norm_fwd_kernel<T, false>), grid, block, 0, stream, a);
    return launch_status();
}

hipError_t launch_layer_norm_fwd(const LayerNormArgs &a, int dtype, hipStream_t stream)
{
    if (a.n <= 0) return hipSuccess;
    return dtype == 0 ? launch_ln_fwd<F16>(a, stream) : dtype == 1 ? launch_ln_fwd<BF16>(a, stream) : launch_ln_fwd<F32>(a, stream);
}

template <class T>
static hipError_t launch_ln_bwd(const LayerNormArgs &a0, hipStream_t stream)
{
    LayerNormArgs a = a0;
    const dim3 block(LN_THREADS);
    if (a.dgamma) {                                     // before dx, which may lie where dy does
        a.chunk = (a.n + a.slabs - 1) / a.slabs;
        const dim3 cols((unsigned)a.slabs, (unsigned)((a.C + 63) / 64));
        DLK_LAUNCH("layer_norm_param_kernel", layer_norm_param_kernel<T>, cols, block, 0, stream, a);
        hipError_t e = launch_status();
        if (e != hipSuccess) return e;
        const dim3 all((unsigned)((2 * (int64_t)a.C + LN_THREADS - 1) / LN_THREADS));
        DLK_LAUNCH("layer_norm_param_sum_kernel", layer_norm_param_sum_kernel, all, block, 0, stream, a.partial, a.slabs, a.C, a.dgamma, a.dbeta);
        e = launch_status();
        if (e != hipSuccess) return e;
    }
    if (a.n <= 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20));
    if (a.joined) DLK_LAUNCH("layer_norm_bwd_kernel", (layer_norm_bwd_kernel<T, true>), grid, block, 0, stream, a);
    else DLK_LAUNCH("layer_norm_bwd_kernel", (layer_norm_bwd_kernel<T, false>), grid, block, 0, stream, a);
    return launch_status();
}

hipError_t launch_layer_norm_bwd(const LayerNormArgs &a, int dtype, hipStream_t stream)
{
    return dtype == 0 ? launch_ln_bwd<F16>(a, stream) : dtype == 1 ? launch_ln_bwd<BF16>(a, stream) : launch_ln_bwd<F32>(a, stream);
}

}  // namespace dlk
