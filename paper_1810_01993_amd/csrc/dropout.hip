// Dropout on a flat tensor, with the mask drawn from a counter-based generator and never stored:
//   y[i] = residual[i] + (u[i] >= t ? scale * x[i] : 0),  u[i] a 16-bit number, t = p * 65536, scale = 65536 / (65536 - t).
// A dropped element is chosen away, not multiplied by zero: an infinity or NaN there does not reach y.  The same kernel
// without a residual on dy is the backward pass.
#include "rows.h"

namespace dlk {

constexpr int DO_THREADS = 256;

template <class T>
__global__ __launch_bounds__(DO_THREADS) void dropout_kernel(const DropoutArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    const Philox rng(p.drop);
    const elem *x = static_cast<const elem *>(p.x), *res = static_cast<const elem *>(p.residual);
    elem *y = static_cast<elem *>(p.y);
    const int64_t blocks = (p.n + 7) / 8;
    for (int64_t b = (int64_t)blockIdx.x * DO_THREADS + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * DO_THREADS) {
        const u32x4_t w = rng((uint64_t)b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t i = 8 * b + e;
            if (i >= p.n) break;
            const float v = philox_field(w, e) >= p.drop.t ? R::get(x[i]) : 0.f;
            y[i] = R::put(res ? fmaf(v, p.drop.scale, R::get(res[i])) : v * p.drop.scale);
        }
    }
}

hipError_t launch_dropout(const DropoutArgs &a, int dtype, hipStream_t stream)
{
    if (a.n <= 0) return hipSuccess;
    const int64_t wgs = ((a.n + 7) / 8 + DO_THREADS - 1) / DO_THREADS;
    const dim3 grid((unsigned)(wgs < 65536 ? wgs : 65536)), block(DO_THREADS);
    if (dtype == 0) DLK_LAUNCH("dropout_kernel", dropout_kernel<F16>, grid, block, 0, stream, a);
    else if (dtype == 1) DLK_LAUNCH("dropout_kernel", dropout_kernel<BF16>, grid, block, 0, stream, a);
    else DLK_LAUNCH("dropout_kernel", dropout_kernel<F32>, grid, block, 0, stream, a);
    return launch_status();
}

}  // namespace dlk
