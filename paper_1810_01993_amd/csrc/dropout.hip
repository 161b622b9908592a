// Dropout on a flat tensor, with the mask drawn from a counter-based generator and never stored:
//   y[i] = residual[i] + (u[i] >= t ? scale * x[i] : 0),  u[i] a 16-bit number, t = p * 65536, scale = 65536 / (65536 - t).
// A dropped element is chosen away, not multiplied by zero: an infinity or NaN there does not reach y.  The same kernel
// without a residual on dy is the backward pass.
//
// Bound by memory: 2 or 3 tensors cross it, and the generator's 20 wide products per 16-byte piece (about two thirds of the
// instructions) fit under that.  A thread has four pieces' loads in flight before it computes the first; one tile of them per
// workgroup, all tiles in the grid (walking the tensor with 1024 workgroups instead: 1769472 x 256 fp16 with a residual 477 us
// against 434, 6.3 TB/s).  Loads carry the hint that the input is not needed again, stores do not, since what follows reads y:
// 56.6 M fp16 elements take 42.0 us without hints, 40.4 with the loads' (5.6 TB/s), 38.8 with both, but together with a kernel that
// reads y 52.6, 53.5 and 56.4 us.
#include <algorithm>

#include "rows.h"

namespace dlk {

// Only the products written as such are fused with an addition: layer_norm.hip forms the same sums.
#pragma clang fp contract(off)

constexpr int DO_THREADS = 256, DO_PIECES = 4;

template <class T, bool RES>
__global__ __launch_bounds__(DO_THREADS) void dropout_kernel(const DropoutArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    constexpr int E = R::E, U = DO_PIECES;
    const Philox rng(p.drop);
    const elem *x = static_cast<const elem *>(p.x), *res = static_cast<const elem *>(p.residual);
    elem *y = static_cast<elem *>(p.y);
    const int64_t pieces = p.n / E;
    auto one = [&](int64_t j, u32x4_t xv, u32x4_t rv) {
        float f[E];
        R::unpack(xv, f);
        uint32_t w[E / 2];
        if (p.drop.t) {
            drop_words<E, true>(rng, (uint64_t)j * E, w);
            drop_select<E>(w, p.drop.limit, f);
        }
        if constexpr (RES) {
            float r[E];
            R::unpack(rv, r);
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = fmaf(f[e], p.drop.scale, r[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] *= p.drop.scale;
        }
        reinterpret_cast<u32x4_t *>(y)[j] = R::pack(f);
    };
    const u32x4_t *xp = reinterpret_cast<const u32x4_t *>(x), *rp = reinterpret_cast<const u32x4_t *>(res);
    for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int64_t first = tile * (U * DO_THREADS) + threadIdx.x;
        if ((tile + 1) * (U * DO_THREADS) <= pieces) {
            u32x4_t xv[U], rv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                xv[u] = __builtin_nontemporal_load(xp + first + u * DO_THREADS);
                if constexpr (RES) rv[u] = __builtin_nontemporal_load(rp + first + u * DO_THREADS);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) one(first + u * DO_THREADS, xv[u], RES ? rv[u] : u32x4_t{});
            continue;
        }
        for (int64_t j = first; j < pieces; j += DO_THREADS) one(j, xp[j], RES ? rp[j] : u32x4_t{});
        const int64_t i = pieces * E + threadIdx.x;     // what is left of the last piece
        if (i < p.n) {
            float f[1] = {R::get(x[i])};
            if (p.drop.t) {
                uint32_t w[1];
                drop_words<1, false>(rng, (uint64_t)i, w);
                drop_select<1>(w, p.drop.limit, f);
            }
            y[i] = R::put(RES ? fmaf(f[0], p.drop.scale, R::get(res[i])) : f[0] * p.drop.scale);
        }
    }
}

template <class T>
static hipError_t dropout_type(const DropoutArgs &a0, hipStream_t stream)
{
    DropoutArgs a = a0;
    const int64_t per = (int64_t)DO_PIECES * DO_THREADS * Row<T>::E;
    a.tiles = (a.n + per - 1) / per;
    const dim3 grid((unsigned)std::min<int64_t>(a.tiles, 1 << 22)), block(DO_THREADS);
    if (a.residual) DLK_LAUNCH("dropout_kernel", (dropout_kernel<T, true>), grid, block, 0, stream, a);
    else DLK_LAUNCH("dropout_kernel", (dropout_kernel<T, false>), grid, block, 0, stream, a);
    return launch_status();
}

hipError_t launch_dropout(const DropoutArgs &a, int dtype, hipStream_t stream)
{
    if (a.n <= 0) return hipSuccess;
    return dtype == 0 ? dropout_type<F16>(a, stream) : dtype == 1 ? dropout_type<BF16>(a, stream) : dropout_type<F32>(a, stream);
}

}  // namespace dlk
