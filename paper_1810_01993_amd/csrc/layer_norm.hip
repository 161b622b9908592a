// Layer norm over the channels of each pixel, and its backward pass, alone or behind a residual add with dropout.
//   forward:   s = residual + dropout(x)  (or x itself);  m = sum_c s / C;  v = sum_c (s - m)^2 / C;  r = 1 / sqrt(v + eps)
//              y = (s - m) r gamma + beta
//   backward:  h = (s - m) r;  g = dy gamma;  a = sum_c g / C;  b = sum_c g h / C
//              ds = r (g - a - h b)  (+ the gradient that reaches s by another way);  dx = dropout's mask and scale on ds
//              dgamma = sum_pixels dy h;  dbeta = sum_pixels dy
// The norm is that of s as stored (rounded), so that the backward pass, which has nothing else, sees the same numbers.
//
// Bound by memory: every tensor crosses it once.  A row stays in registers from its loads to its result, so that the mean can be
// corrected and the variance summed from the deviations themselves (one pass over memory; see ln_delta), and the sums of the backward
// pass's two parameter gradients stay in registers too.  Measured, with the bandwidth of what has to cross (a large copy reaches
// 5.5-5.7 TB/s):
//   forward   1769472 x 256 fp16 319 us (5.7 TB/s), 6912 x 1024 bf16 8.2 us (3.4)
//   backward  110592 x 304 fp16 40 us (5.1), 6912 x 2048 fp32 35 us (4.9), 208297 x 77 bf16 29 us (3.4: too little in flight, see
//             ln_shape)
//   joined    forward 110592 x 256 bf16 38 us (6.0), backward 442368 x 256 bf16 196 us (5.8), 3015 x 512 fp16 10.9 us (1.4: two
//             launches, 8.0 and 2.6 us on their own)
// The second launch of a backward call, which adds the workgroups' sums in a fixed order, shows 2.6 to 4.9 us in these cases; calls
// without parameter gradients and those that one workgroup does alone have none.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace dlk {

// Only the products written as such are fused with an addition: the joined kernels then give the bits of the separate ones.
#pragma clang fp contract(off)

// How the rows are dealt out.  A team of `lanes` lanes of a wave has a row (teams side by side in the wave have neighbouring
// rows), or, WIDE, a whole workgroup has one.  Lane l owns the 16-byte pieces l, l + lanes, ... (V at most) of its row: it reads
// them once, keeps them in registers through both sums and the result, and has the next row's pieces on their way meanwhile.
// Rows that are no whole number of pieces (ODD) end in a piece that reaches back over what the one before it covers: the elements
// that both hold are counted once and, in a team's row, stored twice, with the same bits (in a WIDE one once, see ln_store).  VEC = 1:
// rows shorter than a piece.
//
// Whole pieces are loaded with the hint that nobody reads the line again (backward 110592 x 256 fp16: 35.1 us with it, 38.1
// without); a line that rows share is not.  s and the residual's gradient, which come back a whole block later, are stored with it:
// joined forward 110592 x 256 bf16 37.8 us with it, 43.6 without; backward 442368 x 256 197 and 198 with inputs from memory, 169 and
// 199 where part of them is still in the last-level cache.  y and dx are not, the next kernel reads them: joined forward 110592 x 512
// fp16 72 us, and 90.5 together with a kernel that reads y; with the hint on y too 80.8 and 100.
constexpr int LN_WAVES = 4;                             // of a workgroup whose teams lie within waves
struct LnShape {
    int pieces, lanes, waves, v;                        // of a row; lanes 0: WIDE; pieces a lane has
    int grid;
    int64_t trips;                                      // rows that a team, or a workgroup, goes through
};

template <class T, int VEC, int V, bool ODD> struct LnLane {
    int c0[V], skip;                                    // first element of a piece; elements of the last one that the piece before it has
    bool on[V];
    __device__ __forceinline__ LnLane(int l, int lanes, int pieces, int C)
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = l + v * lanes;
            on[v] = j < pieces;
            c0[v] = on[v] ? ODD ? min(j * VEC, C - VEC) : j * VEC : 0;
        }
        skip = ODD && on[V - 1] ? (l + (V - 1) * lanes) * VEC - c0[V - 1] : 0;
    }
};

// The VEC floats of a parameter from channel c on, four at a time; `none` where there is no parameter.
template <int VEC> __device__ __forceinline__ void ln_param(const float *param, int c, bool on, float none, float (&f)[VEC])
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = none;
    if (!param || !on) return;
    if constexpr (VEC == 1) f[0] = param[c];
    else
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
            const floatx4_t w = *reinterpret_cast<const floatx4_any_t *>(param + c + e);
#pragma unroll
            for (int d = 0; d < 4; ++d) f[e + d] = w[d];
        }
}

// The sums of a piece's channels from element `skip` on.
template <int VEC, bool ODD> __device__ __forceinline__ void ln_put_sums(float *to, int skip, const float (&f)[VEC])
{
    if constexpr (VEC == 1) to[0] = f[0];
    else if (ODD && skip) {
#pragma unroll
        for (int e = 1; e < VEC; ++e)
            if (e >= skip) to[e] = f[e];
    } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 4)
            *reinterpret_cast<floatx4_any_t *>(to + e) = floatx4_any_t{f[e], f[e + 1], f[e + 2], f[e + 3]};
    }
}

// Stores piece v of a row.  The overlap of an ODD row's last piece is stored twice with the same bits by one wave.  In a WIDE row the
// two pieces may lie in different waves, and the output may lie where an input does: a wave that is ahead would overwrite what the
// other has yet to load.  There each element is stored by the one lane that counts it, and what else that lane has loaded is not used.
template <bool WIDE, bool PAST, class T, int VEC, int V, bool ODD>
__device__ __forceinline__ void ln_store(typename Row<T>::elem *row, const LnLane<T, VEC, V, ODD> &at, int v,
                                         typename Piece<T, VEC, ODD>::raw w)
{
    if constexpr (ODD && WIDE)
        if (v == V - 1 && at.skip) {
            const auto parts = __builtin_bit_cast(typename Row<T>::elems, w);
#pragma unroll
            for (int e = 1; e < VEC; ++e)
                if (e >= at.skip) row[at.c0[v] + e] = parts.v[e];
            return;
        }
    Piece<T, VEC, ODD>::template store<PAST>(row + at.c0[v], w);
}

// The second look at a row's mean.  The first, sum * inv, is off by the roundings of the sum and of inv = 1 / C, which a mean far above
// the spread would leave in every deviation from it (240 values of 10000: 1e-3, and y off by 0.3 gamma).  sd and sq are the sums of the
// deviations d from the first mean and of their squares: delta = sd / C is what the first mean lacks, to the roundings of sums of d,
// and sum (d - delta)^2 = sq - sd delta.  Rows of equal values come out exact: each d is the same few steps of the value, and the
// quotient is rounded once (its remainder is added) and so exact too.  Where the row holds an infinity or NaN sd has no finite value and
// the first mean stays.
__device__ __forceinline__ float ln_delta(float &sd, float &sq, float inv, float C)
{
    sd = fabsf(sd) < __builtin_inff() ? sd : 0.f;
    float delta = sd * inv;
    delta = fmaf(fmaf(-delta, C, sd), inv, delta);
    sq = fmaf(-sd, delta, sq);
    sq = sq < 0.f ? 0.f : sq;                           // (NaN stays)
    return delta;
}

// Sums over a row: its team's lanes (FULL: all 64), or the workgroup's waves through red (two arrays used in turn: between two
// uses of one lies the other's barrier).
template <bool FULL, bool WIDE, int N> __device__ __forceinline__ void row_sums(float (&v)[N], int lanes, float *red)
{
    team_sums(v, FULL || WIDE ? 64 : lanes);
    if constexpr (WIDE) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[16 * i + (threadIdx.x >> 6)] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = red[16 * i];
            for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v[i] += red[16 * i + w];
        }
    }
}

// The rows of a team, or of a workgroup: first, first + step, ...  DEPTH - 1 rows' loads are under way while one is computed.  They
// are not conditional (beyond the last row they read that one again, for a piece that the row does not have its first one, and nobody
// uses what comes): the wait for a row's data then counts exactly the loads behind it, where a branch round them would make it a wait
// for all.
template <bool WIDE> struct LnRows {
    int64_t row, step;
    __device__ __forceinline__ LnRows(int lanes)
    {
        const int per = WIDE ? 1 : 64 * LN_WAVES / lanes;
        step = (int64_t)gridDim.x * per;
        row = (int64_t)blockIdx.x * per + (WIDE ? 0 : threadIdx.x / lanes);
    }
};

template <class T, int VEC, int V, int MODE, bool ODD, bool WIDE, bool FULL>
__global__ __launch_bounds__(WIDE ? 512 : 64 * LN_WAVES) void layer_norm_fwd_kernel(const LayerNormArgs p, const LnShape q)
{
    constexpr bool JOINED = MODE > 0, RES = MODE > 1;
    using P = Piece<T, VEC, ODD>;
    using elem = typename P::elem;
    using raw = typename P::raw;
    constexpr int DEPTH = 2;
    __shared__ float red[3][16];
    const int lanes = WIDE ? (int)blockDim.x : FULL ? 64 : q.lanes;
    const int l = threadIdx.x & (lanes - 1);
    const LnLane<T, VEC, V, ODD> at(l, lanes, q.pieces, p.C);
    LnRows<WIDE> it(lanes);
    const elem *x = static_cast<const elem *>(p.x), *res = static_cast<const elem *>(p.residual);
    struct Buf { raw x[V], res[RES ? V : 1]; } buf[DEPTH];
    auto fetch = [&](Buf &b, int64_t r) {
        const int64_t base = min(r, p.n - 1) * p.C;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            b.x[v] = P::load(x + base + at.c0[v]);
            if constexpr (RES) b.res[v] = P::load(res + base + at.c0[v]);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) fetch(buf[d], it.row + d * it.step);
    float gamma[V][VEC], beta[V][VEC];                  // asked for behind the first rows, which are needed first
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ln_param<VEC>(p.gamma, at.c0[v], at.on[v], 1.f, gamma[v]);
        ln_param<VEC>(p.beta, at.c0[v], at.on[v], 0.f, beta[v]);
    }
    const Philox rng(p.drop);
    const float inv = 1.f / (float)p.C;
    auto row = [&](const Buf &b) {
        const int64_t base = it.row * p.C;
        float f[V][VEC], sum[1] = {0.f}, dev[2] = {0.f, 0.f};
        raw out[JOINED ? V : 1];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            P::unpack(b.x[v], f[v]);
            if constexpr (JOINED) {
                if (p.drop.t) {
                    uint32_t w[(VEC + 1) / 2];
                    drop_words<VEC, !ODD && VEC != 1>(rng, (uint64_t)(base + at.c0[v]), w);
                    drop_select<VEC>(w, p.drop.limit, f[v]);
                }
                float r[VEC];
                if constexpr (RES) P::unpack(b.res[v], r);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[v][e] = RES ? fmaf(f[v][e], p.drop.scale, r[e]) : f[v][e] * p.drop.scale;
                out[v] = P::pack(f[v]);
                P::unpack(out[v], f[v]);
            }
            if (at.on[v])
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[0] += !ODD || v < V - 1 || e >= at.skip ? f[v][e] : 0.f;
        }
        row_sums<FULL, WIDE>(sum, lanes, red[0]);
        if constexpr (JOINED)                           // behind the sum, which has waited for all of the row: s may lie where x does
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (at.on[v]) ln_store<WIDE, true>(static_cast<elem *>(p.s) + base, at, v, out[v]);
        const float first = sum[0] * inv;
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[v][e] -= first;
            if (at.on[v])
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = !ODD || v < V - 1 || e >= at.skip ? f[v][e] : 0.f;
                    dev[0] += d;
                    dev[1] = fmaf(d, d, dev[1]);
                }
        }
        row_sums<FULL, WIDE>(dev, lanes, red[1]);
        const float delta = ln_delta(dev[0], dev[1], inv, (float)p.C), mean = first + delta;
        const float rstd = 1.f / sqrtf(fmaf(dev[1], inv, p.eps));
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[v][e] = fmaf((f[v][e] - delta) * rstd, gamma[v][e], beta[v][e]);
            if (at.on[v]) ln_store<WIDE, false>(static_cast<elem *>(p.y) + base, at, v, P::pack(f[v]));
        }
        if (l == 0) {
            if (p.mean) p.mean[it.row] = mean;
            if (p.rstd) p.rstd[it.row] = rstd;
        }
    };
    for (int64_t k = 0; k < q.trips; k += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            fetch(buf[(d + DEPTH - 1) % DEPTH], it.row + (DEPTH - 1) * it.step);
            if (it.row < p.n) row(buf[d]);
            it.row += it.step;
        }
    }
}

// The backward pass.  h is formed first: it lies within sqrt(C) whatever the row's spread, so that no product leaves fp32's range that
// the gradient itself does not leave (r^2 would).  The lanes that hold a channel add up its part of dgamma and dbeta over their rows
// in registers; at the end the teams of a wave, then the waves of the workgroup are added (fixed order) and the workgroup's sums
// written as one slab.
template <class T, int VEC, int V, int MODE, bool ODD, bool WIDE, bool FULL>
__global__ __launch_bounds__(WIDE ? 512 : 64 * LN_WAVES) void layer_norm_bwd_kernel(const LayerNormArgs p, const LnShape q)
{
    constexpr bool JOINED = MODE > 0, RES = MODE > 1;
    using P = Piece<T, VEC, ODD>;
    using elem = typename P::elem;
    using raw = typename P::raw;
    constexpr int DEPTH = 2;
    extern __shared__ float lds[];                      // WIDE: [2][2][16]; otherwise the sums of the workgroup's waves
    const int lanes = WIDE ? (int)blockDim.x : FULL ? 64 : q.lanes;
    const int l = threadIdx.x & (lanes - 1);
    const LnLane<T, VEC, V, ODD> at(l, lanes, q.pieces, p.C);
    LnRows<WIDE> it(lanes);
    const elem *dy = static_cast<const elem *>(p.dy), *s = static_cast<const elem *>(p.x), *ds = static_cast<const elem *>(p.ds);
    struct Buf { raw dy[V], s[V], ds[RES ? V : 1]; float mean, rstd; } buf[DEPTH];
    auto fetch = [&](Buf &b, int64_t r) {
        r = min(r, p.n - 1);
        const int64_t base = r * p.C;
        b.mean = p.mean[r];
        b.rstd = p.rstd[r];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            b.dy[v] = P::load(dy + base + at.c0[v]);
            b.s[v] = P::load(s + base + at.c0[v]);
            if constexpr (RES) b.ds[v] = P::load(ds + base + at.c0[v]);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) fetch(buf[d], it.row + d * it.step);
    float gamma[V][VEC], dg[V][VEC], db[V][VEC];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        ln_param<VEC>(p.gamma, at.c0[v], at.on[v], 1.f, gamma[v]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) dg[v][e] = db[v][e] = 0.f;
    }
    const Philox rng(p.drop);
    const float inv = 1.f / (float)p.C;
    float *red = lds;
    auto row = [&](const Buf &b) {
        const int64_t base = it.row * p.C;
        float g[V][VEC], h[V][VEC], sum[2] = {0.f, 0.f};
        const float mean = b.mean, rstd = b.rstd;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            P::unpack(b.dy[v], g[v]);
            P::unpack(b.s[v], h[v]);
            if (!at.on[v]) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const bool mine = !ODD || v < V - 1 || e >= at.skip;
                h[v][e] = (h[v][e] - mean) * rstd;
                db[v][e] += mine ? g[v][e] : 0.f;
                dg[v][e] = fmaf(mine ? g[v][e] : 0.f, h[v][e], dg[v][e]);
                g[v][e] *= gamma[v][e];
                sum[0] += mine ? g[v][e] : 0.f;
                sum[1] = fmaf(mine ? g[v][e] : 0.f, h[v][e], sum[1]);
            }
        }
        row_sums<FULL, WIDE>(sum, lanes, red);
        if constexpr (WIDE) red = lds + (red == lds ? 32 : 0);
        const float m0 = sum[0] * inv, m1 = sum[1] * inv;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!at.on[v]) continue;
            float d[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] = fmaf(-h[v][e], m1, g[v][e] - m0);
            float r[VEC];
            if constexpr (RES) P::unpack(b.ds[v], r);
#pragma unroll
            for (int e = 0; e < VEC; ++e) d[e] = RES ? fmaf(d[e], rstd, r[e]) : d[e] * rstd;
            if constexpr (JOINED) {
                if (p.dres) ln_store<WIDE, true>(static_cast<elem *>(p.dres) + base, at, v, P::pack(d));
                if (!p.dx) continue;
                if (p.drop.t) {
                    uint32_t w[(VEC + 1) / 2];
                    drop_words<VEC, !ODD && VEC != 1>(rng, (uint64_t)(base + at.c0[v]), w);
                    drop_select<VEC>(w, p.drop.limit, d);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) d[e] *= p.drop.scale;
                }
            }
            ln_store<WIDE, false>(static_cast<elem *>(p.dx) + base, at, v, P::pack(d));
        }
    };
    for (int64_t k = 0; k < q.trips; k += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            fetch(buf[(d + DEPTH - 1) % DEPTH], it.row + (DEPTH - 1) * it.step);
            if (it.row < p.n) row(buf[d]);
            it.row += it.step;
        }
    }
    if (!p.dgamma) return;
    // with one slab the sums are the result
    float *og = q.grid == 1 ? p.dgamma : p.partial + (size_t)blockIdx.x * 2 * p.C, *ob = q.grid == 1 ? p.dbeta : og + p.C;
    if constexpr (WIDE) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (at.on[v]) {
                ln_put_sums<VEC, ODD>(og + at.c0[v], v < V - 1 ? 0 : at.skip, dg[v]);
                ln_put_sums<VEC, ODD>(ob + at.c0[v], v < V - 1 ? 0 : at.skip, db[v]);
            }
    } else {
        // [wave][dgamma, dbeta][v][lane][VEC]: consecutive lanes next to each other
        const int wave = threadIdx.x >> 6, half = V * lanes * VEC;
        float sums[2 * V * VEC];
#pragma unroll
        for (int i = 0; i < V * VEC; ++i) {
            sums[i] = dg[i / VEC][i % VEC];
            sums[V * VEC + i] = db[i / VEC][i % VEC];
        }
        if constexpr (!FULL) cross_sums(sums, lanes);
        if (FULL || (int)(threadIdx.x & 63) < lanes)
#pragma unroll
            for (int i = 0; i < 2 * V * VEC; ++i)
                lds[2 * half * wave + (i / VEC * lanes + l) * VEC + i % VEC] = sums[i];
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * V * lanes; i += 64 * LN_WAVES) {
            const int j = i < V * lanes ? i : i - V * lanes;            // piece (in order of the row)
            if (j >= q.pieces) continue;
            float sum[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                sum[e] = lds[i * VEC + e];
#pragma unroll
                for (int w = 1; w < LN_WAVES; ++w) sum[e] += lds[2 * half * w + i * VEC + e];
            }
            const int c = ODD ? min(j * VEC, p.C - VEC) : j * VEC;
            ln_put_sums<VEC, ODD>((i < V * lanes ? og : ob) + c, ODD ? j * VEC - c : 0, sum);
        }
    }
}

constexpr int LN_THREADS = 256;

template <class F> __device__ __forceinline__ F block_sum(F v, F *red)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();                                    // red may still be read from the sum before
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Rows too long for the registers (more than 16384 16-bit or 8192 fp32 channels): one row per workgroup, each thread the elements
// c = thread, thread + 256, ...; the later passes over a row find it in the caches.  A thread adds up to 4096 elements one after the
// other: the forward pass's sums are in 64 bits, in which equal values (24 bits, 2^20 of them at most) add up exactly.  Simple, and far
// from memory's rate: an element a load, several passes, a block of random numbers an element.  4096 x 16392 fp16 forward 203 us
// (1.3 TB/s; 197 with sums in 32 bits), backward 239 us (1.7), joined 400 and 451 us.
template <class T, bool JOINED>
__global__ __launch_bounds__(LN_THREADS) void layer_norm_long_fwd_kernel(const LayerNormArgs p)
{
    using R = Row<T>;
    using elem = typename R::elem;
    __shared__ double red[4];
    const Philox rng(p.drop);
    for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x) {
        const int64_t base = row * p.C;
        const elem *x = static_cast<const elem *>(p.x) + base;
        const elem *s = x;
        double sum = 0.0;
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
        const double mean = block_sum(sum, red) / p.C;
        double sq = 0.0;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const double d = R::get(s[c]) - mean;
            sq = fma(d, d, sq);
        }
        const float rstd = (float)(1.0 / sqrt(block_sum(sq, red) / p.C + p.eps));
        elem *y = static_cast<elem *>(p.y) + base;
        for (int c = threadIdx.x; c < p.C; c += LN_THREADS) {
            const float h = (float)(R::get(s[c]) - mean) * rstd;
            y[c] = R::put(p.gamma ? fmaf(h, p.gamma[c], p.beta[c]) : h);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = (float)mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <class T, bool JOINED>
__global__ __launch_bounds__(LN_THREADS) void layer_norm_long_bwd_kernel(const LayerNormArgs p)
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
            float d = rstd * fmaf(-(R::get(s[c]) - mean) * rstd, b, g - a);
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

// dgamma and dbeta from the slabs' sums: a workgroup has 16 columns and 64 lanes down the slabs, four of them in a wave.  With U >=
// slabs / 64 all loads go out at once: the kernel is one trip to memory, two lane exchanges, one barrier.
template <int U>
__global__ __launch_bounds__(1024) void layer_norm_param_sum_kernel(const float *partial, int slabs, int C, float *dgamma, float *dbeta)
{
    __shared__ float red[16][16];
    const int col = threadIdx.x & 15, lane = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 16 + col, all = 2 * (int64_t)C;
    float f[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int z = 64 * u + lane;
        f[u] = z < slabs && i < all ? partial[z * all + i] : 0.f;
    }
#pragma unroll
    for (int u = 1; u < U; ++u) f[0] += f[u];
    const float sum = swap32_add(swap16_add(f[0]));
    if ((threadIdx.x & 63) < 16) red[wave][col] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && i < all) {
        float s = red[0][col];
#pragma unroll
        for (int w = 1; w < 16; ++w) s += red[w][col];
        (i < C ? dgamma[i] : dbeta[i - C]) = s;
    }
}

// ---- dispatch ----------------------------------------------------------------
constexpr int CUS = 256;
static int pow2_from(int v) { int p = 1; while (p < v) p <<= 1; return p; }

// Up to 2048 pieces of a row stay in the registers of 8 waves.  (The joined backward pass with ds at four pieces a lane, 12289 to 16384
// 16-bit channels, needs a few more than the 256 there are: 9 to 17 words a lane go through scratch memory.  2000 x 16384 fp16 87 us,
// 3.8 TB/s.)
template <class T> static bool ln_long(int C) { return C > 2048 * Row<T>::E; }

// params: a backward call that is asked for dgamma and dbeta.
template <class T> static LnShape ln_shape(int64_t n, int C, bool bwd, bool params)
{
    constexpr int E = Row<T>::E;
    // The figures are bf16 rows, 64 M elements where no other size is given; forward first.
    const bool large = n * C * (16 / E) >= 64 << 20;
    LnShape q{};
    q.waves = LN_WAVES;
    q.v = 1;
    q.pieces = C < E ? C : (C + E - 1) / E;
    int64_t most;                                       // workgroups
    if (q.pieces <= 192) {
        if (q.pieces <= 8) q.lanes = pow2_from(q.pieces);
        else {
            // The number of pieces a lane that leaves fewest lanes idle, 8 lanes (a 128-byte line) at least: 304 channels 52.9 us with
            // three pieces (48 places for 38), 61.4 with two (64 places); 64 channels 50.0 with one, 54.5 with two and 4 lanes.
            // Where one and two leave the same, two: 256 channels 47.7 and 49.6.  The backward pass has one on short rows (96
            // channels 71.9, with two 82.7).
            const int first = bwd && q.pieces < 32 ? 1 : 2;
            int best = 1 << 30;
            for (int v : {first, 3 - first, 3}) {
                const int lanes = std::max(8, pow2_from((q.pieces + v - 1) / v));
                if (lanes <= 64 && lanes * v < best) {
                    best = lanes * v;
                    q.lanes = lanes;
                    q.v = v;
                }
            }
        }
        // Loads under way, not more: from 64 MB on 8 waves a compute unit with two or three pieces a lane, 16 with one (1769472 x 256
        // fp16 318 us with 8 waves, 367 with 16: fewer rows at a time stay within fewer memory pages); twice that on smaller tensors,
        // where a wave has few rows (8192 x 1024 9.0 us, 9.4 with half).  Backward, where each workgroup's sums are a slab of the
        // workspace, 4 waves (256 slabs) with two pieces or more (65536 x 1024 67.9 us, 70.6 with 512), 12 (768) with one (96 channels
        // 71.9, with 256 116).  Rows that leave many lanes idle have little under way all the same: at 77 channels 10 of 16 lanes hold a
        // piece, 15 KB a compute unit for a row of dy and x each (304 channels: 19 KB, and 5.1 TB/s for 3.4).
        most = bwd ? (q.v == 1 ? 3 : 1) * CUS : (q.v == 1 ? 8 : 4) * CUS / (large ? 2 : 1);
    } else {
        // As few waves a row as its registers allow, since they wait for each other at two barriers (one, backward): up to four
        // pieces a lane (fp16 8192 x 4096 27.6 us with 2 waves, 29.8 with 4, 48.6 with 8), two in the backward pass, which holds
        // the sums of its channels too (44.0 us with 4 waves, 51.9 with 8, 55.0 with 2).  8 waves a compute unit; with one piece a
        // lane and many rows 12 (20971 x 1600 44.7 us, 51.2 with 8; 2048 x 2048 17.7 with 12, 13.9 with 8).
        q.waves = std::min(8, bwd ? std::max(4, pow2_from((q.pieces + 127) / 128)) : pow2_from((q.pieces + 255) / 256));
        q.v = (q.pieces + 64 * q.waves - 1) / (64 * q.waves);
        most = (bwd && q.v == 1 && n >= 16384 ? 12 : 8) * CUS / q.waves;
    }
    const int64_t per = q.lanes ? 64 * LN_WAVES / q.lanes : 1, want = (n + per - 1) / per;
    // One workgroup's sums are the result: where dgamma and dbeta are asked for, a few rows go through it in turns, without the second
    // launch.  (Each call behind another in a graph.)  Four turns of teams: 64 x 256 fp16 5.9 us, 6.3 with four workgroups, joined 7.8
    // and 6.9; two turns 4.9 and 6.6 (8 x 1024), joined 6.0 and 7.3.  Two rows that a workgroup has to itself: 2 x 2048 3.5 and 5.1, 2 x
    // 16384 8.6 and 11.8, joined 12.6 and 14.5; with four of them it does not pay (4 x 16384 13.0 and 12.0, joined 20.8 and 14.7).
    if (params && want <= (q.lanes ? 4 : 2)) most = 1;
    q.grid = (int)std::max<int64_t>(1, std::min(want, most));
    q.trips = (want + q.grid - 1) / q.grid;
    return q;
}

static int ln_long_slabs(int64_t n) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + 63) / 64, 512)); }

int layer_norm_slabs(int64_t n, int C)
{
    const int half = ln_long<F16>(C) ? ln_long_slabs(n) : ln_shape<F16>(n, C, true, true).grid;
    const int whole = ln_long<F32>(C) ? ln_long_slabs(n) : ln_shape<F32>(n, C, true, true).grid;
    return std::max(half, whole);
}

template <class T, int VEC, int V, bool WIDE, bool FULL>
static void ln_launch(const LayerNormArgs &a, const LnShape &q, bool bwd, hipStream_t stream)
{
    const dim3 grid((unsigned)q.grid), block((unsigned)q.waves * 64);
    const size_t lds = (WIDE ? 64 : a.dgamma ? (size_t)LN_WAVES * 2 * V * q.lanes * VEC : 1) * sizeof(float);
    const auto go = [&](auto mode, auto odd) {
        constexpr int MODE = decltype(mode)::value;
        constexpr bool ODD = decltype(odd)::value;
        if (bwd) DLK_LAUNCH("layer_norm_bwd_kernel", (layer_norm_bwd_kernel<T, VEC, V, MODE, ODD, WIDE, FULL>), grid, block, lds, stream, a, q);
        else if constexpr (!WIDE || V > 2) DLK_LAUNCH("layer_norm_fwd_kernel", (layer_norm_fwd_kernel<T, VEC, V, MODE, ODD, WIDE, FULL>), grid, block, 0, stream, a, q);
    };
    const auto mode = [&](auto odd) {
        if (!a.joined) go(std::integral_constant<int, 0>{}, odd);
        else if (!(bwd ? a.ds : a.residual)) go(std::integral_constant<int, 1>{}, odd);
        else go(std::integral_constant<int, 2>{}, odd);
    };
    if constexpr (VEC > 1)
        if (a.C % VEC != 0) return mode(std::true_type{});
    mode(std::false_type{});
}

// (One piece a lane never fills a wave's 64 lanes: two with half of them leave as few idle.  Rows of several waves have three or four
// pieces a lane in the forward pass.)
template <class T>
static hipError_t ln_resident(const LayerNormArgs &a, const LnShape &q, bool bwd, hipStream_t stream)
{
    constexpr int E = Row<T>::E;
    if (a.C < E) ln_launch<T, 1, 1, false, false>(a, q, bwd, stream);
    else if (q.lanes == 64 && q.v == 2) ln_launch<T, E, 2, false, true>(a, q, bwd, stream);
    else if (q.lanes == 64) ln_launch<T, E, 3, false, true>(a, q, bwd, stream);
    else if (q.lanes && q.v == 1) ln_launch<T, E, 1, false, false>(a, q, bwd, stream);
    else if (q.lanes && q.v == 2) ln_launch<T, E, 2, false, false>(a, q, bwd, stream);
    else if (q.lanes) ln_launch<T, E, 3, false, false>(a, q, bwd, stream);
    else if (q.v == 1) ln_launch<T, E, 1, true, false>(a, q, bwd, stream);
    else if (q.v == 2) ln_launch<T, E, 2, true, false>(a, q, bwd, stream);
    else if (q.v == 3) ln_launch<T, E, 3, true, false>(a, q, bwd, stream);
    else ln_launch<T, E, 4, true, false>(a, q, bwd, stream);
    return launch_status();
}

template <class T>
static hipError_t launch_ln_fwd(const LayerNormArgs &a, hipStream_t stream)
{
    if (!ln_long<T>(a.C)) return ln_resident<T>(a, ln_shape<T>(a.n, a.C, false, false), false, stream);
    const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20)), block(LN_THREADS);
    if (a.joined) DLK_LAUNCH("layer_norm_long_fwd_kernel", (layer_norm_long_fwd_kernel<T, true>), grid, block, 0, stream, a);
    else DLK_LAUNCH("layer_norm_long_fwd_kernel", (layer_norm_long_fwd_kernel<T, false>), grid, block, 0, stream, a);
    return launch_status();
}

hipError_t launch_layer_norm_fwd(const LayerNormArgs &a, int dtype, hipStream_t stream)
{
    if (a.n <= 0) return hipSuccess;
    return dtype == 0 ? launch_ln_fwd<F16>(a, stream) : dtype == 1 ? launch_ln_fwd<BF16>(a, stream) : launch_ln_fwd<F32>(a, stream);
}

static hipError_t ln_param_sum(const LayerNormArgs &a, int slabs, hipStream_t stream)
{
    const dim3 grid((unsigned)((2 * (int64_t)a.C + 15) / 16)), block(1024);
    static_assert(3 * CUS <= 64 * 12, "the longest list of slabs");
    if (slabs <= 256) DLK_LAUNCH("layer_norm_param_sum_kernel", layer_norm_param_sum_kernel<4>, grid, block, 0, stream, a.partial, slabs, a.C, a.dgamma, a.dbeta);
    else DLK_LAUNCH("layer_norm_param_sum_kernel", layer_norm_param_sum_kernel<12>, grid, block, 0, stream, a.partial, slabs, a.C, a.dgamma, a.dbeta);
    return launch_status();
}

template <class T>
static hipError_t launch_ln_bwd(const LayerNormArgs &a0, hipStream_t stream)
{
    LayerNormArgs a = a0;
    const dim3 block(LN_THREADS);
    hipError_t e;
    if (a.n > 0 && !ln_long<T>(a.C)) {
        const LnShape q = ln_shape<T>(a.n, a.C, true, a.dgamma);
        e = ln_resident<T>(a, q, true, stream);
        return e != hipSuccess || !a.dgamma || q.grid == 1 ? e : ln_param_sum(a, q.grid, stream);
    }
    if (a.dgamma) {                                     // before dx, which may lie where dy does
        const int slabs = ln_long_slabs(a.n);
        a.chunk = (a.n + slabs - 1) / slabs;
        const dim3 cols((unsigned)slabs, (unsigned)((a.C + 63) / 64));
        DLK_LAUNCH("layer_norm_param_kernel", layer_norm_param_kernel<T>, cols, block, 0, stream, a);
        e = launch_status();
        if (e == hipSuccess) e = ln_param_sum(a, slabs, stream);
        if (e != hipSuccess) return e;
    }
    if (a.n <= 0) return hipSuccess;
    const dim3 grid((unsigned)std::min<int64_t>(a.n, 1 << 20));
    if (a.joined) DLK_LAUNCH("layer_norm_long_bwd_kernel", (layer_norm_long_bwd_kernel<T, true>), grid, block, 0, stream, a);
    else DLK_LAUNCH("layer_norm_long_bwd_kernel", (layer_norm_long_bwd_kernel<T, false>), grid, block, 0, stream, a);
    return launch_status();
}

hipError_t launch_layer_norm_bwd(const LayerNormArgs &a, int dtype, hipStream_t stream)
{
    return dtype == 0 ? launch_ln_bwd<F16>(a, stream) : dtype == 1 ? launch_ln_bwd<BF16>(a, stream) : launch_ln_bwd<F32>(a, stream);
}

}  // namespace dlk
