// What the [pixels][channels] kernels (layer norm, dropout) share: 16-byte pieces of a row in the three storage types, and
// the counter-based generator.
#pragma once
#include "device_common.h"
#include "kernels.h"

namespace dlk {

// fp32 storage beside F16 and BF16.
struct F32 {};

typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element's address
typedef float floatx4_any_t __attribute__((ext_vector_type(4), aligned(4)));

// The fp32 result of a kernel before it is rounded to the storage type.  The compiler may otherwise fuse a multiply-add with its
// rounding to fp16 (v_fma_mixlo_f16, which rounds once) in one kernel and not in the next, and the two then differ in the last bit
// where fp32's rounding falls on a border between two fp16 numbers.
__device__ __forceinline__ float settled(float v)
{
    asm("" : "+v"(v));
    return v;
}

template <class T> struct Row {                        // 16-bit storage
    using elem = uint16_t;
    static constexpr int E = 8;                        // elements of a 16-byte piece
    struct elems { elem v[E]; };
    static __device__ __forceinline__ float get(elem v) { return T::to_float(v); }
    static __device__ __forceinline__ elem put(float v) { return T::from_float(settled(v)); }
    static __device__ __forceinline__ void unpack(u32x4_t w, float (&v)[E])
    {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            v[2 * d] = T::to_float((uint16_t)(w[d] & 0xffffu));
            v[2 * d + 1] = T::to_float((uint16_t)(w[d] >> 16));
        }
    }
    static __device__ __forceinline__ u32x4_t pack(const float (&v)[E])
    {
        u32x4_t w;
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] = T::pack2(settled(v[2 * d]), settled(v[2 * d + 1]));
        return w;
    }
};
template <> struct Row<F32> {
    using elem = float;
    static constexpr int E = 4;
    struct elems { elem v[E]; };
    static __device__ __forceinline__ float get(elem v) { return v; }
    static __device__ __forceinline__ elem put(float v) { return v; }
    static __device__ __forceinline__ void unpack(u32x4_t w, float (&v)[E])
    {
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t u = w[d];                   // (a bit cast of a vector's element would take element 0)
            v[d] = __builtin_bit_cast(float, u);
        }
    }
    static __device__ __forceinline__ u32x4_t pack(const float (&v)[E])
    {
        return u32x4_t{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                       __builtin_bit_cast(uint32_t, v[3])};
    }
};

// The generator: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), ten
// rounds of two 32 x 32 -> 64 bit products on a 128-bit counter.  Nothing is kept between calls, so any element's number can
// be had again in the backward pass without storing a mask.  Block g of a call covers the elements 8g .. 8g+7, 16 bits each:
// one block per 16-byte piece of a 16-bit tensor.  (32 bits an element would double the products, which are a quarter as
// fast as other integer instructions, and the streaming kernels would then wait for them instead of for memory.)
struct Philox {
    uint32_t k0, k1, o0, o1;                           // key and upper half of the counter, the same in every lane
    __device__ __forceinline__ explicit Philox(const DropArgs &d)
    {
        const uint64_t o = d.offset + (d.step ? *d.step : 0);
        k0 = d.k0; k1 = d.k1; o0 = (uint32_t)o; o1 = (uint32_t)(o >> 32);
    }
    __device__ __forceinline__ u32x4_t operator()(uint64_t block) const
    {
        uint32_t a = (uint32_t)block, b = (uint32_t)(block >> 32), c = o0, d = o1, ka = k0, kb = k1;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
            a = (uint32_t)(q >> 32) ^ b ^ ka;
            b = (uint32_t)q;
            c = (uint32_t)(p >> 32) ^ d ^ kb;
            d = (uint32_t)p;
            ka += 0x9E3779B9u;
            kb += 0xBB67AE85u;
        }
        return u32x4_t{a, b, c, d};
    }
};
// The 16 bits of element e of a block.
__device__ __forceinline__ uint32_t philox_field(u32x4_t w, int e) { return (w[e >> 1] >> (16 * (e & 1))) & 0xffffu; }

// The 16-bit numbers of E consecutive elements from element `first` on, two to a word, lowest first.  AT: first is a multiple of E,
// so that a piece lies within one block; otherwise it may end in the next one.
template <int E, bool AT>
__device__ __forceinline__ void drop_words(const Philox &rng, uint64_t first, uint32_t (&w)[(E + 1) / 2])
{
    const u32x4_t lo = rng(first >> 3);
    if constexpr (E == 1) {
        w[0] = philox_field(lo, 0);
        const int f = (int)(first & 7);
#pragma unroll
        for (int e = 1; e < 8; ++e)
            if (f == e) w[0] = philox_field(lo, e);
    } else if constexpr (AT && E == 8) {
#pragma unroll
        for (int d = 0; d < 4; ++d) w[d] = lo[d];
    } else if constexpr (AT) {
        const bool upper = first & 4;
        w[0] = upper ? lo[2] : lo[0];
        w[1] = upper ? lo[3] : lo[1];
    } else {
        const u32x4_t hi = rng((first >> 3) + 1);
        const int f = (int)(first & 7);
        uint32_t s[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        const uint32_t four = f & 4 ? ~0u : 0u, two = f & 2 ? ~0u : 0u;     // (masks: a choice between elements becomes one of addresses)
#pragma unroll
        for (int d = 0; d < E / 2 + 2; ++d) s[d] = (s[d + 2] & four) | (s[d] & ~four);
#pragma unroll
        for (int d = 0; d < E / 2 + 1; ++d) s[d] = (s[d + 1] & two) | (s[d] & ~two);
        const uint32_t by = 16 * (f & 1);
#pragma unroll
        for (int d = 0; d < E / 2; ++d) w[d] = __builtin_amdgcn_alignbit(s[d + 1], s[d], by);
    }
}
// v[e] = 0 where the number of element e is below t; limit = (t << 16) - 1.  (An upper half is compared with its word's lower
// half below it, which cannot carry it over the border.)
template <int E>
__device__ __forceinline__ void drop_select(const uint32_t (&w)[(E + 1) / 2], uint32_t limit, float (&v)[E])
{
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (e & 1 ? w[e >> 1] : w[e >> 1] << 16) > limit ? v[e] : 0.f;
}

// A piece at p: VEC elements.  ANY: p is aligned to an element only.
template <class T, int VEC, bool ANY> struct Piece {
    using elem = typename Row<T>::elem;
    using raw = u32x4_t;
    static __device__ __forceinline__ raw load(const elem *p)
    {
        if constexpr (ANY) return *reinterpret_cast<const u32x4_any_t *>(p);
        else return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
    }
    template <bool PAST> static __device__ __forceinline__ void store(elem *p, raw v)      // PAST: past the caches
    {
        if constexpr (ANY) *reinterpret_cast<u32x4_any_t *>(p) = v;
        else if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(p));
        else *reinterpret_cast<u32x4_t *>(p) = v;
    }
    static __device__ __forceinline__ void unpack(raw w, float (&v)[VEC]) { Row<T>::unpack(w, v); }
    static __device__ __forceinline__ raw pack(const float (&v)[VEC]) { return Row<T>::pack(v); }
};
template <class T, bool ANY> struct Piece<T, 1, ANY> {
    using elem = typename Row<T>::elem;
    using raw = elem;
    static __device__ __forceinline__ raw load(const elem *p) { return *p; }
    template <bool PAST> static __device__ __forceinline__ void store(elem *p, raw v) { *p = v; }
    static __device__ __forceinline__ void unpack(raw w, float (&v)[1]) { v[0] = Row<T>::get(w); }
    static __device__ __forceinline__ raw pack(const float (&v)[1]) { return Row<T>::put(v[0]); }
};

// Sums over a team of `lanes` (a power of two) neighbouring lanes of a wave; every lane of the team gets the same bits, since each
// step adds two numbers that its two halves have both of.  The steps within 16 lanes are lane permutations of the addition itself.
template <int CTRL> __device__ __forceinline__ float dpp_add(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float swap16_add(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float swap32_add(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
#define DLK_STEP(cond, step)                                                 \
    if (cond) {                                                              \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = step(v[i]);     \
    }
template <int N> __device__ __forceinline__ void team_sums(float (&v)[N], int lanes)
{
    DLK_STEP(lanes > 1, dpp_add<0xB1>)                  // quad_perm 1 0 3 2
    DLK_STEP(lanes > 2, dpp_add<0x4E>)                  // quad_perm 2 3 0 1
    DLK_STEP(lanes > 4, dpp_add<0x141>)                 // row_half_mirror
    DLK_STEP(lanes > 8, dpp_add<0x140>)                 // row_mirror
    DLK_STEP(lanes > 16, swap16_add)
    DLK_STEP(lanes > 32, swap32_add)
}
// Sums over the lanes of the wave that hold the same place in their teams: the first team gets them.
template <int N> __device__ __forceinline__ void cross_sums(float (&v)[N], int lanes)
{
    DLK_STEP(lanes <= 32, swap32_add)
    DLK_STEP(lanes <= 16, swap16_add)
    DLK_STEP(lanes <= 8, dpp_add<0x128>)                // row_ror 8, 4, 2, 1
    DLK_STEP(lanes <= 4, dpp_add<0x124>)
    DLK_STEP(lanes <= 2, dpp_add<0x122>)
    DLK_STEP(lanes <= 1, dpp_add<0x121>)
}
#undef DLK_STEP

}  // namespace dlk
