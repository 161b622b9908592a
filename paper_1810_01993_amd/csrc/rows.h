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

template <class T> struct Row {                        // 16-bit storage: 8 elements a piece
    using elem = uint16_t;
    static constexpr int E = 8;
    static __device__ __forceinline__ float get(elem v) { return T::to_float(v); }
    static __device__ __forceinline__ elem put(float v) { return T::from_float(v); }
};
template <> struct Row<F32> {
    using elem = float;
    static constexpr int E = 4;
    static __device__ __forceinline__ float get(elem v) { return v; }
    static __device__ __forceinline__ elem put(float v) { return v; }
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

}  // namespace dlk
