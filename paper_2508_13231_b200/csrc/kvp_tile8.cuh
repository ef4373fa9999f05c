// Layout of the cache held in 8 bits (see "A cache held in 8 bits" in include/kvp.h): a page of one kv-head is page_tokens / 16
// blocks, a block holds 16 tokens as the matrix unit takes them: keys with the dims contiguous in cores of 8 tokens x 16 dims, values
// with the tokens contiguous, a core of 8 dims x 16 tokens after the other. Attention copies both to shared memory as they are.
#pragma once

#include "kvp_tile.cuh"

namespace kvp {

// All offsets in bytes from the start of a block.
template <int D>
struct Tile8 {
    static constexpr uint32_t kKeys = 0;
    static constexpr uint32_t kKeyBytes = 16 * D;
    static constexpr uint32_t kValues = 16 * D;
    static constexpr uint32_t kScale = 32 * D;                 // of the keys, and of the values 4 bytes on
    static constexpr uint32_t kValueBytes = 16 * D + 16;       // values and scales
    static constexpr uint32_t kBytes = 32 * D + 16;
    // dims 16 c .. 16 c + 15 of token i's key
    static __host__ __device__ constexpr uint32_t key(uint32_t i, uint32_t c) { return ((i / 8) * (D / 16) + c) * 128 + i % 8 * 16; }
    // dim d of all 16 tokens
    static __host__ __device__ constexpr uint32_t value(uint32_t d) { return kValues + d * 16; }
};

// two fp32 numbers to e4m3, to the nearest, ties to even, cut to 448; `lo` in the low byte
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 floats_of_e4m3(uint32_t pair)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)pair));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

}  // namespace kvp
