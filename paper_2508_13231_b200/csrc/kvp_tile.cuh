// Layout of the cache held in 4 bits (see "A cache held in 4 bits" in include/kvp.h): a page of one kv-head is page_tokens / 16
// tiles, a tile holds 16 tokens, and inside it keys and values lie in the order in which a warp's matrix fragments take them,
// so that attention reads them with 16-byte loads and no shuffle.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kvp_common.cuh"

namespace kvp {

constexpr uint32_t kTileTokens = 16;

// All offsets in bytes from the start of a tile; N = head_dim / 32 groups.
template <int N>
struct Tile {
    static constexpr uint32_t D = 32 * N;
    static constexpr uint32_t kKeys = 0;                       // [16 tokens][4][N] words of 8 dims
    static constexpr uint32_t kValues = 8 * D;                 // [2][8][4][N][2] half-words of 4 dims
    static constexpr uint32_t kKeyScale = 16 * D;              // [16 tokens][N] fp16
    static constexpr uint32_t kKeyZero = kKeyScale + 32 * N;
    static constexpr uint32_t kValueScale = kKeyZero + 32 * N; // [4][N][4 tokens] fp16
    static constexpr uint32_t kValueZero = kValueScale + 32 * N;
    static constexpr uint32_t kBytes = kValueZero + 32 * N;    // 20 * D

    // word of dims 32 n + 8 t .. + 7 of token i's key; dim 32 n + 8 t + m in bits 4m .. 4m+3
    static __host__ __device__ constexpr uint32_t key_word(uint32_t i, uint32_t t, uint32_t n) { return kKeys + ((i * 4 + t) * N + n) * 4; }
    // half-word of dims 32 n + 4 g .. + 3 of token i's value
    static __host__ __device__ constexpr uint32_t value_half(uint32_t i, uint32_t g, uint32_t n)
    {
        return kValues + ((((((i >> 1) & 1) * 8 + g) * 4 + (i >> 2)) * N + n) * 2 + (i & 1)) * 2;
    }
    static __host__ __device__ constexpr uint32_t key_meta(uint32_t i, uint32_t n) { return kKeyScale + (i * N + n) * 2; }
    static __host__ __device__ constexpr uint32_t value_meta(uint32_t i, uint32_t n) { return kValueScale + (((i >> 2) * N + n) * 4 + (i & 3)) * 2; }
};

inline bool head_dim_served(uint32_t d) { return d == 64 || d == 128 || d == 256; }

}  // namespace kvp
