// Writing and reading the cache held in 4 bits.
//
// A group of 32 dims of one token and head is kept as zero + scale * q: zero = fp16(min), scale = fp16((max - zero) / 15),
// q = the nearest whole number to (x - zero) / scale, 0..15, ties to even. Every operation is one fp32 operation, rounded as
// IEEE 754 asks, so that a plain program gives the same bits. Two roundings to 16 bits are part of the form: zero moves the
// whole group by at most 2^-11 of |min| (a half-step is 1/30 of the range), scale is off by at most 2^-11 of itself (fp16 rather than
// bf16 because the steps' error is 15 times the scale's, and the range of keys and values of a model fits fp16).
#include <cuda_bf16.h>

#include "kvp_tile.cuh"

namespace kvp {

namespace {

struct RowsK {
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;     // strides in elements
    const int64_t* slots;
    uint8_t* cache;
    uint64_t slots_in_cache;                      // pages * page_tokens
    uint32_t tokens, heads, page_tokens;
};

constexpr float kMost = 65504.0f;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// eight neighbouring elements; `aligned`: at a 16-byte boundary
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool aligned, float (&x)[8])
{
    if (aligned) {
        alignas(16) T e[8];
#pragma unroll
        for (uint32_t i = 0; i < sizeof(e) / 16; ++i) reinterpret_cast<uint4*>(e)[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_float(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_float(p[i]);
    }
}

// the tile of a slot, for one head; slot < slots_in_cache
template <int N>
__device__ __forceinline__ uint64_t tile_at(uint64_t slot, uint32_t head, uint32_t heads, uint32_t page_tokens)
{
    const uint64_t page = slot / page_tokens;
    const uint32_t in_page = (uint32_t)(slot - page * page_tokens);
    return ((page * heads + head) * (page_tokens / kTileTokens) + in_page / kTileTokens) * Tile<N>::kBytes;
}

// A thread quantises eight dims; the four threads of a group of 32 dims are neighbours. D / 4 threads serve a (token, head): the
// first half of them its key, the rest its value.
template <int N, typename T>
__global__ void __launch_bounds__(256) append_kernel(const RowsK p, bool aligned)
{
    using L = Tile<N>;
    constexpr uint32_t kPer = 4 * N;                                   // threads of a key or of a value
    const uint64_t at = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const uint64_t row = at / (2 * kPer);
    const uint32_t j = (uint32_t)(at % kPer), n = j / 4, t = j % 4;
    const bool is_value = (at / kPer) & 1;
    const bool in = row < (uint64_t)p.tokens * p.heads;
    const uint32_t token = (uint32_t)(in ? row / p.heads : 0), head = (uint32_t)(in ? row % p.heads : 0);
    float x[8];
    const T* from = is_value ? static_cast<const T*>(p.v) + token * p.v_token + head * p.v_head
                             : static_cast<const T*>(p.k) + token * p.k_token + head * p.k_head;
    load8(from + 8 * j, aligned, x);
    float low = INFINITY, high = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = x[i] != x[i] ? 0.0f : __fadd_rn(fminf(fmaxf(x[i], -kMost), kMost), 0.0f);     // -0 becomes 0
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
        high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, o));
    }
    const __half zero = __float2half_rn(low);
    const float z = __half2float(zero);
    const __half scale = __float2half_rn(fmaxf(__fdiv_rn(__fsub_rn(high, z), 15.0f), 0.0f));
    const float s = __half2float(scale);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = s > 0.0f ? rintf(__fdiv_rn(__fsub_rn(x[i], z), s)) : 0.0f;
        word |= (uint32_t)fminf(fmaxf(q, 0.0f), 15.0f) << (4 * i);
    }
    const int64_t slot = in ? __ldg(p.slots + token) : -1;
    if (slot < 0 || (uint64_t)slot >= p.slots_in_cache) return;
    uint8_t* tile = p.cache + tile_at<N>((uint64_t)slot, head, p.heads, p.page_tokens);
    const uint32_t i = (uint32_t)((uint64_t)slot % kTileTokens);
    if (is_value) {
        *reinterpret_cast<uint16_t*>(tile + L::value_half(i, 2 * t, n)) = (uint16_t)word;
        *reinterpret_cast<uint16_t*>(tile + L::value_half(i, 2 * t + 1, n)) = (uint16_t)(word >> 16);
    } else {
        *reinterpret_cast<uint32_t*>(tile + L::key_word(i, t, n)) = word;
    }
    if (t == 0) {
        __half* meta = reinterpret_cast<__half*>(tile + (is_value ? L::value_meta(i, n) : L::key_meta(i, n)));
        meta[0] = scale;
        meta[(L::kKeyZero - L::kKeyScale) / 2] = zero;
    }
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// The inverse: a thread gives eight dims back. Outputs are [tokens][heads][D]; a token of a slot outside the cache reads as 0.
template <int N, typename T>
__global__ void __launch_bounds__(256) read_kernel(const RowsK p, T* __restrict__ k, T* __restrict__ v)
{
    using L = Tile<N>;
    constexpr uint32_t kPer = 4 * N;
    const uint64_t at = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const uint64_t row = at / (2 * kPer);
    if (row >= (uint64_t)p.tokens * p.heads) return;
    const uint32_t j = (uint32_t)(at % kPer), n = j / 4, t = j % 4;
    const bool is_value = (at / kPer) & 1;
    const uint32_t token = (uint32_t)(row / p.heads), head = (uint32_t)(row % p.heads);
    const int64_t slot = __ldg(p.slots + token);
    uint32_t word = 0;
    float s = 0.0f, z = 0.0f;
    if (slot >= 0 && (uint64_t)slot < p.slots_in_cache) {
        const uint8_t* tile = p.cache + tile_at<N>((uint64_t)slot, head, p.heads, p.page_tokens);
        const uint32_t i = (uint32_t)((uint64_t)slot % kTileTokens);
        word = is_value ? (uint32_t)*reinterpret_cast<const uint16_t*>(tile + L::value_half(i, 2 * t, n)) |
                              (uint32_t)*reinterpret_cast<const uint16_t*>(tile + L::value_half(i, 2 * t + 1, n)) << 16
                        : *reinterpret_cast<const uint32_t*>(tile + L::key_word(i, t, n));
        const __half* meta = reinterpret_cast<const __half*>(tile + (is_value ? L::value_meta(i, n) : L::key_meta(i, n)));
        s = __half2float(meta[0]);
        z = __half2float(meta[(L::kKeyZero - L::kKeyScale) / 2]);
    }
    alignas(16) T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) put(e + i, __fadd_rn(__fmul_rn((float)((word >> (4 * i)) & 15u), s), z));
    uint4* to = reinterpret_cast<uint4*>((is_value ? v : k) + row * L::D + 8 * j);
#pragma unroll
    for (uint32_t i = 0; i < sizeof(e) / 16; ++i) to[i] = reinterpret_cast<const uint4*>(e)[i];
}

template <int N, typename T>
int launch_append(const RowsK& p, bool aligned, cudaStream_t st)
{
    const uint64_t threads = (uint64_t)p.tokens * p.heads * 8 * N, grid = (threads + 255) / 256;
    append_kernel<N, T><<<(uint32_t)grid, 256, 0, st>>>(p, aligned);
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

template <int N, typename T>
int launch_read(const RowsK& p, void* k, void* v, cudaStream_t st)
{
    const uint64_t threads = (uint64_t)p.tokens * p.heads * 8 * N, grid = (threads + 255) / 256;
    read_kernel<N, T><<<(uint32_t)grid, 256, 0, st>>>(p, static_cast<T*>(k), static_cast<T*>(v));
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

int check_rows(const kvp_cache_shape* c, const void* cache, uint32_t tokens, const void* a, const void* b, const int64_t* slots, uint32_t dtype)
{
    if (!c || c->reserved || !c->pages || !c->kv_heads || dtype > KVP_F32) return KVP_ERR_ARG;
    if (!c->page_tokens || c->page_tokens % kTileTokens) return KVP_ERR_ARG;
    if (!head_dim_served(c->head_dim)) return KVP_ERR_RANGE;
    if (tokens && (!cache || !a || !b || !slots)) return KVP_ERR_ARG;
    if ((uint64_t)tokens * c->kv_heads * (c->head_dim / 4) >= (1ull << 31) * 256) return KVP_ERR_RANGE;
    return KVP_OK;
}

#define KVP_BY_SHAPE(CALL)                                                                     \
    switch (c->head_dim * 4 + dtype) {                                                         \
        case 64 * 4 + KVP_BF16: return CALL(2, __nv_bfloat16);                                 \
        case 64 * 4 + KVP_F16: return CALL(2, __half);                                         \
        case 64 * 4 + KVP_F32: return CALL(2, float);                                          \
        case 128 * 4 + KVP_BF16: return CALL(4, __nv_bfloat16);                                \
        case 128 * 4 + KVP_F16: return CALL(4, __half);                                        \
        case 128 * 4 + KVP_F32: return CALL(4, float);                                         \
        case 256 * 4 + KVP_BF16: return CALL(8, __nv_bfloat16);                                \
        case 256 * 4 + KVP_F16: return CALL(8, __half);                                        \
        case 256 * 4 + KVP_F32: return CALL(8, float);                                         \
        default: return KVP_ERR_RANGE;                                                         \
    }

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" uint64_t kvp_cache_page_bytes(uint32_t head_dim, uint32_t page_tokens)
{
    if (!head_dim_served(head_dim) || page_tokens % kTileTokens) return 0;
    return (uint64_t)page_tokens / kTileTokens * 20 * head_dim;
}

extern "C" int kvp_cache_append(const kvp_cache_shape* c, void* cache, uint32_t dtype, uint32_t tokens, const void* k,
                                int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                                int64_t v_head_stride, const int64_t* slots, void* stream)
{
    const int rc = check_rows(c, cache, tokens, k, v, slots, dtype);
    if (rc || !tokens) return rc;
    RowsK p;
    p.k = k; p.v = v;
    p.k_token = k_token_stride; p.k_head = k_head_stride; p.v_token = v_token_stride; p.v_head = v_head_stride;
    p.slots = slots; p.cache = static_cast<uint8_t*>(cache);
    p.slots_in_cache = (uint64_t)c->pages * c->page_tokens;
    p.tokens = tokens; p.heads = c->kv_heads; p.page_tokens = c->page_tokens;
    const uint64_t e = dtype == KVP_F32 ? 4 : 2;
    const uint64_t low = (uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)v | (uint64_t)k_token_stride * e | (uint64_t)k_head_stride * e |
                         (uint64_t)v_token_stride * e | (uint64_t)v_head_stride * e;
    const bool aligned = low % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define KVP_APPEND(N, T) launch_append<N, T>(p, aligned, st)
    KVP_BY_SHAPE(KVP_APPEND)
#undef KVP_APPEND
}

extern "C" int kvp_cache_read(const kvp_cache_shape* c, const void* cache, uint32_t dtype, uint32_t tokens, const int64_t* slots,
                              void* k, void* v, void* stream)
{
    const int rc = check_rows(c, cache, tokens, k, v, slots, dtype);
    if (rc || !tokens) return rc;
    RowsK p = {};
    p.slots = slots; p.cache = static_cast<uint8_t*>(const_cast<void*>(cache));
    p.slots_in_cache = (uint64_t)c->pages * c->page_tokens;
    p.tokens = tokens; p.heads = c->kv_heads; p.page_tokens = c->page_tokens;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define KVP_READ(N, T) launch_read<N, T>(p, k, v, st)
    KVP_BY_SHAPE(KVP_READ)
#undef KVP_READ
}
