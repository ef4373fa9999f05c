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
constexpr uint32_t kRowThreads = 128;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// eight neighbouring elements; `aligned`: at a 16-byte boundary
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool aligned, float* x)
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
__device__ __forceinline__ uint64_t tile_at(uint64_t slot, uint32_t head, const RowsK& p, uint32_t& token)
{
    uint64_t page;
    uint32_t in_page;
    if (p.slots_in_cache <= ~0u) {                                     // a 64-bit division takes as long as the rest of the kernel
        const uint32_t q = (uint32_t)slot / p.page_tokens;
        page = q;
        in_page = (uint32_t)slot - q * p.page_tokens;
    } else {
        page = slot / p.page_tokens;
        in_page = (uint32_t)(slot - page * p.page_tokens);
    }
    token = in_page % kTileTokens;
    return ((page * p.heads + head) * (p.page_tokens / kTileTokens) + in_page / kTileTokens) * Tile<N>::kBytes;
}

// Two neighbouring threads quantise the 32 dims of a group, 16 each: what is done once a thread counts little beside the elements' work, and there are
// threads enough for a decode step. Next to them stand the groups of the token, then the next tokens (whose values fill the same sectors of a
// tile); blockIdx.y is the head, blockIdx.z 0 for keys and 1 for values. What bounds it is instructions (26 an element, 77%
// of the issue slots), so the common way has a multiplication, three additions, a comparison and a pack for an element, and no division:
// y = fl(x inv - z inv) stands for the quotient (x - z) / s; with |z inv| = b it is off from it by less than (b + 16) 2^-21 (the
// roundings of inv, z inv and y, each 2^-24 relative, and that of x - z in the definition). Adding 1.5 * 2^23 rounds y to the nearest whole number, ties to even,
// as the definition rounds the quotient unless y lies that close to a half; the whole number is in the low bits, and a Horner scheme packs eight of
// them (the constant's bits leave by the top). A group in which some y lies near a half (2% of the groups of bf16 values:
// their grid and the scale's often meet in one), or that is to be cut, is done again with a look at each number, and a division where it takes one.
template <int N, typename T>
__global__ void __launch_bounds__(kRowThreads) append_kernel(const RowsK p, bool aligned)
{
    using L = Tile<N>;
    const uint32_t half = threadIdx.x % 2, n = threadIdx.x / 2 % N, row = blockIdx.x * (kRowThreads / (2 * N)) + threadIdx.x / (2 * N), head = blockIdx.y;
    const bool is_value = blockIdx.z, in = row < p.tokens;
    const uint32_t token = in ? row : 0;                               // both threads of a pair are in or out
    const int64_t slot = in ? __ldg(p.slots + token) : -1;
    float x[16];
    {
        const T* from = (is_value ? static_cast<const T*>(p.v) + token * p.v_token + head * p.v_head
                                  : static_cast<const T*>(p.k) + token * p.k_token + head * p.k_head) + 32 * n + 16 * half;
        load8(from, aligned, x);
        load8(from + 8, aligned, x + 8);
    }
    float low, high, odd;                                              // odd: NaN if some x is not finite
    {
        float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[0], x[1], x[2], x[3]}, c[4] = {0, 0, 0, 0};     // four short chains for one long
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            a[i % 4] = fminf(a[i % 4], x[i]);
            b[i % 4] = fmaxf(b[i % 4], x[i]);
            c[i % 4] = fmaf(x[i], 0.0f, c[i % 4]);
        }
        low = fminf(fminf(a[0], a[1]), fminf(a[2], a[3]));
        high = fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3]));
        odd = (c[0] + c[1]) + (c[2] + c[3]);
    }
    if (odd != 0.0f || low < -kMost || high > kMost) {                 // rare: NaN becomes 0, the rest is cut
        low = INFINITY;
        high = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -kMost), kMost);
            low = fminf(low, x[i]);
            high = fmaxf(high, x[i]);
        }
    }
    low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, 1));
    high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, 1));
    const __half zero = __float2half_rn(__fadd_rn(low, 0.0f));         // -0 becomes 0
    const float z = __half2float(zero);
    const __half scale = __float2half_rn(fmaxf(__fdiv_rn(__fsub_rn(high, z), 15.0f), 0.0f));
    const float s = __half2float(scale);
    uint32_t word[2] = {0, 0};
    if (s > 0.0f) {
        constexpr float kRound = 12582912.0f;
        const float inv = __frcp_rn(s), back = -z * inv, room = 0.5f - (fabsf(back) + 16.0f) * 0x1p-21f;
        float most[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 15; i >= 0; --i) {
            const float y = fmaf(x[i], inv, back), r = __fadd_rn(y, kRound);
            most[i / 8] = fmaxf(most[i / 8], fabsf(__fsub_rn(y, __fsub_rn(r, kRound))));
            word[i / 8] = word[i / 8] * 16u + (uint32_t)__float_as_int(r);
        }
        // 0x4B400000 is the whole number 0 here; of the sum of its multiples by powers of 16 only the first three stay within 32 bits
        constexpr uint32_t kZero = 0x4B400000u + 0x4B400000u * 16u + 0x4B400000u * 256u;
        word[0] -= kZero;
        word[1] -= kZero;
        if (!(fmaxf(most[0], most[1]) < room && fmaf(low, inv, back) > -0.25f && fmaf(high, inv, back) < 15.25f)) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                word[w] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = fmaf(x[8 * w + i], inv, back);
                    float r = rintf(y);
                    if (!(fabsf(y - r) < room)) r = rintf(__fdiv_rn(__fsub_rn(x[8 * w + i], z), s));
                    word[w] |= (uint32_t)fminf(fmaxf(r, 0.0f), 15.0f) << (4 * i);
                }
            }
        }
    }
    if (slot < 0 || (uint64_t)slot >= p.slots_in_cache) return;
    uint32_t i;
    uint8_t* tile = p.cache + tile_at<N>((uint64_t)slot, head, p, i);
    if (is_value) {
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g) *reinterpret_cast<uint16_t*>(tile + L::value_half(i, 4 * half + g, n)) = (uint16_t)(word[g / 2] >> (16 * (g & 1)));
    } else {
        *reinterpret_cast<uint32_t*>(tile + L::key_word(i, 2 * half, n)) = word[0];
        *reinterpret_cast<uint32_t*>(tile + L::key_word(i, 2 * half + 1, n)) = word[1];
    }
    __half* meta = reinterpret_cast<__half*>(tile + (is_value ? L::value_meta(i, n) : L::key_meta(i, n)));
    if (half) meta[(L::kKeyZero - L::kKeyScale) / 2] = zero;
    else meta[0] = scale;
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// The inverse, by the same threads. Outputs are [tokens][heads][D]; a token of a slot outside the cache reads as 0.
template <int N, typename T>
__global__ void __launch_bounds__(kRowThreads) read_kernel(const RowsK p, T* __restrict__ k, T* __restrict__ v)
{
    using L = Tile<N>;
    const uint32_t half = threadIdx.x % 2, n = threadIdx.x / 2 % N, row = blockIdx.x * (kRowThreads / (2 * N)) + threadIdx.x / (2 * N), head = blockIdx.y;
    const bool is_value = blockIdx.z, in = row < p.tokens;
    const int64_t slot = in ? __ldg(p.slots + row) : -1;
    uint32_t word[2] = {0, 0};
    float s = 0.0f, z = 0.0f;
    if (slot >= 0 && (uint64_t)slot < p.slots_in_cache) {
        uint32_t i;
        const uint8_t* tile = p.cache + tile_at<N>((uint64_t)slot, head, p, i);
#pragma unroll
        for (uint32_t t = 0; t < 2; ++t)
            word[t] = is_value ? (uint32_t)*reinterpret_cast<const uint16_t*>(tile + L::value_half(i, 4 * half + 2 * t, n)) |
                                     (uint32_t)*reinterpret_cast<const uint16_t*>(tile + L::value_half(i, 4 * half + 2 * t + 1, n)) << 16
                               : *reinterpret_cast<const uint32_t*>(tile + L::key_word(i, 2 * half + t, n));
        const __half* meta = reinterpret_cast<const __half*>(tile + (is_value ? L::value_meta(i, n) : L::key_meta(i, n)));
        s = __half2float(meta[0]);
        z = __half2float(meta[(L::kKeyZero - L::kKeyScale) / 2]);
    }
    constexpr int kPieces = 16 * sizeof(T) / 16;
    uint4 piece[kPieces];
    T* e = reinterpret_cast<T*>(piece);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float q = __uint_as_float(0x4B000000u | (word[i / 8] >> (4 * (i % 8)) & 15u)) - 8388608.0f;    // 2^23 + q, without a conversion
        put(e + i, __fadd_rn(__fmul_rn(q, s), z));
    }
    uint4* to = reinterpret_cast<uint4*>((is_value ? v : k) + ((uint64_t)row * p.heads + head) * L::D + 32 * n);
    if (kPieces == 2) {
        // the pair's four pieces lie side by side: the threads exchange two, so that a store fills whole sectors
        uint4 give = half ? piece[0] : piece[1], got;
        got.x = __shfl_xor_sync(0xFFFFFFFFu, give.x, 1);
        got.y = __shfl_xor_sync(0xFFFFFFFFu, give.y, 1);
        got.z = __shfl_xor_sync(0xFFFFFFFFu, give.z, 1);
        got.w = __shfl_xor_sync(0xFFFFFFFFu, give.w, 1);
        if (in) {
            to[half] = half ? got : piece[0];
            to[2 + half] = half ? piece[1] : got;
        }
    } else if (in) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) to[half * kPieces + i] = piece[i];
    }
}

template <int N, typename T>
int launch_append(const RowsK& p, bool aligned, cudaStream_t st)
{
    constexpr uint32_t kTokens = kRowThreads / (2 * N);
    append_kernel<N, T><<<dim3((p.tokens + kTokens - 1) / kTokens, p.heads, 2), kRowThreads, 0, st>>>(p, aligned);
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

template <int N, typename T>
int launch_read(const RowsK& p, void* k, void* v, cudaStream_t st)
{
    constexpr uint32_t kTokens = kRowThreads / (2 * N);
    read_kernel<N, T><<<dim3((p.tokens + kTokens - 1) / kTokens, p.heads, 2), kRowThreads, 0, st>>>(p, static_cast<T*>(k), static_cast<T*>(v));
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

int check_rows(const kvp_cache_shape* c, const void* cache, uint32_t tokens, const void* a, const void* b, uint32_t rows_align, const int64_t* slots, uint32_t dtype)
{
    if (!c || c->reserved || !c->pages || !c->kv_heads || dtype > KVP_F32) return KVP_ERR_ARG;
    if (!c->page_tokens || c->page_tokens % kTileTokens) return KVP_ERR_ARG;
    if (!head_dim_served(c->head_dim)) return KVP_ERR_RANGE;
    if (tokens && (!cache || !a || !b || !slots)) return KVP_ERR_ARG;
    if (off_by(cache, 16) || off_by(a, rows_align) || off_by(b, rows_align) || off_by(slots, 8)) return KVP_ERR_ARG;
    if (c->kv_heads > 65535 || tokens >= (1u << 31)) return KVP_ERR_RANGE;
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
    const int rc = check_rows(c, cache, tokens, k, v, dtype == KVP_F32 ? 4 : 2, slots, dtype);
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
    const int rc = check_rows(c, cache, tokens, k, v, 16, slots, dtype);
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
