// Writing and reading the cache held in 8 bits.
//
// The keys (and the values) of a block, 16 tokens of one head, are kept as scale * q: q in e4m3 (to the nearest, ties to even), scale
// the smallest power of two 2^e with |x| <= 448 * 2^e for all of them. A power of two costs nothing (e4m3 has the same four bits over 2^15 of its
// range) and makes the form exact to handle: x / scale is exact, and when a token comes that asks for a larger scale, what
// the block holds is divided by a power of two, which rounds only what falls below e4m3's normal numbers (2^-15 of the block's largest).
#include <cuda_bf16.h>

#include "kvp_tile8.cuh"

namespace kvp {

namespace {

struct Rows8K {
    const void *k, *v;
    int64_t k_token, k_head, v_token, v_head;     // strides in elements
    const int64_t* slots;
    uint8_t* cache;
    uint64_t slots_in_cache;                      // pages * page_tokens
    uint32_t tokens, heads, page_tokens;
};

constexpr float kMost = 0x1p100f;                 // larger magnitudes count as this
constexpr int kLeastExp = -100;                   // of a scale

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

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

// the block of a slot, for one head; slot < slots_in_cache
template <int D>
__device__ __forceinline__ uint64_t block_at(uint64_t slot, uint32_t head, const Rows8K& p)
{
    uint64_t page;
    uint32_t in_page;
    if (p.slots_in_cache <= ~0u) {
        page = (uint32_t)slot / p.page_tokens;
        in_page = (uint32_t)slot - (uint32_t)page * p.page_tokens;
    } else {
        page = slot / p.page_tokens;
        in_page = (uint32_t)(slot - page * p.page_tokens);
    }
    return ((page * p.heads + head) * (p.page_tokens / kTileTokens) + in_page / kTileTokens) * Tile8<D>::kBytes;
}

// the smallest power of two, 2^-100 at least, that `most` (at most 2^100) is 448 times of at most; 0 for 0
__device__ __forceinline__ float scale_for(float most)
{
    const int bits = __float_as_int(most), e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);      // 448 = 1.75 * 2^8
    return most > 0.0f ? __int_as_float((max(e, kLeastExp) + 127) << 23) : 0.0f;
}

// four e4m3 numbers times a power of two
__device__ __forceinline__ uint32_t rounded_again(uint32_t four, float by)
{
    const float2 a = floats_of_e4m3(four & 0xFFFFu), b = floats_of_e4m3(four >> 16);
    return e4m3_pair(a.x * by, a.y * by) | e4m3_pair(b.x * by, b.y * by) << 16;
}

struct Run {
    uint64_t block;          // where it lies in the cache
    float old, now;          // scales
    bool begins;             // the block's first token is among them: nothing is held
    uint32_t many;           // places that are written
    uint8_t token[16];       // of each place, counted from the CTA's first; kNobody: not written
};
constexpr uint8_t kNobody = 0xFF;

// A run is the tokens of one block in the call, which stand within 16 tokens of it. A CTA takes the runs that begin among 16 tokens; the last ones may go
// on behind them, so a thread has eight dims of two tokens. blockIdx.y is the head, blockIdx.z 0 for keys and 1 for values. One CTA thus knows the largest magnitude
// of a block's new tokens, and the block's bytes are written by nobody else.
// A run's bytes are gathered in shared memory and written 16 at a time: a token's 16 dims, or a dim of 16 tokens; single values (one byte each) where the
// run does not fill the block and its scale stays.
template <int D, typename T>
__global__ void __launch_bounds__(2 * D) append8_kernel(const Rows8K p, bool aligned)
{
    using L = Tile8<D>;
    constexpr uint32_t kThreads = 2 * D, kPerRow = D / 8;
    __shared__ int64_t slot[48];                                       // of the tokens from 16 before the CTA's first on
    __shared__ uint32_t leads[64];                                     // by the same numbers: the first token of its run; 0: no token
    __shared__ float most[32];
    __shared__ Run runs[16];
    __shared__ uint32_t many_runs;
    __shared__ alignas(16) uint8_t held[32][D];
    const uint32_t tid = threadIdx.x, row = tid / kPerRow, part = tid % kPerRow, head = blockIdx.y, base = blockIdx.x * 16;
    const bool is_value = blockIdx.z;
    const T* const from = is_value ? static_cast<const T*>(p.v) + head * p.v_head + 8 * part : static_cast<const T*>(p.k) + head * p.k_head + 8 * part;
    const int64_t stride = is_value ? p.v_token : p.k_token;
    float x[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[0][i] = x[1][i] = 0.0f;
    if (base + row < p.tokens) load8(from + (base + row) * stride, aligned, x[0]);
    if (tid < 48) {
        const int64_t t = (int64_t)base - 16 + tid;
        int64_t s = -1;
        if (t >= 0 && t < p.tokens) s = __ldg(p.slots + t);
        slot[tid] = s < 0 || (uint64_t)s >= p.slots_in_cache ? -1 : s;
    }
    __syncthreads();
    if (tid < 64) {                                                    // two whole warps
        const int64_t s = tid < 48 ? slot[tid] : -1;
        uint32_t first = tid;
        for (uint32_t j = tid < 16 ? 0 : tid - 15; s >= 0 && j < first; ++j)
            if (slot[j] >= 0 && slot[j] / kTileTokens == s / kTileTokens) first = j;
        leads[tid] = s >= 0 ? first : 0;
    }
    __syncthreads();
    // in a run that begins here?
    const bool in0 = leads[16 + row] >= 16, in1 = leads[32 + row] >= 16 && leads[32 + row] < 32;
    if (in1 && base + 16 + row < p.tokens) load8(from + (base + 16 + row) * stride, aligned, x[1]);
    if (tid < 32) {
        const bool leader = tid < 16 && leads[16 + tid] == 16 + tid;
        const uint32_t all = __ballot_sync(0xFFFFFFFFu, leader), at = __popc(all & ((1u << tid) - 1u));
        if (tid == 0) many_runs = __popc(all);
        if (leader) {
            Run& r = runs[at];
            r.block = block_at<D>((uint64_t)slot[16 + tid], head, p);
            const float old = *reinterpret_cast<const float*>(p.cache + r.block + L::kScale + (is_value ? 4 : 0));
            for (uint32_t i = 0; i < 16; ++i) r.token[i] = kNobody;
            r.many = 0;
            for (uint32_t t = tid; t < tid + 16; ++t)
                if (leads[16 + t] == 16 + tid) {
                    const uint32_t place = (uint32_t)(slot[16 + t] % kTileTokens);
                    r.many += r.token[place] == kNobody;
                    r.token[place] = (uint8_t)t;
                }
            r.begins = r.token[0] != kNobody;
            // a scale that is no power of two is none: nothing is held
            r.old = !r.begins && old >= 0x1p-126f && old < INFINITY && !(__float_as_int(old) & 0x7FFFFF) ? old : 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[u][i] = x[u][i] != x[u][i] ? 0.0f : fminf(fmaxf(x[u][i], -kMost), kMost);
            m = fmaxf(m, fabsf(x[u][i]));
        }
#pragma unroll
        for (uint32_t o = 1; o < kPerRow; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        if (part == 0) most[16 * u + row] = m;
    }
    __syncthreads();
    if (tid < many_runs) {
        Run& r = runs[tid];
        float m = 0.0f;
        for (uint32_t i = 0; i < 16; ++i)
            if (r.token[i] != kNobody) m = fmaxf(m, most[r.token[i]]);
        r.now = fmaxf(r.old, scale_for(m));
        for (uint32_t i = 0; i < 16; ++i)
            if (r.token[i] != kNobody) most[r.token[i]] = r.now;
        if (r.now != r.old || r.begins) *reinterpret_cast<float*>(p.cache + r.block + L::kScale + (is_value ? 4 : 0)) = r.now;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
        if (u ? in1 : in0) {
            const float scale = most[16 * u + row];
            const float by = scale > 0.0f ? __int_as_float((254 << 23) - __float_as_int(scale)) : 0.0f;      // 1 / scale
            uint2 q;
            q.x = e4m3_pair(x[u][0] * by, x[u][1] * by) | e4m3_pair(x[u][2] * by, x[u][3] * by) << 16;
            q.y = e4m3_pair(x[u][4] * by, x[u][5] * by) | e4m3_pair(x[u][6] * by, x[u][7] * by) << 16;
            if (!(scale > 0.0f)) q = make_uint2(0, 0);                 // -0 among them
            *reinterpret_cast<uint2*>(&held[16 * u + row][8 * part]) = q;
        }
    __syncthreads();
    for (uint32_t i = tid; i < many_runs * D; i += kThreads) {
        const Run& r = runs[i / D];
        const uint32_t at = i % D;
        const bool again = !r.begins && r.now != r.old;                // what is there is rounded again
        const float by = r.old > 0.0f ? r.old / r.now : 0.0f;
        if (!is_value) {
            const uint32_t place = at % 16, c = at / 16;
            uint4* to = reinterpret_cast<uint4*>(p.cache + r.block + L::key(place, c));
            if (r.token[place] != kNobody) {
                *to = *reinterpret_cast<const uint4*>(&held[r.token[place]][16 * c]);
            } else if (again) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if (by > 0.0f) {
                    q = *to;
                    q = make_uint4(rounded_again(q.x, by), rounded_again(q.y, by), rounded_again(q.z, by), rounded_again(q.w, by));
                }
                *to = q;
            }
        } else {
            uint8_t* to = p.cache + r.block + L::value(at);
            if (again || r.many == kTileTokens) {
                uint32_t q[4] = {0, 0, 0, 0};
                if (r.many < kTileTokens && by > 0.0f) {
                    const uint4 x = *reinterpret_cast<const uint4*>(to);
                    q[0] = rounded_again(x.x, by);
                    q[1] = rounded_again(x.y, by);
                    q[2] = rounded_again(x.z, by);
                    q[3] = rounded_again(x.w, by);
                }
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j)
                    if (r.token[j] != kNobody) q[j / 4] = q[j / 4] & ~(0xFFu << (8 * (j % 4))) | (uint32_t)held[r.token[j]][at] << (8 * (j % 4));
                *reinterpret_cast<uint4*>(to) = make_uint4(q[0], q[1], q[2], q[3]);
            } else {
                for (uint32_t j = 0; j < 16; ++j)
                    if (r.token[j] != kNobody) to[j] = held[r.token[j]][at];
            }
        }
    }
}

// The inverse. A CTA reads 16 tokens of the call, one head, keys or values; values by way of shared memory, 16 bytes (a dim of 16 tokens) at a
// time where the tokens are a whole block in order.
template <int D, typename T>
__global__ void __launch_bounds__(2 * D) read8_kernel(const Rows8K p, T* __restrict__ k, T* __restrict__ v)
{
    using L = Tile8<D>;
    constexpr uint32_t kThreads = 2 * D, kPerRow = D / 8;
    __shared__ uint64_t block[16];
    __shared__ uint32_t place[16];
    __shared__ float scale[16];                                        // -1: no such token
    __shared__ alignas(16) uint8_t held[16][D + 16];
    __shared__ uint32_t whole;
    const uint32_t tid = threadIdx.x, row = tid / kPerRow, part = tid % kPerRow, head = blockIdx.y, base = blockIdx.x * 16;
    const bool is_value = blockIdx.z;
    if (tid < 32) {
        const uint32_t t = base + tid;
        const int64_t s = tid < 16 && t < p.tokens ? __ldg(p.slots + t) : -1;
        const bool there = s >= 0 && (uint64_t)s < p.slots_in_cache;
        if (tid < 16) {
            float f = -1.0f;
            if (there) {
                block[tid] = block_at<D>((uint64_t)s, head, p);
                place[tid] = (uint32_t)(s % kTileTokens);
                f = *reinterpret_cast<const float*>(p.cache + block[tid] + L::kScale + (is_value ? 4 : 0));
            }
            scale[tid] = f;
        }
        const int64_t first = __shfl_sync(0xFFFFFFFFu, s, 0);
        const bool in_order = __all_sync(0xFFFFFFFFu, tid >= 16 || (there && s == first + tid && first % kTileTokens == 0));
        if (tid == 0) whole = in_order;
    }
    __syncthreads();
    if (is_value) {
        if (whole) {
            for (uint32_t d = tid; d < D; d += kThreads) {
                const uint4 q = __ldg(reinterpret_cast<const uint4*>(p.cache + block[0] + L::value(d)));
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) held[i][d] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
            }
        } else {
            for (uint32_t i = tid; i < 16 * D; i += kThreads) {
                const uint32_t t = i / D, d = i % D;
                if (scale[t] >= 0.0f) held[t][d] = p.cache[block[t] + L::value(d) + place[t]];
            }
        }
        __syncthreads();
    }
    if (base + row >= p.tokens) return;
    const float s = scale[row];
    uint2 q = make_uint2(0, 0);
    if (s >= 0.0f) {
        if (is_value) q = *reinterpret_cast<const uint2*>(&held[row][8 * part]);
        else q = __ldg(reinterpret_cast<const uint2*>(p.cache + block[row] + L::key(place[row], part / 2) + 8 * (part % 2)));
    }
    const float by = fmaxf(s, 0.0f);
    alignas(16) T e[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = floats_of_e4m3((i < 2 ? q.x : q.y) >> (16 * (i % 2)) & 0xFFFFu);
        put(e + 2 * i, f.x * by);
        put(e + 2 * i + 1, f.y * by);
    }
    uint4* to = reinterpret_cast<uint4*>((is_value ? v : k) + ((uint64_t)(base + row) * p.heads + head) * D + 8 * part);
#pragma unroll
    for (uint32_t i = 0; i < sizeof(e) / 16; ++i) to[i] = reinterpret_cast<uint4*>(e)[i];
}

template <int D, typename T>
int launch_append(const Rows8K& p, bool aligned, cudaStream_t st)
{
    append8_kernel<D, T><<<dim3((p.tokens + 15) / 16, p.heads, 2), 2 * D, 0, st>>>(p, aligned);
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

template <int D, typename T>
int launch_read(const Rows8K& p, void* k, void* v, cudaStream_t st)
{
    read8_kernel<D, T><<<dim3((p.tokens + 15) / 16, p.heads, 2), 2 * D, 0, st>>>(p, static_cast<T*>(k), static_cast<T*>(v));
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
        case 64 * 4 + KVP_BF16: return CALL(64, __nv_bfloat16);                                \
        case 64 * 4 + KVP_F16: return CALL(64, __half);                                        \
        case 64 * 4 + KVP_F32: return CALL(64, float);                                         \
        case 128 * 4 + KVP_BF16: return CALL(128, __nv_bfloat16);                              \
        case 128 * 4 + KVP_F16: return CALL(128, __half);                                      \
        case 128 * 4 + KVP_F32: return CALL(128, float);                                       \
        case 256 * 4 + KVP_BF16: return CALL(256, __nv_bfloat16);                              \
        case 256 * 4 + KVP_F16: return CALL(256, __half);                                      \
        case 256 * 4 + KVP_F32: return CALL(256, float);                                       \
        default: return KVP_ERR_RANGE;                                                         \
    }

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" uint64_t kvp_cache8_page_bytes(uint32_t head_dim, uint32_t page_tokens)
{
    if (!head_dim_served(head_dim) || page_tokens % kTileTokens) return 0;
    return (uint64_t)page_tokens / kTileTokens * (32 * head_dim + 16);
}

extern "C" int kvp_cache8_append(const kvp_cache_shape* c, void* cache, uint32_t dtype, uint32_t tokens, const void* k,
                                 int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                                 int64_t v_head_stride, const int64_t* slots, void* stream)
{
    const int rc = check_rows(c, cache, tokens, k, v, dtype == KVP_F32 ? 4 : 2, slots, dtype);
    if (rc || !tokens) return rc;
    Rows8K p;
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
#define KVP_APPEND(D, T) launch_append<D, T>(p, aligned, st)
    KVP_BY_SHAPE(KVP_APPEND)
#undef KVP_APPEND
}

extern "C" int kvp_cache8_read(const kvp_cache_shape* c, const void* cache, uint32_t dtype, uint32_t tokens, const int64_t* slots,
                               void* k, void* v, void* stream)
{
    const int rc = check_rows(c, cache, tokens, k, v, 16, slots, dtype);
    if (rc || !tokens) return rc;
    Rows8K p = {};
    p.slots = slots; p.cache = static_cast<uint8_t*>(const_cast<void*>(cache));
    p.slots_in_cache = (uint64_t)c->pages * c->page_tokens;
    p.tokens = tokens; p.heads = c->kv_heads; p.page_tokens = c->page_tokens;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define KVP_READ(D, T) launch_read<D, T>(p, k, v, st)
    KVP_BY_SHAPE(KVP_READ)
#undef KVP_READ
}
