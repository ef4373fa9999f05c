// Rotary positions (include/kvp.h, kvp_rope): pairs of dims of queries and keys turned by position * frequency.
//
// An angle is kept as a fraction of a turn, in 2^-64 turns: frequency / 2 pi, to 2^-64 turns, times the position, modulo 2^64. A double holds 53 bits of that quotient, which
// is not enough (2^31 tokens at a radian each would be off by 2^-21), so it is two: the product with the double next to 1 / 2 pi, and what that leaves out. An angle is off by 2^-65 turns a token,
// 2^-34 at the farthest. Its upper bits give the quadrant and what is left, at most an eighth of a turn, whose fp32 form is off by 2^-27 turns at most.
//
// What bounds it is memory: a thread computes the sines and cosines of its pairs once and goes through several heads with them,
// 16 bytes at a time, four heads' loads under way. 32768 tokens x 40 heads of 128 dims, bf16 (671 MB): 103 us, 6.5 TB/s; one head's loads at a time 203, elements
// unpacked as they are loaded 184 (120 registers instead of 80). 32 tokens: 2.5 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

#include "kvp_line.cuh"

namespace kvp {

namespace {

struct RopeK {
    const void *q, *k;
    void *q_out, *k_out;
    const int32_t* positions;
    const double* frequencies;
    int64_t q_token, q_head, k_token, k_head, qo_token, qo_head, ko_token, ko_head;
    uint32_t tokens, heads, all_heads, per;       // per: heads of a thread
    uint32_t half;                                // pairs of a head
    uint32_t turned;                              // chunks of a head that are turned; those behind are copied
    Divisor chunks, groups;                       // of a thread's number, of a CTA's
    float scale;
    bool inverse;
};

__device__ __forceinline__ float float_of(float x) { return x; }
__device__ __forceinline__ float float_of(__half x) { return __half2float(x); }
__device__ __forceinline__ float float_of(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void round_to(float* p, float x) { *p = x; }
__device__ __forceinline__ void round_to(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void round_to(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// V elements of a load, kept as they lie: 16 bytes, or one element
template <typename T, int V>
struct Vec {
    uint4 w;
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ uint32_t& word(int i) { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
    __device__ __forceinline__ void get(float* x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = word(i);
            if constexpr (sizeof(T) == 4) {
                x[i] = __uint_as_float(u);
            } else if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(half2_of(u));
                x[2 * i] = f.x;
                x[2 * i + 1] = f.y;
            } else {
                x[2 * i] = __uint_as_float(u << 16);
                x[2 * i + 1] = __uint_as_float(u & 0xFFFF0000u);
            }
        }
    }
    __device__ __forceinline__ void put(const float* x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) word(i) = __float_as_uint(x[i]);
            else word(i) = out_pair<std::is_same<T, __half>::value>(x[2 * i], x[2 * i + 1]);
        }
    }
};
template <typename T>
struct Vec<T, 1> {
    T e;
    __device__ __forceinline__ void load(const T* p) { e = *p; }
    __device__ __forceinline__ void store(T* p) const { *p = e; }
    __device__ __forceinline__ void get(float* x) { x[0] = float_of(e); }
    __device__ __forceinline__ void put(const float* x) { round_to(&e, x[0]); }
};

__device__ __forceinline__ void turn_of(int32_t position, double frequency, float scale, bool inverse, float& c, float& s)
{
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;                // 1 / 2 pi
    const double turns = __dmul_rn(frequency, kTurn), rest = fma(frequency, kTurnRest, fma(frequency, kTurn, -turns));
    const uint64_t part = (uint64_t)__double2ll_rn((turns - rint(turns)) * 0x1p64) + (uint64_t)__double2ll_rn((rest - rint(rest)) * 0x1p64);
    const uint64_t angle = (uint64_t)(int64_t)position * part + (1ull << 61);               // + an eighth, so that quadrants are cut there
    const uint32_t quadrant = (uint32_t)(angle >> 62);
    const int32_t left = (int32_t)((uint32_t)(angle >> 30) ^ 0x80000000u);                            // what is below it, 2^-34 turns, the eighth taken off again
    const float x = (float)left * 0x1p-33f;                                                           // half turns, -1/4 .. 1/4
    float a, b;
    sincospif(x, &a, &b);
    c = (quadrant & 1u) ? a : b;
    s = (quadrant & 1u) ? b : a;
    if (quadrant == 1u || quadrant == 2u) c = -c;
    if (quadrant >= 2u) s = -s;
    c *= scale;
    s *= inverse ? -scale : scale;
}

// V: elements of a load (1: any alignment and sizes). A chunk is V pairs (halves) or V elements, V / 2 pairs, side by side (interleaved); a CTA takes
// `per` heads of 256 chunks, queries before keys.
template <typename T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rope_kernel(const RopeK p)
{
    constexpr int kPairs = INTERLEAVED && V > 1 ? V / 2 : V;
    constexpr bool kTwo = !(INTERLEAVED && V > 1);                     // two loads for a chunk
    constexpr uint32_t kBatch = 4;
    using W = Vec<T, V>;
    let_next_start();
    wait_for_previous();
    const uint32_t block = p.groups.of(blockIdx.x), group = blockIdx.x - block * p.groups.d;       // heads of the same tokens at the same time, as they lie in memory
    const uint32_t i = block * 256 + threadIdx.x, t = p.chunks.of(i), chunk = i - t * p.chunks.d;
    if (t >= p.tokens) return;
    const uint32_t first = group * p.per, last = min(first + p.per, p.all_heads);
    const bool turned = chunk < p.turned;
    uint32_t at0, at1 = 0;
    float c[kPairs], s[kPairs];
    if (turned) {
        const int32_t position = __ldg(p.positions + t);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) turn_of(position, __ldg(p.frequencies + chunk * kPairs + j), p.scale, p.inverse, c[j], s[j]);
        at0 = INTERLEAVED ? (V > 1 ? chunk * V : 2 * chunk) : chunk * V;
        at1 = INTERLEAVED ? at0 + 1 : at0 + p.half;
    } else {
        at0 = 2 * p.half + (chunk - p.turned) * V;
    }
    // Loads of four heads before the first store: results may lie over what is read, so the compiler keeps their order.
    for (uint32_t h0 = first; h0 < last; h0 += kBatch) {
        W x[kBatch], y[kBatch];
#pragma unroll
        for (uint32_t k = 0; k < kBatch; ++k)
            if (h0 + k < last) {
                const uint32_t h = h0 + k;
                const T* from = h < p.heads ? static_cast<const T*>(p.q) + t * p.q_token + h * p.q_head : static_cast<const T*>(p.k) + t * p.k_token + (h - p.heads) * p.k_head;
                x[k].load(from + at0);
                if (kTwo && turned) y[k].load(from + at1);
            }
#pragma unroll
        for (uint32_t k = 0; k < kBatch; ++k)
            if (h0 + k < last) {
                const uint32_t h = h0 + k;
                T* to = h < p.heads ? static_cast<T*>(p.q_out) + t * p.qo_token + h * p.qo_head : static_cast<T*>(p.k_out) + t * p.ko_token + (h - p.heads) * p.ko_head;
                if (turned) {
                    float u[V], v[V];
                    x[k].get(u);
                    if (kTwo) y[k].get(v);
#pragma unroll
                    for (int j = 0; j < kPairs; ++j) {
                        float& a = u[kTwo ? j : 2 * j];
                        float& b = kTwo ? v[j] : u[kTwo ? 0 : 2 * j + 1];
                        const float new_a = a * c[j] - b * s[j], new_b = a * s[j] + b * c[j];
                        a = new_a;
                        b = new_b;
                    }
                    x[k].put(u);
                    if (kTwo) {
                        y[k].put(v);
                        y[k].store(to + at1);
                    }
                }
                x[k].store(to + at0);
            }
    }
}

template <typename T, int V>
int launch_rope(RopeK k, const kvp_rope_params* a, bool copies, cudaStream_t st)
{
    const bool interleaved = a->flags & KVP_ROPE_INTERLEAVED;
    k.turned = interleaved && V > 1 ? a->rotary_dim / V : a->rotary_dim / 2 / V;
    const uint32_t chunks = k.turned + (copies ? (a->head_dim - a->rotary_dim) / V : 0);
    k.chunks = divisor(chunks);
    if ((uint64_t)k.tokens * chunks >= (1ull << 31) - 256) return KVP_ERR_RANGE;
    // As many heads a thread as leave about eight warps for each of an SM's four schedulers: few tokens spread over the GPU (a decode step is latency), many share
    // the sines and cosines of eight heads, two batches of loads.
    const uint64_t threads = (uint64_t)k.tokens * chunks;
    uint64_t per = threads * k.all_heads / (148 * 1024);
    per = per < 1 ? 1 : per < 4 ? per : per < 8 ? 4 : 8;
    k.per = (uint32_t)per;
    k.groups = divisor((k.all_heads + k.per - 1) / k.per);
    const uint64_t grid = (threads + 255) / 256 * k.groups.d;
    if (grid >= (1ull << 31)) return KVP_ERR_RANGE;
    return interleaved ? launch(rope_kernel<T, V, true>, (uint32_t)grid, 256, 0, true, st, k) : launch(rope_kernel<T, V, false>, (uint32_t)grid, 256, 0, true, st, k);
}

template <typename T>
int rope_of(const RopeK& k, const kvp_rope_params* a, bool copies, cudaStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    const uint64_t addresses = (uint64_t)(uintptr_t)k.q | (uint64_t)(uintptr_t)k.k | (uint64_t)(uintptr_t)k.q_out | (uint64_t)(uintptr_t)k.k_out;
    uint64_t strides = k.q_token | k.q_head | k.qo_token | k.qo_head;
    if (k.k) strides |= k.k_token | k.k_head | k.ko_token | k.ko_head;
    const uint32_t piece = a->flags & KVP_ROPE_INTERLEAVED ? a->rotary_dim : a->rotary_dim / 2;
    const bool wide = addresses % 16 == 0 && strides % V == 0 && piece % V == 0 && (a->head_dim - a->rotary_dim) % V == 0;
    return wide ? launch_rope<T, V>(k, a, copies, st) : launch_rope<T, 1>(k, a, copies, st);
}

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" int kvp_rope_frequencies(const kvp_rope_scaling* r, uint32_t rotary_dim, double* frequencies, float* scale)
{
    if (!r || !frequencies || r->reserved || !rotary_dim || rotary_dim % 2 || r->kind > KVP_ROPE_RAMP || !(r->base > 0.0) || !std::isfinite(r->base)) return KVP_ERR_ARG;
    if (r->kind && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return KVP_ERR_ARG;
    if (r->kind >= KVP_ROPE_PARTS && (!(r->original_tokens > 0.0) || !std::isfinite(r->original_tokens) || !(r->low >= 0.0) || !(r->high > r->low) || !std::isfinite(r->high))) return KVP_ERR_ARG;
    if (r->kind == KVP_ROPE_BASE && rotary_dim < 4) return KVP_ERR_ARG;
    const uint32_t half = rotary_dim / 2;
    const double two_pi = 6.283185307179586476925;
    double base = r->base;
    if (r->kind == KVP_ROPE_BASE) base *= std::pow(r->factor, (double)rotary_dim / (rotary_dim - 2));
    if (!std::isnormal(base) || (r->kind == KVP_ROPE_RAMP && !(base > 1.0))) return KVP_ERR_ARG;     // frequencies of 0 or infinity; no borders
    for (uint32_t j = 0; j < half; ++j) {
        double f = std::pow(base, -(double)j / half);
        if (r->kind == KVP_ROPE_LINEAR) f /= r->factor;
        if (r->kind == KVP_ROPE_PARTS) {
            // turns within the original context: kept from `high` on, divided up to `low`, linear in them between
            const double turns = r->original_tokens * f / two_pi;
            double keep = (turns - r->low) / (r->high - r->low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / r->factor * (1.0 - keep);
        }
        if (r->kind == KVP_ROPE_RAMP) {
            // the same borders, but linear in the dim between those that turn `high` and `low` times, rounded outwards to whole dims. The second may lie behind the last pair, which
            // then is not divided in full.
            auto dim_of = [&](double turns) { return half * std::log(r->original_tokens / (turns * two_pi)) / std::log(base); };
            double from = std::floor(dim_of(r->high)), to = r->low > 0.0 ? std::ceil(dim_of(r->low)) : half - 1.0;
            if (!(from > 0.0)) from = 0.0;
            if (!(to > from)) to = from + 0.001;
            double divide = ((double)j - from) / (to - from);
            divide = divide < 0.0 ? 0.0 : divide > 1.0 ? 1.0 : divide;
            f = f * (1.0 - divide) + f / r->factor * divide;
        }
        frequencies[j] = f;
    }
    if (scale) *scale = r->kind == KVP_ROPE_RAMP ? (float)(0.1 * std::log(r->factor) + 1.0) : 1.0f;
    return KVP_OK;
}

extern "C" int kvp_rope(const kvp_rope_params* a, const void* q, void* q_out, const void* k, void* k_out, const int32_t* positions, const double* frequencies,
                        void* stream)
{
    if (!a || a->reserved || a->dtype > KVP_F32 || a->flags & ~(KVP_ROPE_INTERLEAVED | KVP_ROPE_INVERSE)) return KVP_ERR_ARG;
    if (!a->head_dim || !a->rotary_dim || a->rotary_dim % 2 || a->rotary_dim > a->head_dim || !(a->scale > -INFINITY && a->scale < INFINITY)) return KVP_ERR_ARG;
    if (!a->heads && !a->kv_heads) return KVP_ERR_ARG;
    if (a->head_dim > 65536 || (uint64_t)a->heads + a->kv_heads >= (1u << 20) || a->tokens >= (1u << 31)) return KVP_ERR_RANGE;
    if (!a->tokens) return KVP_OK;
    if ((a->heads && (!q || !q_out)) || (a->kv_heads && (!k || !k_out)) || !positions || !frequencies) return KVP_ERR_ARG;
    const uint32_t e = a->dtype == KVP_F32 ? 4 : 2;
    if (off_by(q, e) || off_by(k, e) || off_by(q_out, e) || off_by(k_out, e) || off_by(positions, 4) || off_by(frequencies, 8)) return KVP_ERR_ARG;
    // over the input itself only as it lies
    if ((a->heads && q == q_out && (a->q_token_stride != a->q_out_token_stride || a->q_head_stride != a->q_out_head_stride)) ||
        (a->kv_heads && k == k_out && (a->k_token_stride != a->k_out_token_stride || a->k_head_stride != a->k_out_head_stride))) return KVP_ERR_ARG;
    RopeK p = {};
    p.tokens = a->tokens; p.heads = a->heads; p.all_heads = a->heads + a->kv_heads;
    p.half = a->rotary_dim / 2;
    p.positions = positions; p.frequencies = frequencies;
    p.scale = a->scale;
    p.inverse = a->flags & KVP_ROPE_INVERSE;
    if (a->heads) {
        p.q = q; p.q_out = q_out;
        p.q_token = a->q_token_stride; p.q_head = a->q_head_stride; p.qo_token = a->q_out_token_stride; p.qo_head = a->q_out_head_stride;
    }
    if (a->kv_heads) {
        p.k = k; p.k_out = k_out;
        p.k_token = a->k_token_stride; p.k_head = a->k_head_stride; p.ko_token = a->k_out_token_stride; p.ko_head = a->k_out_head_stride;
    }
    const bool copies = (a->heads && q != q_out) || (a->kv_heads && k != k_out);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == KVP_BF16) return rope_of<__nv_bfloat16>(p, a, copies, st);
    return a->dtype == KVP_F16 ? rope_of<__half>(p, a, copies, st) : rope_of<float>(p, a, copies, st);
}
