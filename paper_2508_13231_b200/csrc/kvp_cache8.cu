// Writing and reading the cache held in 8 bits.
//
// The keys (and the values) of a block, 16 tokens of one head, are kept as scale * q: q in e4m3 (to the nearest, ties to even), scale
// the smallest power of two 2^e with |x| <= 448 * 2^e for all of them. A power of two costs nothing (e4m3 has the same four bits over 2^15 of its
// range) and makes the form exact to handle: x / scale is exact, and when a token comes that asks for a larger scale, what
// the block holds is divided by a power of two, which rounds only what falls below e4m3's normal numbers (2^-15 of the block's largest).
//
// What bounds it, 32768 tokens x 8 heads of 128 dims, bf16 (134 MB of numbers, 67 MB of blocks): writing 63 us, instructions (20 a number, issue slots 66%) and three
// barriers a block, with the next block's loads under way; reading 44 us, the latency of loads at full occupancy. A step of 32 tokens: 6 and 3.5 us, latency.
#include <type_traits>

#include "kvp_line.cuh"
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
    Divisor by_heads;                             // of a CTA's number: heads of the same tokens stand next to each other, as in memory
};

constexpr float kMost = 0x1p100f;                 // larger magnitudes count as this
constexpr int kLeastExp = -100;                   // of a scale

// eight neighbouring elements as they lie; `aligned`: at a 16-byte boundary
template <typename T>
struct Eight {
    static constexpr int kWords = 2 * sizeof(T);
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p, bool aligned)
    {
        if (aligned) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i / 4);
                w[i] = x.x;
                w[i + 1] = x.y;
                w[i + 2] = x.z;
                w[i + 3] = x.w;
            }
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(p[i]);
        } else {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)q[2 * i] | (uint32_t)q[2 * i + 1] << 16;
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __half>::value) return i % 2 ? __high2float(half2_of(w[i / 2])) : __low2float(half2_of(w[i / 2]));
        else return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    // The largest magnitude of what is held, as the bits of an fp32 number: without the signs numbers are in the order of their bits.
    __device__ __forceinline__ uint32_t most(bool& odd) const              // odd: some number is not held as it is
    {
        uint32_t m;
        if constexpr (sizeof(T) == 4) {
            m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        } else {
            m = __vimax3_u16x2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu, w[2] & 0x7FFF7FFFu);
            m = __vimax3_u16x2(m, w[3] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu);
            m = max(m & 0xFFFFu, m >> 16);
            if constexpr (std::is_same<T, __half>::value) m = m >= 0x7C00u ? 0x7F800000u : __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
            else m <<= 16;
        }
        odd = m > __float_as_uint(kMost);
        if (!odd) return m;
        m = 0;                                                         // rare: NaN and what is cut
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(fabsf(held(at(i)))));
        return m;
    }
    static __device__ __forceinline__ float held(float x) { return x != x ? 0.0f : fminf(fmaxf(x, -kMost), kMost); }
};

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

// eight numbers over a power of two, or 0 where that is 0
template <typename T>
__device__ __forceinline__ uint2 rounded(const Eight<T>& x, float scale, bool odd)
{
    if (!(scale > 0.0f)) return make_uint2(0, 0);
    const float by = __int_as_float((254 << 23) - __float_as_int(scale));              // 1 / scale
    uint32_t q[4];
    if (!odd) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = e4m3_pair(x.at(2 * i) * by, x.at(2 * i + 1) * by);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = e4m3_pair(Eight<T>::held(x.at(2 * i)) * by, Eight<T>::held(x.at(2 * i + 1)) * by);
    }
    return make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
}

constexpr uint8_t kNobody = 0xFF;

// The runs that begin in a CTA; a run is the tokens of one block in the call, which stand within 16 tokens of it. [2]: keys, values
struct Runs {
    uint64_t block[16];              // where it lies in the cache
    float old[2][16], now[2][16];    // scales
    alignas(16) uint8_t token[16][16];       // of each place, counted from the CTA's first; kNobody: not written
    uint32_t mask[16];               // of the places that are written
    uint32_t many;
};

// A CTA takes the runs that begin among 16 tokens, of one head, keys and values; the last runs may go on behind the 16, so a thread has eight dims of two
// tokens. One CTA thus knows the largest magnitude of a block's new tokens, and the block's bytes are written by nobody else.
// Where the 16 tokens are a block from its first place to its last, as most of a prompt's are, nothing else is looked at: keys are written as a thread has them
// (two tokens of a warp fill whole sectors), values by way of shared memory, 8 tokens of a dim a thread. Elsewhere a run's bytes are gathered in shared memory and written 16 at a time, or one by one where the run does not fill the block and its scale stays.
template <int D, typename T>
__global__ void __launch_bounds__(2 * D, 1024 / (2 * D)) append8_kernel(const Rows8K p, uint32_t rounds, bool aligned)
{
    using L = Tile8<D>;
    constexpr uint32_t kThreads = 2 * D, kPerRow = D / 8, kStride = D + 8;             // rows eight apart lie in other banks
    __shared__ int64_t slot[48];                                       // of the tokens from 16 before the CTA's first on; -1: none
    __shared__ uint8_t run_of[32];                                     // of the tokens from the CTA's first on
    __shared__ uint32_t most[2][32];                                   // bits of magnitudes
    __shared__ Runs runs;
    __shared__ bool whole;
    __shared__ alignas(16) uint8_t held[2][32][kStride];
    const uint32_t tid = threadIdx.x, lane = tid % 32, row = tid / kPerRow, part = tid % kPerRow;
    // what a round needs from memory is sent for a round ahead: the eight dims of a token, keys and values, and the slots
    Eight<T> raw[2];
    int64_t my_slot = -1;
    const auto from = [&](int u, uint32_t token, uint32_t head) {
        return u ? static_cast<const T*>(p.v) + token * p.v_token + head * p.v_head + 8 * part : static_cast<const T*>(p.k) + token * p.k_token + head * p.k_head + 8 * part;
    };
    const auto fetch = [&](uint32_t round) {
        const uint32_t group = p.by_heads.of(round), head = round - group * p.heads, base = group * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            raw[u].clear();
            if (base + row < p.tokens) raw[u].load(from(u, base + row, head), aligned);
        }
        if (tid < 48) {
            const int64_t t = (int64_t)base - 16 + tid;
            my_slot = t >= 0 && t < p.tokens ? __ldg(p.slots + t) : -1;
        }
    };
    let_next_start();
    wait_for_previous();
    fetch(blockIdx.x);
    for (uint32_t round = blockIdx.x; round < rounds; round += gridDim.x) {
    const uint32_t group = p.by_heads.of(round), head = round - group * p.heads, base = group * 16;
    if (tid < 48) slot[tid] = my_slot < 0 || (uint64_t)my_slot >= p.slots_in_cache ? -1 : my_slot;
    else if (tid < 64) reinterpret_cast<uint4*>(runs.token)[tid - 48] = make_uint4(~0u, ~0u, ~0u, ~0u);
    __syncthreads();
    if (tid < 32) {
        const int64_t s = slot[16 + (lane & 15)], s0 = slot[16];
        const bool all = __all_sync(0xFFFFFFFFu, s0 >= 0 && s0 % kTileTokens == 0 && s == s0 + (lane & 15));
        if (lane == 0) whole = all;
        if (all) {
            if (lane == 0) runs.block[0] = block_at<D>((uint64_t)s0, head, p);
        } else {
            // token 16 + lane: the first of the 15 before it in the same block leads
            const int64_t mine = lane < 31 ? slot[16 + lane] : -1;
            uint32_t first = 16 + lane;
#pragma unroll
            for (uint32_t j = 15; j > 0; --j)
                if (slot[1 + lane + (15 - j)] >= 0 && slot[1 + lane + (15 - j)] / kTileTokens == mine / kTileTokens) first = min(first, 1 + lane + (15 - j));
            const bool leader = mine >= 0 && first < 32 && first == 16 + lane;
            const uint32_t leaders = __ballot_sync(0xFFFFFFFFu, leader);
            // in a run that begins here; a token whose first one is led itself, from further away than allowed, is left out
            const bool here = mine >= 0 && first >= 16 && first < 32 && (leaders >> (first - 16) & 1u);
            const uint32_t run = here ? __popc(leaders & ((1u << (first - 16)) - 1u)) : kNobody;
            run_of[lane] = (uint8_t)run;
            if (here) runs.token[run][mine % kTileTokens] = (uint8_t)lane;
            if (lane == 0) runs.many = __popc(leaders);
            if (leader) {
                const uint64_t at = block_at<D>((uint64_t)mine, head, p);
                const float2 old = *reinterpret_cast<const float2*>(p.cache + at + L::kScale);
                runs.block[run] = at;
                // a scale that is no power of two is none: nothing is held, and -1 is changed whatever comes
                const auto valid = [](float x) { return x == 0.0f || (x >= 0x1p-126f && x < INFINITY && !(__float_as_int(x) & 0x7FFFFF)); };
                runs.old[0][run] = valid(old.x) ? old.x : -1.0f;
                runs.old[1][run] = valid(old.y) ? old.y : -1.0f;
            }
        }
    }
    const Eight<T> x[2] = {raw[0], raw[1]};
    bool odd[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint32_t m = x[u].most(odd[u]);
#pragma unroll
        for (uint32_t o = 1; o < kPerRow; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        if (part == 0) most[u][row] = m;
    }
    if (round + gridDim.x < rounds) fetch(round + gridDim.x);
    __syncthreads();
    if (whole) {
        uint8_t* const block = p.cache + runs.block[0];
        float scale[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            scale[u] = scale_for(__uint_as_float(__reduce_max_sync(0xFFFFFFFFu, most[u][lane % 16])));
        }
        *reinterpret_cast<uint2*>(block + L::key(row, part / 2) + 8 * (part % 2)) = rounded(x[0], scale[0], odd[0]);
        *reinterpret_cast<uint2*>(&held[1][row][8 * part]) = rounded(x[1], scale[1], odd[1]);
        if (tid == 0) *reinterpret_cast<float2*>(block + L::kScale) = make_float2(scale[0], scale[1]);
        __syncthreads();
        const uint32_t d = tid / 2, first = tid % 2 * 8;
        uint32_t q[2] = {0, 0};
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) q[j / 4] |= (uint32_t)held[1][first + j][d] << (8 * (j % 4));
        *reinterpret_cast<uint2*>(block + L::value(d) + first) = make_uint2(q[0], q[1]);
        continue;                                                      // what the next round writes before its first barrier nobody reads any more
    }
    const bool in0 = run_of[row] != kNobody, in1 = row < 15 && run_of[16 + row] != kNobody;
    Eight<T> y[2];                                                     // of the token 16 further on
    bool odder[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        y[u].clear();
        if (in1) y[u].load(from(u, base + 16 + row, head), aligned);
        uint32_t m = y[u].most(odder[u]);
#pragma unroll
        for (uint32_t o = 1; o < kPerRow; o <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        if (part == 0) most[u][16 + row] = m;
    }
    __syncthreads();
    if (tid < 2 * runs.many) {
        const uint32_t run = tid / 2, u = tid % 2;
        const bool begins = runs.token[run][0] != kNobody;             // the block's first token is among them: nothing is held
        const float old = begins ? 0.0f : runs.old[u][run];
        uint32_t m = 0, mask = 0;
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) {
            const uint32_t t = runs.token[run][i];
            m = max(m, t != kNobody ? most[u][t] : 0u);
            mask |= (t != kNobody) << i;
        }
        if (u == 0) runs.mask[run] = mask;
        const float now = fmaxf(fmaxf(old, 0.0f), scale_for(__uint_as_float(m)));
        runs.old[u][run] = old;
        runs.now[u][run] = now;
        if (now != old || begins) *reinterpret_cast<float*>(p.cache + runs.block[run] + L::kScale + 4 * u) = now;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (in0) *reinterpret_cast<uint2*>(&held[u][row][8 * part]) = rounded(x[u], runs.now[u][run_of[row]], odd[u]);
        if (in1) *reinterpret_cast<uint2*>(&held[u][16 + row][8 * part]) = rounded(y[u], runs.now[u][run_of[16 + row]], odder[u]);
    }
    __syncthreads();
    // 2 D pieces of 16 bytes a run: its keys (place, 16 dims), then its values (dim, 16 places)
    for (uint32_t i = tid; i < runs.many * 2 * D; i += kThreads) {
        const uint32_t run = i / (2 * D), u = i / D % 2, at = i % D;
        const uint8_t* token = runs.token[run];
        const float old = runs.old[u][run], now = runs.now[u][run], by = old > 0.0f ? old / now : 0.0f;
        const uint32_t mask = runs.mask[run];
        const bool again = !(mask & 1u) && now != old;                 // what is there is rounded again
        uint8_t* const block = p.cache + runs.block[run];
        if (u == 0) {
            const uint32_t place = at % 16, c = at / 16;
            uint4* to = reinterpret_cast<uint4*>(block + L::key(place, c));
            if (mask >> place & 1u) {
                const uint2* q = reinterpret_cast<const uint2*>(&held[0][token[place]][16 * c]);
                *to = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
            } else if (again) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if (by > 0.0f) {
                    q = *to;
                    q = make_uint4(rounded_again(q.x, by), rounded_again(q.y, by), rounded_again(q.z, by), rounded_again(q.w, by));
                }
                *to = q;
            }
        } else {
            uint8_t* to = block + L::value(at);
            const bool full = mask == 0xFFFFu;
            if (again || full) {
                uint32_t q[4] = {0, 0, 0, 0};
                if (!full && by > 0.0f) {
                    const uint4 x = *reinterpret_cast<const uint4*>(to);
                    q[0] = rounded_again(x.x, by);
                    q[1] = rounded_again(x.y, by);
                    q[2] = rounded_again(x.z, by);
                    q[3] = rounded_again(x.w, by);
                }
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j)
                    if (mask >> j & 1u) q[j / 4] = q[j / 4] & ~(0xFFu << (8 * (j % 4))) | (uint32_t)held[1][token[j]][at] << (8 * (j % 4));
                *reinterpret_cast<uint4*>(to) = make_uint4(q[0], q[1], q[2], q[3]);
            } else {
                for (uint32_t left = mask; left; left &= left - 1u) {
                    const uint32_t j = __ffs(left) - 1u;
                    to[j] = held[1][token[j]][at];
                }
            }
        }
    }
    __syncthreads();
    }
}

// The inverse. A CTA reads 16 tokens of the call, one head; values by way of shared memory, 8 bytes (a dim of 8 tokens) at a time where the tokens are a whole
// block in order.
template <int D, typename T>
__global__ void __launch_bounds__(2 * D) read8_kernel(const Rows8K p, T* __restrict__ k, T* __restrict__ v)
{
    using L = Tile8<D>;
    constexpr uint32_t kThreads = 2 * D, kPerRow = D / 8, kStride = D + 8;
    __shared__ uint64_t block[16];
    __shared__ uint32_t place[16];                                     // ~0: no such token
    __shared__ alignas(16) uint8_t held[16][kStride];
    __shared__ bool whole;
    const uint32_t tid = threadIdx.x, row = tid / kPerRow, part = tid % kPerRow, group = p.by_heads.of(blockIdx.x), head = blockIdx.x - group * p.heads, base = group * 16;
    let_next_start();
    wait_for_previous();
    if (tid < 32) {
        const uint32_t t = base + tid;
        const int64_t s = tid < 16 && t < p.tokens ? __ldg(p.slots + t) : -1;
        const bool there = s >= 0 && (uint64_t)s < p.slots_in_cache;
        if (tid < 16) {
            block[tid] = there ? block_at<D>((uint64_t)s, head, p) : 0;
            place[tid] = there ? (uint32_t)(s % kTileTokens) : ~0u;
        }
        const int64_t first = __shfl_sync(0xFFFFFFFFu, s, 0);
        const bool in_order = __all_sync(0xFFFFFFFFu, tid >= 16 || (there && s == first + tid && first % kTileTokens == 0));
        if (tid == 0) whole = in_order;
    }
    __syncthreads();
    const bool there = place[row] != ~0u;
    const uint8_t* const mine = p.cache + block[row];
    uint2 q[2] = {make_uint2(0, 0), make_uint2(0, 0)};
    float2 scale = make_float2(0.0f, 0.0f);
    if (there) {
        q[0] = __ldg(reinterpret_cast<const uint2*>(mine + L::key(place[row], part / 2) + 8 * (part % 2)));
        scale = __ldg(reinterpret_cast<const float2*>(mine + L::kScale));
    }
    if (whole) {
        const uint32_t d = tid / 2, first = tid % 2 * 8;
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(p.cache + block[0] + L::value(d) + first));
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) held[first + j][d] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j % 4)));
    } else {
        for (uint32_t i = tid; i < 16 * D; i += kThreads) {
            const uint32_t t = i / D, d = i % D;
            if (place[t] != ~0u) held[t][d] = p.cache[block[t] + L::value(d) + place[t]];
        }
    }
    __syncthreads();
    if (base + row >= p.tokens) return;
    if (there) q[1] = *reinterpret_cast<const uint2*>(&held[row][8 * part]);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float by = u ? scale.y : scale.x;
        uint32_t e[2 * sizeof(T)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = floats_of_e4m3((i < 2 ? q[u].x : q[u].y) >> (16 * (i % 2)) & 0xFFFFu);
            if constexpr (sizeof(T) == 4) {
                e[2 * i] = __float_as_uint(f.x * by);
                e[2 * i + 1] = __float_as_uint(f.y * by);
            } else {
                e[i] = out_pair<std::is_same<T, __half>::value>(f.x * by, f.y * by);
            }
        }
        uint4* to = reinterpret_cast<uint4*>((u ? v : k) + ((uint64_t)(base + row) * p.heads + head) * D + 8 * part);
#pragma unroll
        for (uint32_t i = 0; i < sizeof(T) / 2; ++i) to[i] = make_uint4(e[4 * i], e[4 * i + 1], e[4 * i + 2], e[4 * i + 3]);
    }
}

template <int D, typename T>
int launch_append(const Rows8K& p, bool aligned, cudaStream_t st)
{
    // as many CTAs as are resident, each with the next round's loads under way
    const uint32_t rounds = (p.tokens + 15) / 16 * p.heads, resident = 148 * (1024 / (2 * D));
    return launch(append8_kernel<D, T>, rounds < resident ? rounds : resident, 2 * D, 0, true, st, p, rounds, aligned);
}

template <int D, typename T>
int launch_read(const Rows8K& p, void* k, void* v, cudaStream_t st)
{
    return launch(read8_kernel<D, T>, (p.tokens + 15) / 16 * p.heads, 2 * D, 0, true, st, p, static_cast<T*>(k), static_cast<T*>(v));
}

int check_rows(const kvp_cache_shape* c, const void* cache, uint32_t tokens, const void* a, const void* b, uint32_t rows_align, const int64_t* slots, uint32_t dtype)
{
    if (!c || c->reserved || !c->pages || !c->kv_heads || dtype > KVP_F32) return KVP_ERR_ARG;
    if (!c->page_tokens || c->page_tokens % kTileTokens) return KVP_ERR_ARG;
    if (!head_dim_served(c->head_dim)) return KVP_ERR_RANGE;
    if (tokens && (!cache || !a || !b || !slots)) return KVP_ERR_ARG;
    if (off_by(cache, 16) || off_by(a, rows_align) || off_by(b, rows_align) || off_by(slots, 8)) return KVP_ERR_ARG;
    if (c->kv_heads > 65535 || tokens >= (1u << 31) || (uint64_t)(tokens / 16 + 1) * c->kv_heads >= (1u << 31)) return KVP_ERR_RANGE;
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
    p.tokens = tokens; p.heads = c->kv_heads; p.page_tokens = c->page_tokens; p.by_heads = divisor(c->kv_heads);
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
    p.tokens = tokens; p.heads = c->kv_heads; p.page_tokens = c->page_tokens; p.by_heads = divisor(c->kv_heads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define KVP_READ(D, T) launch_read<D, T>(p, k, v, st)
    KVP_BY_SHAPE(KVP_READ)
#undef KVP_READ
}
