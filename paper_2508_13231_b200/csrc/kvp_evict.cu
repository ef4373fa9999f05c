// Eviction by accumulated attention weight (include/kvp.h, kvp_evict) and the placement policy made of it.
//
// Weights are accumulated as whole numbers of 2^-24, so that no order of summation shows, and the units of a group are ranked
// by (accumulated weight, lower index first) through one 64-bit key, acc << 16 | (65535 - index), that no two units share.
#include "kvp_common.cuh"

namespace kvp {

namespace {

constexpr uint64_t kAccMost = (1ull << 48) - 1;
constexpr uint32_t kEvictUnits = 32768;        // units of a group
constexpr uint32_t kEvictThreads = 256;

struct EvictK {
    const float* w;           // [steps][U]
    const int64_t* acc_in;    // [U] or null: zero
    int64_t* acc;             // [U]
    const uint32_t* kept;     // [W32] or null: every unit
    const int32_t* exist;     // [groups] or null: n
    uint32_t* out;            // [steps][W32]
    uint64_t U, W32;
    uint32_t n, steps, budget, sink, recent, decay;
    bool aligned;             // n % 32 == 0: no word is shared by two groups
    bool before;              // a step's row is chosen before its weights are added
};

__device__ __forceinline__ uint64_t fixed_weight(float w)
{
    return w > 0.0f ? (uint64_t)__float2uint_rn(fminf(w, 128.0f) * 16777216.0f) : 0u;   // NaN counts as 0
}
__device__ __forceinline__ uint64_t accumulated(uint64_t acc, uint32_t decay, float w)
{
    if (decay != 65536u) acc = acc * decay >> 16;
    return min(acc + fixed_weight(w), kAccMost);
}
__device__ __forceinline__ uint64_t key_of(uint64_t acc, uint32_t i) { return acc << 16 | (65535u - i); }

__global__ void __launch_bounds__(kEvictThreads) evict_kernel(const EvictK p)
{
    __shared__ uint32_t hist[256], number, need_s;
    __shared__ uint64_t edge;
    const uint32_t g = blockIdx.x, tid = threadIdx.x, lane = tid % 32;
    const uint64_t first = (uint64_t)g * p.n;
    const uint32_t e = p.exist ? (uint32_t)min(max(p.exist[g], 0), (int32_t)p.n) : p.n;
    const uint32_t left = p.budget - min(min(e, p.sink + p.recent), p.budget);
    auto safe = [&](uint32_t i) { return i < p.sink || i + p.recent >= e; };
    auto old = [&](uint32_t i) { return !p.kept || (p.kept[(first + i) >> 5] >> ((first + i) & 31) & 1u); };
    uint64_t* acc = reinterpret_cast<uint64_t*>(p.acc + first);
    for (uint32_t i = tid; i < p.n; i += kEvictThreads) {
        const int64_t a = p.acc_in ? p.acc_in[first + i] : 0;
        acc[i] = a < 0 ? 0u : min((uint64_t)a, kAccMost);
    }
    for (uint32_t s = 0; s < p.steps; ++s) {
        const float* w = p.w + s * p.U + first;
        if (tid == 0) number = 0;
        __syncthreads();
        if (!p.before)
            for (uint32_t i = tid; i < p.n; i += kEvictThreads) acc[i] = accumulated(acc[i], p.decay, w[i]);
        uint32_t here = 0;
        for (uint32_t i = tid; i < e; i += kEvictThreads) here += !safe(i) && old(i);
        atomicAdd(&number, here);
        __syncthreads();
        uint64_t K = 0;
        uint32_t need = left;
        if (left == 0) {
            K = ~0ull;
        } else if (number > left) {
            for (int sh = 56; sh >= 0; sh -= 8) {
                hist[tid] = 0;
                __syncthreads();
                for (uint32_t i = tid; i < e; i += kEvictThreads) {
                    const uint64_t k = key_of(acc[i], i);
                    if (!safe(i) && old(i) && (sh == 56 || k >> (sh + 8) == K >> (sh + 8))) atomicAdd(&hist[k >> sh & 255u], 1u);
                }
                __syncthreads();
                if (tid == 0) {
                    uint32_t d = 255;
                    while (hist[d] < need) need -= hist[d--];
                    need_s = need;
                    edge = K | (uint64_t)d << sh;
                }
                __syncthreads();
                need = need_s;
                K = edge;
                __syncthreads();
            }
        }
        uint32_t* row = p.out + s * p.W32;
        for (uint32_t i = tid; i - lane < p.n; i += kEvictThreads) {
            const bool in = i < e && (safe(i) || (left && old(i) && key_of(acc[i], i) >= K));
            const uint32_t bits = __ballot_sync(0xFFFFFFFFu, in);
            if (lane == 0) {
                const uint64_t at = first + i;
                const uint32_t sh = (uint32_t)at & 31u;
                if (p.aligned) {
                    row[at >> 5] = bits;
                } else {
                    if (bits << sh) atomicOr(row + (at >> 5), bits << sh);
                    if (sh && bits >> (32u - sh)) atomicOr(row + (at >> 5) + 1, bits >> (32u - sh));
                }
            }
        }
        __syncthreads();
        if (p.before)
            for (uint32_t i = tid; i < p.n; i += kEvictThreads) acc[i] = accumulated(acc[i], p.decay, w[i]);
    }
}

int check_evict(const kvp_evict_params* a)
{
    if (!a || a->reserved || !a->groups || !a->units_per_group || !a->steps || a->decay_q > 65536) return KVP_ERR_ARG;
    if ((uint64_t)a->sink + a->recent > a->budget || a->budget > a->units_per_group) return KVP_ERR_ARG;
    if (a->units_per_group > kEvictUnits || (uint64_t)a->groups * a->units_per_group >= (1ull << 31)) return KVP_ERR_RANGE;
    return KVP_OK;
}

int launch_evict(const kvp_evict_params* a, const float* weights, const int64_t* acc_in, int64_t* acc, const uint32_t* kept,
                 const int32_t* exist, uint32_t* rows, bool before, cudaStream_t st)
{
    EvictK k;
    k.w = weights; k.acc_in = acc_in; k.acc = acc; k.kept = kept; k.exist = exist; k.out = rows;
    k.n = a->units_per_group; k.steps = a->steps; k.budget = a->budget; k.sink = a->sink; k.recent = a->recent; k.decay = a->decay_q;
    k.U = (uint64_t)a->groups * k.n;
    k.W32 = (k.U + 31) / 32;
    k.aligned = k.n % 32 == 0;
    k.before = before;
    if (!k.aligned) KVP_CUDA(cudaMemsetAsync(rows, 0, (size_t)a->steps * k.W32 * 4, st));
    evict_kernel<<<a->groups, kEvictThreads, 0, st>>>(k);
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" int kvp_evict(const kvp_evict_params* a, const float* weights, const int64_t* acc_in, int64_t* acc_out,
                         const uint32_t* kept_in, const int32_t* exist, uint32_t* kept_out, void* stream)
{
    const int rc = check_evict(a);
    if (rc) return rc;
    if (!weights || !acc_out || !kept_out) return KVP_ERR_ARG;
    const uint64_t words = ((uint64_t)a->groups * a->units_per_group + 31) / 32;
    if (kept_in && kept_in < kept_out + words * a->steps && kept_out < kept_in + words) return KVP_ERR_ARG;
    return launch_evict(a, weights, acc_in, acc_out, kept_in, exist, kept_out, false, static_cast<cudaStream_t>(stream));
}

extern "C" int kvp_policy_accumulated(kvp_problem* p, const kvp_evict_params* a, const float* weights, uint32_t* schedule, void* stream)
{
    if (!p || !weights || !schedule || p->d_birth) return KVP_ERR_ARG;
    const int rc = check_evict(a);
    if (rc) return rc;
    if (a->steps != p->S || (uint64_t)a->groups * a->units_per_group != p->U) return KVP_ERR_ARG;
    if ((uint64_t)a->groups * a->budget > p->cap) return KVP_ERR_CAPACITY;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int rs = ensure_scratch(p, (size_t)p->U * 8, st);
    if (rs) return rs;
    return launch_evict(a, weights, nullptr, static_cast<int64_t*>(p->d_scratch), nullptr, nullptr, schedule, true, st);
}
