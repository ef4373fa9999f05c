// Eviction by accumulated attention weight (include/kvp.h, kvp_evict) and the placement policy made of it.
//
// Weights are accumulated as whole numbers of 2^-24, so that no order of summation shows; the units of a group are ranked by
// (accumulated weight, lower index first).
//
// Two forms. One pass: a CTA walks the steps of a group with the sums in registers; it reads every weight once and writes a bit for it, but
// a step takes about two microseconds of barriers and latency, which only other groups on the SM hide. Two passes: one thread
// per unit writes the sums of all steps to scratch, and the choices of the steps, independent of each other now, are made by as many CTAs as fit.
#include <algorithm>

#include "kvp_select.cuh"

namespace kvp {

namespace {

constexpr uint64_t kAccMost = (1ull << 48) - 1;
constexpr uint32_t kEvictUnits = 32768;        // units of a group

struct EvictK {
    const float* w;           // [steps][U]
    const int64_t* acc_in;    // [U] or null: zero
    int64_t* acc;             // [U]
    const uint32_t* kept;     // [W32] or null: every unit
    const int32_t* exist;     // [groups] or null: n
    uint32_t* out;            // [steps][W32]
    uint64_t* sums;           // [steps][U], two passes only: the sums that step's choice goes by
    uint64_t U, W32;
    uint32_t n, steps, groups, budget, sink, recent, decay;
    uint32_t chunk;           // steps of a CTA of the second pass
    bool aligned;             // n % 32 == 0: no word is shared by two groups
    bool before;              // a step's row is chosen before its weights are added
    bool carry;               // what a step leaves out is gone for the later ones; exist is [steps][groups] then
};

// NaN and negative weights convert to 0 (fminf would make 128 of NaN)
__device__ __forceinline__ uint32_t fixed_weight(float w) { return min(__float2uint_rn(w * 16777216.0f), 0x80000000u); }
__device__ __forceinline__ uint64_t accumulated(uint64_t acc, uint32_t decay, float w)
{
    if (decay != 65536u) acc = acc * decay >> 16;
    acc += fixed_weight(w);
    return acc < kAccMost ? acc : kAccMost;
}
__device__ __forceinline__ uint64_t first_sum(const EvictK& p, uint64_t u)
{
    const int64_t a = p.acc_in ? p.acc_in[u] : 0;
    return a < 0 ? 0u : min((uint64_t)a, kAccMost);
}

// Lane j's words of round j: the units there are, those that are protected, and those that may be chosen
struct Members {
    uint32_t there, safe, cand, left;
};
__device__ __forceinline__ Members members_of(const EvictK& p, uint32_t g, uint32_t step, uint32_t kept)
{
    const uint32_t e = p.exist ? (uint32_t)min(max(p.exist[(uint64_t)step * p.groups + g], 0), (int32_t)p.n) : p.n;
    Members m;
    m.there = units_there(e);
    m.safe = m.there & (units_there(p.sink) | ~units_there(e - min(e, p.recent)));
    m.cand = kept & m.there & ~m.safe;
    m.left = p.budget - min(min(e, p.sink + p.recent), p.budget);
    return m;
}
// Lane j's word of round j of kept_in; bits behind the group's last unit may be anything
__device__ __forceinline__ uint32_t kept_before(const EvictK& p, uint32_t g)
{
    const uint32_t unit = ((threadIdx.x & 31) * (blockDim.x / 32) + threadIdx.x / 32) * 32;
    if (!p.kept || unit >= p.n) return ~0u;
    const uint64_t at = (uint64_t)g * p.n + unit, w = at >> 5;
    const uint32_t sh = (uint32_t)at & 31u;
    return __funnelshift_r(p.kept[w], sh && w + 1 < p.W32 ? p.kept[w + 1] : 0u, sh);
}

// One pass. The sums of a group, 48 bits each, are in shared memory as lower words and upper half-words (24 KB for 4096 units: five CTAs an SM,
// so that 740 groups of that size are worked on at once); a step's first pass adds its weights. What bounds it is the latency of a step (two barriers,
// the search of the band's bins by one warp) with 17 warps an SM. Walks of 32 steps over 2.6 million units, us, by the units of a group: 2048 246, 2080 308,
// 4064 221, 4096 209, 7000 410, 8192 393, 16384 536, 32768 772; 53 would move the bytes. The weights of the next step in registers meanwhile: 198 at 4096, the
// one length for which they fit without spills (326 otherwise). Twice the threads a group are no faster.
template <int T>
struct SumsRow {
    typedef float Raw;
    static constexpr int kFetch = kBatch;
    static constexpr uint32_t kThreads = T;
    static constexpr bool kWhole = false, kPeeled = true;
    const EvictK& p;
    uint32_t* lo;
    uint16_t* hi;
    uint32_t n;
    const float* w;           // the weights to be added, or null
    bool plain;               // no decay, and no sum can reach 2^48
    __device__ __forceinline__ uint64_t key(uint32_t unit) const { return (uint64_t)hi[unit] << 32 | lo[unit]; }
    // Slots behind the row's end are not looked at: clamped to its last unit, they would read a sum that another warp is adding to.
    __device__ __forceinline__ bool there(uint32_t j) const { return j * T + threadIdx.x < n; }
    template <bool WHOLE>
    __device__ __forceinline__ void keys(uint32_t j0, uint64_t (&k)[kBatch]) const
    {
        const uint32_t* l = lo + j0 * T + threadIdx.x;            // the offsets from them are constants
        const uint16_t* h = hi + j0 * T + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) k[i] = WHOLE || there(j0 + i) ? (uint64_t)h[i * T] << 32 | l[i * T] : 0u;
    }
    __device__ __forceinline__ void again(uint32_t j0, uint64_t (&k)[kBatch]) const { keys<false>(j0, k); }
    template <bool FIRST, bool WHOLE>
    __device__ __forceinline__ void fetch(uint32_t j0, float (&x)[kFetch]) const
    {
        if (FIRST && w) {
            const float* at = w + j0 * T + threadIdx.x;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] = WHOLE || there(j0 + i) ? __ldcs(at + i * T) : 0.0f;
        }
    }
    __device__ __forceinline__ void done() const {}
    template <bool FIRST, bool WHOLE>
    __device__ __forceinline__ void split(uint32_t j0, const float* x, uint64_t least, uint64_t most, uint32_t (&a)[kBatch], uint32_t (&b)[kBatch]) const
    {
        uint64_t k[kBatch];
        if (FIRST && w) {
            uint32_t* const l0 = lo + j0 * T + threadIdx.x;
            uint16_t* const h0 = hi + j0 * T + threadIdx.x;
            if (plain && WHOLE) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const uint32_t add = fixed_weight(x[i]), l = l0[i * T] + add, h = h0[i * T] + (l < add);
                    l0[i * T] = l;
                    if (l < add) h0[i * T] = (uint16_t)h;
                    k[i] = (uint64_t)h << 32 | l;
                }
            } else {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    k[i] = 0;
                    if (WHOLE || there(j0 + i)) {
                        k[i] = accumulated((uint64_t)h0[i * T] << 32 | l0[i * T], p.decay, x[i]);
                        l0[i * T] = (uint32_t)k[i];
                        h0[i * T] = (uint16_t)(k[i] >> 32);
                    }
                }
            }
        } else {
            keys<WHOLE>(j0, k);
        }
        ballots(k, least, most, a, b);
    }
};

template <int T>
__global__ void __launch_bounds__(T, T == 128 ? 5 : 1) evict_kernel(const EvictK p)
{
    extern __shared__ uint32_t sums[];
    __shared__ SelectShared<uint64_t, T> sm;
    __shared__ uint32_t upper;
    const uint32_t g = blockIdx.x, tid = threadIdx.x, rounds = (p.n + T - 1) / T;
    const uint64_t first = (uint64_t)g * p.n;
    if (tid == 0) upper = 0;
    clear(sm);
    Members m = members_of(p, g, 0, kept_before(p, g));
    SumsRow<T> row = {p, sums, reinterpret_cast<uint16_t*>(sums + p.n), p.n, nullptr, false};
    uint32_t most = 0;
    for (uint32_t i = tid; i < p.n; i += T) {
        const uint64_t x = first_sum(p, first + i);
        row.lo[i] = (uint32_t)x;
        row.hi[i] = (uint16_t)(x >> 32);
        most = max(most, (uint32_t)(x >> 32));
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if ((tid & 31) == 0) atomicMax(&upper, most);
    __syncthreads();
    row.plain = p.decay == 65536u && upper + (uint64_t)p.steps / 2 + 1 < 0xFFFFu;             // a step adds 2^31 at most
    Band<uint64_t> band;
    band.valid = band.moved = false;
    // a row that is chosen before its weights are added is what the step before left
    for (uint32_t s = 0; s < p.steps; ++s) {
        const uint32_t adds = p.before ? s - 1 : s;                // the step whose weights are added; none (wraps) before the first choice
        row.w = adds < p.steps ? p.w + adds * p.U + first : nullptr;
        uint32_t word = choose<uint64_t, T>(row, rounds, m.cand, m.left, band, sm, s) | m.safe;
        if (p.carry) {                                             // units that are not there yet are not evicted
            word |= units_there(p.n) & ~m.there;
            if (s + 1 < p.steps) m = members_of(p, g, s + 1, word);
        }
        put_words(p.out + s * p.W32, first, p.n, p.aligned, word);
    }
    if (p.before) return;                                          // a policy: nobody asks for the sums
    for (uint32_t i = tid; i < p.n; i += T) p.acc[first + i] = (int64_t)row.key(i);           // written by this thread
}

// Two passes, the first: the sums that the steps' choices go by.
__global__ void __launch_bounds__(128) sums_kernel(const EvictK p)
{
    const uint64_t u = (uint64_t)blockIdx.x * 128 + threadIdx.x;
    if (u >= p.U) return;
    uint64_t acc = first_sum(p, u);
    constexpr uint32_t kAhead = 32;                                // weights under way while those before are added
    const uint32_t last = p.steps - 1;
    float next[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) next[i] = __ldcs(p.w + min(i, last) * p.U + u);
    for (uint32_t s0 = 0; s0 < p.steps; s0 += kAhead) {
        float x[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) x[i] = next[i];
        if (s0 + kAhead < p.steps) {
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) next[i] = __ldcs(p.w + min(s0 + kAhead + i, last) * p.U + u);
        }
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
            if (s0 + i >= p.steps) break;
            const uint64_t was = acc;
            acc = accumulated(acc, p.decay, x[i]);
            p.sums[(s0 + i) * p.U + u] = p.before ? was : acc;
        }
    }
    if (!p.before) p.acc[u] = (int64_t)acc;
}

// The second: a CTA chooses for some consecutive steps of a group.
template <int T>
struct StoredRow {
    typedef uint64_t Raw;
    static constexpr int kFetch = 2 * kBatch;
    static constexpr uint32_t kThreads = T;
    static constexpr bool kWhole = false, kPeeled = true;
    const uint64_t* from;
    uint32_t n;
    __device__ __forceinline__ void done() const {}
    __device__ __forceinline__ uint64_t key(uint32_t unit) const { return from[unit]; }
    __device__ __forceinline__ void again(uint32_t j0, uint64_t (&k)[kBatch]) const
    {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) k[i] = from[min((j0 + i) * T + threadIdx.x, n - 1)];
    }
    template <bool FIRST, bool WHOLE>
    __device__ __forceinline__ void fetch(uint32_t j0, uint64_t (&x)[kFetch]) const
    {
        const uint64_t* at = from + j0 * T + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kFetch; ++i) x[i] = WHOLE ? at[i * T] : from[min((j0 + i) * T + threadIdx.x, n - 1)];
    }
    template <bool FIRST, bool WHOLE>
    __device__ __forceinline__ void split(uint32_t, const uint64_t* k, uint64_t least, uint64_t most, uint32_t (&a)[kBatch], uint32_t (&b)[kBatch]) const
    {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            a[i] = __ballot_sync(0xFFFFFFFFu, k[i] >= least);
            b[i] = __ballot_sync(0xFFFFFFFFu, k[i] > most);
        }
    }
};

template <int T>
__global__ void __launch_bounds__(T) choose_kernel(const EvictK p)
{
    __shared__ SelectShared<uint64_t, T> sm;
    const uint32_t g = blockIdx.x % p.groups, s0 = blockIdx.x / p.groups * p.chunk, s1 = min(s0 + p.chunk, p.steps);
    const uint32_t rounds = (p.n + T - 1) / T;
    const uint64_t first = (uint64_t)g * p.n;
    clear(sm);
    const Members m = members_of(p, g, 0, kept_before(p, g));
    Band<uint64_t> band;
    band.valid = band.moved = false;
    for (uint32_t s = s0; s < s1; ++s) {
        StoredRow<T> row = {p.sums + s * p.U + first, p.n};
        const uint32_t word = choose<uint64_t, T>(row, rounds, m.cand, m.left, band, sm, s);
        put_words(p.out + s * p.W32, first, p.n, p.aligned, word | m.safe);
    }
}

template <int T>
int launch_choice(const EvictK& k, bool two, cudaStream_t st)
{
    if (two) {
        choose_kernel<T><<<k.groups * ((k.steps + k.chunk - 1) / k.chunk), T, 0, st>>>(k);
        return KVP_OK;
    }
    const uint32_t smem = (k.n * 6 + 15) / 16 * 16;
    if (smem > 40 * 1024) KVP_CUDA(cudaFuncSetAttribute(evict_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    evict_kernel<T><<<k.groups, T, smem, st>>>(k);
    return KVP_OK;
}

int check_evict(const kvp_evict_params* a)
{
    if (!a || (a->flags & ~KVP_EVICT_CARRY) || !a->groups || !a->units_per_group || !a->steps || a->decay_q > 65536) return KVP_ERR_ARG;
    if ((uint64_t)a->sink + a->recent > a->budget || a->budget > a->units_per_group) return KVP_ERR_ARG;
    if (a->units_per_group > kEvictUnits || (uint64_t)a->groups * a->units_per_group >= (1ull << 31)) return KVP_ERR_RANGE;
    return KVP_OK;
}

int launch_evict(const kvp_evict_params* a, const float* weights, const int64_t* acc_in, int64_t* acc, const uint32_t* kept,
                 const int32_t* exist, uint32_t* rows, bool before, cudaStream_t st)
{
    EvictK k = {};
    k.w = weights; k.acc_in = acc_in; k.acc = acc; k.kept = kept; k.exist = exist; k.out = rows;
    k.n = a->units_per_group; k.steps = a->steps; k.budget = a->budget; k.sink = a->sink; k.recent = a->recent; k.decay = a->decay_q;
    k.U = (uint64_t)a->groups * k.n;
    k.W32 = (k.U + 31) / 32;
    k.aligned = k.n % 32 == 0;
    k.before = before;
    k.carry = a->flags & KVP_EVICT_CARRY;
    k.groups = a->groups;
    if (!k.aligned) KVP_CUDA(cudaMemsetAsync(rows, 0, (size_t)a->steps * k.W32 * 4, st));
    const uint32_t n = k.n;
    // Which form is the faster one, in seconds. One pass: a step's latency grows with the units of a group, and with many groups the SMs are full. Two
    // passes: by the bytes. Measured on 461 shapes (128 .. 32768 units, 1 .. 1280 groups, 2 .. 256 steps): the form taken is 1% slower than the other at the
    // mean, 35% at most (1280 groups x 128 units x 4 steps, 36 and 27 us). 8 groups x 2048 units x 256 steps 37 and 754 us in two passes and one, 64 x 4096
    // x 64 107 and 407, 300 x 4096 x 64 354 and 420, 148 x 32768 x 4 188 and 106. One step, or more than 1 GiB of sums: one pass.
    const uint64_t all = k.U * a->steps;
    const size_t bytes = all * 8;
    const double one = std::max(a->steps * (3.5e-6 + n * 0.5e-9), (double)all * (n > 4096 ? 3.2e-12 : 2.0e-12));
    const bool faster = a->steps > 1 && one > 9e-6 + 4.3e-12 * (double)all;
    const uint32_t form = g_hooks.evict_form;                      // test hook
    const bool two = !k.carry && bytes <= ((size_t)1 << 30) && (form ? form == 2 : faster);
    if (two) {
        int dev = 0;
        KVP_CUDA(cudaGetDevice(&dev));
        const int prc = retain_in_pool(dev, bytes);
        if (prc) return prc;
        KVP_CUDA(cudaMallocAsync(&k.sums, bytes, st));
        sums_kernel<<<(uint32_t)((k.U + 127) / 128), 128, 0, st>>>(k);
        k.chunk = select_chunk((uint64_t)k.groups * a->steps);
    }
    const uint32_t threads = select_threads(n);
    const int rc = threads == 32 ? launch_choice<32>(k, two, st) : threads == 128 ? launch_choice<128>(k, two, st) : threads == 256 ? launch_choice<256>(k, two, st)
                 : threads == 512 ? launch_choice<512>(k, two, st) : launch_choice<1024>(k, two, st);
    const cudaError_t le = cudaGetLastError();
    if (two) KVP_CUDA(cudaFreeAsync(k.sums, st));
    if (rc) return rc;
    KVP_CUDA(le);
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
    if (off_by(weights, 4) || off_by(acc_in, 8) || off_by(acc_out, 8) || off_by(kept_in, 4) || off_by(exist, 4) || off_by(kept_out, 4)) return KVP_ERR_ARG;
    const uint64_t words = ((uint64_t)a->groups * a->units_per_group + 31) / 32;
    if (kept_in && kept_in < kept_out + words * a->steps && kept_out < kept_in + words) return KVP_ERR_ARG;
    const uint64_t units = (uint64_t)a->groups * a->units_per_group;
    if (acc_in && acc_in != acc_out && acc_in < acc_out + units && acc_out < acc_in + units) return KVP_ERR_ARG;
    return launch_evict(a, weights, acc_in, acc_out, kept_in, exist, kept_out, false, static_cast<cudaStream_t>(stream));
}

extern "C" int kvp_policy_accumulated(kvp_problem* p, const kvp_evict_params* a, const float* weights, uint32_t* schedule, void* stream)
{
    if (!p || !weights || !schedule || p->d_birth || off_by(weights, 4) || off_by(schedule, 4)) return KVP_ERR_ARG;
    const int rc = check_evict(a);
    if (rc) return rc;
    if (a->flags) return KVP_ERR_ARG;
    if (a->steps != p->S || (uint64_t)a->groups * a->units_per_group != p->U) return KVP_ERR_ARG;
    if ((uint64_t)a->groups * a->budget > p->cap) return KVP_ERR_CAPACITY;
    KVP_CUDA(cudaSetDevice(p->device));
    return launch_evict(a, weights, nullptr, nullptr, nullptr, nullptr, schedule, true, static_cast<cudaStream_t>(stream));
}
