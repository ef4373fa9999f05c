// The `left` largest keys of a row, ties to the lower index, for rows whose threshold moves little from one to the next.
//
// A CTA goes through a row in rounds of T units, unit j * T + tid in round j, so that a warp's ballot in a round is 32 units in order: word
// (j, warp) of the row, kept by lane j. Two thresholds around the expected one split the row in one pass of two comparisons
// and two ballots a key: keys above the band are chosen, those inside it (one or two hundred) are counted in 256 bins of shared memory, a warp
// finds the bin with the threshold, and the lanes look at their words' keys in the band again. Where the threshold has left the band (and on
// the first row), a histogram over all keys finds a new one; where it splits the keys of its bin, these are listed and ranked
// against each other; many equal keys are taken in the order of their words.
#pragma once

#include <type_traits>

#include "kvp_common.cuh"

namespace kvp {

constexpr uint32_t kBins256 = 256;
constexpr uint32_t kListed = 128;             // keys that can be ranked
constexpr uint32_t kFew = 128;                // keys of a band found by the histogram
// A band should hold this many keys, or up to twice as many: sums move steadily, weights by a drift of their own.
template <typename Key>
constexpr uint32_t kBandGoal = sizeof(Key) == 8 ? 32 : 64;

constexpr int kBatch = 8;                     // rounds whose keys are loaded together

template <typename Key, int T>
struct SelectShared {
    uint32_t hist[kBins256];                  // zero between uses
    uint32_t words[T];                        // chosen keys of the list, or ties per word; zero between uses
    uint32_t above[2];                        // keys above the band of this row and the next; zero before a call
    Key list[kListed];
    uint32_t unit[kListed];
    Key edge;                                 // the bin's number
    uint32_t top, low, total, positive, need, equal, inside, listed;
};

// Keys lo .. lo + 2^bits - 1, in 2^max(bits - 8, 0) keys a bin.
template <typename Key>
struct Band {
    Key lo, last;                             // and the threshold found last
    int bits;
    bool valid, moved;                        // moved: `last` is there
};

// A 32-bit number that grows with the key, and spreads keys of very different sizes
__device__ __forceinline__ uint32_t coarse(uint32_t key) { return key; }
__device__ __forceinline__ uint32_t coarse(uint64_t key) { return __float_as_uint(__ull2float_rz(key)); }
// the smallest key with that number or a larger one
__device__ __forceinline__ uint32_t smallest(uint32_t c, uint32_t) { return c; }
__device__ __forceinline__ uint64_t smallest(uint32_t c, uint64_t) { return __float2ull_ru(__uint_as_float(c)); }

__device__ __forceinline__ int bits_needed(uint32_t x) { return 32 - __clz(x); }
__device__ __forceinline__ int bits_needed(uint64_t x) { return 64 - __clzll(x); }

// bin[at] += 1 if `in`: one instruction that no branch surrounds
__device__ __forceinline__ void count_if(bool in, uint32_t bins, uint32_t at)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %0, 0; @p red.shared.add.u32 [%1], 1; }" ::"r"((uint32_t)in), "r"(bins + at * 4u) : "memory");
}

// One warp: the bin from the top in which the need-th key lies -> sm.edge (its number), sm.need (how many of its keys are
// wanted), sm.equal (how many it has); sm.inside: keys in all bins. Leaves the bins zero. need = 0 or need > inside: edge is left alone.
template <typename Key, int T>
__device__ __forceinline__ void find_bin(SelectShared<Key, T>& sm, uint32_t need, uint32_t lane)
{
    uint4* mine = reinterpret_cast<uint4*>(sm.hist) + 2 * lane;    // a lane owns eight neighbouring bins
    const uint4 a = mine[0], b = mine[1];
    mine[0] = mine[1] = make_uint4(0, 0, 0, 0);
    const uint32_t h[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += h[i];
    uint32_t suffix = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_down_sync(0xFFFFFFFFu, suffix, o);
        if (lane + o < 32) suffix += v;
    }
    if (lane == 0) sm.inside = suffix;
    const uint32_t reach = __ballot_sync(0xFFFFFFFFu, suffix >= need);
    if (reach && need && lane == 31u - __clz(reach)) {
        uint32_t higher = suffix - s;
#pragma unroll
        for (int i = 7; i >= 0; --i) {
            if (higher + h[i] >= need) {
                sm.edge = (Key)(8 * lane + i);
                sm.need = need - higher;
                sm.equal = h[i];
                break;
            }
            higher += h[i];
        }
    }
}

// `Row` gives the keys of n units: again(j0, k) those of this thread in rounds j0 .. j0 + 7, key(unit) any unit's, fetch<..>(j0, x) gets
// what kFetch rounds need from memory, done() is called when all rounds of FIRST were, and split<..>(j0, x, lo, hi, a, b) gives the ballots of >= lo and > hi over eight of them, with FIRST for
// the first time (which may change the keys: the weights of a step are added then), WHOLE where all of these rounds hold units, so that nothing is
// looked at and offsets are constants. kWhole: all rounds of the row do; kPeeled: the rounds that do go first, in a loop of their own. Rounds behind the last unit give any key at all: `cand`, lane j's word of the
// candidates in round j, says which count. 32-bit keys: of the units in it, those with key 0 are no candidates either.

// One digit of the search for a band: of the candidates at a distance of at most `span` from its base, counted by distance >> sh.
template <typename Key, int T, typename Row, typename Distance>
__device__ __forceinline__ void one_digit(SelectShared<Key, T>& sm, Row& row, uint32_t rounds, uint32_t cand, int sh, uint64_t span, uint32_t need,
                                          Distance distance)
{
    const uint32_t bins = (uint32_t)__cvta_generic_to_shared(sm.hist), lane = threadIdx.x & 31;
    for (uint32_t j0 = 0; j0 < rounds; j0 += kBatch) {
        Key k[kBatch];
        row.again(j0, k);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t mine = __shfl_sync(0xFFFFFFFFu, cand, (j0 + i) & 31) >> lane & 1u;
            const uint64_t d = distance(k[i]);
            count_if(j0 + i < rounds && mine && (sizeof(Key) == 8 || k[i]) && d <= span, bins, (uint32_t)(d >> sh) & 255u);
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) find_bin(sm, need, threadIdx.x);
    __syncthreads();
}

enum class Found { kAll, kBand, kTies };

// A band that holds the threshold. kAll: there are no more than `left` candidates. kTies: the threshold is band.lo, and more keys
// equal it than can be ranked. Every thread of the CTA calls it.
template <typename Key, int T, typename Row>
__device__ Found find_band(Row& row, uint32_t rounds, uint32_t cand, uint32_t left, Band<Key>& band, SelectShared<Key, T>& sm)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31;
    __syncthreads();
    if (tid == 0) {
        sm.top = 0; sm.low = ~0u; sm.total = 0; sm.positive = 0;
        sm.above[0] = sm.above[1] = 0;
    }
    __syncthreads();
    uint32_t most = 0, least = ~0u, here = 0, positive = 0;
    for (uint32_t j0 = 0; j0 < rounds; j0 += kBatch) {
        Key k[kBatch];
        row.again(j0, k);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t mine = __shfl_sync(0xFFFFFFFFu, cand, (j0 + i) & 31) >> lane & 1u;
            if (j0 + i < rounds && mine && (sizeof(Key) == 8 || k[i])) {
                const uint32_t c = coarse(k[i]);
                most = max(most, c);
                ++here;
                if (c) { least = min(least, c); ++positive; }
            }
        }
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    here = __reduce_add_sync(0xFFFFFFFFu, here);
    positive = __reduce_add_sync(0xFFFFFFFFu, positive);
    if (lane == 0 && here) {
        atomicMax(&sm.top, most);
        atomicMin(&sm.low, least);
        atomicAdd(&sm.total, here);
        atomicAdd(&sm.positive, positive);
    }
    __syncthreads();
    if (sm.total <= left) return Found::kAll;
    if (sm.positive < left) {                                     // the threshold is 0
        band.lo = 0;
        band.bits = 0;
        band.valid = true;
        return Found::kTies;
    }
    uint32_t base = sm.low, need = left, equal = sm.positive;
    const uint32_t top = sm.top;
    int rem = bits_needed(top - base);
    uint64_t span = top - base;
    while (rem > 0 && equal > kFew) {
        const int sh = max(rem - 8, 0);
        one_digit(sm, row, rounds, cand, sh, span, need, [&](Key x) { const uint32_t c = coarse(x); return c < base ? ~0ull : (uint64_t)(c - base); });
        base += (uint32_t)sm.edge << sh;
        need = sm.need;
        equal = sm.equal;
        rem = sh;
        span = (1ull << sh) - 1;
    }
    band.lo = smallest(base, Key());
    const Key hi = smallest((span < top - base ? base + (uint32_t)span : top) + 1u, Key()) - 1;
    band.bits = bits_needed(hi - band.lo);
    band.valid = true;
    if (sizeof(Key) == 8 && equal > kListed) {                    // keys that share their upper 24 bits
        while (band.bits > 0 && equal > kFew) {
            const int sh = max(band.bits - 8, 0);
            const uint64_t wide = (1ull << band.bits) - 1;
            one_digit(sm, row, rounds, cand, sh, wide, need, [&](Key x) { return (uint64_t)(x - band.lo); });
            band.lo += (Key)sm.edge << sh;
            need = sm.need;
            equal = sm.equal;
            band.bits = sh;
        }
    }
    return band.bits == 0 && equal > kListed ? Found::kTies : Found::kBand;
}

// of eight words the one whose number is lane % 8
__device__ __forceinline__ uint32_t own_of(const uint32_t (&x)[kBatch], uint32_t lane)
{
    const uint32_t a = lane & 1u ? x[1] : x[0], b = lane & 1u ? x[3] : x[2], c = lane & 1u ? x[5] : x[4], d = lane & 1u ? x[7] : x[6];
    const uint32_t e = lane & 2u ? b : a, f = lane & 2u ? d : c;
    return lane & 4u ? f : e;
}

// the ballots of keys at hand
template <typename Key>
__device__ __forceinline__ void ballots(const Key (&k)[kBatch], Key lo, Key hi, uint32_t (&a)[kBatch], uint32_t (&b)[kBatch])
{
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
        a[i] = __ballot_sync(0xFFFFFFFFu, k[i] >= lo);
        b[i] = __ballot_sync(0xFFFFFFFFu, k[i] > hi);
    }
}

// Lane j's words of round j: keys from `lo` on and keys above `hi`, of the candidates.
template <bool FIRST, typename Key, typename Row>
__device__ __forceinline__ void split(Row& row, uint32_t rounds, uint32_t cand, Key lo, Key hi, uint32_t& from, uint32_t& above)
{
    const uint32_t lane = threadIdx.x & 31;
    from = above = 0;
    auto some = [&](uint32_t j0, auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        typename Row::Raw x[Row::kFetch];
        row.template fetch<FIRST, kWhole>(j0, x);
#pragma unroll
        for (int i = 0; i < Row::kFetch; i += kBatch) {
            uint32_t a[kBatch], b[kBatch];
            row.template split<FIRST, kWhole>(j0 + i, x + i, lo, hi, a, b);
            const uint32_t c = own_of(a, lane), d = own_of(b, lane);
            if ((lane & ~7u) == j0 + i) {
                from = c;
                above = d;
            }
        }
    };
    uint32_t j0 = 0;
    if constexpr (Row::kPeeled)
        for (; (j0 + Row::kFetch) * Row::kThreads <= row.n; j0 += Row::kFetch) some(j0, std::true_type());
    for (; j0 < rounds; j0 += Row::kFetch) some(j0, std::bool_constant<Row::kWhole>());
    from &= cand;
    above &= cand;
}

// Many keys equal the threshold `at`: the keys above it, and of the equal ones the first in the order of the units.
template <typename Key, int T, typename Row>
__device__ uint32_t choose_ties(Row& row, uint32_t rounds, uint32_t cand, uint32_t left, Key at, SelectShared<Key, T>& sm)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, warps = blockDim.x / 32;
    uint32_t from, word;
    split<false>(row, rounds, cand, at, at, from, word);
    uint32_t ties = from & ~word;
    __syncthreads();
    if (tid == 0) sm.total = 0;
    if (lane < rounds) sm.words[lane * warps + warp] = __popc(ties);
    __syncthreads();
    const uint32_t n = __reduce_add_sync(0xFFFFFFFFu, (uint32_t)__popc(word));
    if (lane == 0) atomicAdd(&sm.total, n);
    if (warp == 0) {                                               // counts before each word, by one warp
        uint32_t run = 0;
        for (uint32_t i = lane; i - lane < rounds * warps; i += 32) {
            const uint32_t mine = i < rounds * warps ? sm.words[i] : 0u;
            uint32_t upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= (uint32_t)o) upto += v;
            }
            if (i < rounds * warps) sm.words[i] = run + upto - mine;
            run += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }
    __syncthreads();
    if (lane < rounds) {
        uint32_t* mine = &sm.words[lane * warps + warp];
        const uint32_t need = left - sm.total, before = *mine;     // equal keys of words before this one are chosen first
        const uint32_t take = need > before ? need - before : 0u;
        while ((uint32_t)__popc(ties) > take) ties &= ~(0x80000000u >> __clz(ties));
        word |= ties;
        *mine = 0;
    }
    if (tid == 0) sm.above[0] = sm.above[1] = 0;
    __syncthreads();
    return word;
}

// -> lane j's word of round j: the chosen units. turn: a number that changes by one from call to call. Every thread of the CTA calls it; when it
// returns, no lane of the warp looks at the warp's keys any more (other warps' keys are never looked at).
template <typename Key, int T, typename Row>
__device__ __forceinline__ uint32_t choose(Row& row, uint32_t rounds, uint32_t cand, uint32_t left, Band<Key>& band, SelectShared<Key, T>& sm,
                                           uint32_t turn)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, warps = T / 32, now = turn & 1;
    bool loaded = false;
    if (left == 0 || !band.valid) {                                // loads only
        uint32_t from, above;
        split<true>(row, rounds, cand, (Key)1, (Key)1, from, above);
        __syncwarp();
        row.done();
        loaded = true;
        if (left == 0) return 0;
    }
    // At most one band that misses, one that is found, and eight narrower ones in it
    for (int attempt = 0; attempt < 12; ++attempt) {
        if (!band.valid) {
            const Found found = find_band(row, rounds, cand, left, band, sm);
            if (found != Found::kBand) {
                band.valid = false;
                if (found == Found::kTies) return choose_ties(row, rounds, cand, left, band.lo, sm);
                if (sizeof(Key) == 8) return cand;
                uint32_t from, above;
                split<false>(row, rounds, cand, (Key)1, (Key)1, from, above);
                return from;
            }
        }
        const Key lo = band.lo, span = ((Key)1 << band.bits) - 1;
        const int sh = max(band.bits - 8, 0);
        uint32_t word, inside;
        if (loaded) split<false>(row, rounds, cand, lo, lo + span, inside, word);
        else split<true>(row, rounds, cand, lo, lo + span, inside, word);
        if (!loaded) row.done();                                   // the next row's keys may be sent for
        loaded = true;
        inside &= ~word;
        __syncwarp();                                              // a lane looks at keys that other lanes of its warp may have written
        const uint32_t first = (lane * warps + warp) * 32;         // unit of the words' bit 0
        for (uint32_t x = inside; x; x &= x - 1u) atomicAdd(&sm.hist[(uint32_t)((row.key(first + __ffs(x) - 1u) - lo) >> sh)], 1u);
        uint32_t above = __reduce_add_sync(0xFFFFFFFFu, (uint32_t)__popc(word));
        if (lane == 0 && above) atomicAdd(&sm.above[now], above);
        __syncthreads();
        above = sm.above[now];
        if (warp == 0) find_bin(sm, left > above ? left - above : 0u, lane);
        if (tid == 0) sm.above[now ^ 1] = 0;                       // last read a row ago, added to on the next one
        __syncthreads();
        const uint32_t in_band = sm.inside;
        if (above > left || left - above > in_band) {              // the threshold is not in the band
            band.valid = false;
            continue;                                              // find_band resets `above` behind a barrier
        }
        const uint32_t need = left - above, wanted = sm.need, equal = sm.equal;
        const Key edge = need ? lo + ((Key)sm.edge << sh) : lo + span + 1, over = edge + ((Key)1 << sh);
        if (need == 0 || wanted == equal) {
            for (uint32_t x = need ? inside : 0u; x; x &= x - 1u)
                if (row.key(first + __ffs(x) - 1u) >= edge) word |= x & (0u - x);
            __syncwarp();                                          // these are other lanes' keys, which those may change once `choose` returns
        } else if (equal <= kListed) {
            // the threshold splits its bin: its keys are ranked
            if (tid == 0) sm.listed = 0;
            __syncthreads();
            for (uint32_t x = inside; x; x &= x - 1u) {
                const uint32_t unit = first + __ffs(x) - 1u;
                const Key k = row.key(unit);
                if (k >= over) {
                    word |= x & (0u - x);
                } else if (k >= edge) {
                    const uint32_t at = atomicAdd(&sm.listed, 1u);
                    sm.list[at] = k;
                    sm.unit[at] = unit;
                }
            }
            __syncthreads();
            for (uint32_t e = tid; e < equal; e += (uint32_t)T) {
                const Key k = sm.list[e];
                const uint32_t u = sm.unit[e];
                uint32_t before = 0;
                for (uint32_t i = 0; i < equal; ++i) {
                    const Key x = sm.list[i];
                    before += x > k || (x == k && sm.unit[i] < u);
                }
                if (before < wanted) atomicOr(&sm.words[u >> 5], 1u << (u & 31));
            }
            __syncthreads();
            if (lane < rounds) {
                uint32_t* mine = &sm.words[lane * warps + warp];
                word |= *mine;
                *mine = 0;
            }
        } else if (sh > 0) {                                       // many keys close together: the bin becomes the band
            if (tid == 0) sm.above[now] = 0;
            band.lo = edge;
            band.bits = sh;
            __syncthreads();
            continue;
        } else {
            band.valid = band.moved = false;
            return choose_ties(row, rounds, cand, left, edge, sm);
        }
        // The next row's band: around the threshold, moved on by as much as it moved last, and wide enough for kBandGoal keys.
        if (in_band < kBandGoal<Key> && band.bits < (int)sizeof(Key) * 8 - 4) ++band.bits;
        else if (in_band > 2 * kBandGoal<Key> && band.bits > 0) --band.bits;
        const Key half = ((Key)1 << band.bits) / 2;
        const Key centre = edge + (sizeof(Key) == 8 && band.moved ? edge - band.last : 0);    // wraps where it moved down
        band.lo = centre > half && centre < (Key)1 << (sizeof(Key) * 8 - 1) ? centre - half : sizeof(Key) == 4;
        band.last = edge;
        band.moved = true;
        return word;
    }
    return 0;                                                      // not reached
}

// Lane j's word of round j: which units there are
__device__ __forceinline__ uint32_t units_there(uint32_t n)
{
    const uint32_t first = ((threadIdx.x & 31) * (blockDim.x / 32) + threadIdx.x / 32) * 32;
    return first >= n ? 0u : n - first >= 32 ? ~0u : (1u << (n - first)) - 1u;
}

template <typename Key, int T>
__device__ __forceinline__ void clear(SelectShared<Key, T>& sm)
{
    sm.words[threadIdx.x] = 0;
    for (uint32_t i = threadIdx.x; i < kBins256; i += T) sm.hist[i] = 0;
    if (threadIdx.x < 2) sm.above[threadIdx.x] = 0;
    __syncthreads();
}

// Writes the words of a row of a bitmap: word (j, warp) stands for units 32 (j T / 32 + warp) .. + 31 of the group that begins at bit `first`.
// aligned: no word is shared by two groups; otherwise the row was cleared before.
__device__ __forceinline__ void put_words(uint32_t* row, uint64_t first, uint32_t n, bool aligned, uint32_t word)
{
    const uint32_t at = ((threadIdx.x & 31) * (blockDim.x / 32) + threadIdx.x / 32) * 32;
    if (at >= n) return;
    uint32_t* to = row + ((first + at) >> 5);
    const uint32_t sh = (uint32_t)(first + at) & 31u;
    if (aligned) {
        *to = word;
    } else {
        if (word << sh) atomicOr(to, word << sh);
        if (sh && word >> (32u - sh)) atomicOr(to + 1, word >> (32u - sh));
    }
}

// Threads of a CTA for rows of n units (at most 32768): 32 rounds at most, 128 threads where that is enough, and a warp (whose barriers
// cost nothing) up to eight rounds.
inline uint32_t select_threads(uint32_t n) { return n <= 256 ? 32 : n <= 4096 ? 128 : n <= 8192 ? 256 : n <= 16384 ? 512 : 1024; }

// Consecutive rows of a CTA: it begins with the search for a band, so some rows together are cheaper once there are CTAs enough for all SMs (ten an SM).
inline uint32_t select_chunk(uint64_t rows) { return rows <= 148 * 10 ? 1 : rows >= 148 * 10 * 7 ? 8 : (uint32_t)(rows / (148 * 10)) + 1; }

}  // namespace kvp
