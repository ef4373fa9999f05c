// The line of tiles that attention over a paged cache is cut from: lengths, bitmaps of units and the search for a CTA's part.
// Templates on the parameters of a kernel, a struct that derives from LineK.
#pragma once

#include <cuda_bf16.h>

#include "kvp_tile.cuh"

namespace kvp {

constexpr int kWarps = 8;
constexpr uint32_t kThreads = kWarps * 32;
constexpr float kNone = -3e38f; // maximum of nothing

// Division by a number known at the launch: n / d = (n * mul) >> (32 + shift) for n < 2^31 (d = 1: mul = 0)
struct Divisor {
    uint32_t d, mul, shift;
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return mul ? __umulhi(n, mul) >> shift : n; }
};

// mul = ceil(2^(32 + shift) / d) with 2^shift < d <= 2^(shift + 1) is below 2^32 and off by e < d; n e / (d 2^(32 + shift)) < 1 / d for n < 2^31
inline Divisor divisor(uint32_t d)
{
    Divisor r = {d, 0, 0};
    if (d <= 1) return r;
    while ((2ull << r.shift) < d) ++r.shift;
    r.mul = (uint32_t)(((1ull << (32 + r.shift)) + d - 1) / d);
    return r;
}

template <uint32_t FIXED>
struct LineK {
    static constexpr uint32_t kFixed = FIXED;   // places before a segment's first tile
    const int32_t* table;
    const int32_t* lens;
    const uint32_t* units;
    uint32_t* counts;        // [batch * heads] tiles to read, where a bitmap says which
    uint64_t unit_words;     // words of the bitmap
    uint32_t batch, queries;
    Divisor heads, group;
    uint32_t rows;           // query rows of a kv-head
    Divisor segs;            // segments of a kv-head
    Divisor page_tiles;
    uint32_t table_pages, pages;
    uint32_t unit, row_units;
    uint32_t ctas, least;    // CTAs of the launch, and the least tiles worth one
    void* out;
    float* lse;
    float* weights;
    float* part;             // [slots][rows of a segment][D] sums of a CTA's share of a segment
    float2* ml;              // [slots][rows] their maximum and their sum of weights
    float* mass;             // [batch * heads][segments of a head][blocks of `sub` tokens][rows] log2 of the weight before the division
    uint64_t row_subs;       // blocks of `sub` tokens of a table row
    uint32_t sub;            // tokens per block of `mass`: min(unit, 16); 0: no weights asked for
    uint32_t unit_log2;      // of a unit of at most 16 tokens; 4 for larger ones
    bool warp_rows;          // segments have few parts: a warp joins a row, not a CTA
};

template <class P>
__device__ __forceinline__ uint32_t length_of(const P& p, uint32_t b)
{
    const int64_t most = (int64_t)p.table_pages * p.page_tiles.d * kTileTokens;
    const int64_t n = __ldg(p.lens + b);
    return (uint32_t)(n < 0 ? 0 : n > most ? most : n);
}
__device__ __forceinline__ uint32_t tiles_of(uint32_t tokens) { return (tokens + kTileTokens - 1) / kTileTokens; }

// The kernels of a call follow each other closely: the next one's CTAs come up while the last ones of this one work, and wait
// here until all of it is done and visible. No CTA ends without having waited: what comes after a call in its stream starts when the last
// kernel has ended, and that must not be before the one in front of it.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// 32 bits of the bitmap from bit `at` on; bits behind its end read as 0
template <class P>
__device__ __forceinline__ uint32_t bits_at(const P& p, uint64_t at)
{
    const uint64_t w = at >> 5;
    const uint32_t lo = w < p.unit_words ? __ldg(p.units + w) : 0u, sh = (uint32_t)at & 31u;
    if (!sh) return lo;
    const uint32_t hi = w + 1 < p.unit_words ? __ldg(p.units + w + 1) : 0u;
    return __funnelshift_r(lo, hi, sh);
}

// The units 32 w .. 32 w + 31 of a row that are to be read, of those that hold one of the first `len` tokens. Units smaller than a
// tile are put together: bit i (a multiple of 16 / unit) stands for a tile.
template <class P>
__device__ __forceinline__ uint32_t unit_word(const P& p, uint32_t bh, uint32_t w, uint32_t units)
{
    uint32_t x = bits_at(p, (uint64_t)bh * p.row_units + 32ull * w);
    const uint32_t left = units - 32u * w;                  // 32 w < units
    if (left < 32u) x &= (1u << left) - 1u;
    if (p.unit < kTileTokens) {
        for (uint32_t k = 1; k < kTileTokens / p.unit; k <<= 1) x |= x >> k;
        x &= p.unit == 1 ? 0x00010001u : p.unit == 2 ? 0x01010101u : p.unit == 4 ? 0x11111111u : 0x55555555u;
    }
    return x;
}
template <class P>
__device__ __forceinline__ uint32_t units_of(const P& p, uint32_t len) { return (len + p.unit - 1) / p.unit; }

// is the tile read for a sequence of `len` tokens, as far as that does not depend on a bitmap
template <class P>
__device__ __forceinline__ bool tile_seen(const P&, uint32_t, uint32_t) { return true; }

// The line of all tiles. An entry is a sequence (no bitmap) or a (sequence, kv-head) pair; the `per` segments of an entry have
// the same number of tiles. A segment with tiles takes kFixed places before its first one: what a CTA spends on a segment whatever
// its length (queries, the first tiles' way from memory, the join) is that of kFixed tiles about. CTA c works on the tiles at places
// c * chunk .. c * chunk + chunk - 1.

struct Line {
    uint32_t before, total;  // places before the entry asked for, and of all
    uint32_t chunk;
    uint32_t count;          // tiles of a segment of that entry
};
template <class P>
__device__ __forceinline__ uint32_t entry_count(const P& p, uint32_t e) { return p.units ? p.counts[e] : tiles_of(length_of(p, e)); }
template <class P>
__device__ __forceinline__ uint32_t line_entries(const P& p) { return p.units ? p.batch * p.heads.d : p.batch; }
template <class P>
__device__ __forceinline__ uint32_t line_per(const P& p) { return p.units ? p.segs.d : p.segs.d * p.heads.d; }
template <class P>
__device__ __forceinline__ uint32_t places_of(uint32_t count, uint32_t per) { return count ? (count + P::kFixed) * per : 0u; }
template <class P>
__device__ __forceinline__ uint32_t entry_places(const P& p, uint32_t e, uint32_t per)
{
    return places_of<P>(entry_count(p, e), per);
}
__device__ __forceinline__ uint32_t sum_upto(uint32_t x, uint32_t lane)       // over the lanes up to this one
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= (uint32_t)o) x += v;
    }
    return x;
}

struct LineSmem {
    uint32_t warp[20], before, entry;
};

// Every thread of the CTA calls it. With a CTA's number: the entry in which its part begins (`entry`; only if it has a part) and the places
// before that entry. With cta = ~0: the places before `entry`. Up to 128 entries every warp goes through them by itself (one load's
// latency, no barrier), more of them are split over the CTA.
template <uint32_t THREADS = kThreads, class P>
__device__ __forceinline__ Line find_in_line(const P& p, uint32_t cta, uint32_t& entry, LineSmem& sm)
{
    const uint32_t E = line_entries(p), per = line_per(p), tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    Line line;
    if (E <= 128) {
        uint32_t c[4], n[4], upto[4], base = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = 32 * i + lane < E ? entry_count(p, 32 * i + lane) : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = places_of<P>(c[i], per);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            upto[i] = 0;
            if (32 * i < (int)E) {
                upto[i] = base + sum_upto(n[i], lane);
                base = __shfl_sync(0xFFFFFFFFu, upto[i], 31);
            }
        }
        line.total = base;
        line.chunk = max((base + p.ctas - 1) / p.ctas, p.least);
        line.before = line.count = 0;
        const uint64_t at = (uint64_t)line.chunk * cta;
        bool found = false;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (32 * i < (int)E && !found) {
                const uint32_t here = __ballot_sync(0xFFFFFFFFu, cta == ~0u ? 32 * i + lane == entry : at < upto[i] && n[i]);
                if (here) {
                    const int l = __ffs(here) - 1;
                    line.before = __shfl_sync(0xFFFFFFFFu, upto[i] - n[i], l);
                    line.count = __shfl_sync(0xFFFFFFFFu, c[i], l);
                    if (cta != ~0u) entry = 32 * i + l;
                    found = true;
                }
            }
        return line;
    }
    const uint32_t each = (E + THREADS - 1) / THREADS, first = min(tid * each, E), last = min(first + each, E);
    uint32_t mine = 0;
    for (uint32_t e = first; e < last; ++e) mine += entry_places(p, e, per);
    const uint32_t upto = sum_upto(mine, lane);
    if (lane == 31) sm.warp[warp] = upto;
    __syncthreads();
    uint32_t base = 0, total = 0;
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 32; ++w) {
        if (w < warp) base += sm.warp[w];
        total += sm.warp[w];
    }
    line.total = total;
    line.chunk = max((total + p.ctas - 1) / p.ctas, p.least);
    uint32_t before = base + upto - mine;
    if (cta == ~0u) {
        if (first <= entry && entry < last) {
            for (uint32_t e = first; e < entry; ++e) before += entry_places(p, e, per);
            sm.before = before;
        }
    } else {
        const uint64_t at = (uint64_t)line.chunk * cta;
        if (before <= at && at < (uint64_t)before + mine) {
            uint32_t e = first;
            for (;; ++e) {
                const uint32_t n = entry_places(p, e, per);
                if (at < (uint64_t)before + n) break;
                before += n;
            }
            sm.before = before;
            sm.entry = e;
        }
    }
    __syncthreads();
    line.before = sm.before;
    if (cta != ~0u) entry = sm.entry;
    if (cta == ~0u || (uint64_t)line.chunk * cta < total) line.count = entry_count(p, entry);
    return line;
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float log2_fast(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t bits_of(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 half2_of(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t pack(float lo, float hi) { return bits_of(__floats2half2_rn(lo, hi)); }
template <bool HALF>
__device__ __forceinline__ uint32_t out_pair(float a, float b)
{
    if (HALF) return pack(a, b);
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// Joins the parts of segments that several CTAs worked on, and turns the blocks' masses into weights.
// Blocks 0 .. batch * heads * rows - 1: one query row each; or, where segments have few parts (warp_rows), blocks 0 .. batch * heads * segs * ROWS / 8 - 1:
// eight rows of a segment, a warp each. The rest: kThreads units of a (sequence, kv-head) each.
template <class P, int N, bool HALF, uint32_t ROWS>
__global__ void __launch_bounds__(kThreads) join_kernel(const P p)
{
    constexpr uint32_t D = 32 * N, kQuads = D / 4;                 // 16-byte pieces of a row
    constexpr uint32_t kOver = kQuads < 32 ? 32 / kQuads : 1;      // parts that a warp's lanes take at a time
    constexpr uint32_t kEach = kQuads > 32 ? kQuads / 32 : 1;      // pieces of a lane
    __shared__ LineSmem sm;
    __shared__ float lse2[64];
    __shared__ float4 sums[kWarps * kOver * kQuads];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid / 32, per = line_per(p);
    const uint32_t per_head = p.warp_rows ? p.segs.d * (ROWS / kWarps) : p.rows, out_blocks = p.batch * p.heads.d * per_head;
    const bool is_out = blockIdx.x < out_blocks;
    const uint32_t chunks = p.weights ? (p.row_units + kThreads - 1) / kThreads : 1;
    const uint32_t bh = is_out ? blockIdx.x / per_head : (blockIdx.x - out_blocks) / chunks;
    const uint32_t b = p.heads.of(bh), h = bh - b * p.heads.d;
    const uint32_t entry0 = p.units ? bh : b;
    uint32_t entry = entry0;
    if (p.units) wait_for_previous();                              // for the rows' counts; lengths were there before
    const Line line = find_in_line(p, ~0u, entry, sm);
    const uint32_t count = line.count;
    // the CTAs that worked on segment seg: first and last
    auto first_cta = [&](uint32_t seg) { return (line.before + (seg - entry0 * per) * (count + P::kFixed) + P::kFixed) / line.chunk; };
    auto last_cta = [&](uint32_t seg) { return (line.before + (seg - entry0 * per + 1) * (count + P::kFixed) - 1) / line.chunk; };
    // a warp joins the maxima and sums of a row's parts
    auto join_row = [&](uint32_t seg, uint32_t r, uint32_t c0, uint32_t c1, float& m, float& l) {
        m = kNone;
        l = 0.0f;
        for (uint32_t c = c0 + lane; c <= c1; c += 32) {
            const float2 x = p.ml[((uint64_t)c + seg) * ROWS + r];
            const float up = fmaxf(m, x.x);
            l = fmaf(l, exp2_fast(m - up), x.y * exp2_fast(x.x - up));
            m = up;
        }
        float top = m;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        l *= exp2_fast(m - top);
        m = top;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    };
    if (is_out && p.warp_rows) {
        const uint32_t row = (blockIdx.x - bh * per_head) * kWarps + warp, seg = bh * p.segs.d + row / ROWS, query = p.group.of(row);
        const uint64_t at = ((uint64_t)b * p.queries + query) * (p.heads.d * p.group.d) + h * p.group.d + (row - query * p.group.d);
        uint2* const out = reinterpret_cast<uint2*>(p.out) + at * kQuads;
        const bool mine = row < p.rows;
        if (!count && mine) {
            for (uint32_t c = lane; c < kQuads; c += 32) out[c] = make_uint2(0u, 0u);
            if (lane == 0 && p.lse) p.lse[at] = -INFINITY;
        }
        if (!p.units) wait_for_previous();
        if (!count || !mine) return;
        const uint32_t c0 = first_cta(seg), c1 = last_cta(seg), piece = lane % kQuads;
        if (c0 == c1) return;                                      // written by its one CTA
        float m, l;
        join_row(seg, row % ROWS, c0, c1, m, l);
        float4 sum[kEach];
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) sum[j] = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (uint32_t c = c0 + lane / kQuads; c <= c1; c += kOver) {
            const float k = exp2_fast(p.ml[((uint64_t)c + seg) * ROWS + row % ROWS].x - m);
#pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) {
                const float4 x = reinterpret_cast<const float4*>(p.part)[(((uint64_t)c + seg) * ROWS + row % ROWS) * kQuads + piece + 32 * j];
                sum[j].x = fmaf(x.x, k, sum[j].x);
                sum[j].y = fmaf(x.y, k, sum[j].y);
                sum[j].z = fmaf(x.z, k, sum[j].z);
                sum[j].w = fmaf(x.w, k, sum[j].w);
            }
        }
        if (kOver == 2) {
            __syncwarp();
            sum[0].x += __shfl_xor_sync(0xFFFFFFFFu, sum[0].x, 16);
            sum[0].y += __shfl_xor_sync(0xFFFFFFFFu, sum[0].y, 16);
            sum[0].z += __shfl_xor_sync(0xFFFFFFFFu, sum[0].z, 16);
            sum[0].w += __shfl_xor_sync(0xFFFFFFFFu, sum[0].w, 16);
        }
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j)
            if (lane < kQuads) out[piece + 32 * j] = make_uint2(out_pair<HALF>(sum[j].x * by, sum[j].y * by), out_pair<HALF>(sum[j].z * by, sum[j].w * by));
        if (lane == 0 && p.lse) p.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        return;
    }
    if (is_out) {
        const uint32_t row = blockIdx.x - bh * p.rows, r = row % ROWS, seg = bh * p.segs.d + row / ROWS, query = p.group.of(row);
        const uint64_t at = ((uint64_t)b * p.queries + query) * (p.heads.d * p.group.d) + h * p.group.d + (row - query * p.group.d);
        if (!count) {
            if (tid < kQuads) reinterpret_cast<uint2*>(p.out)[at * kQuads + tid] = make_uint2(0u, 0u);
            if (tid == 0 && p.lse) p.lse[at] = -INFINITY;
            if (!p.units) wait_for_previous();
            return;
        }
        const uint32_t c0 = first_cta(seg), c1 = last_cta(seg);
        if (!p.units) wait_for_previous();
        if (c0 == c1) return;                                      // written by its one CTA
        const uint32_t piece = lane % kQuads, own = c0 + warp * kOver + lane / kQuads;
        auto part = [&](uint32_t c, uint32_t j) {
            return reinterpret_cast<const float4*>(p.part)[(((uint64_t)c + seg) * ROWS + r) * kQuads + piece + 32 * j];
        };
        constexpr uint32_t kFirst = 5;                             // parts of this lane that are on their way while the maxima are joined
        float4 ahead[kFirst][kEach];
        float top[kFirst];
#pragma unroll
        for (uint32_t i = 0; i < kFirst; ++i) {
            const uint32_t c = own + i * kWarps * kOver, at = min(c, c1);
            top[i] = p.ml[((uint64_t)at + seg) * ROWS + r].x;
            if (c > c1) top[i] = -INFINITY;
#pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) ahead[i][j] = part(at, j);
        }
        float m, l;
        join_row(seg, r, c0, c1, m, l);
        float4 sum[kEach];
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) sum[j] = make_float4(0, 0, 0, 0);
        auto add = [&](float4& to, const float4& x, float k) {
            to.x = fmaf(x.x, k, to.x);
            to.y = fmaf(x.y, k, to.y);
            to.z = fmaf(x.z, k, to.z);
            to.w = fmaf(x.w, k, to.w);
        };
#pragma unroll
        for (uint32_t i = 0; i < kFirst; ++i)
            if (own + i * kWarps * kOver <= c1) {
                const float k = exp2_fast(top[i] - m);
#pragma unroll
                for (uint32_t j = 0; j < kEach; ++j) add(sum[j], ahead[i][j], k);
            }
        for (uint32_t c = own + kFirst * kWarps * kOver; c <= c1; c += kWarps * kOver) {
            const float k = exp2_fast(p.ml[((uint64_t)c + seg) * ROWS + r].x - m);
#pragma unroll
            for (uint32_t j = 0; j < kEach; ++j) add(sum[j], part(c, j), k);
        }
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) sums[(warp * kOver + lane / kQuads) * kQuads + piece + 32 * j] = sum[j];
        __syncthreads();
        if (tid < kQuads) {
            float4 x = sums[tid];
#pragma unroll
            for (uint32_t i = 1; i < kWarps * kOver; ++i) {
                const float4 y = sums[i * kQuads + tid];
                x.x += y.x;
                x.y += y.y;
                x.z += y.z;
                x.w += y.w;
            }
            const float by = l == 0.0f ? 0.0f : 1.0f / l;
            reinterpret_cast<uint2*>(p.out)[at * kQuads + tid] = make_uint2(out_pair<HALF>(x.x * by, x.y * by), out_pair<HALF>(x.z * by, x.w * by));
            if (tid == 0 && p.lse) p.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
        return;
    }
    const uint32_t unit = (blockIdx.x - out_blocks - bh * chunks) * kThreads + tid;
    const uint32_t len = length_of(p, b);
    const uint64_t base = (uint64_t)unit * p.unit;
    bool read = unit < p.row_units && base < len && count;
    if (read && p.units) read = bits_at(p, (uint64_t)bh * p.row_units + unit) & 1u;
    if (!__syncthreads_or(read)) {                                 // none of these units is read
        if (unit < p.row_units) p.weights[(uint64_t)bh * p.row_units + unit] = 0.0f;
        if (!p.units) wait_for_previous();
        return;
    }
    if (!p.units) wait_for_previous();
    float got = 0.0f;
    for (uint32_t row0 = 0; row0 < p.rows; row0 += 64) {           // rows in turns of 64
        const uint32_t rows = min(p.rows - row0, 64u), padded = (rows + 7) / 8 * 8;
        __syncthreads();
        for (uint32_t i = warp; i < padded; i += kWarps) {         // a warp joins a row's sums
            float m = kNone, l = 0.0f;
            if (count && i < rows) {
                const uint32_t seg = bh * p.segs.d + (row0 + i) / ROWS;
                join_row(seg, (row0 + i) % ROWS, first_cta(seg), last_cta(seg), m, l);
            }
            if (lane == 0) lse2[i] = l == 0.0f ? INFINITY : m + log2f(l);
        }
        __syncthreads();
        if (!read) continue;
        const uint64_t last = min((uint64_t)len, base + p.unit);
        for (uint64_t i = base; i < last; i += p.sub) {
            const uint32_t tile = (uint32_t)(i / kTileTokens);
            const int32_t page = __ldg(p.table + (uint64_t)b * p.table_pages + p.page_tiles.of(tile));
            if (page < 0 || (uint32_t)page >= p.pages || !tile_seen(p, len, tile)) continue;
            for (uint32_t r = 0; r < rows; r += 8) {               // a segment's rows lie together; rows that are none have 0
                const float4* x = reinterpret_cast<const float4*>(p.mass + (((uint64_t)bh * p.segs.d + (row0 + r) / ROWS) * p.row_subs + (i >> (p.unit_log2 < 4 ? p.unit_log2 : 4))) * ROWS + (row0 + r) % ROWS);
                const float4 lo = x[0], hi = x[1];
                got += exp2_fast(lo.x - lse2[r]) + exp2_fast(lo.y - lse2[r + 1]) + exp2_fast(lo.z - lse2[r + 2]) + exp2_fast(lo.w - lse2[r + 3]) +
                       exp2_fast(hi.x - lse2[r + 4]) + exp2_fast(hi.y - lse2[r + 5]) + exp2_fast(hi.z - lse2[r + 6]) + exp2_fast(hi.w - lse2[r + 7]);
            }
        }
    }
    if (unit < p.row_units) p.weights[(uint64_t)bh * p.row_units + unit] = got;
}

inline uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }

// `chained`: waits by itself for the end of the kernel before it in the stream, so that it may come up while that one works
template <typename... A>
int launch(void (*kernel)(A...), uint32_t grid, uint32_t threads, uint32_t smem, bool chained, cudaStream_t st, const A&... k)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(grid);
    c.blockDim = dim3(threads);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute a;
    a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &a;
    c.numAttrs = chained ? 1 : 0;
    KVP_CUDA(cudaLaunchKernelEx(&c, kernel, k...));
    return KVP_OK;
}

}  // namespace kvp
