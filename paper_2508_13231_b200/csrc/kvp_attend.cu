// Attention over the cache held in 4 bits, for the last few tokens of each sequence, and the weight that every unit of the
// cache received (include/kvp.h, kvp_attend).
//
// Per query row r (a query token and a query head), over the tokens i that it sees:
//   s_i = scale * q . k_i,  p_i = exp(s_i - lse),  lse = log sum_i exp(s_i),  out = sum_i p_i v_i,
//   weights[unit] = sum over the rows of a kv-head and the tokens of the unit of p_i.
//
// Products. Up to eight rows that share a kv-head are one segment; the matrix instruction m16n8k16 takes 16 tokens x 16 dims of
// keys as its left operand and the rows as its right one, so that no row is padding where eight heads share a kv-head.
// (tcgen05.mma wants 64 or 128 rows of the left operand and 8 columns would use it no better; what bounds this kernel is memory.)
// The 4-bit whole numbers enter as fp16 subnormals (bits 0-3 of a half-word are q 2^-24, bits 4-7 are q 2^-20), which costs one
// AND for two numbers and no conversion; their products with fp16 queries are exact and summed in fp32. Scales act on the sums of
// 32 dims in fp32, the zeros on the sums of the query's dims, which enter as two fp16 terms (22 bits). A row's queries are divided by a power
// of two first, so that bf16 ones fit fp16 whatever their size.
// exp runs in fp32 against a running maximum that moves only when a score passes it by 2^8 (rare), sums are fp32. The weights p
// times the scales of the values are the second product's right operand, in fp16 (11 bits, half a step is 2^-12 of a weight; the
// output has 8 or 11 bits); the scales are divided by a running power of two so that small values lose nothing.
//
// Split. The tiles (16 tokens) of all segments stand in one line that is cut into equal parts, one for each CTA, on the device,
// where the lengths are known: any mix of lengths, and rows of a bitmap with any number of units, keep all SMs busy alike. A CTA
// takes a segment's tiles in turn by its eight warps, which join their sums in shared memory; segments that more than one
// CTA worked on are joined by the second kernel, which also turns what was noted per unit into weights. The order of every sum is
// fixed, so results do not change from run to run.
#include <cuda_bf16.h>

#include "kvp_tile.cuh"

namespace kvp {

namespace {

constexpr int kWarps = 8;
constexpr uint32_t kThreads = kWarps * 32;
constexpr uint32_t kRows = 8;                 // query rows of a segment
constexpr uint32_t kListCap = 1024;           // tiles of a bitmap row that are listed at a time
constexpr float kNone = -3e38f;               // maximum of nothing
constexpr float kLift = 3.0f, kSlack = 8.0f;  // weights are at most 2^(kLift + kSlack), 2^kLift right after the maximum moved

struct AttendK {
    const void* q;
    void* out;
    float* lse;
    float* weights;
    const uint8_t* cache;
    const int32_t* table;
    const int32_t* lens;
    const uint32_t* units;
    float* part;             // [slots][8][D] sums of a CTA's share of a segment
    float2* ml;              // [slots][8] their maximum and their sum of weights
    float* mass;             // [batch * heads][segments of a head][blocks of `sub` tokens][8] log2 of the weight before the division
    uint32_t* counts;        // [batch * heads] tiles to read, where a bitmap says which
    int64_t q_batch, q_query, q_head;
    uint64_t unit_words;     // words of the bitmap
    uint64_t row_subs;       // blocks of `sub` tokens of a table row
    uint32_t batch, queries, heads, group;
    uint32_t rows, segs;     // query rows of a kv-head, segments of a kv-head
    uint32_t page_tiles, table_pages, pages;
    uint32_t unit, row_units;
    uint32_t sub;            // tokens per block of `mass`: min(unit, 16)
    uint32_t ctas, least;    // CTAs of the launch, and the least tiles worth one
    float scale;
    bool bf16;
};

__device__ __forceinline__ uint32_t length_of(const AttendK& p, uint32_t b)
{
    const int64_t most = (int64_t)p.table_pages * p.page_tiles * kTileTokens;
    const int64_t n = __ldg(p.lens + b);
    return (uint32_t)(n < 0 ? 0 : n > most ? most : n);
}
__device__ __forceinline__ uint32_t tiles_of(uint32_t tokens) { return (tokens + kTileTokens - 1) / kTileTokens; }

// 32 bits of the bitmap from bit `at` on; bits behind its end read as 0
__device__ __forceinline__ uint32_t bits_at(const AttendK& p, uint64_t at)
{
    const uint64_t w = at >> 5;
    const uint32_t lo = w < p.unit_words ? __ldg(p.units + w) : 0u, sh = (uint32_t)at & 31u;
    if (!sh) return lo;
    const uint32_t hi = w + 1 < p.unit_words ? __ldg(p.units + w + 1) : 0u;
    return __funnelshift_r(lo, hi, sh);
}

// which of the tiles 32 w .. 32 w + 31 of row bh hold a token that is to be read
__device__ uint32_t tile_word(const AttendK& p, uint32_t bh, uint32_t w, uint32_t tiles)
{
    const uint64_t row = (uint64_t)bh * p.row_units;
    uint32_t bits = 0;
    if (p.unit == kTileTokens) {
        bits = bits_at(p, row + 32ull * w);
    } else if (p.unit < kTileTokens) {
        const uint32_t k = kTileTokens / p.unit, mask = (1u << k) - 1u;
        for (uint32_t i = 0; i < 32; i += 32 / k) {
            const uint32_t x = bits_at(p, row + (32ull * w + i) * k);
            for (uint32_t j = 0; j < 32 / k; ++j) bits |= (uint32_t)(((x >> (j * k)) & mask) != 0) << (i + j);
        }
    } else {
        const uint32_t k = p.unit / kTileTokens, first = 32u * w / k;
        const uint32_t x = bits_at(p, row + first);
        for (uint32_t i = 0; i < 32; ++i) bits |= ((x >> ((32u * w + i) / k - first)) & 1u) << i;
    }
    const uint32_t left = tiles > 32u * w ? tiles - 32u * w : 0u;
    return left >= 32u ? bits : bits & ((1u << left) - 1u);
}

// counts[bh]: one warp per row of the bitmap
__global__ void __launch_bounds__(kThreads) count_kernel(const AttendK p)
{
    const uint32_t bh = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (bh >= p.batch * p.heads) return;
    const uint32_t tiles = tiles_of(length_of(p, bh / p.heads));
    uint32_t n = 0;
    for (uint32_t w = lane; 32u * w < tiles; w += 32) n += __popc(tile_word(p, bh, w, tiles));
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    if (lane == 0) p.counts[bh] = n;
}

// The line of all tiles. An entry is a sequence (no bitmap) or a (sequence, kv-head) pair; the `per` segments of an entry have
// the same number of tiles.
struct Line {
    uint64_t before, total;  // tiles before the entry asked for, and of all
    uint32_t active;         // CTAs that get a part
};
__device__ __forceinline__ uint32_t entry_count(const AttendK& p, uint32_t e) { return p.units ? p.counts[e] : tiles_of(length_of(p, e)); }
__device__ __forceinline__ uint32_t line_entries(const AttendK& p) { return p.units ? p.batch * p.heads : p.batch; }
__device__ __forceinline__ uint32_t line_per(const AttendK& p) { return p.units ? p.segs : p.segs * p.heads; }

struct LineSmem {
    uint64_t warp[32], total, before;
    uint32_t entry;
};

// Every thread of the CTA calls it. `at`: a place in the line as a fraction of the CTAs (part `cta` of `active`), returned as the
// entry there and the tiles before it; or, with cta = ~0, the place of entry `entry`.
__device__ Line find_in_line(const AttendK& p, uint32_t cta, uint32_t& entry, LineSmem& sm)
{
    const uint32_t E = line_entries(p), per = line_per(p), tid = threadIdx.x, T = blockDim.x, lane = tid % 32, warp = tid / 32;
    const uint32_t chunk = (E + T - 1) / T, first = min(tid * chunk, E), last = min(first + chunk, E);
    uint64_t mine = 0;
    for (uint32_t e = first; e < last; ++e) mine += (uint64_t)entry_count(p, e) * per;
    uint64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= (uint32_t)o) upto += v;
    }
    if (lane == 31) sm.warp[warp] = upto;
    __syncthreads();
    uint64_t base = 0, total = 0;
    for (uint32_t w = 0; w < T / 32; ++w) {
        if (w < warp) base += sm.warp[w];
        total += sm.warp[w];
    }
    Line line;
    line.total = total;
    const uint64_t worth = (total + p.least - 1) / p.least;
    line.active = worth < p.ctas ? (uint32_t)worth : p.ctas;
    uint64_t before = base + upto - mine;
    if (cta == ~0u) {
        if (first <= entry && entry < last) {
            for (uint32_t e = first; e < entry; ++e) before += (uint64_t)entry_count(p, e) * per;
            sm.before = before;
        }
    } else if (cta < line.active) {
        const uint64_t at = total * cta / line.active;
        if (before <= at && at < before + mine) {
            uint32_t e = first;
            for (;; ++e) {
                const uint64_t n = (uint64_t)entry_count(p, e) * per;
                if (at < before + n) break;
                before += n;
            }
            sm.before = before;
            sm.entry = e;
        }
    }
    __syncthreads();
    line.before = sm.before;
    if (cta != ~0u) entry = sm.entry;
    return line;
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) { return bits_of(__hmul2(half2_of(a), half2_of(b))); }
__device__ __forceinline__ float over_rows(float x)                 // sum over the lanes that hold other tokens of the same rows
{
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
    return x + __shfl_xor_sync(0xFFFFFFFFu, x, 16);
}

__device__ __forceinline__ float load_q(const AttendK& p, int64_t at)
{
    return p.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[at]) : __half2float(static_cast<const __half*>(p.q)[at]);
}
__device__ __forceinline__ void store_out(const AttendK& p, uint64_t at, float x)
{
    if (p.bf16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(x);
    else static_cast<__half*>(p.out)[at] = __float2half_rn(x);
}

template <int N>
struct Shape {
    static constexpr int kStages = N == 2 ? 8 : 4;                  // tiles of a warp under way
    static constexpr uint32_t kRing = kWarps * kStages * Tile<N>::kBytes;
    static constexpr uint32_t kJoin = kWarps * kRows * 32 * N * 4;
    static constexpr uint32_t kSmem = kRing > kJoin ? kRing : kJoin;
};

struct AttendSmem {
    LineSmem line;
    uint32_t list[kListCap];
    uint32_t scan[kWarps];
    float2 ml[kWarps][kRows];
};

// list[i] = number of the (from + i)-th tile of row bh that is to be read, i < many <= kListCap. Every thread of the CTA calls it.
__device__ void list_tiles(const AttendK& p, uint32_t bh, uint32_t tiles, uint32_t from, uint32_t many, AttendSmem& sm)
{
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    uint32_t seen = 0;
    for (uint32_t w0 = 0; 32u * w0 < tiles && seen < from + many; w0 += kThreads) {
        const uint32_t w = w0 + tid;
        uint32_t bits = 32u * w < tiles ? tile_word(p, bh, w, tiles) : 0u;
        uint32_t upto = __popc(bits);
        const uint32_t mine = upto;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= (uint32_t)o) upto += v;
        }
        if (lane == 31) sm.scan[warp] = upto;
        __syncthreads();
        uint32_t at = seen + upto - mine;
        for (uint32_t i = 0; i < (uint32_t)kWarps; ++i) {
            const uint32_t n = sm.scan[i];
            if (i < warp) at += n;
            seen += n;
        }
        for (; bits; bits &= bits - 1u, ++at)
            if (at >= from && at - from < many) sm.list[at - from] = 32u * w + __ffs(bits) - 1u;
        __syncthreads();
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads, N == 8 ? 1 : 2) attend_kernel(const AttendK p)
{
    using L = Tile<N>;
    using S = Shape<N>;
    constexpr int kStages = S::kStages;
    extern __shared__ __align__(16) uint8_t ring_all[];
    __shared__ AttendSmem sm;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, g = lane >> 2, t = lane & 3;
    uint32_t entry = 0;
    const Line line = find_in_line(p, blockIdx.x, entry, sm.line);
    if (blockIdx.x >= line.active) return;
    uint64_t todo = line.total * (blockIdx.x + 1) / line.active - line.total * blockIdx.x / line.active;
    const uint32_t per = line_per(p), E = line_entries(p);
    uint64_t skip = line.total * blockIdx.x / line.active - line.before;
    uint32_t count = entry_count(p, entry), inner = (uint32_t)(skip / count), off = (uint32_t)(skip % count);
    uint8_t* const ring = ring_all + warp * kStages * L::kBytes;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    // a fragment's row g is token 4 (g / 2) + g % 2 of the tile, its row g + 8 the token two further on: a thread then needs the
    // values of the four tokens 4 t .. 4 t + 3
    const uint32_t tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;

    while (todo) {
        while (inner == per || !count) {
            if (++entry >= E) return;                              // not reached: the line ends with the last part
            count = entry_count(p, entry);
            inner = 0;
        }
        const uint32_t seg = entry * per + inner, bh = seg / p.segs, rt = seg % p.segs, b = bh / p.heads, h = bh % p.heads;
        const uint32_t take = (uint32_t)(todo < count - off ? todo : count - off);
        const uint32_t len = length_of(p, b), tiles = tiles_of(len);
        const int32_t* table = p.table + (uint64_t)b * p.table_pages;

        // queries: this thread's part of row g as the right operand, divided by a power of two; sums over groups for the zeros
        uint32_t qf[N][4], qz[2];
        float f0, f1;
        {
            const uint32_t r = rt * kRows + g;
            const bool real = r < p.rows;
            const int64_t at = real ? b * p.q_batch + (int64_t)(r / p.group) * p.q_query + (int64_t)(h * p.group + r % p.group) * p.q_head : 0;
            float x[N][8], most = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[n][i] = real ? load_q(p, at + n * 32 + t * 8 + i) : 0.0f;
                    most = fmaxf(most, fabsf(x[n][i]));
                }
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            const int e = most > 0.0f && most < INFINITY ? ilogbf(most) - 9 : 0;     // largest magnitude in [2^9, 2^10)
            float sums[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[n][i] = scalbnf(x[n][i], -e);
                    sum += x[n][i];
                }
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
                sums[n] = sum + __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
                qf[n][0] = pack(x[n][0], x[n][4]);
                qf[n][1] = pack(x[n][1] * 0.0625f, x[n][5] * 0.0625f);
                qf[n][2] = pack(x[n][2], x[n][6]);
                qf[n][3] = pack(x[n][3] * 0.0625f, x[n][7] * 0.0625f);
            }
            // columns of the zeros' product: the sums' upper parts, then what they leave
            float col[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = 2 * t + (i & 1) + 8 * (i >> 1);       // column of the operand
                float v = 0.0f;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const float up = __half2float(__float2half_rn(sums[n]));
                    if (c == (uint32_t)n) v = up;
                    if (c == (uint32_t)(N + n)) v = sums[n] - up;
                }
                col[i] = v;
            }
            qz[0] = pack(col[0], col[1]);
            qz[1] = pack(col[2], col[3]);
            const float f = scalbnf(p.scale * 1.4426950408889634f, e);
            f0 = __shfl_sync(0xFFFFFFFFu, f, 8 * t);
            f1 = __shfl_sync(0xFFFFFFFFu, f, 8 * t + 4);
        }
        // rows 2 t and 2 t + 1 see the tokens before these
        int32_t see0, see1, all;
        {
            const int32_t first = (int32_t)len - (int32_t)p.queries + 1;
            see0 = first + (int32_t)((rt * kRows + 2 * t) / p.group);
            see1 = first + (int32_t)((rt * kRows + 2 * t + 1) / p.group);
            see0 = min(see0, (int32_t)len);
            see1 = min(see1, (int32_t)len);
            all = min(first + (int32_t)(rt * kRows / p.group), (int32_t)len);
        }

        float o[2 * N][4], zsum[4] = {0, 0, 0, 0}, m0 = kNone, m1 = kNone, l0 = 0.0f, l1 = 0.0f;
        int ev = -14;                                              // the values' scales are divided by 2^ev
        uint32_t shrink = 0x74007400u;                             // 2^-ev, twice
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;

        for (uint32_t done = 0; done < take;) {
            const uint32_t many = p.units ? min(take - done, kListCap) : take;
            if (p.units) {
                __syncthreads();
                list_tiles(p, bh, tiles, off + done, many, sm);
            }
            const uint32_t mine = many > warp ? (many - warp + kWarps - 1) / kWarps : 0;      // this warp's tiles
            auto tile_no = [&](uint32_t k) { const uint32_t i = warp + k * kWarps; return p.units ? sm.list[i] : off + i; };
            int32_t page = -1;
            uint32_t in_page = 0, bad = 0;
            auto issue = [&](uint32_t k) {
                if (k < mine) {
                    if (k % 32 == 0) {                             // the pages of the next 32 tiles, one a lane
                        page = -1;
                        if (k + lane < mine) {
                            const uint32_t tile = tile_no(k + lane);
                            page = __ldg(table + tile / p.page_tiles);
                            in_page = tile % p.page_tiles;
                        }
                    }
                    const int32_t pg = __shfl_sync(0xFFFFFFFFu, page, k % 32);
                    const uint32_t ip = __shfl_sync(0xFFFFFFFFu, in_page, k % 32), stage = k % kStages;
                    if (pg >= 0 && (uint32_t)pg < p.pages) {
                        const uint8_t* from = p.cache + (((uint64_t)pg * p.heads + h) * p.page_tiles + ip) * L::kBytes;
#pragma unroll
                        for (uint32_t c = 0; c < L::kBytes / 16; c += 32)
                            if (L::kBytes / 16 - c >= 32 || lane < L::kBytes / 16 - c)
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring_at + stage * L::kBytes + (c + lane) * 16),
                                             "l"(from + (c + lane) * 16) : "memory");
                        bad &= ~(1u << stage);
                    } else {
                        bad |= 1u << stage;
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll 1
            for (int k = 0; k < kStages - 1; ++k) issue(k);
#pragma unroll 1
            for (uint32_t k = 0; k < mine; ++k) {
                __syncwarp();                                      // the stage written next was read by all lanes
                issue(k + kStages - 1);
                asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
                __syncwarp();
                if ((bad >> (k % kStages)) & 1u) continue;         // a page that is none: its tokens are not read
                const uint8_t* tile = ring + (k % kStages) * L::kBytes;
                const uint32_t no = tile_no(k);
                const int32_t base = (int32_t)(no * kTileTokens);

                // scores of tokens a and b for rows 2t and 2t + 1
                float s[4] = {0, 0, 0, 0}, z[4] = {0, 0, 0, 0};
                {
                    uint32_t wa[N], wb[N];
                    __half sa[N], sb[N];
#pragma unroll
                    for (int n = 0; n < N; n += N < 4 ? 2 : 4) {
                        if constexpr (N < 4) {
                            *reinterpret_cast<uint2*>(wa) = *reinterpret_cast<const uint2*>(tile + L::key_word(tok_a, t, 0));
                            *reinterpret_cast<uint2*>(wb) = *reinterpret_cast<const uint2*>(tile + L::key_word(tok_b, t, 0));
                        } else {
                            *reinterpret_cast<uint4*>(wa + n) = *reinterpret_cast<const uint4*>(tile + L::key_word(tok_a, t, n));
                            *reinterpret_cast<uint4*>(wb + n) = *reinterpret_cast<const uint4*>(tile + L::key_word(tok_b, t, n));
                        }
                    }
#pragma unroll
                    for (int n = 0; n < N; n += 2) {
                        *reinterpret_cast<uint32_t*>(sa + n) = *reinterpret_cast<const uint32_t*>(tile + L::key_meta(tok_a, n));
                        *reinterpret_cast<uint32_t*>(sb + n) = *reinterpret_cast<const uint32_t*>(tile + L::key_meta(tok_b, n));
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        float acc[4] = {0, 0, 0, 0};
                        mma(acc, wa[n] & 0x000F000Fu, wb[n] & 0x000F000Fu, wa[n] & 0x00F000F0u, wb[n] & 0x00F000F0u, qf[n][0], qf[n][1]);
                        const uint32_t xa = wa[n] >> 8, xb = wb[n] >> 8;
                        mma(acc, xa & 0x000F000Fu, xb & 0x000F000Fu, xa & 0x00F000F0u, xb & 0x00F000F0u, qf[n][2], qf[n][3]);
                        const float fa = __half2float(sa[n]), fb = __half2float(sb[n]);
                        s[0] = fmaf(fa, acc[0], s[0]);
                        s[1] = fmaf(fa, acc[1], s[1]);
                        s[2] = fmaf(fb, acc[2], s[2]);
                        s[3] = fmaf(fb, acc[3], s[3]);
                    }
                    const uint32_t za = *reinterpret_cast<const uint32_t*>(tile + L::kKeyZero + tok_a * 2 * N + (2 * t % N) * 2);
                    const uint32_t zb = *reinterpret_cast<const uint32_t*>(tile + L::kKeyZero + tok_b * 2 * N + (2 * t % N) * 2);
                    const uint32_t zero = 0;
                    if constexpr (N == 8) mma(z, za, zb, za, zb, qz[0], qz[1]);
                    else mma(z, za, zb, zero, zero, qz[0], zero);
                }
                s[0] = f0 * fmaf(s[0], 16777216.0f, z[0]);
                s[1] = f1 * fmaf(s[1], 16777216.0f, z[1]);
                s[2] = f0 * fmaf(s[2], 16777216.0f, z[2]);
                s[3] = f1 * fmaf(s[3], 16777216.0f, z[3]);

                // scales and zeros of the values of tokens 4t .. 4t + 3
                uint32_t vs[N][2], vz0 = 0, vz1 = 0;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const uint2 x = *reinterpret_cast<const uint2*>(tile + L::value_meta(4 * t, n));
                    vs[n][0] = x.x;
                    vs[n][1] = x.y;
                }
                if (g < N) {
                    const uint2 x = *reinterpret_cast<const uint2*>(tile + L::value_meta(4 * t, g) + (L::kValueZero - L::kValueScale));
                    vz0 = x.x;
                    vz1 = x.y;
                }
                const bool parts = p.units && p.unit < kTileTokens;
                if (parts || base + (int32_t)kTileTokens > all) {
                    // some token is not seen by some row. What lies in the cache behind the last token may be anything, also
                    // infinite, so its scales and zeros are cleared too
                    uint32_t bits = ~0u;
                    if (parts) bits = bits_at(p, (uint64_t)bh * p.row_units + base / (int32_t)p.unit);
                    auto seen = [&](uint32_t i) { return base + (int32_t)i < (int32_t)len && (!parts || ((bits >> (i / p.unit)) & 1u)); };
                    const bool a = seen(tok_a), bb = seen(tok_b);
                    if (!a || base + (int32_t)tok_a >= see0) s[0] = -INFINITY;
                    if (!a || base + (int32_t)tok_a >= see1) s[1] = -INFINITY;
                    if (!bb || base + (int32_t)tok_b >= see0) s[2] = -INFINITY;
                    if (!bb || base + (int32_t)tok_b >= see1) s[3] = -INFINITY;
                    const uint32_t k0 = (seen(4 * t) ? 0xFFFFu : 0u) | (seen(4 * t + 1) ? 0xFFFF0000u : 0u);
                    const uint32_t k1 = (seen(4 * t + 2) ? 0xFFFFu : 0u) | (seen(4 * t + 3) ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int n = 0; n < N; ++n) { vs[n][0] &= k0; vs[n][1] &= k1; }
                    vz0 &= k0;
                    vz1 &= k1;
                }
                // has a score passed the maximum by more than the slack, or a scale its power of two?
                uint32_t top = __half2_raw(half2_of(vs[0][0])).x;
                {
                    __half2 v = __hmax2(half2_of(vs[0][0]), half2_of(vs[0][1]));
#pragma unroll
                    for (int n = 1; n < N; ++n) v = __hmax2(v, __hmax2(half2_of(vs[n][0]), half2_of(vs[n][1])));
                    top = __half_as_ushort(__hmax(__low2half(v), __high2half(v)));
                }
                const float t0 = fmaxf(s[0], s[2]), t1 = fmaxf(s[1], s[3]), vmost = __half2float(__ushort_as_half((unsigned short)top));
                const float vlimit = exp2f((float)(ev + 4));
                if (__any_sync(0xFFFFFFFFu, t0 > m0 + kSlack || t1 > m1 + kSlack || vmost > vlimit)) {
                    float n0 = t0, n1 = t1, nv = vmost;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        n0 = fmaxf(n0, __shfl_xor_sync(0xFFFFFFFFu, n0, d));
                        n1 = fmaxf(n1, __shfl_xor_sync(0xFFFFFFFFu, n1, d));
                    }
                    nv = fmaxf(nv, __shfl_xor_sync(0xFFFFFFFFu, nv, 1));
                    nv = fmaxf(nv, __shfl_xor_sync(0xFFFFFFFFu, nv, 2));
                    n0 = fmaxf(m0, n0);
                    n1 = fmaxf(m1, n1);
                    const int en = nv > 0.0f && nv < INFINITY ? max(ev, ilogbf(nv) + 1) : ev;
                    const float c0 = exp2_fast(m0 - n0), c1 = exp2_fast(m1 - n1), ce = exp2f((float)(ev - en));
                    m0 = n0;
                    m1 = n1;
                    ev = en;
                    shrink = bits_of(__float2half2_rn(exp2f((float)-ev)));
                    l0 *= c0;
                    l1 *= c1;
                    zsum[0] *= c0;
                    zsum[1] *= c1;
#pragma unroll
                    for (int i = 0; i < 2 * N; ++i) {
                        o[i][0] *= c0 * ce;
                        o[i][1] *= c1 * ce;
                        o[i][2] *= c0 * ce;
                        o[i][3] *= c1 * ce;
                    }
                }
                const float d0 = m0 - kLift, d1 = m1 - kLift;
                const float e0 = exp2_fast(s[0] - d0), e1 = exp2_fast(s[1] - d1), e2 = exp2_fast(s[2] - d0), e3 = exp2_fast(s[3] - d1);
                l0 += e0 + e2;
                l1 += e1 + e3;
                const uint32_t p0 = transposed(pack(e0, e1)), p1 = transposed(pack(e2, e3));

                // what each block of `sub` tokens received, as log2
                if (p.sub) {
                    float2* mass = reinterpret_cast<float2*>(p.mass) +
                                   (((uint64_t)bh * p.segs + rt) * p.row_subs + (uint64_t)base / p.sub) * (kRows / 2) + t;
                    if (p.sub == 1) {
                        mass[tok_a * (kRows / 2)] = make_float2(s[0], s[1]);
                        mass[tok_b * (kRows / 2)] = make_float2(s[2], s[3]);
                    } else if (p.sub == 2) {
                        float a0 = e0 + __shfl_xor_sync(0xFFFFFFFFu, e0, 4), a1 = e1 + __shfl_xor_sync(0xFFFFFFFFu, e1, 4);
                        float b0 = e2 + __shfl_xor_sync(0xFFFFFFFFu, e2, 4), b1 = e3 + __shfl_xor_sync(0xFFFFFFFFu, e3, 4);
                        if (!(g & 1)) {
                            mass[g * (kRows / 2)] = make_float2(d0 + log2_fast(a0), d1 + log2_fast(a1));
                            mass[(g + 1) * (kRows / 2)] = make_float2(d0 + log2_fast(b0), d1 + log2_fast(b1));
                        }
                    } else {
                        float a0 = e0 + e2, a1 = e1 + e3;
                        for (uint32_t d = 4; d < 2 * p.sub; d <<= 1) {
                            a0 += __shfl_xor_sync(0xFFFFFFFFu, a0, d);
                            a1 += __shfl_xor_sync(0xFFFFFFFFu, a1, d);
                        }
                        const uint32_t same = p.sub / 2;                   // rows g of one block
                        if (g % same == 0) mass[g / same * (kRows / 2)] = make_float2(d0 + log2_fast(a0), d1 + log2_fast(a1));
                    }
                }

                // values: dims 32 n + 4 g + {0, 2} in rows g, {1, 3} in rows g + 8 (16 times too large)
                const uint32_t zero = 0;
                mma(zsum, vz0, zero, vz1, zero, p0, p1);
                uint32_t x[N], y[N];
#pragma unroll
                for (int n = 0; n < N; n += N < 4 ? 2 : 4) {
                    if constexpr (N < 4) {
                        *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(tile + L::value_half(4 * t, g, 0));
                        *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(tile + L::value_half(4 * t + 2, g, 0));
                    } else {
                        *reinterpret_cast<uint4*>(x + n) = *reinterpret_cast<const uint4*>(tile + L::value_half(4 * t, g, n));
                        *reinterpret_cast<uint4*>(y + n) = *reinterpret_cast<const uint4*>(tile + L::value_half(4 * t + 2, g, n));
                    }
                }
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const uint32_t b0 = times(p0, times(vs[n][0], shrink)), b1 = times(p1, times(vs[n][1], shrink));
                    mma(o[2 * n], x[n] & 0x000F000Fu, x[n] & 0x00F000F0u, y[n] & 0x000F000Fu, y[n] & 0x00F000F0u, b0, b1);
                    const uint32_t xx = x[n] >> 8, yy = y[n] >> 8;
                    mma(o[2 * n + 1], xx & 0x000F000Fu, xx & 0x00F000F0u, yy & 0x000F000Fu, yy & 0x00F000F0u, b0, b1);
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            done += many;
        }

        // join the warps
        l0 = over_rows(l0);
        l1 = over_rows(l1);
        __syncthreads();                                           // every warp is done with its ring
        float* join = reinterpret_cast<float*>(ring_all);
        const float up = exp2f((float)(ev + 24)), up16 = exp2f((float)(ev + 20));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float z0 = __shfl_sync(0xFFFFFFFFu, zsum[0], n * 4 + t), z1 = __shfl_sync(0xFFFFFFFFu, zsum[1], n * 4 + t);
            float4 a, c;
            a.x = fmaf(o[2 * n][0], up, z0);
            a.y = fmaf(o[2 * n][2], up16, z0);
            a.z = fmaf(o[2 * n + 1][0], up, z0);
            a.w = fmaf(o[2 * n + 1][2], up16, z0);
            c.x = fmaf(o[2 * n][1], up, z1);
            c.y = fmaf(o[2 * n][3], up16, z1);
            c.z = fmaf(o[2 * n + 1][1], up, z1);
            c.w = fmaf(o[2 * n + 1][3], up16, z1);
            float* to = join + (warp * kRows + 2 * t) * L::D + n * 32 + g * 4;
            *reinterpret_cast<float4*>(to) = a;
            *reinterpret_cast<float4*>(to + L::D) = c;
        }
        if (g == 0) {
            sm.ml[warp][2 * t] = make_float2(m0 - kLift, l0);
            sm.ml[warp][2 * t + 1] = make_float2(m1 - kLift, l1);
        }
        __syncthreads();
        const bool whole = take == count;
        const uint64_t slot = (uint64_t)blockIdx.x + seg;
        for (uint32_t i = tid; i < kRows * L::D; i += kThreads) {
            const uint32_t r = i / L::D, d = i % L::D, row = rt * kRows + r;
            if (row >= p.rows) continue;
            float m = sm.ml[0][r].x;
#pragma unroll
            for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm.ml[w][r].x);
            float sum = 0.0f, l = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float c = exp2_fast(sm.ml[w][r].x - m);
                l = fmaf(sm.ml[w][r].y, c, l);
                sum = fmaf(join[(w * kRows + r) * L::D + d], c, sum);
            }
            if (d == 0) p.ml[slot * kRows + r] = make_float2(m, l);
            if (whole) {
                const uint64_t at = ((uint64_t)b * p.queries + row / p.group) * (p.heads * p.group) + h * p.group + row % p.group;
                store_out(p, at * L::D + d, l == 0.0f ? 0.0f : sum / l);
                if (d == 0 && p.lse) p.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            } else {
                p.part[(slot * kRows + r) * L::D + d] = sum;
            }
        }
        __syncthreads();                                           // the ring is free again
        todo -= take;
        off = 0;
        ++inner;
    }
}

// Joins the parts of segments that several CTAs worked on, and turns the blocks' masses into weights.
// Blocks 0 .. batch * heads * rows - 1: one query row each. The rest: kThreads units of a (sequence, kv-head) each.
template <int N>
__global__ void __launch_bounds__(kThreads) join_kernel(const AttendK p)
{
    constexpr uint32_t D = 32 * N;
    __shared__ LineSmem sm;
    __shared__ float lse2[64];
    __shared__ float2 ml[kThreads];
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, per = line_per(p);
    const uint64_t out_blocks = (uint64_t)p.batch * p.heads * p.rows;
    const bool is_out = blockIdx.x < out_blocks;
    const uint32_t chunks = p.weights ? (p.row_units + kThreads - 1) / kThreads : 1;
    const uint32_t bh = is_out ? blockIdx.x / p.rows : (uint32_t)((blockIdx.x - out_blocks) / chunks);
    const uint32_t b = bh / p.heads, h = bh % p.heads;
    const uint32_t entry0 = p.units ? bh : b;
    uint32_t entry = entry0;
    const Line line = find_in_line(p, ~0u, entry, sm);
    const uint32_t count = entry_count(p, entry0);
    // the CTAs that worked on segment seg: first and last
    auto cta_of = [&](uint64_t tile) { return (uint32_t)(((tile + 1) * line.active - 1) / line.total); };
    auto first_tile = [&](uint32_t seg) { return line.before + (uint64_t)(seg - entry0 * per) * count; };
    if (is_out) {
        const uint32_t row = blockIdx.x % p.rows, rt = row / kRows, r = row % kRows, seg = bh * p.segs + rt;
        const uint64_t at = ((uint64_t)b * p.queries + row / p.group) * (p.heads * p.group) + h * p.group + row % p.group;
        if (!count) {
            for (uint32_t d = tid; d < D; d += kThreads) store_out(p, at * D + d, 0.0f);
            if (tid == 0 && p.lse) p.lse[at] = -INFINITY;
            return;
        }
        const uint32_t c0 = cta_of(first_tile(seg)), c1 = cta_of(first_tile(seg) + count - 1);
        if (c0 == c1) return;                                      // written by its one CTA
        float m = kNone, l = 0.0f, sum = 0.0f;
        for (uint32_t c = c0; c <= c1; c += kThreads) {
            __syncthreads();
            if (c + tid <= c1) ml[tid] = p.ml[((uint64_t)c + tid + seg) * kRows + r];
            __syncthreads();
            const uint32_t many = min(c1 - c + 1, kThreads);
            float up = m;
            for (uint32_t i = 0; i < many; ++i) up = fmaxf(up, ml[i].x);
            const float old = exp2_fast(m - up);
            m = up;
            l *= old;
            sum *= old;
            for (uint32_t i = 0; i < many; ++i) {
                const float k = exp2_fast(ml[i].x - m);
                l = fmaf(ml[i].y, k, l);
                if (tid < D) sum = fmaf(p.part[(((uint64_t)c + i + seg) * kRows + r) * D + tid], k, sum);
            }
        }
        if (tid < D) store_out(p, at * D + tid, l == 0.0f ? 0.0f : sum / l);
        if (tid == 0 && p.lse) p.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        return;
    }
    const uint32_t unit = (uint32_t)((blockIdx.x - out_blocks) % chunks) * kThreads + tid;
    const uint32_t len = length_of(p, b);
    const uint64_t base = (uint64_t)unit * p.unit;
    bool read = unit < p.row_units && base < len && count;
    if (read && p.units) read = bits_at(p, (uint64_t)bh * p.row_units + unit) & 1u;
    float got = 0.0f;
    for (uint32_t row0 = 0; row0 < p.rows; row0 += 64) {           // rows in turns of 64
        const uint32_t rows = min(p.rows - row0, 64u);
        __syncthreads();
        for (uint32_t i = warp; i < rows; i += kWarps) {           // a warp joins a row's sums
            float m = kNone, l = 0.0f;
            if (count) {
                const uint32_t seg = bh * p.segs + (row0 + i) / kRows, r = (row0 + i) % kRows;
                const uint32_t c0 = cta_of(first_tile(seg)), c1 = cta_of(first_tile(seg) + count - 1);
                for (uint32_t c = c0 + lane; c <= c1; c += 32) {
                    const float2 x = p.ml[((uint64_t)c + seg) * kRows + r];
                    const float up = fmaxf(m, x.x);
                    l = fmaf(l, exp2_fast(m - up), x.y * exp2_fast(x.x - up));
                    m = up;
                }
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const float mo = __shfl_xor_sync(0xFFFFFFFFu, m, o), lo = __shfl_xor_sync(0xFFFFFFFFu, l, o);
                    const float up = fmaxf(m, mo);
                    l = l * exp2_fast(m - up) + lo * exp2_fast(mo - up);
                    m = up;
                }
            }
            if (lane == 0) lse2[i] = l == 0.0f ? INFINITY : m + log2f(l);
        }
        __syncthreads();
        if (!read) continue;
        const uint64_t last = min((uint64_t)len, base + p.unit);
        for (uint64_t i = base; i < last; i += p.sub) {
            const uint32_t tile = (uint32_t)(i / kTileTokens);
            const int32_t page = __ldg(p.table + (uint64_t)b * p.table_pages + tile / p.page_tiles);
            if (page < 0 || (uint32_t)page >= p.pages) continue;
            for (uint32_t r = 0; r < rows; ++r)
                got += exp2_fast(p.mass[(((uint64_t)bh * p.segs + (row0 + r) / kRows) * p.row_subs + i / p.sub) * kRows + (row0 + r) % kRows] - lse2[r]);
        }
    }
    if (unit < p.row_units) p.weights[(uint64_t)bh * p.row_units + unit] = got;
}

struct Work {
    uint64_t slots, part, ml, mass, counts, total;     // offsets in bytes
    uint32_t ctas;
};

uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }

// An upper bound of the tiles that can be asked for decides the grid.
Work workspace_of(const kvp_attend_params* a, bool weights, bool bitmap)
{
    Work w;
    const uint64_t rows = (uint64_t)a->queries * a->group, segs = (rows + kRows - 1) / kRows, bh = (uint64_t)a->batch * a->cache.kv_heads;
    const uint64_t tiles = bh * segs * a->table_pages * (a->cache.page_tokens / kTileTokens);
    const uint64_t most = a->cache.head_dim == 256 ? 148 : 296;
    w.ctas = (uint32_t)(tiles < most ? (tiles ? tiles : 1) : most);
    w.slots = w.ctas + bh * segs;
    const uint64_t sub = a->unit_tokens < kTileTokens ? a->unit_tokens : kTileTokens;
    w.part = 0;
    w.ml = up256(w.slots * kRows * a->cache.head_dim * 4);
    w.mass = w.ml + up256(w.slots * kRows * 8);
    w.counts = w.mass + (weights ? up256(bh * segs * ((uint64_t)a->table_pages * a->cache.page_tokens / sub) * kRows * 4) : 0);
    w.total = w.counts + (bitmap ? up256(bh * 4) : 0);
    return w;
}

int check_attend(const kvp_attend_params* a)
{
    if (!a || a->reserved || a->cache.reserved || !a->batch || !a->queries || !a->group || !a->cache.kv_heads || !a->cache.pages) return KVP_ERR_ARG;
    if (!a->table_pages || !a->cache.page_tokens || a->cache.page_tokens % kTileTokens || a->dtype > KVP_F16) return KVP_ERR_ARG;
    const uint32_t u = a->unit_tokens;
    if (!u || a->cache.page_tokens % u || (u < kTileTokens ? kTileTokens % u : u % kTileTokens)) return KVP_ERR_ARG;
    if (!(a->scale > -INFINITY && a->scale < INFINITY)) return KVP_ERR_ARG;
    if (!head_dim_served(a->cache.head_dim)) return KVP_ERR_RANGE;
    const uint64_t rows = (uint64_t)a->queries * a->group, bh = (uint64_t)a->batch * a->cache.kv_heads;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens;
    if (rows > 4096 || a->queries > 1024 || a->batch >= (1u << 24) || bh >= (1u << 24) || tokens >= (1ull << 31)) return KVP_ERR_RANGE;
    if (bh * rows >= (1ull << 30) || bh * ((tokens / u + kThreads - 1) / kThreads) >= (1ull << 30)) return KVP_ERR_RANGE;
    return KVP_OK;
}

template <int N>
int launch_attend(const AttendK& k, cudaStream_t st)
{
    const uint32_t smem = Shape<N>::kSmem;
    KVP_CUDA(cudaFuncSetAttribute(attend_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    if (k.units) {
        count_kernel<<<(k.batch * k.heads + kWarps - 1) / kWarps, kThreads, 0, st>>>(k);
        KVP_CUDA(cudaGetLastError());
    }
    attend_kernel<N><<<k.ctas, kThreads, smem, st>>>(k);
    KVP_CUDA(cudaGetLastError());
    const uint64_t blocks = (uint64_t)k.batch * k.heads * (k.rows + (k.weights ? (k.row_units + kThreads - 1) / kThreads : 0));
    join_kernel<N><<<(uint32_t)blocks, kThreads, 0, st>>>(k);
    KVP_CUDA(cudaGetLastError());
    return KVP_OK;
}

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" int kvp_attend_workspace(const kvp_attend_params* a, int want_weights, int has_units, uint64_t* bytes)
{
    const int rc = check_attend(a);
    if (rc) return rc;
    if (!bytes) return KVP_ERR_ARG;
    *bytes = workspace_of(a, want_weights != 0, has_units != 0).total;
    return KVP_OK;
}

extern "C" int kvp_attend(const kvp_attend_params* a, const void* q, const void* cache, const int32_t* table, const int32_t* lens,
                          const uint32_t* units, void* out, float* lse, float* weights, void* workspace, uint64_t workspace_bytes,
                          void* stream)
{
    const int rc = check_attend(a);
    if (rc) return rc;
    if (!q || !cache || !table || !lens || !out || !workspace) return KVP_ERR_ARG;
    const Work w = workspace_of(a, weights != nullptr, units != nullptr);
    if (workspace_bytes < w.total) return KVP_ERR_ARG;
    AttendK k;
    k.q = q; k.out = out; k.lse = lse; k.weights = weights;
    k.cache = static_cast<const uint8_t*>(cache); k.table = table; k.lens = lens; k.units = units;
    char* ws = static_cast<char*>(workspace);
    k.part = reinterpret_cast<float*>(ws + w.part);
    k.ml = reinterpret_cast<float2*>(ws + w.ml);
    k.mass = reinterpret_cast<float*>(ws + w.mass);
    k.counts = reinterpret_cast<uint32_t*>(ws + w.counts);
    k.q_batch = a->q_batch_stride; k.q_query = a->q_query_stride; k.q_head = a->q_head_stride;
    k.batch = a->batch; k.queries = a->queries; k.heads = a->cache.kv_heads; k.group = a->group;
    k.rows = a->queries * a->group; k.segs = (k.rows + kRows - 1) / kRows;
    k.page_tiles = a->cache.page_tokens / kTileTokens; k.table_pages = a->table_pages; k.pages = a->cache.pages;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens;
    k.unit = a->unit_tokens; k.row_units = (uint32_t)(tokens / a->unit_tokens);
    k.unit_words = ((uint64_t)k.batch * k.heads * k.row_units + 31) / 32;
    const uint32_t sub = k.unit < kTileTokens ? k.unit : kTileTokens;
    k.row_subs = tokens / sub;
    k.sub = weights ? sub : 0;
    k.ctas = w.ctas;
    k.least = kWarps;
    k.scale = a->scale;
    k.bf16 = a->dtype == KVP_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (a->cache.head_dim) {
        case 64: return launch_attend<2>(k, st);
        case 128: return launch_attend<4>(k, st);
        default: return launch_attend<8>(k, st);
    }
}
