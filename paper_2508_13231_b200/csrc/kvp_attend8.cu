// Attention over the cache held in 8 bits, for the last few tokens of each sequence or a chunk of a prompt (include/kvp.h, kvp_attend8).
//
// Per query row r (a query token and a query head), over the tokens i that it sees:
//   s_i = cap(scale * q . k_i) + slope * (i - position of the query),  cap(x) = cap * tanh(x / cap) or x,
//   p_i = exp(s_i - lse),  lse = log sum_i exp(s_i),  out = sum_i p_i v_i,  weights[unit] as in kvp_attend.
//
// Products. Both run on the matrix unit (tcgen05.mma, e4m3) with the cache's bytes as they lie as the left operand: 128 tokens x D dims of keys, then
// D dims x 128 tokens of values. The right operand has a column for each row, or rather for each term of a row: a number with more bits than
// e4m3's four is split into x = t0 + t1 / 32 + t2 / 1024, each the nearest e4m3 to what the ones before leave. A bf16 query is two terms and an fp16 query three,
// exactly (down to 2^-14 of the row's largest, below that to within 2^-22 of it); a weight is three terms, 12 bits (2^-12 of itself), down to 2^-26 of
// the largest. Products of e4m3 numbers are exact and the unit keeps 25 bits of their sums; terms have sums of their own, joined in fp32.
// No byte of the cache goes through a register, and a chunk of a prompt runs at the matrix unit's rate for 16 bits.
//
// exp runs in fp32 against a running maximum that moves only when a score passes it by 2^2 (kSlack). A weight times 2^6 and the scale of its block's values over the
// largest such scale so far is what is split: at most 256.
//
// Split over CTAs as in kvp_attend: one line of all tiles (16 tokens), cut into equal parts on the device; the join is its join.
//
// A CTA: warp 0 sends for tiles (bulk copies; a stage is eight tiles, keys and values), one thread of warp 1 issues the products with keys, one of
// warp 2 those with values, four (or eight) warps turn scores into weights, a token a thread. Every hand-over is a barrier in
// shared memory whose wait ends after two seconds; a CTA that gave up writes NaN.
#include <type_traits>

#include "kvp_line.cuh"
#include "kvp_mma.cuh"
#include "kvp_tile8.cuh"

namespace kvp {

namespace {

constexpr uint32_t kFixed8 = 48;              // what a CTA spends on a segment whatever its length, in tiles
constexpr uint32_t kGroup = 8;                // tiles of a stage
constexpr uint32_t kListCap8 = 1024;          // units of a bitmap row that are listed at a time: 32 words
constexpr float kSlack = 2.0f;
constexpr float kLift = 6.0f;                 // weights are split after a multiplication by 2^kLift
constexpr float kLog2e = 1.4426950408889634f;

struct Attend8K : LineK<kFixed8> {
    const void* q;
    const uint8_t* cache;
    const float* slopes;
    uint32_t* marks;         // [batch * heads][mark_row] tiles of every 32 words of a row of the bitmap
    uint32_t mark_row;
    int64_t q_batch, q_query, q_head;
    float scale, cap;        // cap 0: none
    uint32_t window, sink;   // window 0: none
    bool q_aligned;
};

// Tiles that a sequence's queries see: all, or the first `head` and those from `head + skip` on.
struct Visible {
    uint32_t head, skip;
};
__device__ __forceinline__ Visible visible_tiles(const Attend8K& p, uint32_t len)
{
    Visible v = {0, 0};
    if (p.window) {
        const int64_t from = (int64_t)len - p.queries - p.window + 1;          // first token that the first query sees through the window
        const uint32_t low = from > 0 ? (uint32_t)from / kTileTokens : 0;
        v.head = tiles_of(p.sink < len ? p.sink : len);
        v.skip = low > v.head ? low - v.head : 0;
    }
    return v;
}
__device__ __forceinline__ uint32_t entry_count(const Attend8K& p, uint32_t e)
{
    if (p.units) return p.counts[e];
    const uint32_t len = length_of(p, e);
    return tiles_of(len) - visible_tiles(p, len).skip;
}
__device__ __forceinline__ bool tile_seen(const Attend8K& p, uint32_t len, uint32_t tile)
{
    if (p.units) return true;
    const Visible v = visible_tiles(p, len);
    return tile < v.head || tile >= v.head + v.skip;
}

// counts[bh]: tiles to read of a row of the bitmap, and of every 32 words of it; one CTA per row
__global__ void __launch_bounds__(kThreads) count8_kernel(const Attend8K p)
{
    __shared__ uint32_t sum[kWarps];
    let_next_start();
    const uint32_t bh = blockIdx.x, tid = threadIdx.x;
    const uint32_t len = length_of(p, p.heads.of(bh)), units = units_of(p, len), tiles = tiles_of(len);
    const uint32_t k = p.unit > kTileTokens ? p.unit / kTileTokens : 1;
    uint32_t all = 0;
    for (uint32_t w0 = tid - tid % 32; 32u * w0 < units; w0 += kThreads) {
        const uint32_t w = w0 + tid % 32;
        uint32_t n = 0;
        if (32u * w < units) {
            const uint32_t x = unit_word(p, bh, w, units);
            n = __popc(x) * k;
            if (k > 1 && units - 32u * w <= 32u && (x >> (units - 1u - 32u * w)) & 1u) n -= units * k - tiles;   // the last unit may be cut
        }
        n = __reduce_add_sync(0xFFFFFFFFu, n);
        if (tid % 32 == 0) p.marks[(uint64_t)bh * p.mark_row + w0 / 32] = n;
        all += n;
    }
    if (tid % 32 == 0) sum[tid / 32] = all;
    __syncthreads();
    if (tid == 0) {
        for (uint32_t i = 1; i < (uint32_t)kWarps; ++i) all += sum[i];
        p.counts[bh] = all;
    }
}

// D: dims of a head; ROWS: rows of a segment, 8, 16, 32 or 64, worked on by teams of four warps for 16 rows at most
template <int D_, bool HALF_, uint32_t ROWS_>
struct Shape8 {
    static constexpr int D = D_;
    static constexpr bool HALF = HALF_;
    static constexpr uint32_t ROWS = ROWS_;
    using L = Tile8<D>;
    static constexpr uint32_t kTeams = ROWS > 16 ? ROWS / 16 : 1;      // of four warps
    static constexpr uint32_t kRowsEach = ROWS / kTeams;
    static constexpr uint32_t kBlock = 128 + 128 * kTeams;
    static constexpr uint32_t kQTerms = HALF ? 3 : 2;
    static constexpr uint32_t kQCols = (kQTerms * ROWS + 15) / 16 * 16;
    static constexpr uint32_t kPCols = (3 * ROWS + 15) / 16 * 16;
    static constexpr uint32_t kHalves = D == 256 ? 2 : 1;              // 128 dims of values a product
    static constexpr uint32_t kSumCols = kHalves * kPCols;
    static constexpr uint32_t kScoreBufs = 2 * kQCols + kSumCols <= 512 ? 2 : 1;
    static constexpr uint32_t kColsUsed = kScoreBufs * kQCols + kSumCols;
    static constexpr uint32_t kCols = kColsUsed <= 64 ? 64 : kColsUsed <= 128 ? 128 : kColsUsed <= 256 ? 256 : 512;
    static constexpr uint32_t kStage = kGroup * (L::kKeyBytes + L::kValueBytes);
    static constexpr uint32_t kQBytes = kQCols * D;
    static constexpr uint32_t kPBytes = kPCols * 128;
    static constexpr uint32_t kPad = 2048;                             // D == 64: rows 64 .. 127 of the values' operand are what lies behind
    static constexpr uint32_t kCtas = D <= 128 && ROWS <= 16 ? 2 : 1;  // of an SM
    static constexpr uint32_t kRoom = kCtas == 2 ? 115712 - 2944 : 232448 - 4608;            // less what is declared statically
    static constexpr uint32_t kPBufs = ROWS == 16 && D == 128 ? 1 : 2;
    static constexpr uint32_t kOther = kQBytes + kPBufs * kPBytes + (D == 64 ? kPad : 0);
    static constexpr uint32_t kStagesFit = (kRoom - kOther) / kStage;
    static constexpr uint32_t kStages = kStagesFit < 8 ? kStagesFit : 8;
    static constexpr uint32_t kSmem = kStages * kStage + kOther;
    static_assert(kStages >= 2 && kColsUsed <= 512 && kQCols <= 256 && kPCols <= 256, "does not fit");
};

template <class S>
struct Smem8 {
    uint64_t full[S::kStages], empty[S::kStages];      // a stage has come; its products are done
    uint64_t scored[2], taken[2];                      // scores are in tensor memory; they are in registers
    uint64_t weighed[2], summed[2];                    // weights are in shared memory; the products with values are done
    uint64_t query;                                    // a segment's queries are in shared memory
    uint32_t tensor, gave_up;
    LineSmem line;
    uint32_t tile[S::kStages][kGroup];                 // numbers of a stage's tiles; ~0: not there
    float factor[S::ROWS], slope[S::ROWS];             // per row: what scores are multiplied by, and its bias a token
    int32_t see[S::ROWS];                              // tokens before this one
    float top[S::kTeams][4][S::kRowsEach];             // of the four warps of a team
    float most[S::kTeams][4];
    uint16_t list[kListCap8];                          // units of 32 words of a bitmap's row
};

// The segments of this CTA's part, one after the other; each warp goes through them by itself.
struct Walk {
    uint32_t todo, per, entries, entry, inner, at_place, count;
    uint32_t seg, bh, rt, b, h, len, off, take;
    __device__ __forceinline__ bool next(const Attend8K& p)
    {
        while (todo) {
            while (inner == per || !count) {
                if (++entry >= entries) return false;              // not reached: the line ends with the last part
                count = entry_count(p, entry);
                inner = 0;
            }
            const uint32_t places = min(todo, count + kFixed8 - at_place), at = at_place;
            todo -= places;
            at_place = 0;
            const uint32_t here = inner++;
            if (at + places <= kFixed8) continue;                  // no tile among them
            off = at > kFixed8 ? at - kFixed8 : 0u;
            take = at + places - kFixed8 - off;
            seg = entry * per + here;
            bh = p.segs.of(seg);
            rt = seg - bh * p.segs.d;
            b = p.heads.of(bh);
            h = bh - b * p.heads.d;
            len = length_of(p, b);
            return true;
        }
        return false;
    }
};

__device__ __forceinline__ uint4 load_q8(const Attend8K& p, int64_t at)
{
    const uint16_t* from = static_cast<const uint16_t*>(p.q) + at;
    if (p.q_aligned) return __ldg(reinterpret_cast<const uint4*>(from));
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = __ldg(from + i);
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}
template <bool HALF>
__device__ __forceinline__ void floats_of8(uint32_t x, float* to)
{
    if (HALF) {
        const float2 f = __half22float2(half2_of(x));
        to[0] = f.x;
        to[1] = f.y;
    } else {
        to[0] = __uint_as_float(x << 16);
        to[1] = __uint_as_float(x & 0xFFFF0000u);
    }
}

// the next term of two numbers, and what it leaves, 32 times as large
__device__ __forceinline__ uint32_t next_term(float& a, float& b)
{
    const uint32_t t = e4m3_pair(a, b);
    const float2 f = floats_of_e4m3(t);
    a = (a - f.x) * 32.0f;
    b = (b - f.y) * 32.0f;
    return t;
}

__device__ __forceinline__ bool team_any(bool x, uint32_t team)    // over the four warps of a team
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)x), "r"(team + 1) : "memory");
    return r != 0;
}
__device__ __forceinline__ void team_sync(uint32_t team) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(team + 1) : "memory"); }
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}
__device__ __forceinline__ float warp_max(float x)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

// sums over 2^LOG neighbouring lanes of R numbers each; lane l of them is left with those of rows from(l) on, R >> LOG (one at least) of them
template <int R, int LOG>
__device__ __forceinline__ void sum_neighbours(float (&x)[R], uint32_t lane, uint32_t& from)
{
    from = 0;
    int n = R;
#pragma unroll
    for (int i = LOG - 1; i >= 0; --i) {
        const uint32_t d = 1u << i;
        if (n > 1) {
            n /= 2;
            const bool up = lane & d;
            if (up) from += n;
#pragma unroll
            for (int j = 0; j < R / 2; ++j)
                if (j < n) {
                    const float keep = up ? x[j + n] : x[j], give = up ? x[j] : x[j + n];
                    x[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, d);
                }
        } else {
            x[0] += __shfl_xor_sync(0xFFFFFFFFu, x[0], d);
        }
    }
}

template <class S>
__global__ void __launch_bounds__(S::kBlock, S::kCtas) attend8_kernel(const Attend8K p)
{
    using L = typename S::L;
    constexpr int D = S::D;
    constexpr uint32_t ROWS = S::ROWS, R = S::kRowsEach;
    extern __shared__ __align__(128) uint8_t room[];
    __shared__ Smem8<S> sm;
    static_assert(S::kSmem + sizeof(Smem8<S>) <= (S::kCtas == 2 ? 115712 : 232448), "does not fit");
    let_next_start();
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    wait_for_previous();
    Walk walk;
    {
        uint32_t entry = 0;
        const Line line = find_in_line<S::kBlock>(p, blockIdx.x, entry, sm.line);
        const uint64_t begin = (uint64_t)line.chunk * blockIdx.x;
        if (begin >= line.total) return;
        walk.todo = min(line.chunk, line.total - (uint32_t)begin);     // places
        walk.per = line_per(p);
        walk.entries = line_entries(p);
        walk.entry = entry;
        walk.count = line.count;
        walk.inner = ((uint32_t)begin - line.before) / (line.count + kFixed8);
        walk.at_place = ((uint32_t)begin - line.before) - walk.inner * (line.count + kFixed8);
    }
    uint8_t* const queries = room + S::kStages * S::kStage;
    uint8_t* const weights = queries + S::kQBytes;
    auto keys_of = [&](uint32_t st) { return room + st * S::kStage; };
    auto values_of = [&](uint32_t st) { return room + st * S::kStage + kGroup * L::kKeyBytes; };
    const auto bar = [](uint64_t& b) { return smem_at(&b); };
    if (tid == 0) {
        for (uint32_t i = 0; i < S::kStages; ++i) {
            barrier_init(bar(sm.full[i]), 1);
            barrier_init(bar(sm.empty[i]), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            barrier_init(bar(sm.scored[i]), 1);
            barrier_init(bar(sm.taken[i]), 4 * S::kTeams);
            barrier_init(bar(sm.weighed[i]), 4 * S::kTeams);
            barrier_init(bar(sm.summed[i]), 1);
        }
        barrier_init(bar(sm.query), 4 * S::kTeams);
        sm.gave_up = 0;
        show_to_async();
    }
    if (warp == 1) tensor_alloc<S::kCols>(smem_at(&sm.tensor));
    tensor_before_sync();
    __syncthreads();
    tensor_after_sync();
    const uint32_t scores_at = sm.tensor, sums_at = sm.tensor + S::kScoreBufs * S::kQCols;
    volatile uint32_t* const gave_up = &sm.gave_up;
    uint32_t it = 0;                                                   // groups so far, over all segments

    if (warp == 0) {
        // ---- sends for tiles ----
        bool ok = true;
        while (ok && walk.next(p)) {
            const int32_t* table = p.table + (uint64_t)walk.b * p.table_pages;
            const Visible seen = p.units ? Visible{0, 0} : visible_tiles(p, walk.len);
            // a bitmap's row: `chunk` of 32 words is listed, before it stand `base` tiles of the row, in it `here`
            const uint32_t units = units_of(p, walk.len), k = p.unit > kTileTokens ? p.unit / kTileTokens : 1, fold = p.unit < kTileTokens ? kTileTokens / p.unit : 1;
            uint32_t chunk = 0, base = 0, here = 0;
            const auto list_chunk = [&]() {
                const uint32_t w = 32 * chunk + lane;
                uint32_t bits = 32u * w < units ? unit_word(p, walk.bh, w, units) : 0u;
                const uint32_t mine = __popc(bits), upto = sum_upto(mine, lane);
                __syncwarp();
                for (uint32_t at = upto - mine; bits; bits &= bits - 1u, ++at) sm.list[at] = (uint16_t)(32u * lane + __ffs(bits) - 1u);
                __syncwarp();
                here = p.marks[(uint64_t)walk.bh * p.mark_row + chunk];
            };
            if (p.units) {
                // the chunk with tile `off`
                const uint32_t chunks = (units + 1023) / 1024;
                for (uint32_t c0 = 0;; c0 += 32) {
                    const uint32_t n = c0 + lane < chunks ? p.marks[(uint64_t)walk.bh * p.mark_row + c0 + lane] : 0u, upto = sum_upto(n, lane);
                    const uint32_t found = __ballot_sync(0xFFFFFFFFu, base + upto > walk.off);
                    if (found || c0 + 32 >= chunks) {
                        const int l = found ? __ffs(found) - 1 : 31;
                        chunk = c0 + l;
                        base += __shfl_sync(0xFFFFFFFFu, upto - n, l);
                        break;
                    }
                    base += __shfl_sync(0xFFFFFFFFu, upto, 31);
                }
                list_chunk();
            }
            for (uint32_t g = 0; g < walk.take; g += kGroup, ++it) {
                const uint32_t st = it % S::kStages;
                // which tiles, and where they lie; lanes 8 .. 15 do as 0 .. 7, for the values
                const uint32_t i = walk.off + g + lane % kGroup;
                const bool mine = lane < 2 * kGroup && g + lane % kGroup < walk.take;
                uint32_t tile = 0;
                if (p.units) {
                    bool left = mine;
                    while (true) {
                        if (left && i < base + here) {
                            tile = (1024 * chunk + sm.list[(i - base) / k]) / fold * k + (i - base) % k;
                            left = false;
                        }
                        if (!__any_sync(0xFFFFFFFFu, left)) break;
                        base += here;
                        ++chunk;
                        list_chunk();
                    }
                } else {
                    tile = i < seen.head ? i : i + seen.skip;
                }
                const uint8_t* from = nullptr;
                if (mine) {
                    const uint32_t page = p.page_tiles.of(tile), pg = (uint32_t)__ldg(table + page);
                    if (pg < p.pages) from = p.cache + (((uint64_t)pg * p.heads.d + walk.h) * p.page_tiles.d + (tile - page * p.page_tiles.d)) * L::kBytes;
                }
                if (it >= S::kStages) ok = __all_sync(0xFFFFFFFFu, barrier_wait(bar(sm.empty[st]), (it / S::kStages - 1) & 1, gave_up));
                if (!ok) break;
                const uint32_t many = __popc(__ballot_sync(0xFFFFFFFFu, from != nullptr) & 0xFFu);
                if (lane < kGroup) sm.tile[st][lane] = from ? tile : ~0u;
                __syncwarp();
                if (lane == 0) barrier_arrive_expect(bar(sm.full[st]), many * (L::kKeyBytes + L::kValueBytes));
                __syncwarp();
                if (from) {
                    if (lane < kGroup) copy_bulk(smem_at(keys_of(st)) + lane * L::kKeyBytes, from, L::kKeyBytes, bar(sm.full[st]));
                    else copy_bulk(smem_at(values_of(st)) + (lane - kGroup) * L::kValueBytes, from + L::kValues, L::kValueBytes, bar(sm.full[st]));
                }
            }
        }
        // copies under way end before the CTA does
        for (uint32_t j = it > S::kStages ? it - S::kStages : 0; !ok && j < it; ++j)
            for (uint32_t tries = 0; tries < 1u << 16 && !barrier_try(bar(sm.full[j % S::kStages]), (j / S::kStages) & 1); ++tries) {}
    } else if (warp == 1) {
        // ---- products with keys ----
        if (lane == 0) {
            uint32_t segment = 0;
            bool ok = true;
            for (; ok && walk.next(p); ++segment) {
                ok = barrier_wait(bar(sm.query), segment & 1, gave_up);
                for (uint32_t g = 0; ok && g < walk.take; g += kGroup, ++it) {
                    const uint32_t st = it % S::kStages, sb = it % S::kScoreBufs;
                    ok = barrier_wait(bar(sm.full[st]), (it / S::kStages) & 1, gave_up) &&
                         (it < S::kScoreBufs || barrier_wait(bar(sm.taken[sb]), (it / S::kScoreBufs - 1) & 1, gave_up));
                    if (!ok) break;
                    tensor_after_sync();
                    const uint32_t a = smem_at(keys_of(st)), b = smem_at(queries);
#pragma unroll
                    for (uint32_t k = 0; k < D / 32; ++k)
                        multiply_e4m3(scores_at + sb * S::kQCols, operand(a + 256 * k, 128, 8 * D), operand(b + 256 * k, 128, 8 * D), shape_e4m3(S::kQCols), k > 0);
                    products_arrive(bar(sm.scored[sb]));
                }
            }
        }
    } else if (warp == 2) {
        // ---- products with values ----
        if (lane == 0) {
            bool ok = true;
            while (ok && walk.next(p)) {
                for (uint32_t g = 0; g < walk.take; g += kGroup, ++it) {
                    const uint32_t st = it % S::kStages, pb = it % S::kPBufs, pairs = (min(walk.take - g, kGroup) + 1) / 2;
                    ok = barrier_wait(bar(sm.full[st]), (it / S::kStages) & 1, gave_up) && barrier_wait(bar(sm.weighed[pb]), (it / S::kPBufs) & 1, gave_up);
                    if (!ok) break;
                    tensor_after_sync();
                    const uint32_t a = smem_at(values_of(st)), b = smem_at(weights + pb * S::kPBytes);
                    for (uint32_t k = 0; k < pairs; ++k)
#pragma unroll
                        for (uint32_t half = 0; half < S::kHalves; ++half)
                            multiply_e4m3(sums_at + half * S::kPCols, operand(a + half * 2048 + 2 * k * L::kValueBytes, L::kValueBytes, 128), operand(b + 256 * k, 128, 1024),
                                          shape_e4m3(S::kPCols), g + k > 0);
                    products_arrive(bar(sm.empty[st]));
                    products_arrive(bar(sm.summed[pb]));
                }
            }
        }
    } else if (warp >= 4) {
        // ---- scores to weights: thread `me` of a team has token `me` of a group and rows row0 .. row0 + R - 1 ----
        const uint32_t team = (warp - 4) / 4, part = warp % 4, me = tid % 128, row0 = team * R;
        const uint32_t lanes = part * 32 << 16;                        // of tensor memory
        bool ok = true;
        while (walk.next(p)) {
            // the queries: kEach threads a row
            {
                constexpr uint32_t kFew = 128 * S::kTeams / ROWS, kEach = kFew < D / 8 ? kFew : D / 8, kVecs = D / 8 / kEach;
                const uint32_t t = tid - 128, row = t / kEach, j = t % kEach, r = walk.rt * ROWS + row, query = p.group.of(r);
                const bool mine = row < ROWS;                          // a team's rows are its own
                uint4 raw[kVecs];
#pragma unroll
                for (uint32_t v = 0; v < kVecs; ++v)
                    raw[v] = mine && r < p.rows ? load_q8(p, walk.b * p.q_batch + (int64_t)query * p.q_query +
                                                         (int64_t)(walk.h * p.group.d + (r - query * p.group.d)) * p.q_head + (v * kEach + j) * 8)
                                        : make_uint4(0, 0, 0, 0);
                float most = 0.0f, odd = 0.0f;
#pragma unroll
                for (uint32_t v = 0; v < kVecs; ++v) {
                    const uint32_t w[4] = {raw[v].x, raw[v].y, raw[v].z, raw[v].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x[2];
                        floats_of8<S::HALF>(w[i], x);
                        most = fmaxf(most, fmaxf(fabsf(x[0]), fabsf(x[1])));
                        odd = fmaf(x[0], 0.0f, fmaf(x[1], 0.0f, odd));     // NaN if one is not finite
                    }
                }
#pragma unroll
                for (uint32_t o = 1; o < kEach; o <<= 1) {
                    most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
                    odd += __shfl_xor_sync(0xFFFFFFFFu, odd, o);
                }
                // largest magnitude in [2^7, 2^8); the power of two in two factors, either of them a normal number
                const int e = most > 0.0f && most < INFINITY ? ilogbf(most) - 7 : 0, half_e = -e / 2;
                const float by0 = __int_as_float((half_e + 127) << 23), by1 = __int_as_float((-e - half_e + 127) << 23);
#pragma unroll
                for (uint32_t v = 0; v < kVecs; ++v) {
                    const uint32_t w[4] = {raw[v].x, raw[v].y, raw[v].z, raw[v].w};
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) floats_of8<S::HALF>(w[i], x + 2 * i);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = x[i] * by0 * by1;
                    const uint32_t d = (v * kEach + j) * 8;
#pragma unroll
                    for (uint32_t term = 0; term < S::kQTerms; ++term) {
                        uint2 q;
                        q.x = next_term(x[0], x[1]) | next_term(x[2], x[3]) << 16;
                        q.y = next_term(x[4], x[5]) | next_term(x[6], x[7]) << 16;
                        const uint32_t col = term * ROWS + row;
                        if (mine) *reinterpret_cast<uint2*>(queries + col / 8 * (8 * D) + d / 16 * 128 + col % 8 * 16 + d % 16) = q;
                    }
                }
                if (mine && j == 0) {
                    const float unit = p.cap > 0.0f ? p.scale / p.cap : p.scale * kLog2e;      // scores in units of the cap, or to the base 2
                    sm.factor[row] = scalbnf(unit, e) + odd;
                    sm.slope[row] = p.slopes && r < p.rows ? __ldg(p.slopes + walk.h * p.group.d + (r - query * p.group.d)) * kLog2e : 0.0f;
                    const int32_t see = (int32_t)walk.len - (int32_t)p.queries + 1 + (int32_t)query;
                    sm.see[row] = r < p.rows ? see : INT32_MIN / 2;
                }
                show_to_async();
                __syncwarp();
                if (lane == 0) barrier_arrive(bar(sm.query));
                team_sync(team);
            }
            float m[R], l[R];                                          // running maximum of the team, sums of this thread's weights
            float most_scale = 0.0f;                                   // largest scale of values so far
#pragma unroll
            for (uint32_t r = 0; r < R; ++r) {
                m[r] = kNone;
                l[r] = 0.0f;
            }
            float* const mass = p.mass + (uint64_t)walk.seg * p.row_subs * ROWS + row0;

            for (uint32_t g = 0; g < walk.take; g += kGroup, ++it) {
                const uint32_t st = it % S::kStages, sb = it % S::kScoreBufs, pb = it % S::kPBufs, j = me / 16, many = min(walk.take - g, kGroup);
                ok = ok && barrier_wait(bar(sm.scored[sb]), (it / S::kScoreBufs) & 1, gave_up) && barrier_wait(bar(sm.full[st]), (it / S::kStages) & 1, gave_up);
                __syncwarp();
                tensor_after_sync();
                uint8_t* const block = values_of(st) + j * L::kValueBytes;
                const uint32_t tile = j < many ? sm.tile[st][j] : ~0u;
                const int32_t pos = (int32_t)(tile * kTileTokens + me % 16);
                bool live = tile != ~0u && pos < (int32_t)walk.len;
                if (live && p.units && p.unit < kTileTokens) live = bits_at(p, (uint64_t)walk.bh * p.row_units + ((uint32_t)pos >> p.unit_log2)) & 1u;
                const float2 scales = *reinterpret_cast<const float2*>(block + 16 * D);        // of keys, of values
                float s[R];
#pragma unroll
                for (uint32_t r = 0; r < R; r += 8) {
                    float x[S::kQTerms][8];
#pragma unroll
                    for (uint32_t term = 0; term < S::kQTerms; ++term) tensor_load8(scores_at + lanes + sb * S::kQCols + term * ROWS + row0 + r, x[term]);
                    tensor_wait_load();
#pragma unroll
                    for (uint32_t term = 0; term < S::kQTerms; ++term) tensor_hold8(x[term]);
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) {
                        float y = fmaf(x[1][i], 0x1p-5f, x[0][i]);
                        if (S::kQTerms == 3) y = fmaf(x[S::kQTerms - 1][i], 0x1p-10f, y);
                        s[r + i] = y * (sm.factor[row0 + r + i] * scales.x);
                    }
                }
                tensor_before_sync();
                __syncwarp();
                if (lane == 0) barrier_arrive(bar(sm.taken[sb]));
                if (p.cap > 0.0f) {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) s[r] = tanhf(s[r]) * (p.cap * kLog2e);
                }
                if (p.slopes) {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) s[r] = fmaf(sm.slope[row0 + r], (float)(pos - sm.see[row0 + r] + 1), s[r]);
                }
                bool up = false;                                       // has a score passed the maximum by more than the slack?
#pragma unroll
                for (uint32_t r = 0; r < R; ++r) {
                    const int32_t see = sm.see[row0 + r];
                    const bool seen = live && pos < see && (!p.window || pos >= see - (int32_t)p.window || pos < (int32_t)p.sink);
                    s[r] = seen ? s[r] : -INFINITY;
                    up = up || s[r] > m[r] + kSlack;
                }
                const float scale = live ? scales.y : 0.0f;
                up = up || scale > most_scale;
                if (team_any(up || !ok, team)) {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) {
                        const float x = warp_max(s[r]);
                        if (lane == 0) sm.top[team][part][r] = x;
                    }
                    const float x = warp_max(scale);
                    if (lane == 0) sm.most[team][part] = x;
                    // sums of the group before are to be there, all of them
                    if (g) ok = ok && barrier_wait(bar(sm.summed[(it - 1) % S::kPBufs]), ((it - 1) / S::kPBufs) & 1, gave_up);
                    __syncwarp();
                    if (team_any(!ok, team)) { ok = false; break; }    // also: the maxima are there
                    tensor_after_sync();
                    const float new_scale = fmaxf(most_scale, fmaxf(fmaxf(sm.most[team][0], sm.most[team][1]), fmaxf(sm.most[team][2], sm.most[team][3])));
                    const float by_scale = most_scale > 0.0f ? most_scale / new_scale : 1.0f;
                    most_scale = new_scale;
#pragma unroll
                    for (uint32_t r = 0; r < R; r += 8) {
                        float by[8];
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i) {
                            const float top = fmaxf(m[r + i], fmaxf(fmaxf(sm.top[team][0][r + i], sm.top[team][1][r + i]), fmaxf(sm.top[team][2][r + i], sm.top[team][3][r + i])));
                            by[i] = exp2_fast(m[r + i] - top);
                            l[r + i] *= by[i];
                            by[i] *= by_scale;
                            m[r + i] = top;
                        }
                        if (g) {
#pragma unroll
                            for (uint32_t c = 0; c < 3 * S::kHalves; ++c) {
                                const uint32_t at = sums_at + lanes + c / 3 * S::kPCols + c % 3 * ROWS + row0 + r;
                                float y[8];
                                tensor_load8(at, y);
                                tensor_wait_load();
                                tensor_hold8(y);
#pragma unroll
                                for (uint32_t i = 0; i < 8; ++i) y[i] *= by[i];
                                tensor_store8(at, y);
                            }
                        }
                    }
                    tensor_wait_store();
                    tensor_before_sync();
                    team_sync(team);                                   // the maxima's room is free again
                }
#pragma unroll
                for (uint32_t r = 0; r < R; ++r) {
                    s[r] = exp2_fast(s[r] - m[r]);
                    l[r] += s[r];
                }
                if (p.sub) {                                           // what each block of `sub` tokens received, as log2
                    float x[R];
                    uint32_t from;
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) x[r] = s[r];
                    const auto note = [&](auto log, auto left) {
                        constexpr int LOG = decltype(log)::value, LEFT = decltype(left)::value;
                        sum_neighbours<R, LOG>(x, lane, from);
                        if (tile == ~0u) return;
                        float* to = mass + ((uint64_t)(uint32_t)pos >> LOG) * ROWS + from;
#pragma unroll
                        for (int i = 0; i < LEFT; ++i) {
                            float mx = m[i];
#pragma unroll
                            for (uint32_t r = LEFT; r < R; r += LEFT) mx = from == r ? m[r + i] : mx;
                            to[i] = mx + log2_fast(x[i]);
                        }
                    };
#define KVP_INT(X) std::integral_constant<int, (X)>{}
#define KVP_LEFT(LOG) KVP_INT((R >> LOG) ? (R >> LOG) : 1)
                    switch (p.sub) {
                        case 16: note(KVP_INT(4), KVP_LEFT(4)); break;
                        case 8: note(KVP_INT(3), KVP_LEFT(3)); break;
                        case 4: note(KVP_INT(2), KVP_LEFT(2)); break;
                        case 2: note(KVP_INT(1), KVP_LEFT(1)); break;
                        default: note(KVP_INT(0), KVP_LEFT(0)); break;
                    }
                }
                // the weights as the right operand; the buffer is free when the products with what it held are done
                if (it >= S::kPBufs) ok = ok && barrier_wait(bar(sm.summed[pb]), (it / S::kPBufs - 1) & 1, gave_up);
                const float by = scale > 0.0f ? scale / most_scale * 64.0f : 0.0f;             // 2^kLift
                uint8_t* const to = weights + pb * S::kPBytes + me / 16 * 128 + me % 16;
#pragma unroll
                for (uint32_t r = 0; r < R; r += 2) {
                    float a = s[r] * by, b = s[r + 1] * by;
#pragma unroll
                    for (uint32_t term = 0; term < 3; ++term) {
                        const uint32_t t = next_term(a, b), col = term * ROWS + row0 + r;
                        to[col / 8 * 1024 + col % 8 * 16] = (uint8_t)t;
                        to[col / 8 * 1024 + col % 8 * 16 + 16] = (uint8_t)(t >> 8);
                    }
                }
                // What lies in the cache where no token is may be anything, also NaN, and so may a tile that did not come: its values are cleared.
                const uint32_t lives = __ballot_sync(0xFFFFFFFFu, live) >> (lane & 16u) & 0xFFFFu;
                if (team == 0 && lives != 0xFFFFu && j < (many + 1) / 2 * 2) {
                    uint4 keep;
                    uint32_t* word = &keep.x;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t four = lives >> (4 * i) & 15u;
                        word[i] = (four & 1u ? 0xFFu : 0u) | (four & 2u ? 0xFF00u : 0u) | (four & 4u ? 0xFF0000u : 0u) | (four & 8u ? 0xFF000000u : 0u);
                    }
                    for (uint32_t d = me % 16; d < D; d += 16) {
                        uint4* v = reinterpret_cast<uint4*>(block + d * 16);
                        *v = make_uint4(v->x & keep.x, v->y & keep.y, v->z & keep.z, v->w & keep.w);
                    }
                }
                show_to_async();
                __syncwarp();
                if (lane == 0) barrier_arrive(bar(sm.weighed[pb]));
            }

            // ---- the end of a segment ----
            const uint32_t last = it - 1;
            ok = ok && barrier_wait(bar(sm.summed[last % S::kPBufs]), (last / S::kPBufs) & 1, gave_up);
#pragma unroll
            for (uint32_t r = 0; r < R; ++r) {
                const float x = warp_sum(l[r]);
                if (lane == 0) sm.top[team][part][r] = x;
            }
            if (team_any(!ok, team)) ok = false;
            tensor_after_sync();
            const bool whole = walk.take == walk.count;
            const uint64_t slot = (uint64_t)blockIdx.x + walk.seg;
#pragma unroll
            for (uint32_t r = 0; r < R; ++r) {
                l[r] = (sm.top[team][0][r] + sm.top[team][1][r]) + (sm.top[team][2][r] + sm.top[team][3][r]);
                if (!ok) l[r] = NAN;
            }
            const auto place = [&](uint32_t row) {
                const uint32_t query = p.group.of(row);
                return ((uint64_t)walk.b * p.queries + query) * (p.heads.d * p.group.d) + walk.h * p.group.d + (row - query * p.group.d);
            };
#pragma unroll
            for (uint32_t r = 0; r < R; ++r)
                if (me == r) {
                    const uint32_t row = walk.rt * ROWS + row0 + r;
                    p.ml[slot * ROWS + row0 + r] = make_float2(m[r], l[r]);
                    if (whole && p.lse && row < p.rows) p.lse[place(row)] = l[r] == 0.0f ? -INFINITY : (m[r] + log2f(l[r])) * 0.6931471805599453f;
                }
            const float up = most_scale * 0x1p-6f;
#pragma unroll
            for (uint32_t half = 0; half < S::kHalves; ++half) {
                const uint32_t d = half * 128 + me;
#pragma unroll
                for (uint32_t r = 0; r < R; r += 8) {
                    float x[3][8];
#pragma unroll
                    for (uint32_t c = 0; c < 3; ++c) tensor_load8(sums_at + lanes + half * S::kPCols + c * ROWS + row0 + r, x[c]);
                    tensor_wait_load();
#pragma unroll
                    for (uint32_t c = 0; c < 3; ++c) tensor_hold8(x[c]);
                    if (d < D) {
#pragma unroll
                        for (uint32_t i = 0; i < 8; ++i) {
                            const uint32_t row = walk.rt * ROWS + row0 + r + i;
                            float y = fmaf(fmaf(x[2][i], 0x1p-5f, x[1][i]), 0x1p-5f, x[0][i]) * up;
                            if (row >= p.rows) continue;
                            if (whole) {
                                y = l[r + i] == 0.0f ? 0.0f : y / l[r + i];
                                uint16_t bits;
                                if (S::HALF) bits = __half_as_ushort(__float2half_rn(y));
                                else bits = __bfloat16_as_ushort(__float2bfloat16_rn(y));
                                static_cast<uint16_t*>(p.out)[place(row) * D + d] = bits;
                            } else {
                                p.part[(slot * ROWS + row0 + r + i) * D + d] = y;
                            }
                        }
                    }
                }
            }
            tensor_before_sync();
            team_sync(team);
        }
    }
    tensor_before_sync();
    __syncthreads();
    tensor_after_sync();
    if (warp == 1) tensor_free<S::kCols>(sm.tensor);
}

struct Work8 {
    uint64_t ml, mass, counts, marks, total;           // offsets in bytes; the parts come first
    uint32_t rows, ctas, mark_row;
};

// Rows of a segment: the cache is read once for that many. More rows cost the warps that turn scores into weights more, so no more than there are, in powers of two.
uint32_t segment_rows(const kvp_attend8_params* a)
{
    const uint32_t rows = a->queries * a->group, most = a->cache.head_dim == 256 && a->dtype == KVP_F16 ? 32 : 64;       // what fits shared and tensor memory
    uint32_t r = 8;
    while (r < rows && r < most) r *= 2;
    return r;
}

// An upper bound of the tiles that can be asked for decides the grid.
Work8 workspace_of(const kvp_attend8_params* a, bool weights, bool bitmap)
{
    Work8 w;
    w.rows = segment_rows(a);
    const uint64_t rows = (uint64_t)a->queries * a->group, segs = (rows + w.rows - 1) / w.rows, bh = (uint64_t)a->batch * a->cache.kv_heads;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens, tiles = bh * segs * (tokens / kTileTokens);
    const uint64_t most = a->cache.head_dim == 256 || w.rows > 16 ? 148 : 296;
    w.ctas = (uint32_t)(tiles < most ? (tiles ? tiles : 1) : most);
    const uint64_t slots = w.ctas + bh * segs, sub = a->unit_tokens < kTileTokens ? a->unit_tokens : kTileTokens;
    w.ml = up256(slots * w.rows * a->cache.head_dim * 4);
    w.mass = w.ml + up256(slots * w.rows * 8);
    w.counts = w.mass + (weights ? up256(bh * segs * (tokens / sub) * w.rows * 4) : 0);
    w.marks = w.counts + (bitmap ? up256(bh * 4) : 0);
    w.mark_row = (uint32_t)((tokens / a->unit_tokens + 1023) / 1024);
    w.total = w.marks + (bitmap ? up256(bh * w.mark_row * 4) : 0);
    return w;
}

int check_attend8(const kvp_attend8_params* a)
{
    if (!a || a->reserved || a->cache.reserved || !a->batch || !a->queries || !a->group || !a->cache.kv_heads || !a->cache.pages) return KVP_ERR_ARG;
    if (!a->table_pages || !a->cache.page_tokens || a->cache.page_tokens % kTileTokens || a->dtype > KVP_F16) return KVP_ERR_ARG;
    const uint32_t u = a->unit_tokens;
    if (!u || a->cache.page_tokens % u || (u < kTileTokens ? kTileTokens % u : u % kTileTokens)) return KVP_ERR_ARG;
    if (!(a->scale > -INFINITY && a->scale < INFINITY) || !(a->cap >= 0.0f && a->cap < INFINITY)) return KVP_ERR_ARG;
    if (!head_dim_served(a->cache.head_dim)) return KVP_ERR_RANGE;
    const uint64_t rows = (uint64_t)a->queries * a->group, bh = (uint64_t)a->batch * a->cache.kv_heads;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens;
    if (rows > 4096 || a->queries > 1024 || a->batch >= (1u << 24) || bh >= (1u << 24) || tokens >= (1ull << 30)) return KVP_ERR_RANGE;
    // places in the line are counted in 31 bits
    const uint32_t each = segment_rows(a);
    if (bh * ((rows + each - 1) / each) * (tokens / kTileTokens + kFixed8) >= (1ull << 31)) return KVP_ERR_RANGE;
    if (bh * rows >= (1ull << 30) || bh * ((tokens / u + kThreads - 1) / kThreads) >= (1ull << 30)) return KVP_ERR_RANGE;
    return KVP_OK;
}

template <int D, bool HALF, uint32_t ROWS>
int launch_attend8(const Attend8K& k, cudaStream_t st)
{
    using S = Shape8<D, HALF, ROWS>;
    KVP_CUDA(cudaFuncSetAttribute(attend8_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kSmem));
    int rc = k.units ? launch(count8_kernel, k.batch * k.heads.d, kThreads, 0, false, st, k) : KVP_OK;
    if (!rc) rc = launch(attend8_kernel<S>, k.ctas, S::kBlock, S::kSmem, k.units != nullptr, st, k);
    const uint64_t blocks = (uint64_t)k.batch * k.heads.d * ((k.warp_rows ? k.segs.d * (ROWS / kWarps) : k.rows) + (k.weights ? (k.row_units + kThreads - 1) / kThreads : 0));
    if (!rc) rc = launch(join_kernel<Attend8K, D / 32, HALF, ROWS>, (uint32_t)blocks, kThreads, 0, true, st, k);
    return rc;
}

template <int D, bool HALF>
int attend8_of(const Attend8K& k, uint32_t rows, cudaStream_t st)
{
    switch (rows) {
        case 8: return launch_attend8<D, HALF, 8>(k, st);
        case 16: return launch_attend8<D, HALF, 16>(k, st);
        case 32: return launch_attend8<D, HALF, 32>(k, st);
        default: return launch_attend8<D, HALF, D == 256 && HALF ? 32 : 64>(k, st);
    }
}

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" int kvp_attend8_workspace(const kvp_attend8_params* a, int want_weights, int has_units, uint64_t* bytes)
{
    const int rc = check_attend8(a);
    if (rc) return rc;
    if (!bytes) return KVP_ERR_ARG;
    *bytes = workspace_of(a, want_weights != 0, has_units != 0).total;
    return KVP_OK;
}

extern "C" int kvp_attend8(const kvp_attend8_params* a, const void* q, const void* cache, const int32_t* table, const int32_t* lens,
                           const uint32_t* units, const float* slopes, void* out, float* lse, float* weights, void* workspace, uint64_t workspace_bytes,
                           void* stream)
{
    const int rc = check_attend8(a);
    if (rc) return rc;
    if (!q || !cache || !table || !lens || !out || !workspace) return KVP_ERR_ARG;
    const Work8 w = workspace_of(a, weights != nullptr, units != nullptr);
    if (workspace_bytes < w.total) return KVP_ERR_ARG;
    if (off_by(q, 2) || off_by(cache, 16) || off_by(table, 4) || off_by(lens, 4) || off_by(units, 4) || off_by(slopes, 4) || off_by(out, 8) || off_by(lse, 4) ||
        off_by(weights, 4) || off_by(workspace, 256)) return KVP_ERR_ARG;
    Attend8K k;
    k.q = q; k.out = out; k.lse = lse; k.weights = weights;
    k.cache = static_cast<const uint8_t*>(cache); k.table = table; k.lens = lens; k.units = units; k.slopes = slopes;
    char* ws = static_cast<char*>(workspace);
    k.part = reinterpret_cast<float*>(ws);
    k.ml = reinterpret_cast<float2*>(ws + w.ml);
    k.mass = reinterpret_cast<float*>(ws + w.mass);
    k.counts = reinterpret_cast<uint32_t*>(ws + w.counts);
    k.marks = reinterpret_cast<uint32_t*>(ws + w.marks);
    k.mark_row = w.mark_row;
    k.q_batch = a->q_batch_stride; k.q_query = a->q_query_stride; k.q_head = a->q_head_stride;
    k.batch = a->batch; k.queries = a->queries; k.heads = divisor(a->cache.kv_heads); k.group = divisor(a->group);
    k.rows = a->queries * a->group; k.segs = divisor((k.rows + w.rows - 1) / w.rows);
    k.page_tiles = divisor(a->cache.page_tokens / kTileTokens); k.table_pages = a->table_pages; k.pages = a->cache.pages;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens;
    k.unit = a->unit_tokens; k.row_units = (uint32_t)(tokens / a->unit_tokens);
    k.unit_words = ((uint64_t)k.batch * k.heads.d * k.row_units + 31) / 32;
    const uint32_t sub = k.unit < kTileTokens ? k.unit : kTileTokens;
    k.row_subs = tokens / sub;
    k.sub = weights ? sub : 0;
    k.ctas = w.ctas;
    k.least = kGroup;
    k.unit_log2 = k.unit == 1 ? 0 : k.unit == 2 ? 1 : k.unit == 4 ? 2 : k.unit == 8 ? 3 : 4;
    k.scale = a->scale; k.cap = a->cap;
    const uint32_t far = 1u << 30;
    k.window = a->window < far ? a->window : 0; k.sink = a->sink < far ? a->sink : far;
    k.warp_rows = (uint64_t)k.batch * k.heads.d * k.segs.d * w.rows >= k.ctas / 4 * 8;
    k.q_aligned = ((uint64_t)(uintptr_t)q | (uint64_t)(a->q_batch_stride * 2) | (uint64_t)(a->q_query_stride * 2) | (uint64_t)(a->q_head_stride * 2)) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == KVP_F16) {
        switch (a->cache.head_dim) {
            case 64: return attend8_of<64, true>(k, w.rows, st);
            case 128: return attend8_of<128, true>(k, w.rows, st);
            default: return attend8_of<256, true>(k, w.rows, st);
        }
    }
    switch (a->cache.head_dim) {
        case 64: return attend8_of<64, false>(k, w.rows, st);
        case 128: return attend8_of<128, false>(k, w.rows, st);
        default: return attend8_of<256, false>(k, w.rows, st);
    }
}
