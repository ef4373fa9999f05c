// Attention over the cache held in 8 bits, for the last few tokens of each sequence or a chunk of a prompt (include/kvp.h, kvp_attend8).
//
// Per query row r (a query token and a query head), over the tokens i that it sees:
//   s_i = cap(scale * q . k_i) + slope * (i - position of the query),  cap(x) = cap * tanh(x / cap) or x,
//   p_i = exp(s_i - lse),  lse = log sum_i exp(s_i),  out = sum_i p_i v_i,  weights[unit] as in kvp_attend.
//
// Products. Both run on the matrix unit (tcgen05.mma, e4m3) with the cache's bytes as they lie as the left operand: 128 tokens x D dims of keys, then
// D dims x 128 tokens of values. The right operand has a column for each row, or rather for each term of a row: a number with more bits than
// e4m3's four is split into x = t0 + t1 / 32 + t2 / 1024, each the nearest e4m3 to what the ones before leave. A bf16 query is two terms and an fp16 query three,
// exactly (down to 2^-14 of the row's largest, below that to within 2^-22 of it); a weight is three terms to within 2^-13 of itself (the third's
// half step 2^-14, and what the first one leaves is rounded to fp16), down to 2^-26 of the largest. Products of e4m3 numbers are exact and the unit keeps 25 bits of their sums; terms have sums of their own, joined in fp32.
// No byte of the cache goes through a register, and a chunk of a prompt reads it once for 64 rows.
//
// exp runs in fp32 against a running maximum M of s_i + e_i - E, with 2^e_i the scale of token i's values, over the tokens that the row sees: 2^(s_i - M) times 2^(6 - E) and the scale is
// what is split. It is at most 64, and 256 before M moves: that happens only when a token passes it by 2^2 (kSlack). So neither values behind a row's mask nor large ones that get no
// weight take bits from the others. The weights' sum has the same M and so is 2^(E - e) times as large as with the largest score for M: fp32 has room for scales of 2^-90 to 2^92 (beside the
// largest, weights below 2^-27 of the row's largest are 0). E, a number once for all (kE), keeps s_i - M small, and as exact as s_i, for values of size 1; of size 2^x it is off by 2^-24 |x|.
// E taken from the values of each segment made a chunk of a prompt 822 us instead of 797 and a batch 68.6 instead of 66.5.
//
// Split over CTAs as in kvp_attend: one line of all tiles (16 tokens), cut into equal parts on the device; the join is its join.
//
// A CTA: warp 0 sends for tiles (bulk copies; a stage is eight tiles, keys and values), one thread of warp 1 issues the products with keys, one of
// warp 2 those with values, teams of four warps turn scores into weights, a token a thread. Every hand-over is a barrier in
// shared memory whose wait ends after two seconds; a CTA that gave up writes NaN.
//
// What bounds it. 131072 tokens x 8 heads of 128 dims x 8 queries with weights (270 MB, 42 us at the rate of a copy) take 57 us: 12 until the first groups are through (line,
// queries and first tiles, and the instructions' first fetch), then memory at 5.6 TB/s, 3 for the join; issue slots 37%, matrix unit 6% busy. A chunk of 512 queries x
// 4 heads over 32768 tokens x 8 heads: 797 us, 345 TFLOP/s, issue slots 61%, matrix unit 20%: 26 instructions of a warp a score, a third of them for the terms
// (a weight rounded to fp16 before it is split, 2^-11 of itself instead of 2^-13: 774).
#include <type_traits>

#include "kvp_line.cuh"
#include "kvp_mma.cuh"
#include "kvp_tile8.cuh"

namespace kvp {

namespace {

// What a CTA spends on a segment whatever its length, in tiles. Us with 16, 32, 48, 96, 144: 32 sequences of up to 8192 tokens x 8 heads of 128 dims 75, 71, 69, 74, 79 (capped), of
// 64 dims 59, 56, 57, 61, 67, of 256 114, 110, 110, 113, 116; 64 of up to 2048 60, 56, 55, 57, 60; four of up to 8192 23.4 to 21.4.
constexpr uint32_t kFixed8 = 48;
constexpr uint32_t kGroup = 8;                // tiles of a stage
constexpr uint32_t kOthers = 3;               // warps that are in no team
constexpr uint32_t kListCap8 = 1024;          // units of a bitmap row that are listed at a time: 32 words
constexpr float kSlack = 2.0f;
constexpr int kE = -7;                        // log2 of the scale of a block of normal values
constexpr float kUnit = 64.0f * (1 << -kE);   // 2^(6 - E)
constexpr float kLeastPower = -83.0f;         // e_i - E counts as no less where the maximum is looked for, also where a scale is 0
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
    wait_for_previous();
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

// D: dims of a head; ROWS: rows of a segment, 8, 16, 32 or 64. A team is four warps that turn the scores of a group (eight tiles, 128 tokens) into
// weights, a token a thread, for 16 rows at most. Teams share a group's rows (kRowTeams) and take groups in turn (kTurns): one group takes a warp 2000 cycles, most of them
// latency, so several groups are under way, in two CTAs of an SM or in turns of one, as registers allow without spills. Each turn has scores, weights and sums of its own.
// Us, 131072 tokens x 8 heads of 128 dims x 8 rows: two CTAs without turns 57.5, with two (spills) 60.5; 16 sequences of 8192 tokens x 4 heads of 128 x 12 rows: one CTA of two
// row teams and two turns 48, two CTAs with turns (spills) 59; the windowed case, 64 dims x 12 rows: 29.6 and 28.3.
__host__ __device__ constexpr bool two_ctas(uint32_t d, uint32_t rows) { return d <= 128 && (rows <= 8 || (rows == 16 && d == 64)); }
template <int D_, bool HALF_, uint32_t ROWS_>
struct Shape8 {
    static constexpr int D = D_;
    static constexpr bool HALF = HALF_;
    static constexpr uint32_t ROWS = ROWS_;
    using L = Tile8<D>;
    static constexpr uint32_t kQTerms = HALF ? 3 : 2;
    static constexpr uint32_t kQCols = (kQTerms * ROWS + 15) / 16 * 16;
    static constexpr uint32_t kPCols = (3 * ROWS + 15) / 16 * 16;
    static constexpr uint32_t kHalves = D == 256 ? 2 : 1;              // 128 dims of values a product
    static constexpr uint32_t kSumCols = kHalves * kPCols;
    static constexpr uint32_t kCtas = two_ctas(D, ROWS) ? 2 : 1;       // of an SM
    static constexpr uint32_t kRowTeams = ROWS > 16 ? ROWS / 16 : ROWS == 16 && kCtas == 1 ? 2 : 1;
    static constexpr uint32_t kTurns = (ROWS > 8 || kCtas == 1) && ROWS <= 32 && 2 * (kQCols + kSumCols) <= 512 ? 2 : 1;
    static constexpr uint32_t kTeams = kRowTeams * kTurns;
    static constexpr uint32_t kRowsEach = ROWS / kRowTeams;
    static constexpr uint32_t kBlock = 32 * kOthers + 128 * kTeams;
    static constexpr uint32_t kScoreBufs = kTurns == 2 || 2 * kQCols + kSumCols <= 512 ? 2 : 1;
    static constexpr uint32_t kColsUsed = kScoreBufs * kQCols + kTurns * kSumCols;
    static constexpr uint32_t kCols = kColsUsed <= 64 ? 64 : kColsUsed <= 128 ? 128 : kColsUsed <= 256 ? 256 : 512;
    // shared memory: a stage of keys is free when the scores are there, one of values when the sums are
    static constexpr uint32_t kKeyStage = kGroup * L::kKeyBytes, kValueStage = kGroup * L::kValueBytes;
    static constexpr uint32_t kQBytes = kQCols * D;
    static constexpr uint32_t kPBytes = kPCols * 128;
    static constexpr uint32_t kPad = D == 64 ? 2048 : 0;               // rows 64 .. 127 of the values' operand are what lies behind
    static constexpr uint32_t kStatic = kCtas == 2 ? 4096 : 6144;      // declared statically, at most
    static constexpr uint32_t kRoom = (kCtas == 2 ? 115712 : 232448) - kStatic - kQBytes - 2 * kPBytes - kPad;
    static constexpr uint32_t kKeyStages = 2;
    static constexpr uint32_t kValueFit = (kRoom - kKeyStages * kKeyStage) / kValueStage;
    static constexpr uint32_t kValueStages = kValueFit < 6 ? kValueFit : 6;
    static constexpr uint32_t kSmem = kKeyStages * kKeyStage + kValueStages * kValueStage + kQBytes + 2 * kPBytes + kPad;
    static_assert(kValueStages >= 2 && kColsUsed <= 512 && kQCols <= 256 && kPCols <= 256, "does not fit");
};

// The segments of this CTA's part, one after the other; each of the warps that are in no team goes through them by itself, the teams together.
struct Walk {
    uint32_t todo, per, entries, entry, inner, at_place, count;
    uint32_t seg, bh, rt, b, h, len, off, take, tiles;
    template <uint32_t ROWS>
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
            tiles = take;                                          // of these, those that some row sees
            if (!p.units && !p.sub && p.queries > 1) {
                const int32_t see = (int32_t)len - (int32_t)p.queries + 1 + (int32_t)p.group.of(min(rt * ROWS + ROWS, p.rows) - 1);
                const Visible v = visible_tiles(p, len);
                uint32_t last = see > 0 ? tiles_of((uint32_t)see) : 0;
                if (last > v.head) last = max(v.head, last - min(last, v.skip));
                tiles = last > off ? min(take, last - off) : 0u;
            }
            return true;
        }
        return false;
    }
};

template <class S>
struct Smem8 {
    uint64_t keys[S::kKeyStages], keys_free[S::kKeyStages];            // a stage has come; its products are done
    uint64_t values[S::kValueStages], values_free[S::kValueStages];
    uint64_t scored[2], taken[2];                      // scores are in tensor memory; they are in registers
    uint64_t weighed[2], summed[2];                    // weights are in shared memory; the products with values are done
    uint64_t query;                                    // the queries of a segment with tiles are in shared memory
    uint32_t tensor, gave_up;
    LineSmem line;
    Walk walk[2];                                      // the teams': this segment, and the next one
    bool more[2];
    uint32_t tile[S::kValueStages][kGroup];            // numbers of a stage's tiles; ~0: not there
    alignas(16) float factor[S::ROWS];                 // per row: what scores are multiplied by,
    float slope[S::ROWS];                              // its bias a token,
    int32_t see[S::ROWS];                              // the tokens that it sees are before this one
    alignas(16) float low[S::kTeams][S::kRowsEach];    // what is added to scores: less the running maximum, 0 before a row has seen a token
    alignas(16) float by[S::kTeams][S::kRowsEach];     // how far it moves; at the end of a segment [0] is below 0 for a team that had no group
    float peak[S::kTeams][4][S::kRowsEach];            // of each warp: how far its scores pass it; at the end its sum of weights
    float gone[S::kTeams][4];                          // at the end of a segment: NaN from a warp that gave up
    float2 last[S::kTeams][S::kRowsEach];              // of each turn's row: its factor, and the reciprocal of the row's sum
    uint16_t list[kListCap8];                          // units of 32 words of a bitmap's row
};

// Number of a ring's place and the parity of its turn.
template <uint32_t N>
struct Ring {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next()
    {
        if (++at == N) {
            at = 0;
            parity ^= 1u;
        }
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

// two fp32 numbers at a time
struct F2 {
    uint64_t v;
    __device__ __forceinline__ F2() {}
    __device__ __forceinline__ F2(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ void get(float& lo, float& hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
};
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 operator+(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// The first term of two fp32 numbers of at most 256, and what it leaves, 32 times as large, rounded to fp16: 2^-16 of them at most. The remainder itself is exact.
__device__ __forceinline__ uint32_t first_term(F2 x, uint32_t& left)
{
    float a, b;
    x.get(a, b);
    const uint32_t t = e4m3_pair(a, b);
    const float2 f = floats_of_e4m3(t);
    fma2(F2(f.x, f.y), F2(-32.0f, -32.0f), x * F2(32.0f, 32.0f)).get(a, b);
    left = pack(a, b);
    return t;
}
// the next term of four fp16 numbers, and what it leaves, 32 times as large; both are exact
__device__ __forceinline__ uint32_t next_term(uint32_t& a, uint32_t& b)
{
    uint32_t t, x, y;
    asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f16x2 lo, %3;\n\tcvt.rn.satfinite.e4m3x2.f16x2 hi, %4;\n\tmov.b32 %0, {lo, hi};\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, lo;\n\tcvt.rn.f16x2.e4m3x2 %2, hi;\n\t}" : "=r"(t), "=r"(x), "=r"(y) : "r"(a), "r"(b));
    const __half2 by = __float2half2_rn(32.0f), less = __float2half2_rn(-32.0f);
    a = bits_of(__hfma2(half2_of(x), less, __hmul2(half2_of(a), by)));
    b = bits_of(__hfma2(half2_of(y), less, __hmul2(half2_of(b), by)));
    return t;
}
__device__ __forceinline__ uint32_t last_term(uint32_t a, uint32_t b)
{
    uint32_t t;
    asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f16x2 lo, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 hi, %2;\n\tmov.b32 %0, {lo, hi};\n\t}" : "=r"(t) : "r"(a), "r"(b));
    return t;
}
// of two fp32 numbers
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
__device__ __forceinline__ float warp_max(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));
    return y;
}
template <uint32_t TEAMS>
__device__ __forceinline__ void teams_sync() { asm volatile("barrier.cta.sync 15, %0;" ::"n"(128 * TEAMS) : "memory"); }

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
    static_assert(sizeof(Smem8<S>) <= S::kStatic, "does not fit");
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const auto bar = [](uint64_t& b) { return smem_at(&b); };
    if (tid == 0) {
        for (uint32_t i = 0; i < S::kKeyStages; ++i) {
            barrier_init(bar(sm.keys[i]), 1);
            barrier_init(bar(sm.keys_free[i]), 1);
        }
        for (uint32_t i = 0; i < S::kValueStages; ++i) {
            barrier_init(bar(sm.values[i]), 1);
            barrier_init(bar(sm.values_free[i]), 1);
        }
        for (uint32_t i = 0; i < 2; ++i) {
            barrier_init(bar(sm.scored[i]), 1);
            barrier_init(bar(sm.taken[i]), 4 * S::kRowTeams);
            barrier_init(bar(sm.weighed[i]), 4 * S::kRowTeams);
            barrier_init(bar(sm.summed[i]), 1);
        }
        barrier_init(bar(sm.query), 4 * S::kTeams);
        sm.gave_up = 0;
        show_to_async();
    }
    wait_for_previous();
    let_next_start();                                                  // not sooner: the join looks at the lengths, and fills rows that see nothing, before it waits
    if (warp == 1) tensor_alloc<S::kCols>(smem_at(&sm.tensor));        // not sooner: the kernel before may still have to ask for its own
    Walk walk;
    {
        uint32_t entry = 0;
        const Line line = find_in_line<S::kBlock>(p, blockIdx.x, entry, sm.line);
        const uint64_t begin = (uint64_t)line.chunk * blockIdx.x;
        walk.todo = begin < line.total ? min(line.chunk, line.total - (uint32_t)begin) : 0u;       // places
        walk.per = line_per(p);
        walk.entries = line_entries(p);
        walk.entry = entry;
        walk.count = line.count;
        if (walk.todo) {
            walk.inner = ((uint32_t)begin - line.before) / (line.count + kFixed8);
            walk.at_place = ((uint32_t)begin - line.before) - walk.inner * (line.count + kFixed8);
        }
    }
    bool more = walk.next<ROWS>(p);
    if (tid == 0) {
        sm.walk[0] = walk;
        sm.more[0] = more;
    }
    uint8_t* const value_room = room + S::kKeyStages * S::kKeyStage;
    uint8_t* const queries = value_room + S::kValueStages * S::kValueStage;
    uint8_t* const weights = queries + S::kQBytes;
    tensor_before_sync();
    __syncthreads();
    tensor_after_sync();
    const uint32_t scores_at = sm.tensor, sums_at = sm.tensor + S::kScoreBufs * S::kQCols;
    volatile uint32_t* const gave_up = &sm.gave_up;

    if (warp < kOthers) {
        if (warp == 0) {
            // ---- sends for tiles ----
            bool ok = true;
            uint32_t it = 0;
            Ring<S::kKeyStages> ks;
            Ring<S::kValueStages> vs;
            for (; ok && more; more = walk.next<ROWS>(p)) {
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
                if (p.units && walk.tiles) {
                    // the chunk with the last tile of this part
                    const uint32_t chunks = (units + 1023) / 1024;
                    for (uint32_t c0 = 0;; c0 += 32) {
                        const uint32_t n = c0 + lane < chunks ? p.marks[(uint64_t)walk.bh * p.mark_row + c0 + lane] : 0u, upto = sum_upto(n, lane);
                        const uint32_t found = __ballot_sync(0xFFFFFFFFu, base + upto > walk.off + walk.tiles - 1);
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
                // Which tiles, and their pages, a lane each, 32 ahead of where they are needed: under load an entry of the table takes 2 us. The last ones come first: a
                // bias by distance favours them, and the maximum then seldom moves.
                const auto look = [&](uint32_t n0, uint32_t& tile, uint32_t& page) {
                    const bool mine = n0 + lane < walk.tiles;
                    const uint32_t i = walk.off + walk.tiles - 1 - (n0 + lane);
                    tile = 0;
                    if (p.units) {
                        bool left = mine;
                        while (true) {
                            if (left && i >= base) {
                                tile = (1024 * chunk + sm.list[(i - base) / k]) / fold * k + (i - base) % k;
                                left = false;
                            }
                            if (!__any_sync(0xFFFFFFFFu, left)) break;
                            --chunk;
                            list_chunk();
                            base -= here;
                        }
                    } else {
                        tile = i < seen.head ? i : i + seen.skip;
                    }
                    page = mine ? (uint32_t)__ldg(table + p.page_tiles.of(tile)) : ~0u;
                };
                uint32_t tiles = 0, pages = 0, next_tiles = 0, next_pages = 0;
                if (walk.tiles) look(0, next_tiles, next_pages);
                for (uint32_t g = 0; g < walk.tiles; g += kGroup, ++it) {
                    if (g % 32 == 0) {
                        tiles = next_tiles;
                        pages = next_pages;
                        if (g + 32 < walk.tiles) look(g + 32, next_tiles, next_pages);
                    }
                    // lanes 8 .. 15 do as 0 .. 7, for the values
                    const uint32_t tile = __shfl_sync(0xFFFFFFFFu, tiles, g % 32 + lane % kGroup), page = __shfl_sync(0xFFFFFFFFu, pages, g % 32 + lane % kGroup);
                    const uint8_t* from = nullptr;
                    if (lane < 2 * kGroup && page < p.pages)
                        from = p.cache + (((uint64_t)page * p.heads.d + walk.h) * p.page_tiles.d + (tile - p.page_tiles.of(tile) * p.page_tiles.d)) * L::kBytes;
                    const uint32_t many = __popc(__ballot_sync(0xFFFFFFFFu, from != nullptr) & 0xFFu);
                    if (it >= S::kKeyStages) ok = __all_sync(0xFFFFFFFFu, barrier_wait(bar(sm.keys_free[ks.at]), ks.parity ^ 1u, gave_up));
                    if (!ok) break;
                    if (lane == 0) barrier_arrive_expect(bar(sm.keys[ks.at]), many * L::kKeyBytes);
                    __syncwarp();
                    if (from && lane < kGroup) copy_bulk(smem_at(room + ks.at * S::kKeyStage) + lane * L::kKeyBytes, from, L::kKeyBytes, bar(sm.keys[ks.at]));
                    ks.next();
                    if (it >= S::kValueStages) ok = __all_sync(0xFFFFFFFFu, barrier_wait(bar(sm.values_free[vs.at]), vs.parity ^ 1u, gave_up));
                    if (!ok) break;
                    if (lane < kGroup) sm.tile[vs.at][lane] = from ? tile : ~0u;
                    __syncwarp();
                    if (lane == 0) barrier_arrive_expect(bar(sm.values[vs.at]), many * L::kValueBytes);
                    __syncwarp();
                    if (from && lane >= kGroup)
                        copy_bulk(smem_at(value_room + vs.at * S::kValueStage) + (lane - kGroup) * L::kValueBytes, from + L::kValues, L::kValueBytes, bar(sm.values[vs.at]));
                    vs.next();
                }
            }
            // copies under way end before the CTA does: the phase that a stage is in, or the one before, ends
            if (!ok) {
                for (uint32_t i = 0; i < S::kKeyStages; ++i, ks.next())
                    for (uint32_t tries = 0; tries < 1u << 14 && !barrier_try(bar(sm.keys[ks.at]), ks.parity ^ 1u); ++tries) {}
                for (uint32_t i = 0; i < S::kValueStages; ++i, vs.next())
                    for (uint32_t tries = 0; tries < 1u << 14 && !barrier_try(bar(sm.values[vs.at]), vs.parity ^ 1u); ++tries) {}
            }
        } else if (warp == 1 && lane == 0) {
            // ---- products with keys ----
            uint32_t it = 0, turn = 0;
            bool ok = true;
            Ring<S::kKeyStages> ks;
            Ring<S::kScoreBufs> sb;
            for (; ok && more; more = walk.next<ROWS>(p)) {
                if (!walk.tiles) continue;                             // nobody arrives for it either
                ok = barrier_wait(bar(sm.query), turn, gave_up);
                turn ^= 1u;
                for (uint32_t g = 0; ok && g < walk.tiles; g += kGroup, ++it) {
                    ok = barrier_wait(bar(sm.keys[ks.at]), ks.parity, gave_up) && (it < S::kScoreBufs || barrier_wait(bar(sm.taken[sb.at]), sb.parity ^ 1u, gave_up));
                    if (!ok) break;
                    tensor_after_sync();
                    const uint32_t a = smem_at(room + ks.at * S::kKeyStage), b = smem_at(queries);
#pragma unroll
                    for (uint32_t k = 0; k < D / 32; ++k)
                        multiply_e4m3(scores_at + sb.at * S::kQCols, operand(a + 256 * k, 128, 8 * D), operand(b + 256 * k, 128, 8 * D), shape_e4m3(S::kQCols), k > 0);
                    products_arrive(bar(sm.scored[sb.at]));
                    products_arrive(bar(sm.keys_free[ks.at]));
                    ks.next();
                    sb.next();
                }
            }
        } else if (warp == 2 && lane == 0) {
            // ---- products with values ----
            bool ok = true;
            Ring<S::kValueStages> vs;
            Ring<2> pb;
            for (; ok && more; more = walk.next<ROWS>(p)) {
                for (uint32_t g = 0; g < walk.tiles; g += kGroup) {
                    const uint32_t pairs = (min(walk.tiles - g, kGroup) + 1) / 2;
                    ok = barrier_wait(bar(sm.values[vs.at]), vs.parity, gave_up) && barrier_wait(bar(sm.weighed[pb.at]), pb.parity, gave_up);
                    if (!ok) break;
                    tensor_after_sync();
                    const uint32_t a = smem_at(value_room + vs.at * S::kValueStage), b = smem_at(weights + pb.at * S::kPBytes);
                    const uint32_t sums = sums_at + (S::kTurns == 2 ? pb.at * S::kSumCols : 0u);
                    for (uint32_t k = 0; k < pairs; ++k)
#pragma unroll
                        for (uint32_t half = 0; half < S::kHalves; ++half)
                            multiply_e4m3(sums + half * S::kPCols, operand(a + half * 2048 + 2 * k * L::kValueBytes, L::kValueBytes, 128), operand(b + 512 * k, 128, 2048),
                                          shape_e4m3(S::kPCols) | kColumnsContiguous, g >= S::kTurns * kGroup || k > 0);
                    products_arrive(bar(sm.values_free[vs.at]));
                    products_arrive(bar(sm.summed[pb.at]));
                    vs.next();
                    pb.next();
                }
            }
        }
        __syncwarp();
    } else {
        // ---- scores to weights: thread `me` of a team has token `me` of a group and rows row0 .. row0 + R - 1 ----
        const uint32_t team = (warp - kOthers) / 4, turn = team % S::kTurns, row0 = team / S::kTurns * R, part = warp % 4, me = part * 32 + lane;
        const uint32_t lanes = part * 32 << 16;                        // of tensor memory
        const uint32_t scores = scores_at + lanes + row0, sums = sums_at + lanes + turn * S::kSumCols + row0;
        float* const lows = sm.low[team];
        const bool plain = !(p.cap > 0.0f) && !p.slopes;
        bool ok = true;
        uint32_t it = 0;                                               // groups so far, all teams'
        Ring<S::kValueStages> vs;
        Ring<S::kScoreBufs> sb;
        Ring<2> pb;
        for (uint32_t side = 0; sm.more[side]; side ^= 1u) {
            const Walk& walk = sm.walk[side];                  // not in registers: the loop over groups needs them
            if (tid == 32 * kOthers) {
                Walk ahead = walk;
                sm.more[side ^ 1u] = ahead.next<ROWS>(p);
                sm.walk[side ^ 1u] = ahead;
            }
            // the queries: kEach threads a row
            {
                constexpr uint32_t kFew = 128 * S::kTeams / ROWS, kEach = kFew < D / 8 ? kFew : D / 8, kVecs = D / 8 / kEach;
                const uint32_t t = tid - 32 * kOthers, row = t / kEach, j = t % kEach, r = walk.rt * ROWS + row, query = p.group.of(min(r, p.rows - 1));     // rows that are none see what the last one does
                const bool mine = row < ROWS;
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
                // largest magnitude in [2^7, 2^8), or below it where it is not a normal number; the power of two in two factors, either of them a normal number
                const int e = (__float_as_int(most) >> 23) - 127 - 7, half_e = -e / 2;
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
                    sm.factor[row] = unit * __int_as_float((127 - half_e) << 23) * __int_as_float((127 + e + half_e) << 23) + odd;
                    sm.slope[row] = p.slopes && r < p.rows ? __ldg(p.slopes + walk.h * p.group.d + (r - query * p.group.d)) * kLog2e : 0.0f;
                    sm.see[row] = (int32_t)walk.len - (int32_t)p.queries + 1 + (int32_t)query;
                }
                // Only where products follow: the teams then wait for their scores, and are never more than one such segment ahead of the thread that looks at the parity.
                show_to_async();
                __syncwarp();
                if (lane == 0 && walk.tiles) barrier_arrive(bar(sm.query));
                if (me < R) lows[me] = 0.0f;
                teams_sync<S::kTeams>();
            }
            const uint32_t tiles = walk.tiles, len = walk.len;
            float l[R];                                                // sums of this thread's weights
            bool any = false;                                          // has this team had a group of the segment?
            bool first = true, unset = true;                           // row `me` has not seen a token; some row has not
            const int32_t see_least = sm.see[row0], see_most = sm.see[row0 + R - 1];       // later rows are those of later queries
            const int32_t window = p.window ? (int32_t)p.window : INT32_MAX / 2, sink = (int32_t)p.sink;
#pragma unroll
            for (uint32_t r = 0; r < R; ++r) l[r] = 0.0f;
            float* const mass = p.mass + (uint64_t)walk.seg * p.row_subs * ROWS + row0;

            for (uint32_t g = 0; g < tiles; g += kGroup, ++it, vs.next(), sb.next(), pb.next()) {
                if (S::kTurns == 2 && it % 2 != turn) continue;
                const uint32_t j = me / 16, many = min(tiles - g, kGroup);
                ok = ok && barrier_wait(bar(sm.values[vs.at]), vs.parity, gave_up);
                uint8_t* const block = value_room + vs.at * S::kValueStage + j * L::kValueBytes;
                const uint32_t tile = j < many ? sm.tile[vs.at][j] : ~0u;
                const int32_t pos = (int32_t)(tile * kTileTokens + me % 16);
                const float2 scales = *reinterpret_cast<const float2*>(block + 16 * D);        // of keys, of values
                bool live = tile != ~0u && pos < (int32_t)len;
                if (live && p.units && p.unit < kTileTokens) live = bits_at(p, (uint64_t)walk.bh * p.row_units + ((uint32_t)pos >> p.unit_log2)) & 1u;
                const float scale = live ? scales.y : 0.0f, power = fmaxf((float)((__float_as_int(scale) >> 23) - 127 - kE), kLeastPower);
                // does every row see every token of the warp?
                const bool all_seen = __all_sync(0xFFFFFFFFu, live && pos < see_least && (pos >= see_most - window || pos < sink));
                ok = ok && barrier_wait(bar(sm.scored[sb.at]), sb.parity, gave_up);
                __syncwarp();
                tensor_after_sync();
                float s[R];                                            // scores, less the maximum, then weights
#pragma unroll
                for (uint32_t r = 0; r < R; r += 8) {
                    float x[S::kQTerms][8];
#pragma unroll
                    for (uint32_t term = 0; term < S::kQTerms; ++term) tensor_load(scores + sb.at * S::kQCols + term * ROWS + r, x[term]);
                    tensor_wait_load();
#pragma unroll
                    for (uint32_t term = 0; term < S::kQTerms; ++term) tensor_hold(x[term]);
                    const F2 one(scales.x, scales.x), small(scales.x * 0x1p-5f, scales.x * 0x1p-5f), least(scales.x * 0x1p-10f, scales.x * 0x1p-10f);
#pragma unroll
                    for (uint32_t i = 0; i < 8; i += 2) {
                        F2 y = F2(x[0][i], x[0][i + 1]) * one;
                        y = fma2(F2(x[1][i], x[1][i + 1]), small, y);
                        if (S::kQTerms == 3) y = fma2(F2(x[S::kQTerms - 1][i], x[S::kQTerms - 1][i + 1]), least, y);
                        y.get(s[r + i], s[r + i + 1]);
                    }
                }
                tensor_before_sync();
                __syncwarp();
                if (lane == 0) barrier_arrive(bar(sm.taken[sb.at]));
                if (plain) {
#pragma unroll
                    for (uint32_t r = 0; r < R; r += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(sm.factor + row0 + r), low = *reinterpret_cast<const float4*>(lows + r);
                        fma2(F2(s[r], s[r + 1]), F2(f.x, f.y), F2(low.x, low.y)).get(s[r], s[r + 1]);
                        fma2(F2(s[r + 2], s[r + 3]), F2(f.z, f.w), F2(low.z, low.w)).get(s[r + 2], s[r + 3]);
                    }
                } else {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) {
                        s[r] *= sm.factor[row0 + r];
                        if (p.cap > 0.0f) s[r] = tanhf(s[r]) * (p.cap * kLog2e);
                        if (p.slopes) s[r] = fmaf(sm.slope[row0 + r], (float)(pos - sm.see[row0 + r] + 1), s[r]);
                        s[r] += lows[r];
                    }
                }
                if (!all_seen) {
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) {
                        const int32_t see = sm.see[row0 + r];
                        s[r] = live && pos < see && (pos >= see - window || pos < sink) ? s[r] : -INFINITY;
                    }
                }
                float over = -INFINITY;                                // with `power`: how far tokens pass the maximum
#pragma unroll
                for (uint32_t r = 0; r < R; r += 2) over = fmaxf(over, fmaxf(s[r], s[r + 1]));
                if (team_any(over + power > kSlack || unset || !ok, team)) {
                    float x = 0.0f;
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) {
                        const float y = warp_max(__fadd_ru(s[r], power));              // never less than it is, however large scores are
                        if (lane == r) x = y;
                    }
                    if (lane < R) sm.peak[team][part][lane] = x;
                    // the sums of the team's group before are to be there, all of them
                    if (any) ok = ok && barrier_wait(bar(sm.summed[S::kTurns == 2 ? pb.at : pb.at ^ 1u]), S::kTurns == 2 || pb.at == 0 ? pb.parity ^ 1u : pb.parity, gave_up);
                    __syncwarp();
                    if (team_any(!ok, team)) { ok = false; break; }    // also: the maxima are there
                    tensor_after_sync();
                    bool none = false;                                 // has row `me` not seen a token?
                    if (me < R) {
                        float up = fmaxf(fmaxf(sm.peak[team][0][me], sm.peak[team][1][me]), fmaxf(sm.peak[team][2][me], sm.peak[team][3][me]));
                        if (first) up = fmaxf(up, kNone);              // the first maximum, whatever its sign
                        else up = fmaxf(up, 0.0f);
                        none = up == kNone;
                        first = none;
                        if (none) up = 0.0f;
                        // what the maximum moves by once it is rounded is what the sums are told
                        const float low = lows[me], now = __fsub_rd(low, up);
                        sm.by[team][me] = low - now;
                        lows[me] = now;
                    }
                    unset = team_any(none, team);                      // also: the new maxima are there
                    if (any) {
#pragma unroll 1
                        for (uint32_t c = 0; c < 3 * S::kHalves; ++c)
#pragma unroll
                            for (uint32_t r = 0; r < R; r += 8) {
                                const uint32_t at = sums + c / 3 * S::kPCols + c % 3 * ROWS + r;
                                float y[8];
                                tensor_load(at, y);
                                tensor_wait_load();
                                tensor_hold(y);
#pragma unroll
                                for (uint32_t i = 0; i < 8; ++i) y[i] *= exp2_fast(fminf(-sm.by[team][r + i], 0.0f));
                                tensor_store(at, y);
                            }
                        tensor_wait_store();
                        tensor_before_sync();
                    }
#pragma unroll
                    for (uint32_t r = 0; r < R; ++r) {
                        const float up = sm.by[team][r];
                        s[r] -= up;
                        l[r] *= exp2_fast(fminf(-up, 0.0f));           // a first maximum may be below 0; the sums are 0 then
                    }
                }
                any = true;
#pragma unroll
                for (uint32_t r = 0; r < R; r += 2) {
                    s[r] = exp2_fast(s[r]);
                    s[r + 1] = exp2_fast(s[r + 1]);
                    (F2(l[r], l[r + 1]) + F2(s[r], s[r + 1])).get(l[r], l[r + 1]);
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
                        for (int i = 0; i < LEFT; ++i) to[i] = log2_fast(x[i]) - lows[from + i];
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
                if (it >= 2) ok = ok && barrier_wait(bar(sm.summed[pb.at]), pb.parity ^ 1u, gave_up);
                const float by = scale * kUnit;
                uint8_t* const to = weights + pb.at * S::kPBytes + me * 16;
                uint32_t term[3][R / 4];
#pragma unroll
                for (uint32_t r = 0; r < R; r += 4) {
                    const F2 both(by, by);
                    uint32_t a, b;
                    term[0][r / 4] = first_term(F2(s[r], s[r + 1]) * both, a) | first_term(F2(s[r + 2], s[r + 3]) * both, b) << 16;
                    term[1][r / 4] = next_term(a, b);
                    term[2][r / 4] = last_term(a, b);
                }
                if constexpr (ROWS == 8) {
                    *reinterpret_cast<uint4*>(to) = make_uint4(term[0][0], term[0][1], term[1][0], term[1][1]);
                    *reinterpret_cast<uint2*>(to + 2048) = make_uint2(term[2][0], term[2][1]);
                } else if constexpr (R == 8) {
#pragma unroll
                    for (uint32_t i = 0; i < 3; ++i)
                        *reinterpret_cast<uint2*>(to + (i * ROWS + row0) / 16 * 2048 + row0 % 16) = make_uint2(term[i][0], term[i][1]);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 3; ++i)
                        *reinterpret_cast<uint4*>(to + (i * ROWS + row0) / 16 * 2048) = make_uint4(term[i][0], term[i][1], term[i][2], term[i][3]);
                }
                // What lies in the cache where no token is may be anything, also NaN, and so may a tile that did not come: its values are cleared.
                const uint32_t lives = __ballot_sync(0xFFFFFFFFu, live) >> (lane & 16u) & 0xFFFFu;
                if (row0 == 0 && !all_seen && lives != 0xFFFFu && j < (many + 1) / 2 * 2) {
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
                if (lane == 0) barrier_arrive(bar(sm.weighed[pb.at]));
            }

            // ---- the end of a segment: the turns' sums are joined, each team writes some of the rows ----
            if (any) {
                // the last group of this team: pb stands behind the segment's last group
                const bool mine_last = S::kTurns == 1 || (it - 1) % 2 == turn;
                const uint32_t behind = S::kTurns == 1 || mine_last ? 1u : 2u;             // groups since
                const uint32_t at = (pb.at + 2 - behind) % 2, parity = behind > pb.at ? pb.parity ^ 1u : pb.parity;
                ok = ok && barrier_wait(bar(sm.summed[at]), parity, gave_up);
            }
            __syncwarp();
            {
                uint32_t from;
                sum_neighbours<R, 5>(l, lane, from);                   // R <= 16: one row a lane is left
                sm.peak[team][part][from] = l[0];                      // the same from lanes of the same row
            }
            if (lane == 0) sm.gone[team][part] = ok ? 0.0f : NAN;
            teams_sync<S::kTeams>();
            tensor_after_sync();
            const bool whole = walk.take == walk.count;
            const uint64_t slot = (uint64_t)blockIdx.x + walk.seg;
            constexpr uint32_t F = R / S::kTurns;                      // rows of a team now
            const uint32_t mine = turn * F, team0 = team - turn, row_at = walk.rt * ROWS + row0 + mine;
            const auto place = [&](uint32_t row) {
                const uint32_t query = p.group.of(row);
                return ((uint64_t)walk.b * p.queries + query) * (p.heads.d * p.group.d) + walk.h * p.group.d + (row - query * p.group.d);
            };
            if (me < F) {
                // row mine + me: its maximum and sum over the turns. Sums come with powers of two of their own (the scales of the values at the maximum): such a power goes over to
                // the maximum, so that those of other turns and other parts can be compared with it.
                float m = kNone, sum = 0.0f, one[S::kTurns], high[S::kTurns];
#pragma unroll
                for (uint32_t u = 0; u < S::kTurns; ++u) {
                    const float* x = &sm.peak[team0 + u][0][mine + me];
                    const float* gone = sm.gone[team0 + u];
                    one[u] = ((x[0] + x[R]) + (x[2 * R] + x[3 * R])) + ((gone[0] + gone[1]) + (gone[2] + gone[3]));
                    const int power = min(max((__float_as_int(one[u]) >> 23 & 0xFF) - 127, -126), 126);
                    high[u] = (float)power - sm.low[team0 + u][mine + me];
                    if (one[u] != 0.0f) m = fmaxf(m, high[u]);
                    one[u] *= __int_as_float((127 - power) << 23);
                }
#pragma unroll
                for (uint32_t u = 0; u < S::kTurns; ++u) {
                    const bool some = one[u] != 0.0f;
                    sum = fmaf(one[u], some ? exp2_fast(high[u] - m) : 0.0f, sum);
                    sm.last[team0 + u][mine + me].x = some ? 1.0f / kUnit * exp2_fast(-sm.low[team0 + u][mine + me] - m) : 0.0f;
                }
                const float by = whole ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
                sm.last[team0][mine + me].y = by;
                p.ml[slot * ROWS + row0 + mine + me] = make_float2(m, sum);
                if (whole && p.lse && row_at + me < p.rows) p.lse[place(row_at + me)] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
            }
            if (me == 0) sm.by[team][0] = any ? 0.0f : -1.0f;
            teams_sync<S::kTeams>();
#pragma unroll 1
            for (uint32_t i = 0; i < S::kHalves * F / 4; ++i) {
                const uint32_t half = i / (F / 4), r = mine + i % (F / 4) * 4, d = half * 128 + me;
                float y[4] = {0, 0, 0, 0};
#pragma unroll
                for (uint32_t u = 0; u < S::kTurns; ++u) {
                    if (sm.by[team0 + u][0] < 0.0f) continue;          // uniform: nothing was written there
                    float x[3][4];
#pragma unroll
                    for (uint32_t c = 0; c < 3; ++c) tensor_load(sums_at + lanes + u * S::kSumCols + half * S::kPCols + c * ROWS + row0 + r, x[c]);
                    tensor_wait_load();
#pragma unroll
                    for (uint32_t c = 0; c < 3; ++c) tensor_hold(x[c]);
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)
                        y[k] = fmaf(fmaf(fmaf(x[2][k], 0x1p-5f, x[1][k]), 0x1p-5f, x[0][k]), sm.last[team0 + u][r + k].x, y[k]);
                }
                if (d < D) {
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k) {
                        const uint32_t row = walk.rt * ROWS + row0 + r + k;
                        const float x = y[k] * sm.last[team0][r + k].y;
                        if (!whole) p.part[(slot * ROWS + row0 + r + k) * D + d] = x;
                        else if (row < p.rows) static_cast<uint16_t*>(p.out)[place(row) * D + d] = S::HALF ? __half_as_ushort(__float2half_rn(x)) : __bfloat16_as_ushort(__float2bfloat16_rn(x));
                    }
                }
            }
            tensor_before_sync();
            teams_sync<S::kTeams>();
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
    const uint64_t most = two_ctas(a->cache.head_dim, w.rows) ? 296 : 148;
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
    // scores in units of the cap, and the cap to the base 2, are normal numbers
    if (a->cap > 0.0f && (!(fabsf(a->scale / a->cap) < INFINITY) || !(a->cap * kLog2e < INFINITY) || (a->scale != 0.0f && fabsf(a->scale / a->cap) < 0x1p-126f))) return KVP_ERR_ARG;
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
    int rc = k.units ? launch(count8_kernel, k.batch * k.heads.d, kThreads, 0, true, st, k) : KVP_OK;
    if (!rc) rc = launch(attend8_kernel<S>, k.ctas, S::kBlock, S::kSmem, true, st, k);
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
