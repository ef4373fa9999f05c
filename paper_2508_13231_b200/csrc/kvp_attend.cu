// Attention over the cache held in 4 bits, for the last few tokens of each sequence, and the weight that every unit of the
// cache received (include/kvp.h, kvp_attend).
//
// Per query row r (a query token and a query head), over the tokens i that it sees:
//   s_i = scale * q . k_i,  p_i = exp(s_i - lse),  lse = log sum_i exp(s_i),  out = sum_i p_i v_i,
//   weights[unit] = sum over the rows of a kv-head and the tokens of the unit of p_i.
//
// Products. Up to eight rows that share a kv-head are one segment; the matrix instruction m16n8k16 takes 16 tokens x 16 dims of
// keys as its left operand and the rows as its right one, so that no row is padding where eight heads share a kv-head.
// (tcgen05.mma takes 64 or 128 rows of tokens and eight columns at least, as far as decoding goes: its operands would have to be unpacked to shared memory first,
// and the tensor pipe is 23% busy as it is. A chunk of a prompt, with hundreds of rows a kv-head, would fill it; here it reads the cache once for every eight rows.)
// The 4-bit whole numbers enter as fp16 subnormals, two by one AND and no conversion (values as they lie, q 2^-24 and q 2^-20; keys shifted to bits 4 .. 7
// of a significand, q 2^-20, because leading zeros cost bits of the sum); products with fp16 queries are exact and summed in fp32. Scales act on the sums of
// 32 dims in fp32, the zeros on the sums of the query's dims, which enter as two fp16 terms (22 bits). A row's queries are divided by a power
// of two first, so that bf16 ones fit fp16 whatever their size.
// exp runs in fp32 against a running maximum that moves only when a score passes it by 2^2 (kSlack; seldom behind the first tiles), sums are fp32. The weights p
// times the scales of the values are the second product's right operand, in fp16 (11 bits, half a step is 2^-11 of a weight at most; the
// output has 8 or 11 bits). So that the product keeps them, a weight enters as up to 2^13 .. 2^15, and scales of which none so far
// reached 2^-7 are multiplied by a power of two that brings the largest to 1 .. 2; larger ones than 2 take as much off the weights.
//
// Split. The tiles (16 tokens) of all segments stand in one line that is cut into equal parts, one for each CTA, on the device,
// where the lengths are known: any mix of lengths, and rows of a bitmap with any number of units, keep all SMs busy alike. A CTA
// takes a segment's tiles in turn by its eight warps, which join their sums in shared memory; segments that more than one
// CTA worked on are joined by the second kernel, which also turns what was noted per unit into weights. The order of every sum is
// fixed, so results do not change from run to run.
//
// What bounds it. A warp works on two tiles at a time (346 instructions a tile, all of a call's counted; two share the exchange of maxima, the loads of queries
// and the loop), with two more on their way through cp.async, 16 warps an SM at 128 registers: latency at that number of warps, with issue slots 55% and DRAM
// half busy. 8 x 131072 tokens x 8 heads of 128 dims x 8 queries, 1.34 GB, take 251 us (5.3 TB/s; 274 with weights), one such sequence 45 us where 26 would move
// its bytes: 6 us until the first tiles are there, 3 for the join of the warps, and CTAs that end at different times. Fewer registers and more
// warps spill; 4 warps a CTA were faster on batches (45 instead of 48 us) and slower here (51).
#include "kvp_line.cuh"

namespace kvp {

namespace {

constexpr uint32_t kRows = 8;                 // query rows of a segment
constexpr uint32_t kListCap = 1024;           // tiles of a bitmap row that are listed at a time
constexpr uint32_t kNibble = 0x00F000F0u;     // bits 4 .. 7 of two fp16 significands
constexpr float kLift = 13.0f, kSlack = 2.0f; // weights are at most 2^(kLift + kSlack), 2^kLift right after the maximum moved
constexpr float kRaise = 15.0f;               // scales of values are multiplied by at most 2^15, which fp16 holds
constexpr int kSmall = -7;                    // and only if none of them reached 2^-7
constexpr uint32_t kFrom2 = 0x40004000u, kFromSmall = 0x60006000u;   // bits that one of two fp16 numbers has from 2 on, and from 2^-7 on

// What a CTA spends on a segment whatever its length, in tiles.
// Us with kFixed 16, 32, 48, 64, 96: 32 sequences of up to 8192 tokens x 8 heads of 128 dims 56, 53, 53, 54, 57, of 64 dims 39, 37, 37, 39, 41, of 256 105, 98,
// 95, 97, 100; 64 of up to 2048 43, 39, 39, 41, 42 (64 dims 31, 29, 30, 31, 32); one of 131072 45, 44, 43, 43, 43; four of up to 8192 14.5 to 15.1.
constexpr uint32_t kFixed = 48;

struct AttendK : LineK<kFixed> {
    const void* q;
    const uint8_t* cache;
    int64_t q_batch, q_query, q_head;
    float scale;
    bool q_aligned;          // every eight dims of a query lie at a 16-byte boundary
};

// counts[bh]: tiles to read of a row of the bitmap; one CTA per row
__global__ void __launch_bounds__(kThreads) count_kernel(const AttendK p)
{
    __shared__ uint32_t sum[kWarps];
    let_next_start();
    const uint32_t bh = blockIdx.x, tid = threadIdx.x;
    const uint32_t len = length_of(p, p.heads.of(bh)), units = units_of(p, len), tiles = tiles_of(len);
    const uint32_t k = p.unit > kTileTokens ? p.unit / kTileTokens : 1;
    uint32_t n = 0;
    for (uint32_t w = tid; 32u * w < units; w += kThreads) {
        const uint32_t x = unit_word(p, bh, w, units);
        n += __popc(x) * k;
        if (k > 1 && units - 32u * w <= 32u && (x >> (units - 1u - 32u * w)) & 1u) n -= units * k - tiles;   // the last unit may be cut
    }
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    if (tid % 32 == 0) sum[tid / 32] = n;
    __syncthreads();
    if (tid == 0) {
        for (uint32_t i = 1; i < (uint32_t)kWarps; ++i) n += sum[i];
        p.counts[bh] = n;
    }
}

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0,
                                    float c1, float c2, float c3)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    mma(c, a0, a1, a2, a3, b0, b1, c[0], c[1], c[2], c[3]);
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t times(uint32_t a, uint32_t b) { return bits_of(__hmul2(half2_of(a), half2_of(b))); }
__device__ __forceinline__ float over_rows(float x)                 // sum over the lanes that hold other tokens of the same rows
{
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
    return x + __shfl_xor_sync(0xFFFFFFFFu, x, 16);
}

// eight dims of a query
__device__ __forceinline__ uint4 load_q(const AttendK& p, int64_t at, bool real)
{
    uint4 x = make_uint4(0, 0, 0, 0);
    if (real) {
        const uint16_t* from = static_cast<const uint16_t*>(p.q) + at;
        if (p.q_aligned) {
            x = __ldg(reinterpret_cast<const uint4*>(from));
        } else {
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __ldg(from + i);
            x = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
    }
    return x;
}
template <bool HALF>
__device__ __forceinline__ void floats_of(uint32_t x, float* to)
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
template <int N>
struct Shape {
    static constexpr int kStages = N == 2 ? 8 : 4;                  // tiles of a warp under way, two of them worked on
    static constexpr uint32_t kRing = kWarps * kStages * Tile<N>::kBytes;
    static constexpr uint32_t kJoin = kWarps * kRows * 32 * N * 4;
    static constexpr uint32_t kSmem = kRing > kJoin ? kRing : kJoin;
};

struct AttendSmem {
    LineSmem line;
    uint32_t list[kListCap];
    uint32_t scan[kWarps];
    float2 ml[kWarps][kRows];
    float share[kWarps][kRows];
    alignas(16) uint4 query[8][32];          // per group of 32 dims: each lane's fragments
    float sums[8][kRows], factor[kRows];     // of the scaled queries per group and row; what scores are multiplied by
};

// list[i] = number of the (from + i)-th tile of row bh that is to be read, i < many <= kListCap. Every thread of the CTA calls it.
__device__ __forceinline__ void list_tiles(const AttendK& p, uint32_t bh, uint32_t len, uint32_t from, uint32_t many, AttendSmem& sm)
{
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, units = units_of(p, len), tiles = tiles_of(len);
    const uint32_t k = p.unit > kTileTokens ? p.unit / kTileTokens : 1, fold = p.unit < kTileTokens ? kTileTokens / p.unit : 1;
    uint32_t seen = 0;
    for (uint32_t w0 = 0; 32u * w0 < units && seen < from + many; w0 += kThreads) {
        const uint32_t w = w0 + tid;
        uint32_t bits = 32u * w < units ? unit_word(p, bh, w, units) : 0u;
        uint32_t mine = __popc(bits) * k;                    // the last unit may be cut, but nothing stands behind it
        uint32_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= (uint32_t)o) upto += v;
        }
        if (lane == 31) sm.scan[warp] = upto;
        __syncthreads();
        uint32_t at = seen + upto - mine;
#pragma unroll
        for (uint32_t i = 0; i < (uint32_t)kWarps; ++i) {
            const uint32_t n = sm.scan[i];
            if (i < warp) at += n;
            seen += n;
        }
        if (at < from + many && at + mine > from)
            for (; bits; bits &= bits - 1u) {
                const uint32_t tile = (32u * w + __ffs(bits) - 1u) / fold * k;
                for (uint32_t j = 0; j < k; ++j, ++at)
                    if (at >= from && at - from < many && tile + j < tiles) sm.list[at - from] = tile + j;
            }
        __syncthreads();
    }
}

// HALF: fp16 queries and outputs, else bf16. fp16 outputs keep three more bits, so there the weights enter the second product as two fp16
// terms (22 bits).
template <int N, bool HALF>
__global__ void __launch_bounds__(kThreads, N == 8 ? 1 : 2) attend_kernel(const AttendK p)
{
    using L = Tile<N>;
    using S = Shape<N>;
    constexpr int kStages = S::kStages;
    extern __shared__ __align__(16) uint8_t ring_all[];
    __shared__ AttendSmem sm;
    let_next_start();
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, g = lane >> 2, t = lane & 3;
    wait_for_previous();
    uint32_t entry = 0;
    const Line line = find_in_line(p, blockIdx.x, entry, sm.line);
    const uint64_t begin = (uint64_t)line.chunk * blockIdx.x;
    if (begin >= line.total) return;
    uint32_t todo = min(line.chunk, line.total - (uint32_t)begin);  // places
    const uint32_t per = line_per(p), E = line_entries(p);
    uint32_t count = line.count, inner = ((uint32_t)begin - line.before) / (count + kFixed);
    uint32_t at_place = ((uint32_t)begin - line.before) - inner * (count + kFixed);      // in the segment
    uint8_t* const ring = ring_all + warp * kStages * L::kBytes;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    // a fragment's row g is token 4 (g / 2) + g % 2 of the tile, its row g + 8 the token two further on: a thread then needs the
    // values of the four tokens 4 t .. 4 t + 3
    const uint32_t tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;

    for (; todo; ++inner, at_place = 0) {
        while (inner == per || !count) {
            if (++entry >= E) return;                              // not reached: the line ends with the last part
            count = entry_count(p, entry);
            inner = 0;
        }
        const uint32_t places = min(todo, count + kFixed - at_place);
        todo -= places;
        if (at_place + places <= kFixed) continue;                 // no tile among them
        const uint32_t off = at_place > kFixed ? at_place - kFixed : 0u, take = at_place + places - kFixed - off;
        const uint32_t seg = entry * per + inner, bh = p.segs.of(seg), rt = seg - bh * p.segs.d, b = p.heads.of(bh), h = bh - b * p.heads.d;
        const uint32_t len = length_of(p, b);
        const int32_t* table = p.table + (uint64_t)b * p.table_pages;

        uint32_t done = 0, many = 0, mine = 0, where = ~0u, bad = 0;   // this chunk of the segment's tiles, and this warp's part of it
        auto tile_no = [&](uint32_t k) { const uint32_t i = warp + k * kWarps; return p.units ? sm.list[i] : off + i; };
        auto issue = [&](uint32_t k) {
            const uint32_t stage = k % kStages;
            if (k % 32 == 0) {                                 // where the next 32 tiles lie, one a lane
                where = ~0u;
                if (k + lane < mine) {
                    const uint32_t tile = tile_no(k + lane), page = p.page_tiles.of(tile);
                    const uint32_t pg = (uint32_t)__ldg(table + page);
                    if (pg < p.pages) where = (pg * p.heads.d + h) * p.page_tiles.d + (tile - page * p.page_tiles.d);
                }
            }
            const uint32_t at = __shfl_sync(0xFFFFFFFFu, where, k % 32);
            if (at != ~0u) {
                const uint8_t* from = p.cache + (uint64_t)at * L::kBytes + lane * 16;
                const uint32_t to = ring_at + stage * L::kBytes + lane * 16;
#pragma unroll
                for (uint32_t c = 0; c < L::kBytes / 16; c += 32)
                    if (L::kBytes / 16 - c >= 32 || lane < L::kBytes / 16 - c)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + c * 16), "l"(from + c * 16) : "memory");
                bad &= ~(1u << stage);
            } else {
                bad |= 1u << stage;                            // no tile, or in a page that is none
            }
        };
        auto send = [&](int from, int to) {
#pragma unroll 1
            for (int k = from; k < to; k += 2) {
                if (k < (int)mine) { issue(k); issue(k + 1); }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        };
        auto begin_chunk = [&]() {                                 // lists its tiles and sends for the first two
            many = p.units ? min(take - done, kListCap) : take;
            if (p.units) {
                __syncthreads();
                list_tiles(p, bh, len, off + done, many, sm);
            }
            mine = many > warp ? (many - warp + kWarps - 1) / kWarps : 0;
            where = ~0u;
            bad = 0;
            send(0, 2);
        };
        uint4 raw[N];                                              // this thread's part of row g's query: on their way before the tiles
        {
            const uint32_t r = rt * kRows + g, query = p.group.of(r);
            const int64_t at = b * p.q_batch + (int64_t)query * p.q_query + (int64_t)(h * p.group.d + (r - query * p.group.d)) * p.q_head + t * 8;
#pragma unroll
            for (int n = 0; n < N; ++n) raw[n] = load_q(p, at + n * 32, r < p.rows);
        }
        begin_chunk();

        // The queries as the right operand, divided by a power of two, and their sums over groups for the zeros. A warp prepares one group for
        // all; they stay in shared memory, which is read once for two tiles: 16 registers more would be too many.
        {
            float most = 0.0f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float x[8];
                floats_of<HALF>(raw[n].x, x);
                floats_of<HALF>(raw[n].y, x + 2);
                floats_of<HALF>(raw[n].z, x + 4);
                floats_of<HALF>(raw[n].w, x + 6);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
            }
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            // largest magnitude in [2^6, 2^7); the power of two in two factors, either of them a normal number
            const int e = most > 0.0f && most < INFINITY ? ilogbf(most) - 6 : 0, half_e = -e / 2;
            const float by0 = __int_as_float((half_e + 127) << 23), by1 = __int_as_float((-e - half_e + 127) << 23);
            if (warp < N) {
                uint4 mine = raw[0];
#pragma unroll
                for (int n = 1; n < N; ++n) mine = warp == (uint32_t)n ? raw[n] : mine;
                float x[8], sum = 0.0f;
                floats_of<HALF>(mine.x, x);
                floats_of<HALF>(mine.y, x + 2);
                floats_of<HALF>(mine.z, x + 4);
                floats_of<HALF>(mine.w, x + 6);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = x[i] * by0 * by1;
                    sum += x[i];
                }
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
                sm.query[warp][lane] = make_uint4(pack(x[0], x[4]), pack(x[1], x[5]), pack(x[2], x[6]), pack(x[3], x[7]));
                if (t == 0) sm.sums[warp][g] = sum;
            }
            if (warp == 0 && t == 0) sm.factor[g] = scalbnf(p.scale * 1.4426950408889634f, e);
        }
        __syncthreads();
        uint32_t qz[N == 8 ? 2 : 1];
        // the right operand of the zeros' product, 2 N columns: the upper parts of the sums and what those leave
#pragma unroll
        for (int j = 0; j < (N == 8 ? 2 : 1); ++j) {
            float col[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t c = 8 * j + 2 * t + i, kind = c / N;
                const float sum = sm.sums[c % N][g], up = __half2float(__float2half_rn(sum)), part = kind & 1 ? sum - up : up;
                col[i] = kind > 1 ? 0.0f : part;
            }
            qz[j] = pack(col[0], col[1]);
        }
        const float f0 = sm.factor[2 * t], f1 = sm.factor[2 * t + 1];
        // rows 2 t and 2 t + 1 see the tokens before these, all rows those before `all`
        int32_t see0, see1, all;
        {
            const int32_t first = (int32_t)len - (int32_t)p.queries + 1;
            see0 = min(first + (int32_t)p.group.of(rt * kRows + 2 * t), (int32_t)len);
            see1 = min(first + (int32_t)p.group.of(rt * kRows + 2 * t + 1), (int32_t)len);
            all = min(first + (int32_t)p.group.of(rt * kRows), (int32_t)len);
        }
        float* const mass = p.mass + (uint64_t)seg * p.row_subs * kRows + 2 * t;

        float o[2 * N][4], zsum[4] = {0, 0, 0, 0}, m0 = kNone, m1 = kNone, l0 = 0.0f, l1 = 0.0f;
        // weights are 2^(s - d), d = m - min(lift, kLift); scales of values are multiplied by 2^(lift - kLift) where that is more than 1
        float lift = kLift, d0 = kNone, d1 = kNone;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;

        auto rescale_sums = [&](float c0, float c1) {
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) {
                o[i][0] *= c0;
                o[i][1] *= c1;
                o[i][2] *= c0;
                o[i][3] *= c1;
            }
        };
        auto rescale_weights = [&](float c0, float c1) {
            l0 *= c0;
            l1 *= c1;
            zsum[0] *= c0;
            zsum[1] *= c1;
        };

        while (true) {
            send(2, kStages);                                      // not sooner: the first two tiles of every warp are to come first
#pragma unroll 1
            for (uint32_t k = 0; k < mine; k += 2) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kStages / 2 - 1) : "memory");
                __syncwarp();
                const uint32_t stage = k % kStages;
                const uint8_t* const tile0 = ring + stage * L::kBytes;
                const uint32_t none = bad >> stage & 3u;           // of the two tiles, those that are not there
                const uint32_t no0 = tile_no(k), no1 = k + 1 < mine ? tile_no(k + 1) : no0;

                // scores of tokens a and b for rows 2t and 2t + 1
                float s[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint8_t* tile = tile0 + u * L::kBytes;
                    uint32_t wa[N], wb[N], sa[N / 2], sb[N / 2];
                    float z[4], sum[4] = {0, 0, 0, 0};
                    if constexpr (N == 2) {
                        *reinterpret_cast<uint2*>(wa) = *reinterpret_cast<const uint2*>(tile + L::key_word(tok_a, t, 0));
                        *reinterpret_cast<uint2*>(wb) = *reinterpret_cast<const uint2*>(tile + L::key_word(tok_b, t, 0));
                        sa[0] = *reinterpret_cast<const uint32_t*>(tile + L::key_meta(tok_a, 0));
                        sb[0] = *reinterpret_cast<const uint32_t*>(tile + L::key_meta(tok_b, 0));
                    } else {
#pragma unroll
                        for (int n = 0; n < N; n += 4) {
                            *reinterpret_cast<uint4*>(wa + n) = *reinterpret_cast<const uint4*>(tile + L::key_word(tok_a, t, n));
                            *reinterpret_cast<uint4*>(wb + n) = *reinterpret_cast<const uint4*>(tile + L::key_word(tok_b, t, n));
                            *reinterpret_cast<uint2*>(sa + n / 2) = *reinterpret_cast<const uint2*>(tile + L::key_meta(tok_a, n));
                            *reinterpret_cast<uint2*>(sb + n / 2) = *reinterpret_cast<const uint2*>(tile + L::key_meta(tok_b, n));
                        }
                    }
                    {
                        const uint8_t* meta = tile + L::kKeyZero + (2 * t % N) * 2;
                        const uint32_t za = *reinterpret_cast<const uint32_t*>(meta + tok_a * 2 * N);
                        const uint32_t zb = *reinterpret_cast<const uint32_t*>(meta + tok_b * 2 * N);
                        if constexpr (N == 8) mma(z, za, zb, za, zb, qz[0], qz[1], 0.0f, 0.0f, 0.0f, 0.0f);
                        else mma(z, za, zb, 0u, 0u, qz[0], 0u, 0.0f, 0.0f, 0.0f, 0.0f);
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        float acc[4];
                        const uint4 qn = sm.query[n][lane];
                        mma(acc, wa[n] * 16u & kNibble, wb[n] * 16u & kNibble, wa[n] & kNibble, wb[n] & kNibble, qn.x, qn.y,
                            0.0f, 0.0f, 0.0f, 0.0f);
                        const uint32_t xa = wa[n] >> 8, xb = wb[n] >> 8;
                        mma(acc, xa * 16u & kNibble, xb * 16u & kNibble, xa & kNibble, xb & kNibble, qn.z, qn.w);
                        const float2 pa = __half22float2(half2_of(sa[n / 2])), pb = __half22float2(half2_of(sb[n / 2]));
                        const float fa = n & 1 ? pa.y : pa.x, fb = n & 1 ? pb.y : pb.x;
                        sum[0] = fmaf(fa, acc[0], sum[0]);
                        sum[1] = fmaf(fa, acc[1], sum[1]);
                        sum[2] = fmaf(fb, acc[2], sum[2]);
                        sum[3] = fmaf(fb, acc[3], sum[3]);
                    }
                    s[u][0] = f0 * fmaf(sum[0], 0x1p20f, z[0]);
                    s[u][1] = f1 * fmaf(sum[1], 0x1p20f, z[1]);
                    s[u][2] = f0 * fmaf(sum[2], 0x1p20f, z[2]);
                    s[u][3] = f1 * fmaf(sum[3], 0x1p20f, z[3]);
                }

                uint32_t live = ~0u;                               // tokens of the two tiles that some row sees
                const bool parts = p.units && p.unit < kTileTokens;
                if (none || parts || (int32_t)(max(no0, no1) * kTileTokens + kTileTokens) > all) {
                    // Some token is not seen by some row. What lies in the cache behind the last token, or in the ring where there was
                    // no tile, may be anything, also infinite, so its scales and zeros are cleared below.
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int32_t base = (int32_t)((u ? no1 : no0) * kTileTokens);
                        uint32_t bits = 0xFFFFu;                   // of the tile's tokens
                        if (parts) {
                            const uint32_t x = bits_at(p, (uint64_t)bh * p.row_units + (base >> p.unit_log2));
                            bits = 0;
                            for (uint32_t i = 0; i < kTileTokens; ++i) bits |= (x >> (i >> p.unit_log2) & 1u) << i;
                        }
                        const int32_t left = (int32_t)len - base;
                        if (left < (int32_t)kTileTokens) bits &= left > 0 ? (1u << left) - 1u : 0u;
                        if (none >> u & 1u) bits = 0;
                        const bool a = bits >> tok_a & 1u, c = bits >> tok_b & 1u;
                        if (!a || base + (int32_t)tok_a >= see0) s[u][0] = -INFINITY;
                        if (!a || base + (int32_t)tok_a >= see1) s[u][1] = -INFINITY;
                        if (!c || base + (int32_t)tok_b >= see0) s[u][2] = -INFINITY;
                        if (!c || base + (int32_t)tok_b >= see1) s[u][3] = -INFINITY;
                        live = u ? live & 0xFFFFu | bits << 16 : live & 0xFFFF0000u | bits;
                    }
                }
                // has a score passed the maximum by more than the slack?
                const float t0 = fmaxf(fmaxf(s[0][0], s[0][2]), fmaxf(s[1][0], s[1][2])), t1 = fmaxf(fmaxf(s[0][1], s[0][3]), fmaxf(s[1][1], s[1][3]));
                if (__any_sync(0xFFFFFFFFu, t0 > m0 + kSlack || t1 > m1 + kSlack)) {
                    float n0 = t0, n1 = t1;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        n0 = fmaxf(n0, __shfl_xor_sync(0xFFFFFFFFu, n0, d));
                        n1 = fmaxf(n1, __shfl_xor_sync(0xFFFFFFFFu, n1, d));
                    }
                    n0 = fmaxf(m0, n0);
                    n1 = fmaxf(m1, n1);
                    const float c0 = exp2_fast(m0 - n0), c1 = exp2_fast(m1 - n1);
                    rescale_sums(c0, c1);
                    rescale_weights(c0, c1);
                    m0 = n0;
                    m1 = n1;
                    d0 = m0 - fminf(lift, kLift);
                    d1 = m1 - fminf(lift, kLift);
                }
                float e[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    e[u][0] = exp2_fast(s[u][0] - d0);
                    e[u][1] = exp2_fast(s[u][1] - d1);
                    e[u][2] = exp2_fast(s[u][2] - d0);
                    e[u][3] = exp2_fast(s[u][3] - d1);
                }
                float a0 = e[0][0] + e[0][2], a1 = e[0][1] + e[0][3], b0 = e[1][0] + e[1][2], b1 = e[1][1] + e[1][3];
                l0 += a0 + b0;
                l1 += a1 + b1;

                // what each block of `sub` tokens received, as log2
                if (p.sub == kTileTokens) {
                    // four sums over the eight rows: after two exchanges a lane holds one of them, of tile (lane / 16) and row 2 t + lane / 8 % 2
                    const bool up = lane & 16, odd = lane & 8;
                    float x0 = up ? b0 : a0, x1 = up ? b1 : a1;
                    x0 += __shfl_xor_sync(0xFFFFFFFFu, up ? a0 : b0, 16);
                    x1 += __shfl_xor_sync(0xFFFFFFFFu, up ? a1 : b1, 16);
                    float x = (odd ? x1 : x0) + __shfl_xor_sync(0xFFFFFFFFu, odd ? x0 : x1, 8);
                    x += __shfl_xor_sync(0xFFFFFFFFu, x, 4);
                    if (!(lane & 4) && !(none >> (up ? 1 : 0) & 1u))
                        mass[(uint64_t)(up ? no1 : no0) * kRows + (odd ? 1 : 0)] = (odd ? d1 : d0) + log2_fast(x);
                } else if (p.sub) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const bool there = !(none >> u & 1u);
                        float2* to = reinterpret_cast<float2*>(mass) + (uint64_t)((u ? no1 : no0) << (4 - p.unit_log2)) * (kRows / 2);
                        if (p.sub == 1) {
                            if (there) {
                                to[tok_a * (kRows / 2)] = make_float2(s[u][0], s[u][1]);
                                to[tok_b * (kRows / 2)] = make_float2(s[u][2], s[u][3]);
                            }
                        } else if (p.sub == 2) {
                            float x[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = e[u][i] + __shfl_xor_sync(0xFFFFFFFFu, e[u][i], 4);
                            if (there && !(g & 1)) {
                                to[g * (kRows / 2)] = make_float2(d0 + log2_fast(x[0]), d1 + log2_fast(x[1]));
                                to[(g + 1) * (kRows / 2)] = make_float2(d0 + log2_fast(x[2]), d1 + log2_fast(x[3]));
                            }
                        } else {                                    // 4 or 8 tokens: rows 2 j, 2 j + 1, or four of them
                            float x0 = u ? b0 : a0, x1 = u ? b1 : a1;
                            x0 += __shfl_xor_sync(0xFFFFFFFFu, x0, 4);
                            x1 += __shfl_xor_sync(0xFFFFFFFFu, x1, 4);
                            const float y0 = __shfl_xor_sync(0xFFFFFFFFu, x0, 8), y1 = __shfl_xor_sync(0xFFFFFFFFu, x1, 8);
                            if (p.sub == 8) { x0 += y0; x1 += y1; }
                            if (there && !(g & (p.sub / 2 - 1))) to[g / (p.sub / 2) * (kRows / 2)] = make_float2(d0 + log2_fast(x0), d1 + log2_fast(x1));
                        }
                    }
                }

                // values: dims 32 n + 4 g + {0, 2} in rows g, {1, 3} in rows g + 8 (16 times too large)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint8_t* tile = tile0 + u * L::kBytes;
                    uint32_t vs[N][2], vz0 = 0, vz1 = 0;           // scales and zeros of the values of tokens 4t .. 4t + 3
#pragma unroll
                    for (int n = 0; n < N; n += 2) {
                        const uint4 x = *reinterpret_cast<const uint4*>(tile + L::value_meta(4 * t, n));
                        vs[n][0] = x.x;
                        vs[n][1] = x.y;
                        vs[n + 1][0] = x.z;
                        vs[n + 1][1] = x.w;
                    }
                    if (g < N) {
                        const uint2 x = *reinterpret_cast<const uint2*>(tile + L::value_meta(4 * t, g) + (L::kValueZero - L::kValueScale));
                        vz0 = x.x;
                        vz1 = x.y;
                    }
                    if (live != ~0u) {
                        const uint32_t four = live >> (16 * u + 4 * t);
                        const uint32_t k0 = (four & 1u ? 0xFFFFu : 0u) | (four & 2u ? 0xFFFF0000u : 0u);
                        const uint32_t k1 = (four & 4u ? 0xFFFFu : 0u) | (four & 8u ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int n = 0; n < N; ++n) { vs[n][0] &= k0; vs[n][1] &= k1; }
                        vz0 &= k0;
                        vz1 &= k1;
                    }
                    // A weight times a scale has to stay below 2^16. Up to scales of 2 the lift sees to that; larger ones (values
                    // that span more than 30) take as much off the lift, for good. Nor should it sink below fp16's normal numbers: where the
                    // first tile has small scales only (or none), scales are raised until larger ones come.
                    uint32_t large = vs[0][0] | vs[0][1];
#pragma unroll
                    for (int n = 1; n < N; ++n) large |= vs[n][0] | vs[n][1];
                    if (u == 0 && k + done == 0 && !__any_sync(0xFFFFFFFFu, large & kFromSmall)) lift = kLift + kRaise;
                    if (__any_sync(0xFFFFFFFFu, lift > kLift ? large : large & kFrom2)) {
                        __half2 v = __hmax2(half2_of(vs[0][0]), half2_of(vs[0][1]));
#pragma unroll
                        for (int n = 1; n < N; ++n) v = __hmax2(v, __hmax2(half2_of(vs[n][0]), half2_of(vs[n][1])));
                        float most = __half2float(__hmax(__low2half(v), __high2half(v)));
                        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
                        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
                        const int size = most < INFINITY ? ilogbf(most) : 15;
                        const float room = size > 0 || size < kSmall ? fminf(kLift - (float)size, kLift + kRaise) : kLift;
                        if (room < lift) {
                            const float all = exp2f(room - lift), c = exp2f(fminf(room, kLift) - fminf(lift, kLift));
                            rescale_sums(all, all);
                            rescale_weights(c, c);
#pragma unroll
                            for (int i = 0; i < 4; ++i) { e[0][i] *= c; e[1][i] *= c; }
                            lift = room;
                            d0 = m0 - fminf(lift, kLift);
                            d1 = m1 - fminf(lift, kLift);
                        }
                        if (lift > kLift) {                        // exact: fp16 holds a scale below 2 times the power of two
                            const uint32_t by = bits_of(__float2half2_rn(exp2f(lift - kLift)));
#pragma unroll
                            for (int n = 0; n < N; ++n) { vs[n][0] = times(vs[n][0], by); vs[n][1] = times(vs[n][1], by); }
                        }
                    }
                    const uint32_t h0 = pack(e[u][0], e[u][1]), h1 = pack(e[u][2], e[u][3]), p0 = transposed(h0), p1 = transposed(h1);
                    uint32_t r0 = 0, r1 = 0;                       // what the fp16 weights leave
                    mma(zsum, vz0, 0u, vz1, 0u, p0, p1);
                    if constexpr (HALF) {
                        const float2 q0 = __half22float2(half2_of(h0)), q1 = __half22float2(half2_of(h1));
                        r0 = transposed(pack(e[u][0] - q0.x, e[u][1] - q0.y));
                        r1 = transposed(pack(e[u][2] - q1.x, e[u][3] - q1.y));
                        mma(zsum, vz0, 0u, vz1, 0u, r0, r1);
                    }
                    uint32_t x[N], y[N];
                    if constexpr (N == 2) {
                        *reinterpret_cast<uint2*>(x) = *reinterpret_cast<const uint2*>(tile + L::value_half(4 * t, g, 0));
                        *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(tile + L::value_half(4 * t + 2, g, 0));
                    } else {
#pragma unroll
                        for (int n = 0; n < N; n += 4) {
                            *reinterpret_cast<uint4*>(x + n) = *reinterpret_cast<const uint4*>(tile + L::value_half(4 * t, g, n));
                            *reinterpret_cast<uint4*>(y + n) = *reinterpret_cast<const uint4*>(tile + L::value_half(4 * t + 2, g, n));
                        }
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        const uint32_t w0 = times(p0, vs[n][0]), w1 = times(p1, vs[n][1]);
                        const uint32_t a[4] = {x[n] & 0x000F000Fu, x[n] & 0x00F000F0u, y[n] & 0x000F000Fu, y[n] & 0x00F000F0u};
                        const uint32_t xx = x[n] >> 8, yy = y[n] >> 8;
                        const uint32_t c[4] = {xx & 0x000F000Fu, xx & 0x00F000F0u, yy & 0x000F000Fu, yy & 0x00F000F0u};
                        mma(o[2 * n], a[0], a[1], a[2], a[3], w0, w1);
                        mma(o[2 * n + 1], c[0], c[1], c[2], c[3], w0, w1);
                        if constexpr (HALF) {
                            const uint32_t low0 = bits_of(__hfma2(half2_of(r0), half2_of(vs[n][0]), __hfma2(half2_of(p0), half2_of(vs[n][0]), __hneg2(half2_of(w0)))));
                            const uint32_t low1 = bits_of(__hfma2(half2_of(r1), half2_of(vs[n][1]), __hfma2(half2_of(p1), half2_of(vs[n][1]), __hneg2(half2_of(w1)))));
                            mma(o[2 * n], a[0], a[1], a[2], a[3], low0, low1);
                            mma(o[2 * n + 1], c[0], c[1], c[2], c[3], low0, low1);
                        }
                    }
                }
                __syncwarp();                                      // all lanes have read the two stages
                if (k + kStages < mine) { issue(k + kStages); issue(k + kStages + 1); }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            done += many;
            if (done >= take) break;
            begin_chunk();
        }

        // join the warps; a row's 16-byte pieces are shuffled by its number, so that eight lanes write to eight banks
        l0 = over_rows(l0);
        l1 = over_rows(l1);
        __syncthreads();                                           // every warp is done with its ring
        const float up = 0x1p24f * exp2f(fminf(kLift - lift, 0.0f)), up16 = up * 0x1p-4f;
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
            float4* to = reinterpret_cast<float4*>(ring_all) + (warp * kRows + 2 * t) * (L::D / 4) + ((n * 8 + g) ^ (2 * t));
            to[0] = a;
            to[L::D / 4] = c;
        }
        if (g == 0) {
            sm.ml[warp][2 * t] = make_float2(d0, l0);
            sm.ml[warp][2 * t + 1] = make_float2(d1, l1);
        }
        __syncthreads();
        const bool whole = take == count;
        const uint64_t slot = (uint64_t)blockIdx.x + seg;
        auto place = [&](uint32_t row) {
            const uint32_t query = p.group.of(row);
            return ((uint64_t)b * p.queries + query) * (p.heads.d * p.group.d) + h * p.group.d + (row - query * p.group.d);
        };
        if (tid < kRows * kWarps) {                                // a row's warps in eight neighbouring lanes
            const uint32_t r = tid / kWarps, w = tid % kWarps, row = rt * kRows + r;
            const float2 x = sm.ml[w][r];
            float m = x.x;
#pragma unroll
            for (int o = 1; o < kWarps; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            const float k = exp2_fast(x.x - m);
            float l = x.y * k;
#pragma unroll
            for (int o = 1; o < kWarps; o <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
            sm.share[w][r] = whole ? (l == 0.0f ? 0.0f : k / l) : k;
            if (w == 0) {
                p.ml[slot * kRows + r] = make_float2(m, l);
                if (whole && p.lse && row < p.rows) p.lse[place(row)] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
        }
        __syncthreads();
        for (uint32_t i = tid; i < kRows * L::D / 4; i += kThreads) {
            const uint32_t r = i / (L::D / 4), c = i % (L::D / 4), row = rt * kRows + r;
            if (row >= p.rows) continue;
            float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float4 x = reinterpret_cast<const float4*>(ring_all)[(w * kRows + r) * (L::D / 4) + (c ^ (r & 6))];
                const float k = sm.share[w][r];
                sum.x = fmaf(x.x, k, sum.x);
                sum.y = fmaf(x.y, k, sum.y);
                sum.z = fmaf(x.z, k, sum.z);
                sum.w = fmaf(x.w, k, sum.w);
            }
            if (whole) reinterpret_cast<uint2*>(p.out)[place(row) * (L::D / 4) + c] = make_uint2(out_pair<HALF>(sum.x, sum.y), out_pair<HALF>(sum.z, sum.w));
            else reinterpret_cast<float4*>(p.part)[(slot * kRows + r) * (L::D / 4) + c] = sum;
        }
        if (todo) __syncthreads();                                 // the ring is free again
    }
}

struct Work {
    uint64_t slots, part, ml, mass, counts, total;     // offsets in bytes
    uint32_t ctas;
};

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
    // places in the line (31 bits) and tiles of the cache are counted in 32 bits
    if (bh * ((rows + kRows - 1) / kRows) * (tokens / kTileTokens + kFixed) >= (1ull << 31) || (uint64_t)a->cache.pages * a->cache.kv_heads * (a->cache.page_tokens / kTileTokens) >= (1ull << 32) - 1) return KVP_ERR_RANGE;
    if (bh * rows >= (1ull << 30) || bh * ((tokens / u + kThreads - 1) / kThreads) >= (1ull << 30)) return KVP_ERR_RANGE;
    return KVP_OK;
}

template <int N, bool HALF>
int launch_attend(const AttendK& k, cudaStream_t st)
{
    const uint32_t smem = Shape<N>::kSmem;
    KVP_CUDA(cudaFuncSetAttribute(attend_kernel<N, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    int rc = k.units ? launch(count_kernel, k.batch * k.heads.d, kThreads, 0, false, st, k) : KVP_OK;
    if (!rc) rc = launch(attend_kernel<N, HALF>, k.ctas, kThreads, smem, k.units != nullptr, st, k);
    const uint64_t blocks = (uint64_t)k.batch * k.heads.d * ((k.warp_rows ? k.segs.d : k.rows) + (k.weights ? (k.row_units + kThreads - 1) / kThreads : 0));
    if (!rc) rc = launch(join_kernel<AttendK, N, HALF, kRows>, (uint32_t)blocks, kThreads, 0, true, st, k);
    return rc;
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
    if (off_by(q, 2) || off_by(cache, 16) || off_by(table, 4) || off_by(lens, 4) || off_by(units, 4) || off_by(out, 8) || off_by(lse, 4) || off_by(weights, 4) ||
        off_by(workspace, 256)) return KVP_ERR_ARG;
    AttendK k;
    k.q = q; k.out = out; k.lse = lse; k.weights = weights;
    k.cache = static_cast<const uint8_t*>(cache); k.table = table; k.lens = lens; k.units = units;
    char* ws = static_cast<char*>(workspace);
    k.part = reinterpret_cast<float*>(ws + w.part);
    k.ml = reinterpret_cast<float2*>(ws + w.ml);
    k.mass = reinterpret_cast<float*>(ws + w.mass);
    k.counts = reinterpret_cast<uint32_t*>(ws + w.counts);
    k.q_batch = a->q_batch_stride; k.q_query = a->q_query_stride; k.q_head = a->q_head_stride;
    k.batch = a->batch; k.queries = a->queries; k.heads = divisor(a->cache.kv_heads); k.group = divisor(a->group);
    k.rows = a->queries * a->group; k.segs = divisor((k.rows + kRows - 1) / kRows);
    k.page_tiles = divisor(a->cache.page_tokens / kTileTokens); k.table_pages = a->table_pages; k.pages = a->cache.pages;
    const uint64_t tokens = (uint64_t)a->table_pages * a->cache.page_tokens;
    k.unit = a->unit_tokens; k.row_units = (uint32_t)(tokens / a->unit_tokens);
    k.unit_words = ((uint64_t)k.batch * k.heads.d * k.row_units + 31) / 32;
    const uint32_t sub = k.unit < kTileTokens ? k.unit : kTileTokens;
    k.row_subs = tokens / sub;
    k.sub = weights ? sub : 0;
    k.ctas = w.ctas;
    k.least = kWarps;
    k.unit_log2 = k.unit == 1 ? 0 : k.unit == 2 ? 1 : k.unit == 4 ? 2 : k.unit == 8 ? 3 : 4;
    k.scale = a->scale;
    // Segments of few parts are joined by a warp a row, others by a CTA. Us by warps and by CTAs in 296 parts, head dim 128: 1 sequence x 8 heads 47.5, 43.2; 2 x 8
    // 31.0, 28.9; 4 x 8 20.7, 20.7; 40 x 1 20.4, 18.6; 8 x 8 18.6, 18.6; 16 x 8 31.6, 31.9; 32 x 8 52.7, 55.3; 128 x 4 30.9, 36.0. In 148, head dim 256: 4 x 8
    // 32.9, 31.0; 40 x 1 29.0, 28.9; 8 x 8 24.8, 24.5; 16 x 8 60.1, 61.6; 128 x 4 54.3, 59.2.
    k.warp_rows = (uint64_t)k.batch * k.heads.d * k.segs.d >= k.ctas / 4;
    k.q_aligned = ((uint64_t)(uintptr_t)q | (uint64_t)(a->q_batch_stride * 2) | (uint64_t)(a->q_query_stride * 2) | (uint64_t)(a->q_head_stride * 2)) % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == KVP_F16) {
        switch (a->cache.head_dim) {
            case 64: return launch_attend<2, true>(k, st);
            case 128: return launch_attend<4, true>(k, st);
            default: return launch_attend<8, true>(k, st);
        }
    }
    switch (a->cache.head_dim) {
        case 64: return launch_attend<2, false>(k, st);
        case 128: return launch_attend<4, false>(k, st);
        default: return launch_attend<8, false>(k, st);
    }
}
