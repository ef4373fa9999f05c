// Block tables and slot maps from the lengths of requests (include/kvp.h, kvp_block_tables).
//
// Whole numbers and prefix sums over the requests. One CTA goes through the requests (a chunk of its threads at a time): who is granted
// its pages is decided by one pair of running sums, what it gets by a second. Tokens then find their request by a binary search in `starts`: in the same
// CTA where there are few of them (a decode step is one launch), else in a second kernel over all tokens, which writes 16 bytes each.
// 256 requests with a token each take 3.3 us, latency of three rounds of loads and sums; 6.8 where some of them give back pages (a third round of sums, then
// loads and stores of their rows); 64 prompts of 131072 tokens in all 11.7.
#include "kvp_line.cuh"

namespace kvp {

namespace {

struct TablesK {
    const int32_t *new_tokens, *lens, *state;
    int32_t *table, *ring, *lens_out, *state_out, *granted, *starts, *page_starts, *positions, *rows;
    int64_t* slots;
    uint32_t batch, table_pages, tokens;
    Divisor page;            // tokens of a page
    uint32_t pages;
    bool fours;              // rows of the table can be read 16 bytes at a time
};

constexpr uint32_t kScanThreads = 1024, kScanWarps = 32;
constexpr uint32_t kAlone = 4096;                  // tokens that the CTA of the sums still serves by itself: four a thread
constexpr uint32_t kSharedStarts = 2048;           // requests whose `starts` a CTA of the second kernel takes to shared memory
constexpr uint32_t kFull = 0x7FFFFFFFu;            // running sums of what is asked for stay here

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kFull); }       // of two that are at most kFull

struct Pair {
    uint32_t a, b;
};
// running sums over the CTA's threads, this one's included, and of all; every thread calls it
template <bool SATURATE>
__device__ __forceinline__ Pair sum_over(Pair x, Pair& all, Pair* sm)
{
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    auto add = [](uint32_t u, uint32_t v) { return SATURATE ? sat_add(u, v) : u + v; };
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, x.a, o), b = __shfl_up_sync(0xFFFFFFFFu, x.b, o);
        if (lane >= (uint32_t)o) {
            x.a = add(x.a, a);
            x.b = add(x.b, b);
        }
    }
    __syncthreads();                                            // sm is free
    if (lane == 31) sm[warp] = x;
    __syncthreads();
    Pair w = lane < warps ? sm[lane] : Pair{0, 0};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t a = __shfl_up_sync(0xFFFFFFFFu, w.a, o), b = __shfl_up_sync(0xFFFFFFFFu, w.b, o);
        if (lane >= (uint32_t)o) {
            w.a = add(w.a, a);
            w.b = add(w.b, b);
        }
    }
    all.a = __shfl_sync(0xFFFFFFFFu, w.a, 31);
    all.b = __shfl_sync(0xFFFFFFFFu, w.b, 31);
    const uint32_t before = warp ? warp - 1 : 0;
    const uint32_t a = __shfl_sync(0xFFFFFFFFu, w.a, before), b = __shfl_sync(0xFFFFFFFFu, w.b, before);
    if (warp) {
        x.a = add(x.a, a);
        x.b = add(x.b, b);
    }
    return x;
}

__device__ __forceinline__ uint32_t pages_of(const TablesK& p, uint32_t tokens) { return p.page.of(tokens + p.page.d - 1); }
// entries j .. j + 3 of a row (j a multiple of 4), of the first `many`: those that name no page are -1; w: how many do
struct Four {
    int32_t page[4];
    uint32_t w;
};
__device__ __forceinline__ Four good_pages(const TablesK& p, const int32_t* row, uint32_t j, uint32_t many)
{
    Four x = {{-1, -1, -1, -1}, 0};
    if (j >= many) return x;
    int32_t e[4];
    if (p.fours) {                                                             // the row has a multiple of four entries
        const int4 v = *reinterpret_cast<const int4*>(row + j);
        e[0] = v.x;
        e[1] = v.y;
        e[2] = v.z;
        e[3] = v.w;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) e[i] = j + i < many ? row[j + i] : -1;
    }
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const bool good = j + i < many && (uint32_t)e[i] < p.pages;
        x.page[i] = good ? e[i] : -1;
        x.w += good;
    }
    return x;
}
__device__ __forceinline__ uint32_t around(uint32_t at, uint32_t pages) { return at >= pages ? at - pages : at; }       // at < 2 pages

// Token t of the call: its request, position and slot; a page that begins with it goes into the table. `head`: of the ring, before the call.
__device__ __forceinline__ void place_token(const TablesK& p, uint32_t t, const int32_t* starts, const int32_t* page_starts, const int32_t* lens_out, uint32_t head)
{
    if (t >= (uint32_t)starts[p.batch]) {
        p.slots[t] = -1;
        p.positions[t] = 0;
        p.rows[t] = -1;
        return;
    }
    uint32_t low = 0, high = p.batch;                           // starts[low] <= t < starts[high]
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if ((uint32_t)starts[mid] <= t) low = mid;
        else high = mid;
    }
    const uint32_t row = low, first = starts[row], before = (uint32_t)lens_out[row] - (starts[row + 1] - first), pos = before + t - first;
    const uint32_t j = p.page.of(pos), had = pages_of(p, before);
    int32_t* entry = p.table + (uint64_t)row * p.table_pages + j;
    int32_t page;
    if (j >= had) {
        page = p.ring[around(head + around(page_starts[row] + j - had, p.pages), p.pages)];
        if (pos == j * p.page.d) *entry = page;                 // no other token reads it: the entry is new
    } else {
        page = *entry;
    }
    p.slots[t] = page >= 0 && (uint32_t)page < p.pages ? (int64_t)page * p.page.d + (pos - j * p.page.d) : -1;
    p.positions[t] = (int32_t)pos;
    p.rows[t] = (int32_t)row;
}

__global__ void __launch_bounds__(kScanThreads) tables_kernel(const TablesK p, bool alone)
{
    __shared__ Pair sm[kScanWarps];
    __shared__ struct { int32_t starts[kScanThreads + 1], page_starts[kScanThreads], lens[kScanThreads]; } near;      // of the last chunk
    __shared__ struct { uint32_t upto[kScanThreads], many[kScanThreads], warp[kScanWarps]; } gone;       // of a chunk: items up to a request, its pages
    let_next_start();
    wait_for_previous();
    const uint32_t tid = threadIdx.x, lane = tid % 32;
    const uint32_t head = (uint32_t)p.state[0] % p.pages, count = min((uint32_t)max(p.state[1], 0), p.pages);
    const uint32_t most = p.table_pages * p.page.d;
    Pair asked = {0, 0}, given = {0, 0};                        // pages and tokens so far: asked for, given
    uint32_t back = 0;                                          // pages given back so far
    for (uint32_t base = 0; base < p.batch; base += blockDim.x) {
        const uint32_t i = base + tid;
        const bool in = i < p.batch;
        const int32_t n = in ? p.new_tokens[i] : 0;
        const uint32_t len = in ? min((uint32_t)max(p.lens[i], 0), most) : 0, had = pages_of(p, len);
        const bool leaves = n < 0, fits = in && !leaves && (uint32_t)n <= most - len;
        const uint32_t need = fits ? pages_of(p, len + n) - had : 0;
        Pair all;
        Pair sum = sum_over<true>(Pair{need, fits ? (uint32_t)n : 0u}, all, sm);
        const bool yes = fits && (!need || sat_add(asked.a, sum.a) <= count) && (!n || sat_add(asked.b, sum.b) <= p.tokens);
        asked.a = sat_add(asked.a, all.a);
        asked.b = sat_add(asked.b, all.b);
        const Pair mine = {yes ? need : 0u, yes ? (uint32_t)n : 0u};
        sum = sum_over<false>(mine, all, sm);
        if (in) {
            p.starts[i] = (int32_t)(given.b + sum.b - mine.b);
            p.page_starts[i] = (int32_t)(given.a + sum.a - mine.a);
            p.granted[i] = yes || leaves;
            p.lens_out[i] = leaves ? 0 : (int32_t)(len + mine.b);
            near.starts[tid] = (int32_t)(given.b + sum.b - mine.b);
            near.page_starts[tid] = (int32_t)(given.a + sum.a - mine.a);
            near.lens[tid] = leaves ? 0 : (int32_t)(len + mine.b);
        }
        given.a += all.a;
        given.b += all.b;
        if (__syncthreads_or(leaves)) {
            // Pages given back: entries of the rows that leave, 128 to an item, four items a warp at a time, so that the loads of 512 entries are under way together.
            // Items are in the order of requests and entries, and a place in the ring is the number of pages before.
            const uint32_t many = leaves ? had : 0u;
            sum = sum_over<false>(Pair{(many + 127) / 128, 0}, all, sm);
            gone.upto[tid] = sum.a;
            gone.many[tid] = many;
            __syncthreads();
            const uint32_t warp = tid / 32, warps = blockDim.x / 32, rows = min(blockDim.x, p.batch - base);
            for (uint32_t i0 = 0; i0 < all.a; i0 += 4 * warps) {
                Four x[4];
                uint32_t upto[4], mine = 0;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const uint32_t item = i0 + 4 * warp + k;
                    x[k] = Four{{-1, -1, -1, -1}, 0};
                    if (item < all.a) {
                        uint32_t low = 0, high = rows;                  // the first row with upto > item is in low .. high - 1
                        while (high - low > 1) {
                            const uint32_t mid = (low + high) / 2;
                            if (gone.upto[mid - 1] > item) high = mid;
                            else low = mid;
                        }
                        const uint32_t first = low ? gone.upto[low - 1] : 0u;
                        x[k] = good_pages(p, p.table + (uint64_t)(base + low) * p.table_pages, (item - first) * 128 + 4 * lane, gone.many[low]);
                    }
                }
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    upto[k] = mine + sum_upto(x[k].w, lane);
                    mine = __shfl_sync(0xFFFFFFFFu, upto[k], 31);
                }
                if (lane == 0) gone.warp[warp] = mine;
                __syncthreads();
                const uint32_t w = sum_upto(lane < warps ? gone.warp[lane] : 0u, lane), before = __shfl_sync(0xFFFFFFFFu, w, warp) - mine, total = __shfl_sync(0xFFFFFFFFu, w, 31);
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    uint32_t at = (head + count + back + before + upto[k] - x[k].w) % p.pages;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        if (x[k].page[i] >= 0) {
                            p.ring[at] = x[k].page[i];
                            if (++at == p.pages) at = 0;
                        }
                }
                back += total;
                __syncthreads();                                        // the warps' numbers are free
            }
        }
    }
    if (tid == 0) {
        p.starts[p.batch] = (int32_t)given.b;
        if (p.batch <= blockDim.x) near.starts[p.batch] = (int32_t)given.b;
        p.page_starts[p.batch] = (int32_t)given.a;
        p.state_out[0] = (int32_t)around(head + given.a, p.pages);
        p.state_out[1] = (int32_t)min(count - given.a + back, p.pages);
    }
    if (!alone) return;
    __syncthreads();
    const bool here = p.batch <= blockDim.x;                    // what the tokens look up is in shared memory too
    for (uint32_t t = tid; t < p.tokens; t += blockDim.x)
        place_token(p, t, here ? near.starts : p.starts, here ? near.page_starts : p.page_starts, here ? near.lens : p.lens_out, head);
}

__global__ void __launch_bounds__(256) tokens_kernel(const TablesK p)
{
    __shared__ int32_t near[kSharedStarts + 1];
    const uint32_t tid = threadIdx.x;
    let_next_start();
    wait_for_previous();
    const int32_t* starts = p.starts;
    if (p.batch <= kSharedStarts) {
        for (uint32_t i = tid; i <= p.batch; i += 256) near[i] = p.starts[i];
        __syncthreads();
        starts = near;
    }
    const uint32_t head = around((uint32_t)p.state_out[0] + p.pages - p.page_starts[p.batch], p.pages);
    for (uint32_t t = blockIdx.x * 256 + tid; t < p.tokens; t += gridDim.x * 256) place_token(p, t, starts, p.page_starts, p.lens_out, head);
}

}  // namespace

}  // namespace kvp

using namespace kvp;

extern "C" int kvp_block_tables(const kvp_tables_params* a, const int32_t* new_tokens, const int32_t* lens, int32_t* lens_out, int32_t* table, int32_t* ring,
                                const int32_t* state, int32_t* state_out, int64_t* slots, int32_t* positions, int32_t* rows, int32_t* starts,
                                int32_t* page_starts, int32_t* granted, void* stream)
{
    if (!a || a->reserved || !a->batch || !a->table_pages || !a->pages || !a->page_tokens) return KVP_ERR_ARG;
    if (!new_tokens || !lens || !lens_out || !table || !ring || !state || !state_out || !starts || !page_starts || !granted) return KVP_ERR_ARG;
    if (a->tokens && (!slots || !positions || !rows)) return KVP_ERR_ARG;
    if (off_by(new_tokens, 4) || off_by(lens, 4) || off_by(lens_out, 4) || off_by(table, 4) || off_by(ring, 4) || off_by(state, 4) || off_by(state_out, 4) ||
        off_by(slots, 8) || off_by(positions, 4) || off_by(rows, 4) || off_by(starts, 4) || off_by(page_starts, 4) || off_by(granted, 4)) return KVP_ERR_ARG;
    // a length and a page more, pages given and a ring's index twice around are counted in 31 bits
    if ((uint64_t)a->table_pages * a->page_tokens >= (1ull << 30) || a->page_tokens >= (1u << 30) || a->pages >= (1u << 30) || a->tokens >= (1u << 30) ||
        a->batch >= (1u << 24)) return KVP_ERR_RANGE;
    TablesK k;
    k.new_tokens = new_tokens; k.lens = lens; k.state = state;
    k.table = table; k.ring = ring; k.lens_out = lens_out; k.state_out = state_out; k.granted = granted; k.starts = starts; k.page_starts = page_starts;
    k.positions = positions; k.rows = rows; k.slots = slots;
    k.batch = a->batch; k.table_pages = a->table_pages; k.tokens = a->tokens; k.page = divisor(a->page_tokens); k.pages = a->pages;
    k.fours = a->table_pages % 4 == 0 && !off_by(table, 16);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool alone = a->tokens <= kAlone;
    const uint32_t wide = a->batch > a->tokens ? a->batch : a->tokens, threads = wide >= kScanThreads ? kScanThreads : (wide + 31) / 32 * 32;
    int rc = launch(tables_kernel, 1, alone ? threads : kScanThreads, 0, true, st, k, alone);
    if (!rc && !alone) rc = launch(tokens_kernel, (a->tokens + 1023) / 1024, 256, 0, true, st, k);
    return rc;
}
