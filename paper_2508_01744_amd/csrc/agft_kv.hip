// agft_kv.hip -- tables, writes and exports of a serving node's paged cache.
// agft_kv.h states the rules and the layout.

#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "agft_kv_common.h"

namespace agft_kv_detail {

struct PlanArgs {
    const int32_t *add;
    const int32_t *counters, *lengths;
    int32_t *table, *ring;
    int32_t *out_counters, *starts, *granted, *out_lengths, *tiles, *need, *touched, *back, *sums, *arrived, *runs;
    Work *works;
    Item *items;
    int64_t *slots;
    int32_t requests, row_pages, pages, page, shift, group, heads, max_tokens;
    int32_t tile_units, tile_slots;    // of a head: compute units, workgroups that run at once
};

__device__ __forceinline__ int32_t pages_of(int32_t n, int32_t page, int32_t shift) { return (n + page - 1) >> shift; }

// ---- tables ----
//
// A window's table work is prefix sums over the requests and a search for every
// token's request: a few hundred KB at most, so latency is all of it.  Up to
// 1,024 requests every workgroup makes all the prefix sums for itself, in LDS,
// and then its own tokens' slots: one launch, no workgroup waits for
// another.  Beyond that one launch makes the sums of 1,024 requests per
// workgroup, and a second adds the other chunks' totals while it makes the
// slots.  One request 4.9 us (9.7 in two launches), 264 requests with 39,295 new
// tokens 9.0 us (12.9), 16,384 requests with 245,365 tokens 18.4 us.
constexpr int kPlanThreads = 256;
constexpr int kSumsThreads = 1024;                     // of a workgroup that makes one chunk's sums
template <int THREADS>
constexpr int plan_per = kPlanChunk / THREADS;         // requests of a thread
constexpr int kPlanTokens = 256;                       // tokens of a workgroup at a time
constexpr int kPlanNear = 1024;                        // requests whose starts it keeps in LDS

// What a request asks of the window, from its own lengths alone.
struct Ask {
    int32_t past, held, need;
    uint32_t tokens;
    bool wants, ends;
};

__device__ __forceinline__ Ask ask_of(const PlanArgs &p, int32_t past, int32_t add) {
    Ask a;
    const int32_t cap = p.row_pages << p.shift;
    a.past = past < 0 ? 0 : past > cap ? cap : past;
    a.wants = add > 0;
    a.ends = add < 0;
    a.held = pages_of(a.past, p.page, p.shift);
    a.tokens = add > 0 && add <= cap - a.past ? add : 0;
    a.need = pages_of(a.past + (int32_t)a.tokens, p.page, p.shift) - a.held;
    return a;
}

// Sums of what is asked may pass 32 bits; saturated ones compare alike (every
// limit is below 2^31), and a saturated sum less one request's share is still
// above every limit.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int THREADS>
struct PlanLds {
    uint32_t asked[3][THREADS / 64];
    int32_t sums[kPlanSums][THREADS / 64];
    float cost[THREADS / 64];
};

// Sums over the threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ void plan_scan(const int32_t *mine, int32_t *before, int32_t *all, PlanLds<THREADS> &lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t in[kPlanSums];
#pragma unroll
    for (int k = 0; k < kPlanSums; ++k) in[k] = mine[k];
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
#pragma unroll
        for (int k = 0; k < kPlanSums; ++k) {
            const int32_t x = __shfl_up(in[k], s, 64);
            if (lane >= s) in[k] += x;
        }
    __syncthreads();                        // (an earlier scan's sums have been read)
#pragma unroll
    for (int k = 0; k < kPlanSums; ++k)
        if (lane == 63) lds.sums[k][wave] = in[k];
    __syncthreads();
    constexpr int W = THREADS / 64;
#pragma unroll
    for (int k = 0; k < kPlanSums; ++k) {
        before[k] = in[k] - mine[k];
        if constexpr (W <= 4) {
            all[k] = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (w < wave) before[k] += lds.sums[k][w];
                all[k] += lds.sums[k][w];
            }
        } else {
            // many wavefronts: their sums a lane each (read one by one they cost
            // spilled registers, or 6 us of waiting)
            int32_t v = lane < W ? lds.sums[k][lane] : 0;
#pragma unroll
            for (int s = 1; s < W; s *= 2) {
                const int32_t x = __shfl_up(v, s, 64);
                if (lane >= s) v += x;
            }
            const int32_t to_here = __shfl(v, wave > 0 ? wave - 1 : 0, 64);
            if (wave > 0) before[k] += to_here;
            all[k] = __shfl(v, W - 1, 64);
        }
    }
}

// The requests [r0 + plan_per * thread, ..) of one thread.
template <int THREADS>
struct PlanPart {
    static constexpr int PER = plan_per<THREADS>;
    int32_t past[PER], held[PER], granted[PER], after[PER], first[PER], need[PER];
    int32_t tiles[PER];                // tiles of many rows
    int32_t sums[kPlanSums][PER];      // sums over the chunk's earlier requests
    int32_t all[kPlanSums];                 // over the chunk
    int32_t few_rows;                       // rows up to which a request counts as one of few
    uint32_t tokens;                        // asked by the chunk and all before it
};

// Units, for one head, of a request of more than kFewRows and up to kMidRows rows,
// if it gets what it asks for.
__device__ __forceinline__ uint32_t mid_units(const PlanArgs &p, const Ask &a) {
    const int64_t rows = (int64_t)a.tokens * p.group;
    if (rows <= kFewRows || rows > kMidRows) return 0;
    return ((uint32_t)(a.past + (int32_t)a.tokens + kUnit - 1) / kUnit) * (((uint32_t)rows + kRowTile - 1) / kRowTile);
}

// Prefix sums over a chunk, behind requests that ask for need0 pages and tok0
// tokens.  (Requests of up to kMidRows rows are told apart by their work where
// one chunk is all there is.)
template <int THREADS>
__device__ __forceinline__ void plan_chunk(const PlanArgs &p, int r0, uint32_t need0, uint32_t tok0, int32_t free_pages,
                                           PlanLds<THREADS> &lds, PlanPart<THREADS> &o) {
    constexpr int W = THREADS / 64, PER = plan_per<THREADS>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i0 = r0 + threadIdx.x * PER;
    Ask a[PER];
    uint32_t need = 0, tok = 0, mid = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool live = i0 + j < p.requests;
        a[j] = ask_of(p, live ? p.lengths[i0 + j] : 0, live ? p.add[i0 + j] : 0);
        need = add_sat(need, a[j].need), tok = add_sat(tok, a[j].tokens), mid = add_sat(mid, mid_units(p, a[j]));
    }
    uint32_t need_in = need, tok_in = tok;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const uint32_t x = __shfl_up(need_in, s, 64), y = __shfl_up(tok_in, s, 64);
        mid = add_sat(mid, __shfl_xor(mid, s, 64));
        if (lane >= s) need_in = add_sat(need_in, x), tok_in = add_sat(tok_in, y);
    }
    if (lane == 63) lds.asked[0][wave] = need_in, lds.asked[1][wave] = tok_in, lds.asked[2][wave] = mid;
    uint32_t need_at = __shfl_up(need_in, 1, 64), tok_at = __shfl_up(tok_in, 1, 64);
    if (lane == 0) need_at = 0, tok_at = 0;
    __syncthreads();
    need_at = add_sat(need_at, need0), tok_at = add_sat(tok_at, tok0);
    o.tokens = tok0;
    mid = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        mid = add_sat(mid, lds.asked[2][w]);
        if (w < wave) need_at = add_sat(need_at, lds.asked[0][w]), tok_at = add_sat(tok_at, lds.asked[1][w]);
        o.tokens = add_sat(o.tokens, lds.asked[1][w]);
    }
    o.few_rows = p.requests <= kPlanChunk && mid <= (uint32_t)(kMidUnits / p.heads) ? kMidRows : kFewRows;
    int32_t mine[kPlanSums] = {};
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const uint32_t need_to = add_sat(need_at, a[j].need), tok_to = add_sat(tok_at, a[j].tokens);
        const bool ok = a[j].tokens > 0 && (a[j].need == 0 || need_to <= (uint32_t)free_pages) &&
                        tok_to <= (uint32_t)p.max_tokens;
        const int32_t limit = p.max_tokens;
        o.past[j] = a[j].past, o.held[j] = a[j].held;
        o.granted[j] = ok ? (int32_t)a[j].tokens : 0;
        o.after[j] = a[j].ends ? 0 : a[j].past + o.granted[j];
        o.first[j] = tok_at < (uint32_t)limit ? (int32_t)tok_at : limit;
        o.need[j] = need_at < (uint32_t)free_pages ? (int32_t)need_at : free_pages;
        const int32_t last = tok_to < (uint32_t)limit ? (int32_t)tok_to : limit;
        // what the window's kernels have to do for it
        const int32_t rows = last - o.first[j];                         // rows of the window's tensors
        const int64_t wide = (int64_t)rows * p.group;
        const bool few = wide <= o.few_rows;
        o.tiles[j] = rows == 0 || few ? 0 : (int32_t)((wide + kTileRows - 1) / kTileRows);
        const int32_t v[kPlanSums] = {
            ok ? pages_of(o.after[j], p.page, p.shift) - (a[j].past >> p.shift) : 0,    // pages written to
            // units of few rows: every 16 rows read the request's tokens (one unit where there are none)
            rows == 0 || !few ? 0 : (ok ? (o.after[j] + kUnit - 1) / kUnit : 1) *
                                        (((int32_t)wide + kRowTile - 1) / kRowTile),
            o.tiles[j],                                                                 // tiles of many rows
            a[j].ends ? a[j].held : 0,                                                  // pages given back
            a[j].wants && !ok ? 1 : 0,
            ok ? a[j].need : 0,
        };
#pragma unroll
        for (int k = 0; k < kPlanSums; ++k) {
            o.sums[k][j] = mine[k];
            mine[k] += v[k];
        }
        need_at = need_to, tok_at = tok_to;
    }
    int32_t before[kPlanSums];
    plan_scan(mine, before, o.all, lds);
#pragma unroll
    for (int k = 0; k < kPlanSums; ++k)
#pragma unroll
        for (int j = 0; j < PER; ++j) o.sums[k][j] += before[k];
}

// Many rows: in which order the workgroups take their tiles, the longest first
// (by a factor of two), and which tiles several workgroups share, so that few
// tiles over many tokens fill the chip.  Parts cover at least kPartTiles key
// tiles where that gives every compute unit a workgroup (4 / 8 / 16: chunks of up
// to 134 tokens of 14 requests over up to 3,341, 4 heads of 256 numbers, 58 / 52 /
// 61 us; 128 rows of 8 requests over 4,000 tokens, 128 numbers, 33 / 33 / 35), and
// at least kSecondTiles where it would give it a second one (8 / 16 / 24: 2,774
// tokens of 7 query heads on one head of 64 36 / 28 / 32 us; 128 rows of 64
// requests over 1,000 tokens, 256 tiles, 40 / 33 / 33).  For up to kPlanChunk
// requests; beyond, tiles go by request, in one part (64 tokens of 16 query heads
// over 131,000: 1,830 us in a table of 1,025 rows, 115 in one of 1,024; 10 chunks of
// 512 over 3,000 316 and 326).
constexpr int kPartTiles = 8;
constexpr int kSecondTiles = 16;
constexpr int kMaxParts = 64;

__device__ __forceinline__ void plan_order(const PlanArgs &p, const PlanPart<kPlanThreads> &o,
                                           PlanLds<kPlanThreads> &lds, int32_t *base, int32_t *parts,
                                           int32_t *items) {
    constexpr int PER = plan_per<kPlanThreads>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float cost = 0.0f;                                                  // key tiles of all tiles
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (o.tiles[j] > 0) cost += (float)o.tiles[j] * (float)((o.after[j] + kUnit - 1) / kUnit);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) cost += __shfl_xor(cost, s, 64);
    if (lane == 0) lds.cost[wave] = cost;
    __syncthreads();
    cost = 0.0f;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) cost += lds.cost[w];
    const float once = ceilf(cost / (float)p.tile_units), even = ceilf(cost / (float)p.tile_slots);
    const float least = fmaxf((float)kPartTiles, fminf(once, fmaxf((float)kSecondTiles, even)));
    int32_t mine[kPlanSums] = {}, at[PER], kind[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int32_t keys = o.granted[j] > 0 ? (o.after[j] + kUnit - 1) / kUnit : 1;
        const float share = ceilf((float)keys / least);
        parts[j] = share > (float)kMaxParts ? kMaxParts : share > 1.0f ? (int32_t)share : 1;
        kind[j] = parts[j] > 1 ? 0 : keys >= 64 ? 1 : keys >= 32 ? 2 : keys >= 16 ? 3 : keys >= 8 ? 4 : 5;
        at[j] = 0;
#pragma unroll
        for (int k = 0; k < kPlanSums; ++k)
            if (k == kind[j]) at[j] = mine[k], mine[k] += o.tiles[j] * parts[j];
    }
    int32_t before[kPlanSums], all[kPlanSums];
    plan_scan(mine, before, all, lds);
    *items = 0;
#pragma unroll
    for (int k = 0; k < kPlanSums; ++k) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (k == kind[j]) base[j] = *items + before[k] + at[j];
        *items += all[k];
    }
}

// The item(s) of the tile that begins with one of token k's rows, if one does;
// a request's last tile, which sees the most tokens, comes first.
__device__ __forceinline__ void plan_items(const PlanArgs &p, int32_t i, int32_t k, int32_t tiles, int32_t base,
                                           int32_t parts) {
    const int64_t row = (int64_t)k * p.group, tile = (row + kTileRows - 1) / kTileRows;
    if (tiles == 0 || tile * kTileRows >= row + p.group) return;
    Item *item = p.items + base + (int64_t)(tiles - 1 - tile) * parts;
    for (int32_t z = 0; z < parts; ++z) item[z] = Item{i, (int32_t)tile, z, parts};
}

// The window's totals: ends of the prefix sums, and the counters.
__device__ __forceinline__ void plan_totals(const PlanArgs &p, uint32_t tokens, const int32_t *all, int32_t head,
                                            int32_t free_pages) {
    const int32_t total = tokens < (uint32_t)p.max_tokens ? (int32_t)tokens : p.max_tokens;
    p.starts[p.requests] = total;
    p.works[p.requests] = Work{all[1], all[2], total, 0, 0, {0, 0, 0}};
    p.runs[0] = all[0];
    int32_t *c = p.out_counters;
    c[0] = (int32_t)(((int64_t)head + all[5]) % p.pages);
    c[1] = free_pages - all[5] + all[3];
    c[2] = total;
    c[3] = all[4];
    c[4] = all[5];
    c[5] = all[3];
    c[6] = c[7] = 0;
}

// Nobody has arrived yet at the joins of the window's attention.
__device__ __forceinline__ void plan_arrived(const PlanArgs &p) {
    for (int k = threadIdx.x; k < kArrivals; k += kPlanThreads) p.arrived[k] = 0;
}

// place k of the ring from its head on
__device__ __forceinline__ int32_t ring_at(const PlanArgs &p, int32_t head, int64_t k) {
    const int64_t at = head + k;
    return (int32_t)(at < p.pages ? at : at - p.pages < p.pages ? at - p.pages : at % p.pages);
}

// Token t's slot, its run's place where it starts one, and its page's entry in
// the table where it is the page's first.  base: pages taken before its
// request's, run: runs before its request's.
__device__ __forceinline__ void plan_token(const PlanArgs &p, int64_t t, int32_t i, int32_t past, int32_t k, int32_t base,
                                           int32_t run, int32_t head) {
    const int32_t pos = past + k, n = pos >> p.shift, held = pages_of(past, p.page, p.shift), off = pos & (p.page - 1);
    int32_t id;
    if (n >= held) {
        id = p.ring[ring_at(p, head, (int64_t)base + n - held)];
        if (off == 0) p.table[(int64_t)i * p.row_pages + n] = id;
    } else {
        id = p.table[(int64_t)i * p.row_pages + n];
    }
    if (k == 0 || off == 0) p.runs[1 + run + n - (past >> p.shift)] = (int32_t)t;
    p.slots[t] = ((int64_t)id << p.shift) + off;
}

// Pages of the requests of this wavefront that end (a lane per request) go
// behind the ring's tail.
__device__ __forceinline__ void plan_give_back(const PlanArgs &p, bool ends, int32_t i, int32_t held, int32_t before,
                                               int32_t head, int32_t free_pages) {
    constexpr int AHEAD = 4;    // entries of a lane on their way at once
    const int lane = threadIdx.x & 63;
    for (uint64_t left = __ballot(ends && held > 0); left != 0; left &= left - 1) {
        const int l = __ffsll((unsigned long long)left) - 1;
        const int32_t r = __shfl(i, l, 64), n = __shfl(held, l, 64), b = __shfl(before, l, 64);
        const int32_t *row = p.table + (int64_t)r * p.row_pages;
        for (int32_t k0 = lane; k0 < n; k0 += 64 * AHEAD) {
            int32_t id[AHEAD];
#pragma unroll
            for (int z = 0; z < AHEAD; ++z)
                if (k0 + 64 * z < n) id[z] = row[k0 + 64 * z];
#pragma unroll
            for (int z = 0; z < AHEAD; ++z)
                if (k0 + 64 * z < n) p.ring[ring_at(p, head, (int64_t)free_pages + b + k0 + 64 * z)] = id[z];
        }
    }
}

// the last i in [lo, hi) with a[i] <= x (a[lo] <= x, a ascending)
__device__ __forceinline__ int32_t last_at_most(const int32_t *a, int32_t lo, int32_t hi, int32_t x) {
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kPlanThreads) void agft_kv_plan_kernel(PlanArgs p) {
    constexpr int PER = plan_per<kPlanThreads>;
    __shared__ PlanLds<kPlanThreads> lds;
    __shared__ int32_t s_first[kPlanChunk], s_past[kPlanChunk], s_granted[kPlanChunk], s_need[kPlanChunk],
        s_touched[kPlanChunk], s_back[kPlanChunk], s_tiles[kPlanChunk], s_items[kPlanChunk], s_parts[kPlanChunk];
    const int32_t head = p.counters[0], free_pages = p.counters[1];
    PlanPart<kPlanThreads> o;
    plan_chunk(p, 0, 0, 0, free_pages, lds, o);
    const int i0 = threadIdx.x * PER;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        s_first[i0 + j] = o.first[j], s_past[i0 + j] = o.past[j], s_granted[i0 + j] = o.granted[j];
        s_need[i0 + j] = o.need[j], s_touched[i0 + j] = o.sums[0][j], s_back[i0 + j] = o.sums[3][j];
    }
    if (o.all[2] > 0) {
        int32_t base[PER], parts[PER];
        plan_order(p, o, lds, base, parts, &o.all[2]);
#pragma unroll
        for (int j = 0; j < PER; ++j) s_tiles[i0 + j] = o.tiles[j], s_items[i0 + j] = base[j], s_parts[i0 + j] = parts[j];
    }
    if (blockIdx.x == 0) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = i0 + j;
            if (i >= p.requests) continue;
            p.starts[i] = o.first[j], p.granted[i] = o.granted[j], p.out_lengths[i] = o.after[j];
            p.works[i] = Work{o.sums[1][j], 0, o.first[j], o.granted[j], o.after[j], {0, 0, 0}};
        }
        if (threadIdx.x == 0) plan_totals(p, o.tokens, o.all, head, free_pages);
        plan_arrived(p);
    }
    __syncthreads();
    const int32_t total = o.tokens < (uint32_t)p.max_tokens ? (int32_t)o.tokens : p.max_tokens;
    for (int64_t t0 = (int64_t)blockIdx.x * kPlanTokens; t0 < p.max_tokens; t0 += (int64_t)gridDim.x * kPlanTokens)
        for (int64_t t = t0 + threadIdx.x; t < t0 + kPlanTokens && t < p.max_tokens; t += kPlanThreads) {
            const int32_t i = t < total ? last_at_most(s_first, 0, p.requests, (int32_t)t) : 0;
            if (t < total && o.all[2] > 0) plan_items(p, i, (int32_t)t - s_first[i], s_tiles[i], s_items[i], s_parts[i]);
            if (t < total && s_granted[i] > 0)
                plan_token(p, t, i, s_past[i], (int32_t)t - s_first[i], s_need[i], s_touched[i], head);
            else
                p.slots[t] = -1;
        }
    // pages given back, one after another over all threads
    for (int32_t k = blockIdx.x * kPlanThreads + threadIdx.x; k < o.all[3]; k += gridDim.x * kPlanThreads) {
        const int32_t i = last_at_most(s_back, 0, p.requests, k);
        p.ring[ring_at(p, head, (int64_t)free_pages + k)] = p.table[(int64_t)i * p.row_pages + k - s_back[i]];
    }
}

// More than kPlanChunk requests, first launch: a workgroup per chunk.
__global__ __launch_bounds__(kSumsThreads) void agft_kv_plan_sums_kernel(PlanArgs p) {
    constexpr int PER = plan_per<kSumsThreads>;
    __shared__ PlanLds<kSumsThreads> lds;
    __shared__ uint32_t s_before[2][kSumsThreads / 64];
    const int32_t free_pages = p.counters[1];
    const int r0 = blockIdx.x * kPlanChunk, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t need0 = 0, tok0 = 0;
    constexpr int AHEAD = 16;                  // earlier requests of a thread on their way at once
    for (int i0 = threadIdx.x; i0 < r0; i0 += AHEAD * kSumsThreads) {
        int32_t past[AHEAD], add[AHEAD];
#pragma unroll
        for (int z = 0; z < AHEAD; ++z) {
            const int i = i0 + z * kSumsThreads;
            past[z] = i < r0 ? p.lengths[i] : 0, add[z] = i < r0 ? p.add[i] : 0;
        }
#pragma unroll
        for (int z = 0; z < AHEAD; ++z) {
            const Ask a = ask_of(p, past[z], add[z]);
            need0 = add_sat(need0, a.need), tok0 = add_sat(tok0, a.tokens);
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        need0 = add_sat(need0, __shfl_xor(need0, s, 64));
        tok0 = add_sat(tok0, __shfl_xor(tok0, s, 64));
    }
    if (lane == 0) s_before[0][wave] = need0, s_before[1][wave] = tok0;
    __syncthreads();
    need0 = tok0 = 0;
    for (int w = 0; w < kSumsThreads / 64; ++w) need0 = add_sat(need0, s_before[0][w]), tok0 = add_sat(tok0, s_before[1][w]);
    PlanPart<kSumsThreads> o;
    plan_chunk(p, r0, need0, tok0, free_pages, lds, o);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = r0 + threadIdx.x * PER + j;
        if (i >= p.requests) continue;
        p.starts[i] = o.first[j], p.granted[i] = o.granted[j], p.out_lengths[i] = o.after[j], p.need[i] = o.need[j];
        p.touched[i] = o.sums[0][j], p.tiles[i] = o.sums[2][j], p.back[i] = o.sums[3][j];
        p.works[i] = Work{o.sums[1][j], 0, o.first[j], o.granted[j], o.after[j], {0, 0, 0}};
    }
    if (threadIdx.x == 0) {
        for (int k = 0; k < kPlanSums; ++k) p.sums[blockIdx.x * kPlanSums + k] = o.all[k];
        if (blockIdx.x == gridDim.x - 1)
            p.starts[p.requests] = o.tokens < (uint32_t)p.max_tokens ? (int32_t)o.tokens : p.max_tokens;
    }
}

// Second launch: slots, with the chunks' totals added where they are needed.
__global__ __launch_bounds__(kPlanThreads) void agft_kv_plan_slots_kernel(PlanArgs p) {
    constexpr int kMaxChunks = 65536 / kPlanChunk;
    static_assert(kMaxChunks <= 64, "a wavefront's lanes hold the chunks' totals");
    __shared__ int32_t s_off[kPlanSums][kMaxChunks], s_all[kPlanSums], s_first[kPlanNear], s_range[2];
    const int32_t head = p.counters[0], free_pages = p.counters[1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int chunks = (p.requests + kPlanChunk - 1) / kPlanChunk;
    for (int k = wave; k < kPlanSums; k += kPlanThreads / 64) {
        const int32_t v = lane < chunks ? p.sums[lane * kPlanSums + k] : 0;
        int32_t in = v;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int32_t x = __shfl_up(in, s, 64);
            if (lane >= s) in += x;
        }
        s_off[k][lane] = in - v;
        if (lane == 63) s_all[k] = in;
    }
    __syncthreads();
    const int32_t total = p.starts[p.requests];
    if (blockIdx.x == 0) plan_arrived(p);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        int32_t all[kPlanSums];
        for (int k = 0; k < kPlanSums; ++k) all[k] = s_all[k];
        plan_totals(p, (uint32_t)total, all, head, free_pages);
    }
    // 16 requests per wavefront: sums that other kernels read become sums over
    // all requests, and pages come back
    for (int r0 = (blockIdx.x * (kPlanThreads / 64) + wave) * 16; r0 < p.requests; r0 += gridDim.x * (kPlanThreads / 64) * 16) {
        const int i = r0 + lane;
        const bool live = lane < 16 && i < p.requests;
        if (live) p.works[i].few += s_off[1][i / kPlanChunk];
        const bool ends = live && p.add[i] < 0;
        const Ask a = ask_of(p, ends ? p.lengths[i] : 0, 0);
        plan_give_back(p, ends, i, a.held, ends ? p.back[i] + s_off[3][i / kPlanChunk] : 0, head, free_pages);
    }
    for (int64_t t0 = (int64_t)blockIdx.x * kPlanTokens; t0 < p.max_tokens; t0 += (int64_t)gridDim.x * kPlanTokens) {
        // the requests of these tokens
        __syncthreads();
        if (wave < 2) {
            const int64_t t = wave == 0 ? t0 : t0 + kPlanTokens - 1;
            const int32_t i = total == 0 ? 0 : find_last([&](int k) { return p.starts[k]; }, p.requests, t < total ? (int32_t)t : total - 1);
            if (lane == 0) s_range[wave] = i;
        }
        __syncthreads();
        const int32_t lo = s_range[0], hi = s_range[1] + 1;
        const bool near = hi - lo <= kPlanNear;      // (requests without tokens may lie between)
        for (int i = lo + threadIdx.x; near && i < hi; i += kPlanThreads) s_first[i - lo] = p.starts[i];
        __syncthreads();
        for (int64_t t = t0 + threadIdx.x; t < t0 + kPlanTokens && t < p.max_tokens; t += kPlanThreads) {
            int32_t i = 0;
            if (t < total)
                i = near ? lo + last_at_most(s_first, 0, hi - lo, (int32_t)t) : last_at_most(p.starts, lo, hi, (int32_t)t);
            if (t < total && s_all[2] > 0) {
                const int32_t first = p.starts[i], rows = p.starts[i + 1] - first;
                const int64_t wide = (int64_t)rows * p.group;
                const int32_t tiles = wide <= kFewRows ? 0 : (int32_t)((wide + kTileRows - 1) / kTileRows);
                plan_items(p, i, (int32_t)t - first, tiles, s_off[2][i / kPlanChunk] + p.tiles[i], 1);
            }
            if (t < total && p.granted[i] > 0)
                plan_token(p, t, i, ask_of(p, p.lengths[i], 0).past, (int32_t)t - p.starts[i], p.need[i],
                           p.touched[i] + s_off[0][i / kPlanChunk], head);
            else
                p.slots[t] = -1;
        }
    }
}

__global__ __launch_bounds__(256) void agft_kv_reset_kernel(int32_t *counters, int32_t *lengths, int32_t *table,
                                                            int32_t *ring, int32_t requests, int64_t entries,
                                                            int32_t pages) {
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id < 8) counters[id] = id == 1 ? pages : 0;
    for (int64_t j = id; j < requests; j += stride) lengths[j] = 0;
    for (int64_t j = id; j < entries; j += stride) table[j] = 0;
    for (int64_t j = id; j < pages; j += stride) ring[j] = (int32_t)j;
}

__global__ __launch_bounds__(256) void agft_kv_commit_kernel(int32_t *counters, int32_t *lengths,
                                                             const int32_t *new_counters, const int32_t *new_lengths,
                                                             int32_t requests) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < 2) counters[i] = new_counters[i];
    if (i < requests) lengths[i] = new_lengths[i];
}

// ---- writes ----

template <int TYPE>
struct Dense;
template <>
struct Dense<AGFT_KV_BF16> {
    // 16 numbers from p (16-byte aligned)
    static __device__ __forceinline__ void load16(const void *p, float *x) {
        const uint4 *q = static_cast<const uint4 *>(p);
        const uint4 a = q[0], b = q[1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    using type = __hip_bfloat16;
    static __device__ __forceinline__ type from(float x) { return __float2bfloat16(x); }
};
template <>
struct Dense<AGFT_KV_FP16> {
    static __device__ __forceinline__ void load16(const void *p, float *x) {
        const uint4 *q = static_cast<const uint4 *>(p);
        const uint4 v[2] = {q[0], q[1]};
        const _Float16 *h = reinterpret_cast<const _Float16 *>(v);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (float)h[i];
    }
    using type = _Float16;
    static __device__ __forceinline__ type from(float x) { return (_Float16)x; }
};
template <>
struct Dense<AGFT_KV_FP32> {
    static __device__ __forceinline__ void load16(const void *p, float *x) {
        const float4 *q = static_cast<const float4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 a = q[i];
            x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = a.z, x[4 * i + 3] = a.w;
        }
    }
    using type = float;
    static __device__ __forceinline__ type from(float x) { return x; }
};

struct AppendArgs {
    char *codes;
    int32_t *exps;
    const int32_t *runs, *counters;
    const int64_t *slots;
    const void *data[2];
    int64_t token_stride[2], head_stride[2];   // bytes
    int64_t pool_tokens;
    int32_t heads, page, shift;
};

// One workgroup per run (tokens of one page), head and side; one wavefront per
// 16 tokens of the page.  Lane 16 g + m holds token m's numbers 16 g..16 g + 15
// of each 64: the layout's key entry, and what a value entry is turned from.
// 17,641 tokens of 8 heads of 128 numbers, bf16 to e4m3, 24.8 us, 4.4 TB/s of
// numbers and codes (reading and writing reach 6.2; the values' turn through LDS is
// a byte at a time); single tokens are a chain of loads, 4.5 us.
template <int FORM, int TYPE, int DIM>
__global__ void agft_kv_append_kernel(AppendArgs p) {
    constexpr int DG = DIM / kBlockDims;
    __shared__ float s_top[8];
    __shared__ uint32_t s_turn[8][kBlockBytes / 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, m = lane & 15;
    const int head = blockIdx.y, side = blockIdx.z;
    // A single token's write is a chain of loads, so whatever can be asked for
    // at once is: the run, the slots about its first token, then numbers,
    // exponent and older codes together.
    const int32_t runs = p.runs[0], t0 = p.runs[1 + blockIdx.x], total = p.counters[2];
    if ((int)blockIdx.x >= runs) return;
    int64_t near[2];                            // slots of tokens t0 + lane, t0 + 64 + lane
#pragma unroll
    for (int z = 0; z < 2; ++z) near[z] = t0 + 64 * z + lane < total ? p.slots[t0 + 64 * z + lane] : -1;
    const int64_t slot0 = __shfl(near[0], 0, 64);
    if (slot0 < 0 || slot0 >= p.pool_tokens) return;
    const int64_t page_id = slot0 >> p.shift;
    const int off = (int)(slot0 & (p.page - 1));
    // this lane's token
    const int pos = 16 * wave + m, k = pos - off;
    const int64_t at0 = __shfl(near[0], k & 63, 64), at1 = __shfl(near[1], k & 63, 64);
    const bool live = k >= 0 && (k < 64 ? at0 : at1) == slot0 + k;
    const bool older = off > 16 * wave;         // tokens of earlier windows among these 16
    int32_t *ep = p.exps + (page_id * p.heads + head) * 2 + side;
    uint4 *block = reinterpret_cast<uint4 *>(p.codes + ((page_id * p.heads + head) * 2 + side) * p.page * DIM) +
                   (size_t)wave * DG * 64;
    const int old = off > 0 ? *ep : kMinExp;
    uint4 held[DG];
#pragma unroll
    for (int dg = 0; dg < DG; ++dg) {
        held[dg] = make_uint4(0, 0, 0, 0);
        if (older) held[dg] = block[dg * 64 + lane];
    }
    float x[DG][16];
    float top = 0.0f;
    if (live) {
        const char *row = static_cast<const char *>(p.data[side]) + (t0 + k) * p.token_stride[side] +
                          head * p.head_stride[side];
#pragma unroll
        for (int dg = 0; dg < DG; ++dg) {
            Dense<TYPE>::load16(row + (size_t)(dg * kBlockDims + 16 * g) * (TYPE == AGFT_KV_FP32 ? 4 : 2), x[dg]);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float a = fabsf(x[dg][j]);
                if (a < INFINITY) top = fmaxf(top, a);   // NaN and infinities: not counted
            }
        }
    } else {
#pragma unroll
        for (int dg = 0; dg < DG; ++dg)
#pragma unroll
            for (int j = 0; j < 16; ++j) x[dg][j] = 0.0f;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s, 64));
    if (lane == 0) s_top[wave] = top;
    asm volatile("" ::"v"(old));               // the old exponent has arrived before anyone writes the new one
    __syncthreads();
    top = s_top[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) top = fmaxf(top, s_top[w]);
    int e = exponent<FORM>(top);
    if (e < old) e = old;
    const int drop = off > 0 ? e - old : 0;    // how far the older codes' exponent rises
    if (threadIdx.x == 0) *ep = e;
    const bool any = __ballot(live) != 0;
    if (!any && !(older && drop > 0)) return;
    const float inv = pow2(-e), fall = drop > 126 ? 0.0f : pow2(-drop);
#pragma unroll
    for (int dg = 0; dg < DG; ++dg) {
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float z = x[dg][4 * j + i] * inv;
                y[i] = z == z ? fminf(fmaxf(z, -Code<FORM>::kMax), Code<FORM>::kMax) : 0.0f;
            }
            c[j] = Code<FORM>::pack4(y[0], y[1], y[2], y[3]);
        }
        if (older && drop > 0) {
            uint32_t h[4] = {held[dg].x, held[dg].y, held[dg].z, held[dg].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float y[4];
                Code<FORM>::unpack4(h[j], y);
                h[j] = Code<FORM>::pack4(y[0] * fall, y[1] * fall, y[2] * fall, y[3] * fall);
            }
            held[dg] = make_uint4(h[0], h[1], h[2], h[3]);
        }
        if (side == 0) {
            block[dg * 64 + lane] = live ? make_uint4(c[0], c[1], c[2], c[3]) : held[dg];
        } else {
            // values: byte (m % 4) of word g of entry 16 (m / 4) + number
            uint8_t *turn = reinterpret_cast<uint8_t *>(s_turn[wave]);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < 16; ++j)
                turn[((m >> 2) * 16 + j) * 16 + g * 4 + (m & 3)] = (uint8_t)(c[j >> 2] >> (8 * (j & 3)));
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const uint4 fresh = reinterpret_cast<const uint4 *>(s_turn[wave])[lane];
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            // entry 16 g + m: tokens 4 g..4 g + 3
            uint32_t mask = 0;
            const uint64_t lives = __ballot(live);
#pragma unroll
            for (int i = 0; i < 4; ++i) mask |= (lives >> (4 * g + i)) & 1 ? 255u << (8 * i) : 0u;
            block[dg * 64 + lane] = make_uint4((fresh.x & mask) | (held[dg].x & ~mask), (fresh.y & mask) | (held[dg].y & ~mask),
                                               (fresh.z & mask) | (held[dg].z & ~mask), (fresh.w & mask) | (held[dg].w & ~mask));
        }
    }
}

// ---- exports ----

struct ExportArgs {
    const char *codes;
    const int32_t *exps;
    const int64_t *slots;
    void *data[2];
    int64_t token_stride[2], head_stride[2];   // numbers
    int64_t n, pool_tokens;
    int32_t heads, page, shift;
};

// Four threads per slot, a head and a side per workgroup; a thread takes 16
// numbers of each 64: one key entry, or one byte of each of 16 value entries
// (which neighbouring slots' threads read too, from the same lines).
// 17,800 slots of 8 heads of 128 numbers, e4m3 to bf16, 30.6 us, 3.6 TB/s of codes
// and numbers (reading and writing reach 6.2; a thread per key and value: 87 us for the write and
// the export of such prompts, 55 so).
constexpr int kExportSlots = 64;

template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(4 * kExportSlots) void agft_kv_export_kernel(ExportArgs p) {
    using T = typename Dense<TYPE>::type;
    const int part = threadIdx.x & 3, head = blockIdx.y, side = blockIdx.z;
    const int64_t t = (int64_t)blockIdx.x * kExportSlots + (threadIdx.x >> 2);
    if (t >= p.n) return;
    const int64_t slot = p.slots[t];
    const bool here = slot >= 0 && slot < p.pool_tokens;
    const int64_t base = ((here ? slot >> p.shift : 0) * p.heads + head) * 2 + side;
    const int pos = (int)(slot & (p.page - 1)), m = pos & 15;
    const char *block = p.codes + base * p.page * DIM + (pos >> 4) * (kBlockTokens * DIM);
    const float f = here ? pow2(p.exps[base]) : 0.0f;
    T *dst = static_cast<T *>(p.data[side]) + t * p.token_stride[side] + head * p.head_stride[side] + 16 * part;
#pragma unroll
    for (int dg = 0; dg < DIM / kBlockDims; ++dg) {
        uint32_t w[4] = {0, 0, 0, 0};
        if (here && side == 0) {
            const uint4 v = *reinterpret_cast<const uint4 *>(block + dg * kBlockBytes + (16 * part + m) * 16);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else if (here) {
            const uint8_t *v = reinterpret_cast<const uint8_t *>(block) + dg * kBlockBytes + (m >> 2) * 256 + 4 * part + (m & 3);
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j >> 2] |= (uint32_t)v[16 * j] << (8 * (j & 3));
        }
        __attribute__((aligned(16))) T out[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x[4];
            Code<FORM>::unpack4(w[j], x);
#pragma unroll
            for (int i = 0; i < 4; ++i) out[4 * j + i] = Dense<TYPE>::from(x[i] * f);
        }
#pragma unroll
        for (int j = 0; j < (int)sizeof(out) / 16; ++j)
            reinterpret_cast<uint4 *>(dst + dg * kBlockDims)[j] = reinterpret_cast<const uint4 *>(out)[j];
    }
}

// ---- host side ----

template <typename F>
int by_form_type_dim(const agft_kv_config *c, int32_t type, F f) {
    const auto dims = [&](auto form, auto ty) {
        if (c->dim == 64) return f(form, ty, std::integral_constant<int, 64>{});
        if (c->dim == 128) return f(form, ty, std::integral_constant<int, 128>{});
        return f(form, ty, std::integral_constant<int, 256>{});
    };
    const auto types = [&](auto form) {
        if (type == AGFT_KV_BF16) return dims(form, std::integral_constant<int, AGFT_KV_BF16>{});
        if (type == AGFT_KV_FP16) return dims(form, std::integral_constant<int, AGFT_KV_FP16>{});
        return dims(form, std::integral_constant<int, AGFT_KV_FP32>{});
    };
    if (c->form == AGFT_KV_E4M3) return types(std::integral_constant<int, AGFT_KV_E4M3>{});
    return types(std::integral_constant<int, AGFT_KV_INT8>{});
}

}  // namespace agft_kv_detail

using namespace agft_kv_detail;

extern "C" {

size_t agft_kv_tables_bytes(const agft_kv_config *cfg) {
    return config_status(cfg) == AGFT_OK ? tables_layout(cfg).total : 0;
}

size_t agft_kv_step_bytes(const agft_kv_config *cfg, int32_t max_tokens) {
    return config_status(cfg) == AGFT_OK && tokens_ok(max_tokens) ? step_layout(cfg, max_tokens).total : 0;
}

size_t agft_kv_cache_bytes(const agft_kv_config *cfg) {
    return config_status(cfg) == AGFT_OK ? cache_layout(cfg).total : 0;
}

int agft_kv_tables_at(const agft_kv_config *cfg, void *d_tables, size_t nbytes, agft_kv_tables_view *out) {
    const int st = config_status(cfg);
    if (st != AGFT_OK) return st;
    const TablesLayout L = tables_layout(cfg);
    if (!buffer_ok(d_tables, nbytes, L.total) || out == nullptr) return AGFT_E_INVAL;
    char *base = static_cast<char *>(d_tables);
    out->counters = reinterpret_cast<int32_t *>(base + L.counters);
    out->lengths = reinterpret_cast<int32_t *>(base + L.lengths);
    out->table = reinterpret_cast<int32_t *>(base + L.table);
    out->ring = reinterpret_cast<int32_t *>(base + L.ring);
    return AGFT_OK;
}

int agft_kv_step_at(const agft_kv_config *cfg, int32_t max_tokens, void *d_step, size_t nbytes,
                    agft_kv_step_view *out) {
    const int st = config_status(cfg);
    if (st != AGFT_OK) return st;
    if (!tokens_ok(max_tokens) || out == nullptr) return AGFT_E_INVAL;
    const StepLayout L = step_layout(cfg, max_tokens);
    if (!buffer_ok(d_step, nbytes, L.total)) return AGFT_E_INVAL;
    char *base = static_cast<char *>(d_step);
    out->counters = reinterpret_cast<int32_t *>(base + L.counters);
    out->lengths = reinterpret_cast<int32_t *>(base + L.lengths);
    out->granted = reinterpret_cast<int32_t *>(base + L.granted);
    out->starts = reinterpret_cast<int32_t *>(base + L.starts);
    out->slots = reinterpret_cast<int64_t *>(base + L.slots);
    return AGFT_OK;
}

int agft_kv_reset(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, void *stream) {
    agft_kv_tables_view v;
    const int st = agft_kv_tables_at(cfg, d_tables, tables_bytes, &v);
    if (st != AGFT_OK) return st;
    hipLaunchKernelGGL(agft_kv_reset_kernel, dim3(1024), dim3(256), 0, static_cast<hipStream_t>(stream), v.counters,
                       v.lengths, v.table, v.ring, cfg->requests, (int64_t)cfg->requests * cfg->row_pages, cfg->pages);
    return launched();
}

int agft_kv_plan(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_add,
                 void *d_step, size_t step_bytes, int32_t max_tokens, void *stream) {
    agft_kv_tables_view tv;
    agft_kv_step_view sv;
    int st = agft_kv_tables_at(cfg, d_tables, tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_kv_step_at(cfg, max_tokens, d_step, step_bytes, &sv);
    if (st != AGFT_OK) return st;
    if (d_add == nullptr || reinterpret_cast<uintptr_t>(d_add) % 4 != 0) return AGFT_E_INVAL;
    const StepLayout L = step_layout(cfg, max_tokens);
    char *base = static_cast<char *>(d_step);
    const auto part = [&](size_t at) { return reinterpret_cast<int32_t *>(base + at); };
    PlanArgs p;
    p.add = d_add;
    p.counters = tv.counters, p.lengths = tv.lengths, p.table = tv.table, p.ring = tv.ring;
    p.out_counters = sv.counters, p.starts = sv.starts, p.granted = sv.granted, p.out_lengths = sv.lengths;
    p.works = reinterpret_cast<Work *>(base + L.works), p.need = part(L.need), p.touched = part(L.touched), p.tiles = part(L.tiles);
    p.back = part(L.back), p.sums = part(L.sums), p.arrived = part(L.arrived), p.runs = part(L.runs), p.slots = sv.slots;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages, p.page = cfg->page;
    p.shift = log2_of(cfg->page), p.group = cfg->group, p.heads = cfg->heads, p.max_tokens = max_tokens;
    // (a compute unit has the registers for two such workgroups, of heads of 256 numbers for one)
    p.tile_units = per_head(kTileUnits, cfg->heads);
    p.tile_slots = cfg->dim > 128 ? p.tile_units : per_head(kTileSlots, cfg->heads);
    p.items = reinterpret_cast<Item *>(base + L.items);
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const int64_t by_tokens = ((int64_t)max_tokens + kPlanTokens - 1) / kPlanTokens;
    const auto grid = [&](int64_t most) { return dim3((unsigned)(by_tokens < most ? by_tokens : most)); };
    if (cfg->requests <= kPlanChunk) {
        // (every workgroup makes all the sums, so no more of them than run at once)
        hipLaunchKernelGGL(agft_kv_plan_kernel, grid(512), dim3(kPlanThreads), 0, hs, p);
        return launched();
    }
    const dim3 chunks((unsigned)((cfg->requests + kPlanChunk - 1) / kPlanChunk));
    hipLaunchKernelGGL(agft_kv_plan_sums_kernel, chunks, dim3(kSumsThreads), 0, hs, p);
    st = launched();
    if (st != AGFT_OK) return st;
    hipLaunchKernelGGL(agft_kv_plan_slots_kernel, grid(2048), dim3(kPlanThreads), 0, hs, p);
    return launched();
}

int agft_kv_commit(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const void *d_step,
                   size_t step_bytes, int32_t max_tokens, void *stream) {
    agft_kv_tables_view tv;
    agft_kv_step_view sv;
    int st = agft_kv_tables_at(cfg, d_tables, tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_kv_step_at(cfg, max_tokens, const_cast<void *>(d_step), step_bytes, &sv);
    if (st != AGFT_OK) return st;
    hipLaunchKernelGGL(agft_kv_commit_kernel, dim3((unsigned)((cfg->requests + 255) / 256)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), tv.counters, tv.lengths, sv.counters, sv.lengths,
                       cfg->requests);
    return launched();
}

int agft_kv_append(const agft_kv_config *cfg, void *d_cache, size_t cache_bytes, const void *d_step,
                   size_t step_bytes, int32_t max_tokens, const agft_kv_dense *k, const agft_kv_dense *v,
                   void *stream) {
    agft_kv_step_view sv;
    const int st = agft_kv_step_at(cfg, max_tokens, const_cast<void *>(d_step), step_bytes, &sv);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    if (!dense_ok(k) || !dense_ok(v) || k->type != v->type) return AGFT_E_INVAL;
    const StepLayout L = step_layout(cfg, max_tokens);
    AppendArgs p;
    p.codes = static_cast<char *>(d_cache) + C.codes;
    p.exps = reinterpret_cast<int32_t *>(static_cast<char *>(d_cache) + C.exps);
    p.runs = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_step) + L.runs);
    p.counters = sv.counters;
    p.slots = sv.slots;
    const agft_kv_dense *in[2] = {k, v};
    for (int s = 0; s < 2; ++s) {
        p.data[s] = in[s]->data;
        p.token_stride[s] = in[s]->token_stride * (int64_t)type_bytes(k->type);
        p.head_stride[s] = in[s]->head_stride * (int64_t)type_bytes(k->type);
    }
    p.pool_tokens = (int64_t)cfg->pages * cfg->page;
    p.heads = cfg->heads, p.page = cfg->page, p.shift = log2_of(cfg->page);
    const dim3 grid((unsigned)run_cap(cfg, max_tokens), (unsigned)cfg->heads, 2), block((unsigned)cfg->page * 4);
    return by_form_type_dim(cfg, k->type, [&](auto form, auto type, auto dim) {
        agft_kv_append_kernel<form(), type(), dim()><<<grid, block, 0, static_cast<hipStream_t>(stream)>>>(p);
        return launched();
    });
}

int agft_kv_export(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const int64_t *d_slots,
                   int64_t n, const agft_kv_dense *k, const agft_kv_dense *v, void *stream) {
    const int st = config_status(cfg);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    if (n < 0 || n > (int64_t)1 << 30) return AGFT_E_INVAL;
    if (n == 0) return AGFT_OK;
    if (d_slots == nullptr || reinterpret_cast<uintptr_t>(d_slots) % 8 != 0) return AGFT_E_INVAL;
    if (!dense_ok(k) || !dense_ok(v) || k->type != v->type) return AGFT_E_INVAL;
    if (!apart(k, n, cfg->heads) || !apart(v, n, cfg->heads)) return AGFT_E_INVAL;
    ExportArgs p;
    p.codes = static_cast<const char *>(d_cache) + C.codes;
    p.exps = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_cache) + C.exps);
    p.slots = d_slots;
    p.data[0] = k->data, p.data[1] = v->data;
    p.token_stride[0] = k->token_stride, p.token_stride[1] = v->token_stride;
    p.head_stride[0] = k->head_stride, p.head_stride[1] = v->head_stride;
    p.n = n;
    p.pool_tokens = (int64_t)cfg->pages * cfg->page;
    p.heads = cfg->heads, p.page = cfg->page, p.shift = log2_of(cfg->page);
    const dim3 grid((unsigned)((n + kExportSlots - 1) / kExportSlots), (unsigned)cfg->heads, 2);
    return by_form_type_dim(cfg, k->type, [&](auto form, auto type, auto dim) {
        agft_kv_export_kernel<form(), type(), dim()><<<grid, dim3(4 * kExportSlots), 0, static_cast<hipStream_t>(stream)>>>(p);
        return launched();
    });
}

}  // extern "C"
