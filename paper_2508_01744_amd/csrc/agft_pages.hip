// agft_pages.hip -- which requests hold which pages of a serving node's cache:
// forks, trims, compaction, and the copies of pages that they ask for.
// agft_pages.h states the rules.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "agft_kv_common.h"
#include "agft_pages.h"

namespace agft_pages_detail {

using namespace agft_kv_detail;

constexpr int kThreads = 256;
constexpr int kChunks = 1024;          // workgroups, at most, that share the requests of a trim
constexpr int kChunkRequests = 64;     // requests of one, at most: a lane each
constexpr int kForksOnce = 1024;       // forks whose prefix sums every workgroup makes for itself
constexpr int kRowPart = 1024;         // entries of a table's row that a workgroup copies
constexpr int kMaxRequests = 65536;
constexpr int kNearPages = 1 << 18;    // pages whose free bits a workgroup keeps in LDS
constexpr int kChunkWords = 1024;      // words of 32 free bits whose prefix sums one workgroup makes

enum { kHead, kFree, kExtra, kRefused, kTaken, kGiven, kEntries, kKind };
// of the tables' counters, behind the first three: pages have owners that nobody counted
constexpr int kUncounted = 3;
// what the commit needs beside: owners beyond the first before the edit; held pages and moves of a compaction
enum { kExtraBefore, kHeld, kMoves };

struct EditLayout {
    size_t counters, info, lengths, past, granted, moves, rows, sums, flags, bits, prefix, before, total;
};

inline bool moves_ok(int32_t n) { return n >= 1 && n <= 1 << 27; }

inline int32_t words_of(int32_t pages) { return (int32_t)(((int64_t)pages + 31) / 32); }
inline int32_t word_chunks(int32_t pages) { return (words_of(pages) + kChunkWords - 1) / kChunkWords; }

inline EditLayout edit_layout(const agft_kv_config *c, int32_t max_moves) {
    EditLayout L;
    size_t at = 0;
    const size_t row = align_up((size_t)c->requests * 4), words = align_up((size_t)words_of(c->pages) * 4);
    L.counters = at, at += align_up(8 * 4);
    L.info = at, at += align_up(8 * 4);
    L.lengths = at, at += row;
    L.past = at, at += row;
    L.granted = at, at += align_up((size_t)max_moves * 4);
    L.moves = at, at += align_up((size_t)max_moves * 8);
    L.rows = at, at += align_up((size_t)(max_moves < kMaxRequests ? max_moves : kMaxRequests) * 16);
    L.sums = at, at += align_up((size_t)(3 * kChunks > word_chunks(c->pages) ? 3 * kChunks : word_chunks(c->pages)) * 4);
    L.flags = at, at += align_up((size_t)c->requests * c->row_pages);
    L.bits = at, at += words;
    L.prefix = at, at += words;
    L.before = at, at += words;
    L.total = at;
    return L;
}

struct EditArgs {
    // the tables'
    int32_t *counters, *lengths, *table, *ring, *owners;
    int2 *marks;
    // the edit's
    int32_t *out, *info, *out_lengths, *past, *granted;
    int2 *moves;
    int4 *rows;
    int32_t *sums;
    uint8_t *flags;
    uint32_t *bits;
    int32_t *prefix, *before;
    // the call's
    const int32_t *src, *dst, *tokens, *keep;
    int32_t n, max_moves;
    int32_t requests, row_pages, pages, page, shift;
    int32_t per;            // requests of a chunk
};

__device__ __forceinline__ int32_t pages_of(const EditArgs &p, int32_t n) { return (n + p.page - 1) >> p.shift; }
__device__ __forceinline__ int32_t held_to(const EditArgs &p, int32_t n) {
    const int32_t most = p.row_pages << p.shift;
    return n < 0 ? 0 : n > most ? most : n;
}
__device__ __forceinline__ int32_t page_at(const EditArgs &p, int32_t id) {
    return (uint32_t)id < (uint32_t)p.pages ? id : p.pages - 1;
}
// place k of the ring from its head on
__device__ __forceinline__ int32_t ring_at(const EditArgs &p, int32_t head, int64_t k) {
    return (int32_t)(((int64_t)(uint32_t)head + k) % p.pages);
}
__device__ __forceinline__ int32_t free_of(const EditArgs &p) {
    const int32_t n = p.counters[kFree];
    return n < 0 ? 0 : n > p.pages ? p.pages : n;
}

// the sum over the lanes up to this one
__device__ __forceinline__ int32_t up_to(int32_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int32_t y = __shfl_up(x, s, 64);
        if (lane >= s) x += y;
    }
    return x;
}

// The sum over the threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ int32_t before_me(int32_t x, int32_t *all, int32_t *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t to = up_to(x);
    __syncthreads();                        // (an earlier scan's sums have been read)
    if (lane == 63) lds[wave] = to;
    __syncthreads();
    int32_t before = to - x;
    *all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += lds[w];
        *all += lds[w];
    }
    return before;
}

// N sums over all threads.
template <int THREADS, int N>
__device__ __forceinline__ void sums_of(int32_t *x, int32_t *lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int s = 1; s < 64; s *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += __shfl_xor(x[k], s, 64);
    __syncthreads();                        // (an earlier scan's sums have been read)
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (lane == 0) lds[k * (THREADS / 64) + wave] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        x[k] = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) x[k] += lds[k * (THREADS / 64) + w];
    }
}

// Lengths before and after an edit that leaves them.
__device__ __forceinline__ void keep_lengths(const EditArgs &p, const uint32_t *but) {
    for (int32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < p.requests; i += gridDim.x * blockDim.x) {
        const int32_t n = held_to(p, p.lengths[i]);
        p.past[i] = n;
        if (but == nullptr || !(but[i >> 5] >> (i & 31) & 1)) p.out_lengths[i] = n;
    }
}

// ---- forks ----
//
// Which forks are granted is one prefix sum over the fresh pages that they need;
// the rest is a copy of table entries.  Both are latency: a chain of loads (src and
// dst, lengths, an entry, the ring) and a launch.  Nothing that the sums depend on
// changes before the commit, so up to kForksOnce forks every workgroup makes them
// all for itself and copies its share of the rows.  Beyond, one workgroup goes
// over the forks, 1,024 at a time, and a second launch copies.

struct Fork {
    int32_t src, dst, tokens;       // tokens asked for, 0 if none can be
    int32_t full, fresh;            // whole pages; the fresh page or -1
    bool ok;
};

struct ForkLds {
    uint32_t seen[kMaxRequests / 32], twice[kMaxRequests / 32];
    int32_t sums[16];
};

// Note who is named in dst, once and more than once.
__device__ __forceinline__ void fork_note(const EditArgs &p, int32_t j, ForkLds &lds) {
    if (j >= p.n) return;
    const int32_t d = p.dst[j];
    if ((uint32_t)d >= (uint32_t)p.requests) return;
    const uint32_t bit = 1u << (d & 31);
    if (atomicOr(&lds.seen[d >> 5], bit) & bit) atomicOr(&lds.twice[d >> 5], bit);
}

__device__ __forceinline__ void fork_clear(const EditArgs &p, uint32_t *words) {
    for (int k = threadIdx.x; k < (p.requests + 31) / 32; k += blockDim.x) words[k] = 0;
}

struct Wish {
    int32_t src, dst, have, there, tokens;
};
__device__ __forceinline__ Wish fork_read(const EditArgs &p, int32_t j) {
    Wish w{-1, -1, 0, 0, 0};
    if (j >= p.n) return w;
    w.src = p.src[j], w.dst = p.dst[j];
    w.tokens = p.tokens == nullptr ? INT32_MAX : p.tokens[j];
    if ((uint32_t)w.src < (uint32_t)p.requests && (uint32_t)w.dst < (uint32_t)p.requests)
        w.have = held_to(p, p.lengths[w.src]), w.there = p.lengths[w.dst];
    return w;
}
__device__ __forceinline__ Fork fork_ask(const EditArgs &p, const Wish &w, const ForkLds &lds) {
    Fork f{w.src, w.dst, 0, 0, -1, false};
    const int32_t t = w.tokens < w.have ? w.tokens : w.have;
    if (t > 0 && w.src != w.dst && w.there == 0 && !(lds.twice[w.dst >> 5] >> (w.dst & 31) & 1))
        f.tokens = t, f.full = t >> p.shift;
    return f;
}
__device__ __forceinline__ bool fork_needs(const EditArgs &p, const Fork &f) { return (f.tokens & (p.page - 1)) != 0; }

// need0: pages that earlier forks need
__device__ __forceinline__ void fork_grant(const EditArgs &p, Fork &f, int32_t need0, int32_t head, int32_t free_pages) {
    const bool needs = fork_needs(p, f);
    f.ok = f.tokens > 0 && (!needs || need0 < free_pages);
    if (f.ok && needs) f.fresh = page_at(p, p.ring[ring_at(p, head, need0)]);
}

__device__ __forceinline__ void fork_put(const EditArgs &p, int32_t j, const Fork &f) {
    p.granted[j] = f.ok ? f.tokens : 0;
    p.moves[j] = f.fresh >= 0 ? make_int2(page_at(p, p.table[(int64_t)f.src * p.row_pages + f.full]), f.fresh) : make_int2(-1, -1);
    p.rows[j] = make_int4(f.src, f.dst, f.ok ? f.full : 0, f.fresh);
    if (f.ok) p.out_lengths[f.dst] = f.tokens;
}

__device__ __forceinline__ void fork_totals(const EditArgs &p, int32_t need, int32_t shared, int32_t granted, int32_t head,
                                            int32_t free_pages) {
    const int32_t taken = need < free_pages ? need : free_pages, extra = p.counters[kExtra];
    int32_t *c = p.out;
    c[kHead] = ring_at(p, head, taken), c[kFree] = free_pages - taken, c[kExtra] = extra + shared;
    c[kRefused] = p.n - granted, c[kTaken] = taken, c[kGiven] = 0, c[kEntries] = p.n, c[kKind] = AGFT_PAGES_FORK;
    p.info[kExtraBefore] = extra;
}

// Part `part` of a fork's row.
__device__ __forceinline__ void fork_row(const EditArgs &p, int32_t src, int32_t dst, int32_t full, int32_t fresh,
                                         int64_t part) {
    const int32_t *from = p.table + (int64_t)src * p.row_pages;
    int32_t *to = p.table + (int64_t)dst * p.row_pages;
    const int64_t c0 = part * kRowPart;
    int32_t id[kRowPart / kThreads];
#pragma unroll
    for (int z = 0; z < kRowPart / kThreads; ++z) {
        const int64_t c = c0 + z * kThreads + threadIdx.x;
        if (c < full) id[z] = from[c];
    }
#pragma unroll
    for (int z = 0; z < kRowPart / kThreads; ++z) {
        const int64_t c = c0 + z * kThreads + threadIdx.x;
        if (c < full) to[c] = id[z];
    }
    if (part == 0 && threadIdx.x == 0 && fresh >= 0) to[full] = fresh;
}

__global__ __launch_bounds__(kThreads) void agft_pages_fork_kernel(EditArgs p, int32_t parts) {
    constexpr int PER = kForksOnce / kThreads;
    __shared__ ForkLds lds;
    __shared__ uint32_t got[kMaxRequests / 32];
    __shared__ int4 s_rows[kForksOnce];
    const int32_t head = p.counters[kHead], free_pages = free_of(p);
    fork_clear(p, lds.seen), fork_clear(p, lds.twice), fork_clear(p, got);
    const int32_t j0 = threadIdx.x * PER;
    Wish w[PER];
#pragma unroll
    for (int z = 0; z < PER; ++z) w[z] = fork_read(p, j0 + z);
    __syncthreads();
#pragma unroll
    for (int z = 0; z < PER; ++z) fork_note(p, j0 + z, lds);
    __syncthreads();
    Fork f[PER];
    int32_t need = 0, all_need, all_shared, all_ok;
#pragma unroll
    for (int z = 0; z < PER; ++z) f[z] = fork_ask(p, w[z], lds), need += fork_needs(p, f[z]);
    int32_t at = before_me<kThreads>(need, &all_need, lds.sums), shared = 0, ok = 0;
#pragma unroll
    for (int z = 0; z < PER; ++z) {
        fork_grant(p, f[z], at, head, free_pages);
        at += fork_needs(p, f[z]);
        if (f[z].ok) {
            shared += f[z].full, ++ok;
            atomicOr(&got[f[z].dst >> 5], 1u << (f[z].dst & 31));
        }
        s_rows[j0 + z] = make_int4(f[z].src, f[z].dst, f[z].ok ? f[z].full : 0, f[z].fresh);
    }
    if (blockIdx.x == 0) {
        before_me<kThreads>(shared, &all_shared, lds.sums);
        before_me<kThreads>(ok, &all_ok, lds.sums);
#pragma unroll
        for (int z = 0; z < PER; ++z)
            if (j0 + z < p.n) fork_put(p, j0 + z, f[z]);
        if (threadIdx.x == 0) fork_totals(p, all_need, all_shared, all_ok, head, free_pages);
    }
    __syncthreads();
    keep_lengths(p, got);
    for (int64_t x = blockIdx.x; x < (int64_t)p.n * parts; x += gridDim.x) {
        const int4 r = s_rows[x / parts];
        const int64_t part = x % parts;
        if (part * kRowPart < r.z || (part == 0 && r.w >= 0)) fork_row(p, r.x, r.y, r.z, r.w, part);
    }
}

// More than kForksOnce forks, first launch: one workgroup.
__global__ __launch_bounds__(1024) void agft_pages_fork_scan_kernel(EditArgs p) {
    __shared__ ForkLds lds;
    __shared__ uint32_t got[kMaxRequests / 32];
    const int32_t head = p.counters[kHead], free_pages = free_of(p);
    fork_clear(p, lds.seen), fork_clear(p, lds.twice), fork_clear(p, got);
    __syncthreads();
    for (int32_t j = threadIdx.x; j < p.n; j += 1024) fork_note(p, j, lds);
    __syncthreads();
    int32_t need0 = 0, shared = 0, ok = 0;
    for (int32_t j0 = 0; j0 < p.n; j0 += 1024) {
        const int32_t j = j0 + threadIdx.x;
        Fork f = fork_ask(p, fork_read(p, j), lds);
        int32_t all;
        const int32_t at = need0 + before_me<1024>(fork_needs(p, f), &all, lds.sums);
        need0 += all;
        fork_grant(p, f, at, head, free_pages);
        if (f.ok) {
            shared += f.full, ++ok;
            atomicOr(&got[f.dst >> 5], 1u << (f.dst & 31));
        }
        if (j < p.n) fork_put(p, j, f);
    }
    int32_t all_shared, all_ok;
    before_me<1024>(shared, &all_shared, lds.sums);
    before_me<1024>(ok, &all_ok, lds.sums);
    if (threadIdx.x == 0) fork_totals(p, need0, all_shared, all_ok, head, free_pages);
    __syncthreads();
    keep_lengths(p, got);
}

__global__ __launch_bounds__(kThreads) void agft_pages_fork_rows_kernel(EditArgs p, int32_t parts) {
    for (int64_t x = blockIdx.x; x < (int64_t)p.n * parts; x += gridDim.x) {
        const int4 r = p.rows[x / parts];
        const int64_t part = x % parts;
        if (part * kRowPart < r.z || (part == 0 && r.w >= 0)) fork_row(p, r.x, r.y, r.z, r.w, part);
    }
}

// ---- trims ----
//
// The entries that the requests let go, in order, are one list.  A page with one
// owner goes back where its entry stands; one with several goes back if as many
// entries of the list name it as it has owners, where the last of them stands.  So:
// count the entries of each shared page, and its last request (marks); flag the
// entries that go back and count them by chunk of requests; put them behind the
// ring's tail.  The last launch sets the marks back to 0.  Where no page is shared,
// the first launch is empty and the second reads no entries.

struct TrimLds {
    int32_t past[kChunkRequests], to[kChunkRequests], first[kChunkRequests], at[kChunkRequests + 1];
    int32_t refused;
    int32_t sums[16];
};

// The chunk's requests, a lane of the first wavefront each.  PLAN: from what is
// asked for, else from the edit's lengths.
template <bool PLAN>
__device__ __forceinline__ void trim_chunk(const EditArgs &p, bool extra, TrimLds &lds) {
    if (threadIdx.x < 64) {
        const int32_t lane = threadIdx.x, i = blockIdx.x * p.per + lane;
        const bool here = lane < p.per && i < p.requests;
        int32_t past = 0, to = 0;
        bool refused = false;
        const bool uncounted = PLAN && p.counters[kUncounted] != 0;
        if (here) {
            if constexpr (PLAN) {
                past = held_to(p, p.lengths[i]);
                const int32_t k = p.keep[i];
                to = k >= 0 && k < past ? k : past;
                if (uncounted) refused = to < past;
                else if (extra && to < past && (to & (p.page - 1)) != 0)
                    refused = p.owners[page_at(p, p.table[(int64_t)i * p.row_pages + (to >> p.shift)])] > 0;
                if (refused) to = past;
            } else {
                past = held_to(p, p.past[i]), to = held_to(p, p.out_lengths[i]);
                if (to > past) to = past;
            }
        }
        const int32_t first = pages_of(p, to), gone = pages_of(p, past) - first, end = up_to(gone);
        lds.past[lane] = past, lds.to[lane] = to, lds.first[lane] = first, lds.at[lane + 1] = end;
        const int32_t all_refused = __popcll(__ballot(refused));
        if (lane == 0) lds.at[0] = 0, lds.refused = all_refused;
    }
    __syncthreads();
}

// Entry e of the chunk's list: its request's place in the chunk, and its place in the table.
__device__ __forceinline__ int trim_entry(const EditArgs &p, const TrimLds &lds, int32_t e, int64_t *idx) {
    int lo = 0, hi = kChunkRequests;
#pragma unroll
    for (int s = 0; s < 6; ++s) {
        const int mid = (lo + hi) >> 1;
        if (lds.at[mid] <= e) lo = mid;
        else hi = mid;
    }
    *idx = (int64_t)(blockIdx.x * p.per + lo) * p.row_pages + lds.first[lo] + e - lds.at[lo];
    return lo;
}

__global__ __launch_bounds__(kThreads) void agft_pages_trim_mark_kernel(EditArgs p) {
    __shared__ TrimLds lds;
    if (p.counters[kExtra] == 0) return;
    trim_chunk<true>(p, true, lds);
    const int32_t total = lds.at[kChunkRequests];
    for (int32_t e = threadIdx.x; e < total; e += kThreads) {
        int64_t idx;
        const int r = trim_entry(p, lds, e, &idx);
        const int32_t id = page_at(p, p.table[idx]);
        if (p.owners[id] > 0) {
            atomicAdd(&p.marks[id].x, 1);
            atomicMax(&p.marks[id].y, (int32_t)(blockIdx.x * p.per) + r + 1);
        }
    }
}

__global__ __launch_bounds__(kThreads) void agft_pages_trim_flag_kernel(EditArgs p) {
    __shared__ TrimLds lds;
    const bool extra = p.counters[kExtra] != 0;
    trim_chunk<true>(p, extra, lds);
    const int32_t total = lds.at[kChunkRequests];
    int32_t given = 0;
    for (int32_t e = threadIdx.x; extra && e < total; e += kThreads) {
        int64_t idx;
        const int r = trim_entry(p, lds, e, &idx);
        const int32_t id = page_at(p, p.table[idx]), more = p.owners[id];
        bool back = true;
        if (more > 0) {
            const int2 mark = p.marks[id];
            back = mark.x == more + 1 && mark.y == (int32_t)(blockIdx.x * p.per) + r + 1;
        }
        p.flags[idx] = back;
        given += back;
    }
    int32_t all = total;
    if (extra) before_me<kThreads>(given, &all, lds.sums);
    if (threadIdx.x == 0) {
        p.sums[blockIdx.x] = all;
        p.sums[kChunks + blockIdx.x] = lds.refused;
        p.sums[2 * kChunks + blockIdx.x] = total;
    }
}

__global__ __launch_bounds__(kThreads) void agft_pages_trim_give_kernel(EditArgs p) {
    __shared__ TrimLds lds;
    const int32_t head = p.counters[kHead], free_pages = free_of(p), extra = p.counters[kExtra];
    trim_chunk<true>(p, extra != 0, lds);
    const int32_t total = lds.at[kChunkRequests];
    int32_t sum[4] = {};                    // given back before this chunk, and in all; refused; let go
    for (int32_t k = threadIdx.x; k < (int32_t)gridDim.x; k += kThreads) {
        const int32_t g = p.sums[k];
        if (k < (int32_t)blockIdx.x) sum[0] += g;
        sum[1] += g, sum[2] += p.sums[kChunks + k], sum[3] += p.sums[2 * kChunks + k];
    }
    sums_of<kThreads, 4>(sum, lds.sums);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int32_t room = p.pages - free_pages, given = sum[1] < room ? sum[1] : room;
        int32_t *c = p.out;
        c[kHead] = head, c[kFree] = free_pages + given, c[kExtra] = extra - (sum[3] - sum[1]);
        c[kRefused] = sum[2], c[kTaken] = 0, c[kGiven] = given, c[kEntries] = 0, c[kKind] = AGFT_PAGES_TRIM;
        p.info[kExtraBefore] = extra;
    }
    if (threadIdx.x < 64) {
        const int32_t lane = threadIdx.x, i = blockIdx.x * p.per + lane;
        if (lane < p.per && i < p.requests) p.past[i] = lds.past[lane], p.out_lengths[i] = lds.to[lane];
    }
    int32_t at = sum[0];
    for (int32_t e0 = 0; e0 < total; e0 += kThreads) {
        const int32_t e = e0 + threadIdx.x;
        int64_t idx = 0;
        int32_t id = 0;
        bool back = false;
        if (e < total) {
            trim_entry(p, lds, e, &idx);
            id = page_at(p, p.table[idx]);
            back = extra == 0 || p.flags[idx] != 0;
            if (extra != 0 && p.owners[id] > 0) p.marks[id] = make_int2(0, 0);
        }
        int32_t all;
        const int64_t k = (int64_t)at + before_me<kThreads>(back, &all, lds.sums);
        if (back && free_pages + k < p.pages) p.ring[ring_at(p, head, free_pages + k)] = id;
        at += all;
    }
}

// ---- compaction ----
//
// Free pages are bits; a page's rank among the free (held) ones is a prefix sum of
// their counts, and ranks pair the moves.  Up to kNearPages every workgroup makes
// all the bits and sums for itself, in LDS, from the ring; beyond, launches follow
// one another: bits cleared, bits set, sums by chunk, moves.

__device__ __forceinline__ int32_t held_pages(const EditArgs &p) { return p.pages - free_of(p); }

// Free pages below page x, from the word's bits and the free pages before it.
__device__ __forceinline__ int32_t free_below(uint32_t word, int32_t before, int32_t x) {
    return before + __popc(word & ((1u << (x & 31)) - 1u));
}

// Page x's place in the moves, if it has one.
__device__ __forceinline__ void compact_page(const EditArgs &p, int32_t x, uint32_t word, int32_t before, int32_t n,
                                             int32_t below, int32_t moves) {
    const bool is_free = word >> (x & 31) & 1;
    const int32_t rank = free_below(word, before, x);
    if (is_free && x < n && rank < moves) p.moves[rank].y = x;
    const int32_t held = (x - rank) - (n - below);
    if (!is_free && x >= n && held < moves) p.moves[held].x = x;
}

// below: free pages below n; all: free pages
__device__ __forceinline__ int32_t compact_moves(const EditArgs &p, int32_t n, int32_t below, int32_t all) {
    const int32_t above = (p.pages - n) - (all - below);
    const int32_t m = below < above ? below : above;
    return m < p.max_moves ? m : p.max_moves;
}

__device__ __forceinline__ void compact_rest(const EditArgs &p, int32_t n, int32_t moves) {
    keep_lengths(p, nullptr);
    for (int32_t k = moves + blockIdx.x * blockDim.x + threadIdx.x; k < p.max_moves; k += gridDim.x * blockDim.x)
        p.moves[k] = make_int2(-1, -1);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        int32_t *c = p.out;
        c[kHead] = n % p.pages, c[kFree] = p.pages - n, c[kExtra] = p.counters[kExtra];
        c[kRefused] = c[kTaken] = c[kGiven] = 0, c[kEntries] = moves, c[kKind] = AGFT_PAGES_COMPACT;
        p.info[kExtraBefore] = p.counters[kExtra], p.info[kHeld] = n, p.info[kMoves] = moves;
    }
}

__global__ __launch_bounds__(1024) void agft_pages_compact_kernel(EditArgs p) {
    constexpr int PER = kNearPages / 32 / 1024;
    __shared__ uint32_t s_bits[kNearPages / 32];
    __shared__ int32_t s_before[kNearPages / 32], s_sums[16];
    const int32_t head = p.counters[kHead], free_pages = free_of(p), n = p.pages - free_pages;
    const int32_t words = (p.pages + 31) >> 5;
    for (int k = threadIdx.x; k < words; k += 1024) s_bits[k] = 0;
    __syncthreads();
    constexpr int AHEAD = 8;                   // entries of a thread on their way at once
    for (int32_t k0 = threadIdx.x; k0 < free_pages; k0 += 1024 * AHEAD) {
        int32_t id[AHEAD];
#pragma unroll
        for (int z = 0; z < AHEAD; ++z) id[z] = k0 + 1024 * z < free_pages ? p.ring[ring_at(p, head, k0 + 1024 * z)] : -1;
#pragma unroll
        for (int z = 0; z < AHEAD; ++z)
            if ((uint32_t)id[z] < (uint32_t)p.pages) atomicOr(&s_bits[id[z] >> 5], 1u << (id[z] & 31));
    }
    __syncthreads();
    uint32_t word[PER];
    int32_t mine = 0, all;
#pragma unroll
    for (int z = 0; z < PER; ++z) {
        const int k = threadIdx.x * PER + z;
        word[z] = k < words ? s_bits[k] : 0;
        mine += __popc(word[z]);
    }
    int32_t at = before_me<1024>(mine, &all, s_sums);
#pragma unroll
    for (int z = 0; z < PER; ++z) {
        const int k = threadIdx.x * PER + z;
        if (k < words) s_before[k] = at;
        at += __popc(word[z]);
    }
    __syncthreads();
    const int32_t below = n == p.pages ? all : free_below(s_bits[n >> 5], s_before[n >> 5], n);
    const int32_t moves = compact_moves(p, n, below, all);
    for (int32_t x = blockIdx.x * 1024 + threadIdx.x; x < p.pages; x += gridDim.x * 1024) {
        const uint32_t w = s_bits[x >> 5];
        const int32_t b = s_before[x >> 5];
        compact_page(p, x, w, b, n, below, moves);
        if ((x & 31) == 0) p.bits[x >> 5] = w, p.before[x >> 5] = b;
    }
    compact_rest(p, n, moves);
}

__global__ __launch_bounds__(kThreads) void agft_pages_bits_clear_kernel(EditArgs p) {
    for (int32_t k = blockIdx.x * kThreads + threadIdx.x; k < (int32_t)(((int64_t)p.pages + 31) >> 5); k += gridDim.x * kThreads)
        p.bits[k] = 0;
}

__global__ __launch_bounds__(kThreads) void agft_pages_bits_set_kernel(EditArgs p) {
    const int32_t head = p.counters[kHead], free_pages = free_of(p);
    for (int32_t k = blockIdx.x * kThreads + threadIdx.x; k < free_pages; k += gridDim.x * kThreads) {
        const int32_t id = p.ring[ring_at(p, head, k)];
        if ((uint32_t)id < (uint32_t)p.pages) atomicOr(&p.bits[id >> 5], 1u << (id & 31));
    }
}

// Free pages before each word of the chunk, and in the chunk.
__global__ __launch_bounds__(kChunkWords) void agft_pages_bits_sum_kernel(EditArgs p) {
    __shared__ int32_t s_sums[16];
    const int32_t k = blockIdx.x * kChunkWords + threadIdx.x, words = (int32_t)(((int64_t)p.pages + 31) >> 5);
    int32_t all;
    const int32_t at = before_me<kChunkWords>(k < words ? __popc(p.bits[k]) : 0, &all, s_sums);
    if (k < words) p.prefix[k] = at;
    if (threadIdx.x == 0) p.sums[blockIdx.x] = all;
}

__global__ __launch_bounds__(1024) void agft_pages_bits_move_kernel(EditArgs p) {
    __shared__ int32_t s_sums[3 * 16];
    const int32_t n = held_pages(p), chunk = blockIdx.x, chunk_n = n / (32 * kChunkWords);
    int32_t sum[3] = {};                       // free pages before this chunk, before n's, and in all
    for (int32_t k = threadIdx.x; k < (int32_t)gridDim.x; k += 1024) {
        const int32_t s = p.sums[k];
        if (k < chunk) sum[0] += s;
        if (k < chunk_n) sum[1] += s;
        sum[2] += s;
    }
    sums_of<1024, 3>(sum, s_sums);
    const int32_t below = n == p.pages ? sum[2] : sum[1] + free_below(p.bits[n >> 5], p.prefix[n >> 5], n);
    const int32_t moves = compact_moves(p, n, below, sum[2]);
    const int64_t first = (int64_t)chunk * 32 * kChunkWords;
    for (int64_t x = first + threadIdx.x; x < p.pages && x < first + 32 * kChunkWords; x += 1024) {
        const uint32_t w = p.bits[x >> 5];
        const int32_t b = sum[0] + p.prefix[x >> 5];
        compact_page(p, (int32_t)x, w, b, n, below, moves);
        if ((x & 31) == 0) p.before[x >> 5] = b;
    }
    compact_rest(p, n, moves);
}

// ---- commits ----
//
// What a commit takes from the edit's memory as a place is held to what it is a place of.

// Workgroups (blockIdx.y) that share a chunk's entries.
constexpr int kCommitParts = 4;

__global__ __launch_bounds__(kThreads) void agft_pages_commit_kernel(EditArgs p) {
    __shared__ TrimLds lds;
    const int32_t kind = p.out[kKind], group = blockIdx.y * gridDim.x + blockIdx.x, groups = gridDim.x * gridDim.y;
    const int32_t thread = group * kThreads + threadIdx.x, threads = groups * kThreads;
    if (thread < 3) p.counters[thread] = p.out[thread];
    if (kind == AGFT_PAGES_FORK) {
        const int32_t most = p.max_moves < kMaxRequests ? p.max_moves : kMaxRequests;
        const int32_t n = p.out[kEntries] < most ? p.out[kEntries] : most;
        for (int32_t j = group; j < n; j += groups) {
            const int4 r = p.rows[j];
            if ((uint32_t)r.y >= (uint32_t)p.requests) continue;
            const int32_t *row = p.table + (int64_t)r.y * p.row_pages, full = r.z < p.row_pages ? r.z : p.row_pages;
            for (int32_t c = threadIdx.x; c < full; c += kThreads) atomicAdd(&p.owners[page_at(p, row[c])], 1);
        }
    } else if (kind == AGFT_PAGES_TRIM) {
        if (p.info[kExtraBefore] != 0) {
            trim_chunk<false>(p, true, lds);
            const int32_t total = lds.at[kChunkRequests];
            for (int32_t e = blockIdx.y * kThreads + threadIdx.x; e < total; e += kCommitParts * kThreads) {
                int64_t idx;
                trim_entry(p, lds, e, &idx);
                // (of an entry whose page goes back, the page's last owner: none beyond the first is left)
                if (p.flags[idx] == 0) atomicAdd(&p.owners[page_at(p, p.table[idx])], -1);
            }
        }
    } else if (kind == AGFT_PAGES_COMPACT) {
        const int32_t n = p.info[kHeld];
        const int32_t moves = (uint32_t)n < (uint32_t)p.pages ? p.info[kMoves] < p.max_moves ? p.info[kMoves] : p.max_moves : 0;
        const int32_t below = moves > 0 ? free_below(p.bits[n >> 5], p.before[n >> 5], n) : 0;
        for (int32_t k = thread; k < moves; k += threads) {
            const int2 m = p.moves[k];
            if ((uint32_t)m.x < (uint32_t)p.pages && (uint32_t)m.y < (uint32_t)p.pages) p.owners[m.y] = p.owners[m.x], p.owners[m.x] = 0;
        }
        for (int32_t k = thread; k < p.pages; k += threads) p.ring[k] = k;
        // every entry in use
        if (threadIdx.x < 64) {
            const int32_t lane = threadIdx.x, i = blockIdx.x * p.per + lane;
            const int32_t held = lane < p.per && i < p.requests ? pages_of(p, held_to(p, p.past[i])) : 0, end = up_to(held);
            lds.first[lane] = 0, lds.at[lane + 1] = end;
            if (lane == 0) lds.at[0] = 0;
        }
        __syncthreads();
        const int32_t total = moves > 0 ? lds.at[kChunkRequests] : 0;
        for (int32_t e = blockIdx.y * kThreads + threadIdx.x; e < total; e += kCommitParts * kThreads) {
            int64_t idx;
            trim_entry(p, lds, e, &idx);
            const int32_t id = p.table[idx];
            if ((uint32_t)id >= (uint32_t)p.pages || id < n) continue;
            const int32_t rank = (id - free_below(p.bits[id >> 5], p.before[id >> 5], id)) - (n - below);
            if ((uint32_t)rank < (uint32_t)moves) p.table[idx] = p.moves[rank].y;
        }
    }
    for (int32_t i = thread; i < p.requests; i += threads) p.lengths[i] = p.out_lengths[i];
}

// ---- copies ----
//
// Memory's rate: every byte read once and written once, 16 bytes a lane, four of
// them on their way (2 / 8: 637 / 623 us for 620), a workgroup a piece of a page at a time:
// 11,964 pages of 128 KB 609 us, 5.2 TB/s (a large copy of the library's 4.7), 1,177 of 32
// KB 15.8 us.  Workgroups up to 16,384 (2,048 / 4,096 / 16,384 / 65,536: 627 / 620 / 609 /
// 602; those without a move have to come and go).  Stores past the caches save 2 us of the
// 15.8 and cost whoever reads the pages next 14.
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr int kCopyAhead = 4;
constexpr int kCopyGroups = 16384;
constexpr int kCopyBytes = kThreads * 16 * kCopyAhead;

__global__ __launch_bounds__(kThreads) void agft_pages_copy_kernel(char *codes, int32_t *exps, const int32_t *counters,
                                                                   const int2 *moves, int32_t max_moves, int64_t page_bytes,
                                                                   int32_t page_exps, int32_t parts, int32_t pages) {
    const int32_t all = counters[kEntries] < max_moves ? counters[kEntries] : max_moves;
    for (int64_t x = blockIdx.x; x < (int64_t)all * parts; x += gridDim.x) {
        const int2 m = moves[x / parts];
        const int32_t part = (int32_t)(x % parts);
        if ((uint32_t)m.x >= (uint32_t)pages || (uint32_t)m.y >= (uint32_t)pages) continue;
        const int64_t at = (int64_t)part * kCopyBytes + threadIdx.x * 16;
        const char *from = codes + m.x * page_bytes + at;
        char *to = codes + m.y * page_bytes + at;
        uint4v v[kCopyAhead];
#pragma unroll
        for (int z = 0; z < kCopyAhead; ++z)
            v[z] = at + z * kThreads * 16 < page_bytes ? *reinterpret_cast<const uint4v *>(from + z * kThreads * 16) : (uint4v){};
#pragma unroll
        for (int z = 0; z < kCopyAhead; ++z)
            if (at + z * kThreads * 16 < page_bytes)
                *reinterpret_cast<uint4v *>(to + z * kThreads * 16) = v[z];
        if (part == 0)
            for (int k = threadIdx.x; k < page_exps; k += kThreads)
                exps[(int64_t)m.y * page_exps + k] = exps[(int64_t)m.x * page_exps + k];
    }
}

// ---- host side ----

inline int edit_args(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, void *d_edit, size_t edit_bytes,
                     int32_t max_moves, EditArgs *p) {
    agft_kv_tables_view tv;
    agft_pages_view ev;
    int st = agft_kv_tables_at(cfg, d_tables, tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_pages_edit_at(cfg, max_moves, d_edit, edit_bytes, &ev);
    if (st != AGFT_OK) return st;
    const TablesLayout T = tables_layout(cfg);
    const EditLayout L = edit_layout(cfg, max_moves);
    char *t = static_cast<char *>(d_tables), *e = static_cast<char *>(d_edit);
    const auto part = [&](size_t at) { return reinterpret_cast<int32_t *>(e + at); };
    *p = EditArgs{};
    p->counters = tv.counters, p->lengths = tv.lengths, p->table = tv.table, p->ring = tv.ring;
    p->owners = reinterpret_cast<int32_t *>(t + T.owners), p->marks = reinterpret_cast<int2 *>(t + T.marks);
    p->out = ev.counters, p->info = part(L.info), p->out_lengths = ev.lengths, p->past = part(L.past);
    p->granted = ev.granted, p->moves = reinterpret_cast<int2 *>(ev.moves), p->rows = reinterpret_cast<int4 *>(e + L.rows);
    p->sums = part(L.sums), p->flags = reinterpret_cast<uint8_t *>(e + L.flags);
    p->bits = reinterpret_cast<uint32_t *>(e + L.bits), p->prefix = part(L.prefix), p->before = part(L.before);
    p->max_moves = max_moves;
    p->requests = cfg->requests, p->row_pages = cfg->row_pages, p->pages = cfg->pages, p->page = cfg->page;
    p->shift = log2_of(cfg->page);
    p->per = (cfg->requests + kChunks - 1) / kChunks;
    return AGFT_OK;
}

inline bool ints_ok(const int32_t *p) { return p != nullptr && reinterpret_cast<uintptr_t>(p) % 4 == 0; }

inline dim3 chunks_of(const EditArgs &p, unsigned y = 1) { return dim3((unsigned)((p.requests + p.per - 1) / p.per), y); }

}  // namespace agft_pages_detail

using namespace agft_pages_detail;

extern "C" {

size_t agft_pages_edit_bytes(const agft_kv_config *cfg, int32_t max_moves) {
    return config_status(cfg) == AGFT_OK && moves_ok(max_moves) ? edit_layout(cfg, max_moves).total : 0;
}

int agft_pages_edit_at(const agft_kv_config *cfg, int32_t max_moves, void *d_edit, size_t nbytes, agft_pages_view *out) {
    const int st = config_status(cfg);
    if (st != AGFT_OK) return st;
    if (!moves_ok(max_moves) || out == nullptr) return AGFT_E_INVAL;
    const EditLayout L = edit_layout(cfg, max_moves);
    if (!buffer_ok(d_edit, nbytes, L.total)) return AGFT_E_INVAL;
    char *base = static_cast<char *>(d_edit);
    out->counters = reinterpret_cast<int32_t *>(base + L.counters);
    out->lengths = reinterpret_cast<int32_t *>(base + L.lengths);
    out->granted = reinterpret_cast<int32_t *>(base + L.granted);
    out->moves = reinterpret_cast<int32_t *>(base + L.moves);
    return AGFT_OK;
}

int agft_pages_owners_at(const agft_kv_config *cfg, void *d_tables, size_t nbytes, int32_t **out) {
    agft_kv_tables_view tv;
    const int st = agft_kv_tables_at(cfg, d_tables, nbytes, &tv);
    if (st != AGFT_OK) return st;
    if (out == nullptr) return AGFT_E_INVAL;
    *out = reinterpret_cast<int32_t *>(static_cast<char *>(d_tables) + tables_layout(cfg).owners);
    return AGFT_OK;
}

int agft_pages_fork(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_src,
                    const int32_t *d_dst, const int32_t *d_tokens, int32_t n, void *d_edit, size_t edit_bytes,
                    int32_t max_moves, void *stream) {
    EditArgs p;
    int st = edit_args(cfg, d_tables, tables_bytes, d_edit, edit_bytes, max_moves, &p);
    if (st != AGFT_OK) return st;
    if (!ints_ok(d_src) || !ints_ok(d_dst) || (d_tokens != nullptr && !ints_ok(d_tokens))) return AGFT_E_INVAL;
    if (n < 1 || n > max_moves || n > kMaxRequests) return AGFT_E_INVAL;
    p.src = d_src, p.dst = d_dst, p.tokens = d_tokens, p.n = n;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    const int32_t parts = (cfg->row_pages + kRowPart - 1) / kRowPart;
    const int64_t all = (int64_t)n * parts;
    if (n <= kForksOnce) {
        // (every workgroup makes all the sums, so no more of them than run at once)
        agft_pages_fork_kernel<<<dim3((unsigned)(all < 512 ? all : 512)), kThreads, 0, hs>>>(p, parts);
        return launched();
    }
    agft_pages_fork_scan_kernel<<<dim3(1), 1024, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_fork_rows_kernel<<<dim3((unsigned)(all < 8192 ? all : 8192)), kThreads, 0, hs>>>(p, parts);
    return launched();
}

int agft_pages_trim(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const int32_t *d_keep, void *d_edit,
                    size_t edit_bytes, int32_t max_moves, void *stream) {
    EditArgs p;
    int st = edit_args(cfg, d_tables, tables_bytes, d_edit, edit_bytes, max_moves, &p);
    if (st != AGFT_OK) return st;
    if (!ints_ok(d_keep)) return AGFT_E_INVAL;
    p.keep = d_keep;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    agft_pages_trim_mark_kernel<<<chunks_of(p), kThreads, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_trim_flag_kernel<<<chunks_of(p), kThreads, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_trim_give_kernel<<<chunks_of(p), kThreads, 0, hs>>>(p);
    return launched();
}

int agft_pages_compact(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, void *d_edit, size_t edit_bytes,
                       int32_t max_moves, void *stream) {
    EditArgs p;
    int st = edit_args(cfg, d_tables, tables_bytes, d_edit, edit_bytes, max_moves, &p);
    if (st != AGFT_OK) return st;
    if (max_moves < cfg->pages / 2) return AGFT_E_INVAL;
    const hipStream_t hs = static_cast<hipStream_t>(stream);
    if (cfg->pages <= kNearPages) {
        agft_pages_compact_kernel<<<dim3((unsigned)((cfg->pages + 4095) / 4096)), 1024, 0, hs>>>(p);
        return launched();
    }
    const unsigned chunks = (unsigned)word_chunks(cfg->pages);
    agft_pages_bits_clear_kernel<<<dim3(chunks), kThreads, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_bits_set_kernel<<<dim3(2048), kThreads, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_bits_sum_kernel<<<dim3(chunks), kChunkWords, 0, hs>>>(p);
    st = launched();
    if (st != AGFT_OK) return st;
    agft_pages_bits_move_kernel<<<dim3(chunks), 1024, 0, hs>>>(p);
    return launched();
}

int agft_pages_copy(const agft_kv_config *cfg, void *d_cache, size_t cache_bytes, const void *d_edit, size_t edit_bytes,
                    int32_t max_moves, void *stream) {
    agft_pages_view ev;
    const int st = agft_pages_edit_at(cfg, max_moves, const_cast<void *>(d_edit), edit_bytes, &ev);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    const int64_t page_bytes = (int64_t)cfg->heads * 2 * cfg->page * cfg->dim;
    const int32_t parts = (int32_t)((page_bytes + kCopyBytes - 1) / kCopyBytes);
    const int64_t all = (int64_t)max_moves * parts;
    char *base = static_cast<char *>(d_cache);
    agft_pages_copy_kernel<<<dim3((unsigned)(all < kCopyGroups ? all : kCopyGroups)), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
        base + C.codes, reinterpret_cast<int32_t *>(base + C.exps), ev.counters, reinterpret_cast<const int2 *>(ev.moves),
        max_moves, page_bytes, cfg->heads * 2, parts, cfg->pages);
    return launched();
}

int agft_pages_commit(const agft_kv_config *cfg, void *d_tables, size_t tables_bytes, const void *d_edit,
                      size_t edit_bytes, int32_t max_moves, void *stream) {
    EditArgs p;
    const int st = edit_args(cfg, d_tables, tables_bytes, const_cast<void *>(d_edit), edit_bytes, max_moves, &p);
    if (st != AGFT_OK) return st;
    agft_pages_commit_kernel<<<chunks_of(p, kCommitParts), kThreads, 0, static_cast<hipStream_t>(stream)>>>(p);
    return launched();
}

}  // extern "C"
