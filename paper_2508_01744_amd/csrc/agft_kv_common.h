// agft_kv_common.h -- what the cache's kernels share: the configuration's
// checks, where the parts of the caller's buffers lie, and the 8-bit codes.
#ifndef AGFT_KV_COMMON_H
#define AGFT_KV_COMMON_H

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "agft.h"
#include "agft_kv.h"

namespace agft_kv_detail {

constexpr size_t kAlign = 256;
constexpr int kBlockTokens = 16;   // tokens of a layout block
constexpr int kBlockDims = 64;     // numbers of a layout block
constexpr int kBlockBytes = kBlockTokens * kBlockDims;
constexpr int kUnit = 64;          // tokens of a unit of attention work
constexpr int kRowTile = 16;       // query rows (tokens x group) of a tile of the attention over few rows
// Query rows of a request up to which that takes it: kFewRows, or kMidRows while
// the requests of more than kFewRows rows are little work in all.  Reading the
// tokens again for every 16 rows is soon dearer than tiles of 128 that are part
// empty, which are dearer for a few tokens (us, by rows / in tiles: one head of 64
// numbers, 200 requests of 16 to 64 rows, 2,230 units, 20.5 / 29.0; 2 heads of 256,
// 9 requests of up to 20 rows over up to 3,726 tokens 22.5 / 46.2; 4 heads of 128,
// 8 requests x 32 rows x 4,000 tokens, 4,032 units, 29.8 / 23.6; 64 x 32 x 1,000,
// 8,192 units, 33.5 / 26.2; 200 x 64 x 2,000, 300 / 132).
constexpr int kFewRows = 16;
constexpr int kMidRows = 64;
constexpr int kMidUnits = 3584;    // units (for all heads) that are little work
constexpr int kTileRows = 128;     // query rows of a tile of the attention over many rows
constexpr int kFewGroups = 1024;   // workgroups, at most, that share the work of few rows
constexpr int kTileUnits = 256;    // compute units
constexpr int kTileSlots = 2 * kTileUnits;  // workgroups, at most, of the attention over many rows that run at once
constexpr int kTileParts = 2 * kTileSlots;  // of them, at most, that share rows with others
constexpr int kArrivals = 3 * kFewGroups + kTileParts;   // counters of a window's joins
constexpr int kPlanChunk = 1024;   // requests whose prefix sums one workgroup makes
constexpr int kPlanSums = 6;       // prefix sums per request that count granted tokens only
constexpr int kMinExp = -64;

inline size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

// AGFT_OK, or what is wrong with the configuration
inline int config_status(const agft_kv_config *c) {
    if (c == nullptr) return AGFT_E_INVAL;
    if (c->requests < 1 || c->requests > 65536 || c->row_pages < 1) return AGFT_E_INVAL;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return AGFT_E_INVAL;
    if ((int64_t)c->row_pages * c->page >= (int64_t)1 << 30) return AGFT_E_INVAL;
    if (c->pages < 1 || c->pages > 1 << 28) return AGFT_E_INVAL;
    if (c->heads < 1 || c->heads > 256 || c->group < 1 || c->group > 128) return AGFT_E_INVAL;
    if (c->form != AGFT_KV_E4M3 && c->form != AGFT_KV_INT8) return AGFT_E_INVAL;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256)
        return c->dim >= 1 ? AGFT_E_UNSUPPORTED : AGFT_E_INVAL;
    return AGFT_OK;
}

inline bool tokens_ok(int32_t max_tokens) { return max_tokens >= 1 && max_tokens <= 1 << 30; }

struct TablesLayout {
    size_t counters, lengths, table, ring, total;
};

inline TablesLayout tables_layout(const agft_kv_config *c) {
    TablesLayout L;
    size_t at = 0;
    L.counters = at, at += align_up(8 * 4);
    L.lengths = at, at += align_up((size_t)c->requests * 4);
    L.table = at, at += align_up((size_t)c->requests * c->row_pages * 4);
    L.ring = at, at += align_up((size_t)c->pages * 4);
    L.total = at;
    return L;
}

// What the attention reads of a request, in one place: a wavefront that knows
// the request has everything after one round trip to memory.  The last entry,
// behind the requests', holds the totals and the last start.
struct __attribute__((aligned(16))) Work {
    int32_t few;      // units of few rows of the requests before this one
    int32_t items;    // in the last entry: items of many rows
    int32_t start;    // first row
    int32_t granted, length;
    int32_t pad[3];
};

// One workgroup's task, per head, in the attention over many rows: part `part`
// of `parts` of the tokens that tile `tile` of the request's rows sees.
struct __attribute__((aligned(16))) Item {
    int32_t request, tile, part, parts;
};

// Tiles of many rows: the rows' own and a last one of each request that has
// more than kFewRows.
inline int64_t tile_cap(const agft_kv_config *c, int64_t max_tokens) {
    const int64_t rows = max_tokens * c->group, many = rows / (kFewRows + 1);
    return many == 0 ? 0 : rows / kTileRows + (many < c->requests ? many : c->requests);
}

// Items run per head; a share of the chip's slots is a head's.
inline int32_t per_head(int32_t slots, int32_t heads) { return heads < slots ? slots / heads : 1; }

// (parts come to at most one per tile and one per slot)
inline int64_t item_cap(const agft_kv_config *c, int64_t max_tokens) {
    const int64_t tiles = tile_cap(c, max_tokens);
    return tiles == 0 ? 0 : tiles + per_head(kTileSlots, c->heads);
}

struct StepLayout {
    size_t counters, starts, granted, lengths, works, tiles, need, touched, back, sums, arrived, items, runs, slots, total;
};

// Runs of one page's tokens in a window: a request's n tokens touch at most
// 2 + (n - 2) / page pages.
inline int64_t run_cap(const agft_kv_config *c, int32_t max_tokens) {
    const int64_t by_page = 2 * (int64_t)c->requests + max_tokens / c->page;
    return by_page < max_tokens ? by_page : max_tokens;
}

inline StepLayout step_layout(const agft_kv_config *c, int32_t max_tokens) {
    StepLayout L;
    size_t at = 0;
    const size_t row = align_up(((size_t)c->requests + 1) * 4);
    L.counters = at, at += align_up(8 * 4);
    L.starts = at, at += row;
    L.granted = at, at += row;
    L.lengths = at, at += row;
    L.works = at, at += align_up(((size_t)c->requests + 1) * sizeof(Work));
    L.tiles = at, at += row;
    L.need = at, at += row;
    L.touched = at, at += row;
    L.back = at, at += row;
    L.sums = at, at += align_up((size_t)kPlanSums * ((c->requests + kPlanChunk - 1) / kPlanChunk) * 4);
    L.arrived = at, at += align_up((size_t)kArrivals * 4);
    L.items = at, at += align_up((size_t)item_cap(c, max_tokens) * sizeof(Item));
    L.runs = at, at += align_up(((size_t)run_cap(c, max_tokens) + 1) * 4);
    L.slots = at, at += align_up((size_t)max_tokens * 8);
    L.total = at;
    return L;
}

struct CacheLayout {
    size_t codes, exps, total;
};

inline CacheLayout cache_layout(const agft_kv_config *c) {
    CacheLayout L;
    L.codes = 0;
    L.exps = align_up((size_t)c->pages * c->heads * 2 * c->page * c->dim);
    L.total = L.exps + align_up((size_t)c->pages * c->heads * 2 * 4);
    return L;
}

inline bool buffer_ok(const void *p, size_t have, size_t need) {
    return p != nullptr && reinterpret_cast<uintptr_t>(p) % kAlign == 0 && have >= need;
}

inline size_t type_bytes(int32_t type) { return type == AGFT_KV_FP32 ? 4 : 2; }

// rows of numbers that can be moved 16 bytes at a time
inline bool dense_ok(const agft_kv_dense *t) {
    if (t == nullptr || t->data == nullptr) return false;
    if (t->type != AGFT_KV_BF16 && t->type != AGFT_KV_FP16 && t->type != AGFT_KV_FP32) return false;
    const int64_t per = 16 / (int64_t)type_bytes(t->type);
    return reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->token_stride >= 0 && t->head_stride >= 0 &&
           t->token_stride % per == 0 && t->head_stride % per == 0;
}

// and of which each has memory of its own
inline bool apart(const agft_kv_dense *t, int64_t tokens, int64_t heads) {
    return (t->token_stride > 0 || tokens == 1) && (t->head_stride > 0 || heads == 1);
}

inline int log2_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

inline int launched() { return hipGetLastError() == hipSuccess ? AGFT_OK : AGFT_E_HIP; }

// ---- device side ----

// 2^e for e in -126..127
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The last i in [0, n) with at(i) <= x, at(0) <= x and at ascending; the whole
// wavefront looks, 64 places at a time.
template <typename F>
__device__ __forceinline__ int find_last(F at, int n, int32_t x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + 63) >> 6, k = lane * step;
        const bool below = k < len && at(lo + k) <= x;
        const int hits = __popcll(__ballot(below));
        const int skip = (hits < 1 ? 0 : hits - 1) * step;
        lo += skip;
        len = len - skip < step ? len - skip : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

template <int FORM>
struct Code;

template <>
struct Code<AGFT_KV_E4M3> {
    static constexpr float kMax = 448.0f;
    // four numbers within the range to four codes, to nearest even
    static __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    static __device__ __forceinline__ void unpack4(uint32_t w, float *x) {
        x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
        x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
        x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
        x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
    }
    // smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8)
    static __device__ __forceinline__ int need(uint32_t bits) {
        return (int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x600000u ? 8 : 7);
    }
};

template <>
struct Code<AGFT_KV_INT8> {
    static constexpr float kMax = 127.0f;
    static __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
        return ((uint32_t)(int)rintf(a) & 255u) | ((uint32_t)(int)rintf(b) & 255u) << 8 |
               ((uint32_t)(int)rintf(c) & 255u) << 16 | (uint32_t)(int)rintf(d) << 24;
    }
    static __device__ __forceinline__ void unpack4(uint32_t w, float *x) {
        x[0] = (float)(int8_t)w;
        x[1] = (float)(int8_t)(w >> 8);
        x[2] = (float)(int8_t)(w >> 16);
        x[3] = (float)(int8_t)(w >> 24);
    }
    // smallest e with top <= 127 * 2^e = 1.984375 * 2^(e + 6)
    static __device__ __forceinline__ int need(uint32_t bits) {
        return (int)(bits >> 23) - 127 - ((bits & 0x7fffffu) <= 0x7e0000u ? 6 : 5);
    }
};

// The exponent that holds top (finite, >= 0).
template <int FORM>
__device__ __forceinline__ int exponent(float top) {
    const int e = Code<FORM>::need(__float_as_uint(top));
    return e < kMinExp ? kMinExp : e;
}

}  // namespace agft_kv_detail

#endif
