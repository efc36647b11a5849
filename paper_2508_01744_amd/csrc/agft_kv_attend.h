// agft_kv_attend.h -- what the kernels of attention over the paged cache share:
// queries' types and decoded codes, how the work of few query rows is cut, and how
// workgroups meet.
#ifndef AGFT_KV_ATTEND_H
#define AGFT_KV_ATTEND_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "agft_kv_common.h"

namespace agft_kv_detail {

struct AttendArgs {
    const char *codes;
    const int32_t *exps, *table;
    const Work *works;
    const Item *items;
    const char *q;
    char *out;
    float *lse, *partial;
    int32_t *arrived;
    int64_t q_token, q_head, out_token, out_head;   // numbers
    float scale;
    int32_t requests, row_pages, pages, page, shift, heads, group;
    int32_t few_blocks;     // workgroups ahead of the tiles' that take few rows
    bool alone;             // no launch for tiles of many rows
};

typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 fp16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 fp16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 fp16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Queries' types, and codes turned into them: every code of either form is a
// number of at most eight significant bits within fp16's range.
template <int TYPE>
struct Half;
template <>
struct Half<AGFT_KV_BF16> {
    using x8 = bf16x8;
    static __device__ __forceinline__ uint2 pack4(float a, float b, float c, float d) {
        const bf16x2 x = {(__bf16)a, (__bf16)b}, y = {(__bf16)c, (__bf16)d};
        return make_uint2(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y));
    }
    template <int FORM>
    static __device__ __forceinline__ x8 decode(uint32_t lo, uint32_t hi) {
        uint32_t w[4];
        if constexpr (FORM == AGFT_KV_E4M3) {
            w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
            w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
            w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
            w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
        } else {
            // (exact in fp32's upper half)
            float x[8];
            Code<FORM>::unpack4(lo, x);
            Code<FORM>::unpack4(hi, x + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
        }
        return __builtin_bit_cast(x8, (uint4v){w[0], w[1], w[2], w[3]});
    }
    static __device__ __forceinline__ float4v mfma(x8 a, x8 b, float4v c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Half<AGFT_KV_FP16> {
    using x8 = fp16x8;
    static __device__ __forceinline__ uint2 pack4(float a, float b, float c, float d) {
        const fp16x2 x = {(_Float16)a, (_Float16)b}, y = {(_Float16)c, (_Float16)d};
        return make_uint2(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y));
    }
    template <int FORM>
    static __device__ __forceinline__ x8 decode(uint32_t lo, uint32_t hi) {
        uint32_t w[4];
        if constexpr (FORM == AGFT_KV_E4M3) {
            w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
            w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
            w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
            w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
        } else {
            // c + 128 as the low byte of 1024 + (c + 128), less 1152
            lo ^= 0x80808080u, hi ^= 0x80808080u;
            w[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
            w[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
            w[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
            w[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
            const fp16x2 base = {(_Float16)1152.0f, (_Float16)1152.0f};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(fp16x2, w[j]) - base);
        }
        return __builtin_bit_cast(x8, (uint4v){w[0], w[1], w[2], w[3]});
    }
    static __device__ __forceinline__ float4v mfma(x8 a, x8 b, float4v c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// max (or sum) over the lanes that share lane % 32, and over those that share
// lane % 16: halves (rows of 16) change places between two copies
__device__ __forceinline__ float2 halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float2 quarters(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_max(float x) {
    const float2 y = halves(x);
    return fmaxf(y.x, y.y);
}
__device__ __forceinline__ float halves_sum(float x) {
    const float2 y = halves(x);
    return y.x + y.y;
}
__device__ __forceinline__ float across_max(float x) {
    const float2 y = quarters(x);
    return halves_max(fmaxf(y.x, y.y));
}
__device__ __forceinline__ float across_sum(float x) {
    const float2 y = quarters(x);
    return halves_sum(y.x + y.y);
}

typedef float float16v __attribute__((ext_vector_type(16)));

template <int TYPE>
__device__ __forceinline__ float16v mfma32(typename Half<TYPE>::x8 a, typename Half<TYPE>::x8 b, float16v c) {
    if constexpr (TYPE == AGFT_KV_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

constexpr int kFewWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The requests' works as a wavefront sees them: those of 64 requests, a lane
// each, from request `from` on.
struct Works {
    const Work *w;
    int n, from;
    int4 a;             // few, items, start, granted of request from + lane
    int length;
    int4 total;
    __device__ __forceinline__ Works(const Work *works, int requests) : w(works), n(requests), from(0) {
        total = *reinterpret_cast<const int4 *>(w + n);
        if (n <= 64) read();
    }
    __device__ __forceinline__ void read() {
        const int lane = threadIdx.x & 63, k = from + lane < n ? from + lane : n - 1;
        a = *reinterpret_cast<const int4 *>(w + k);
        length = w[k].length;
    }
    // the requests about unit x, for more requests than lanes
    __device__ __forceinline__ void look(int32_t x) {
        if (n <= 64) return;
        from = find_last([&](int k) { return w[k].few; }, n, x);
        read();
    }
    __device__ __forceinline__ void look_at(int request) {
        if (n <= 64) return;
        from = __builtin_amdgcn_readfirstlane(request);
        read();
    }
    // whether unit x's request and the next one are among the 64
    __device__ __forceinline__ bool has(int32_t x) const {
        return n <= 64 || from + 64 >= n || __builtin_amdgcn_readlane(a.x, 63) > x;
    }
    // the request with unit x: its number, entry, length, and the next one's entry
    __device__ __forceinline__ int get(int32_t x, int4 &own, int &len, int4 &next) const {
        const int lane = threadIdx.x & 63;
        const int hits = __popcll(__ballot(from + lane < n && a.x <= x));
        const int i = __builtin_amdgcn_readfirstlane(hits < 1 ? 0 : hits - 1);
        const auto at = [&](int v, int k) { return __builtin_amdgcn_readlane(v, k); };
        own = make_int4(at(a.x, i), at(a.y, i), at(a.z, i), at(a.w, i));
        len = at(length, i);
        next = from + i + 1 < n ? make_int4(at(a.x, i + 1), 0, at(a.z, i + 1), 0) : total;
        return from + i;
    }
};

// Little work: a workgroup per piece, each of one request's rows alone, so that
// nobody goes through two of them one after the other.
struct Piece {
    int32_t first, last;    // units of the work
    int owner, pieces;      // the workgroup with the rows' first piece, and their pieces
    int request;
};

// A request's rows in tiles of 16, and the units of each, from the entries of
// the request and the next one.
__device__ __forceinline__ void tiles_of(const AttendArgs &p, int few, int start, int few_next, int start_next, int &tiles,
                                         int &units) {
    const int all = few_next - few, rows = (start_next - start) * p.group;
    tiles = all > 0 ? (rows + kRowTile - 1) / kRowTile : 0;
    units = tiles > 0 ? all / tiles : 0;
}

// Piece `in` of request i's: tiles of `units` units, cut into `pieces` each.
__device__ __forceinline__ Piece piece_at(const AttendArgs &p, int i, int few, int units, int pieces, int in, int block) {
    const int row = in / pieces, part = in - row * pieces;
    const int32_t from = few * p.heads + row * units;
    return Piece{from + units * part / pieces, from + units * (part + 1) / pieces, block - part, pieces, i};
}

// The piece of workgroup `block` (last = first: none) where rows of `units`
// units are cut into ceil(units / share) even pieces; false if that takes more
// than `groups` workgroups.  For up to 64 requests, a lane each.
__device__ __forceinline__ bool piece_of(const AttendArgs &p, const Works &works, int share, int groups, int block, Piece *o) {
    const int lane = threadIdx.x & 63;
    const int few_next = __shfl_down(works.a.x, 1, 64), start_next = __shfl_down(works.a.z, 1, 64);
    const bool end = lane + 1 >= works.n;
    int tiles, units;
    tiles_of(p, works.a.x, works.a.z, end ? works.total.x : few_next, end ? works.total.z : start_next, tiles, units);
    if (lane >= works.n) tiles = 0;
    const int pieces = (units + share - 1) / share, mine = tiles * pieces * p.heads;
    int to = mine;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int x = __shfl_up(to, s, 64);
        if (lane >= s) to += x;
    }
    if (__builtin_amdgcn_readlane(to, 63) > groups) return false;
    const int i = __popcll(__ballot(to <= block));
    if (i >= works.n) {
        *o = Piece{0, 0, 0, 1, 0};
        return true;
    }
    const auto at = [&](int v) { return __builtin_amdgcn_readlane(v, i); };
    *o = piece_at(p, i, at(works.a.x), at(units), at(pieces), block - (at(to) - at(mine)), block);
    return true;
}

// The same for up to kEvenRequests requests, by the whole workgroup.
constexpr int kEvenPer = 4;
constexpr int kEvenRequests = 64 * kFewWaves * kEvenPer;
struct EvenLds {
    int sums[kFewWaves];
    Piece piece;
};
__device__ __forceinline__ bool piece_of(const AttendArgs &p, const Works &works, int share, int groups, int block, EvenLds &lds,
                                         Piece *o) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i0 = threadIdx.x * kEvenPer;
    int4 w[kEvenPer + 1];
#pragma unroll
    for (int j = 0; j <= kEvenPer; ++j) w[j] = *reinterpret_cast<const int4 *>(works.w + (i0 + j < works.n ? i0 + j : works.n));
    int tiles[kEvenPer], units[kEvenPer];
#pragma unroll
    for (int j = 0; j < kEvenPer; ++j) tiles_of(p, w[j].x, w[j].z, w[j + 1].x, w[j + 1].z, tiles[j], units[j]);
    for (int attempt = 0; attempt < 2; ++attempt, share += 2) {
        int mine = 0, at[kEvenPer];
#pragma unroll
        for (int j = 0; j < kEvenPer; ++j) {
            at[j] = mine;
            mine += tiles[j] * ((units[j] + share - 1) / share) * p.heads;
        }
        int to = mine;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const int x = __shfl_up(to, s, 64);
            if (lane >= s) to += x;
        }
        if (lane == 63) lds.sums[wave] = to;
        __syncthreads();
        int before = to - mine, all = 0;
#pragma unroll
        for (int z = 0; z < kFewWaves; ++z) {
            if (z < wave) before += lds.sums[z];
            all += lds.sums[z];
        }
        if (all <= groups) {
            if (block >= all) {
                if (threadIdx.x == 0) lds.piece = Piece{0, 0, 0, 1, 0};
            } else if (before <= block && block < before + mine) {
                int j = 0;
#pragma unroll
                for (int z = 1; z < kEvenPer; ++z)
                    if (before + at[z] <= block) j = z;
#pragma unroll
                for (int z = 0; z < kEvenPer; ++z)
                    if (z == j)
                        lds.piece = piece_at(p, i0 + z, w[z].x, units[z], (units[z] + share - 1) / share,
                                             block - before - at[z], block);
            }
        }
        __syncthreads();
        if (all <= groups) {
            *o = lds.piece;
            return true;
        }
    }
    return false;
}

// The rows that unit x of the work belongs to, and its place among their units.
struct Segment {
    int request, head, row, first, rows, units, at, granted, length;
};
__device__ __forceinline__ Segment segment_of(const AttendArgs &p, Works &works, int32_t x) {
    Segment s;
    int4 own, next;
    if (!works.has(x / p.heads)) works.look(x / p.heads);
    s.request = works.get(x / p.heads, own, s.length, next);
    const int32_t base = own.x, all = next.x - base;
    s.first = own.z, s.granted = own.w;
    const int rows = (next.z - own.z) * p.group;
    const int tiles = (rows + kRowTile - 1) / kRowTile;
    if (all <= 0 || tiles <= 0 || all < tiles) {
        s.units = 0;
        return s;
    }
    s.units = all / tiles;
    const int32_t rest = x - base * p.heads;
    s.head = rest / all;
    const int32_t in = rest - s.head * all, tile = in / s.units;
    s.row = tile * kRowTile;
    s.rows = rows - s.row < kRowTile ? rows - s.row : kRowTile;
    s.at = in - tile * s.units;
    return s;
}

// Pieces cross between workgroups, which may sit on XCDs with caches of their
// own.  They are written and read past those caches word by word (relaxed
// atomics of the whole GPU's scope), and a workgroup's arrival is counted once
// its words are acknowledged: a fence would write back and drop the whole L2
// every time (measured: 64 tokens over 100..8,192 tokens 166 us with fences).
__device__ __forceinline__ void put(float *p, float x) {
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float get(const float *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put2(float *p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float *p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Counts this workgroup's arrival at a join of `parties`; true in the last one,
// which also sets the counter back for the next layer's call.
__device__ __forceinline__ bool last_to_arrive(int32_t *counter, int parties, int *s_last) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup"); // (no word is moved past the wait)
    __builtin_amdgcn_s_waitcnt(0x0f70);                    // this wavefront's words are out: vmcnt(0)
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parties - 1;
        if (last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *s_last = last;
    }
    __syncthreads();
    return *s_last != 0;
}

}  // namespace agft_kv_detail

#endif
