// agft_diff.hip -- differential attention over a serving node's 8-bit paged cache.
// agft_diff.h states the rules, agft_kv.h the cache's.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "agft_diff.h"
#include "agft_kv_attend.h"

namespace agft_diff_detail {

using namespace agft_kv_detail;

// (heads: the pairs, which the work is cut by)
struct DiffArgs : AttendArgs {
    const float *lambda, *weight;
    int64_t lambda_token, lambda_head;
    float eps, gain;
};

constexpr int kManyPieces = 32;            // more are joined in groups first
constexpr int kRaise = 15;

// Two halves of a value row meet the same probabilities, and each page has a scale
// for either.  The larger one, 2^e, goes into the probabilities' exponent as the
// one scale of agft_kv_attend does; a half's codes come to fp16 times 2^(ev - e +
// lift), lift being what fp16's range leaves above the largest code.  They are whole
// there while their smallest step (2^-9; 1) comes to fp16's, 2^-24, or more.
template <int FORM>
constexpr int lift() {
    return FORM == AGFT_KV_E4M3 ? 7 : 5;   // 448 * 2^7; 1152 * 2^5 (the integers' offset below)
}

// Eight codes, the first four times 2^a and the others times 2^b, as fp16.
template <int FORM>
__device__ __forceinline__ fp16x8 decode_scaled(uint32_t lo, uint32_t hi, float a, float b) {
    uint32_t w[4];
    if constexpr (FORM == AGFT_KV_E4M3) {
        w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, a, false));
        w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, a, true));
        w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, b, false));
        w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, b, true));
    } else {
        // c + 128 as the low byte of 1024 + (c + 128), less 1152, in one fused step with the scale
        lo ^= 0x80808080u, hi ^= 0x80808080u;
        w[0] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u);
        w[1] = __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u);
        w[2] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u);
        w[3] = __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u);
        const fp16x2 f[2] = {{(_Float16)a, (_Float16)a}, {(_Float16)b, (_Float16)b}};
        const fp16x2 base = {(_Float16)-1152.0f, (_Float16)-1152.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(fp16x2, w[j]), f[j >> 1],
                                                                          base * f[j >> 1]));
    }
    return __builtin_bit_cast(fp16x8, (uint4v){w[0], w[1], w[2], w[3]});
}

// 2^(ev - e + lift), e the larger of a page's two value exponents
template <int FORM>
__device__ __forceinline__ float value_scale(int ev, int e) {
    const int k = ev - e + lift<FORM>();
    return pow2(k < -126 ? -126 : k);
}

// gain weight / sqrt(mean(y^2) + eps) without the weight, of a row of WIDE numbers
template <int WIDE>
__device__ __forceinline__ float row_factor(const DiffArgs &p, float squares) {
    return p.weight == nullptr ? p.gain : p.gain / sqrtf(squares * (1.0f / WIDE) + p.eps);
}
__device__ __forceinline__ float4v weight_at(const DiffArgs &p, int d) {
    return p.weight == nullptr ? (float4v){1, 1, 1, 1} : *reinterpret_cast<const float4v *>(p.weight + d);
}
__device__ __forceinline__ float square4(float4v y) { return (y[0] * y[0] + y[1] * y[1]) + (y[2] * y[2] + y[3] * y[3]); }

// a f - b, the product rounded as the other map's was: equal maps leave zero
__device__ __forceinline__ float4v less(float4v a, float f, float4v b) {
#pragma clang fp contract(off)
    a *= f;
    return a - b;
}

template <int TYPE>
__device__ __forceinline__ void store4(const DiffArgs &p, int first, int pair, int r, int d, float4v o) {
    const int t = first + r / p.group, h = pair * p.group + r % p.group;
    uint2 *dst = reinterpret_cast<uint2 *>(p.out + (t * p.out_token + h * p.out_head + d) * 2);
    *dst = Half<TYPE>::pack4(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ void store_lse(const DiffArgs &p, int first, int pair, int map, int r, float m, float l) {
    if (p.lse == nullptr) return;
    const int t = first + r / p.group, hq = (2 * pair + map) * p.group + r % p.group;
    // (no keys: m is -infinity and l 0; scores that are all NaN leave m there too, and l tells them)
    p.lse[(int64_t)t * p.heads * 2 * p.group + hq] = (m + __log2f(l)) * kLn2;
}

__device__ __forceinline__ float lambda_of(const DiffArgs &p, int first, int pair, int r) {
    return p.lambda[(first + r / p.group) * p.lambda_token + (pair * p.group + r % p.group) * p.lambda_head];
}

// Rows that no map has keys for: x in out, `lse` in d_lse.
template <int TYPE, int WIDE, int THREADS>
__device__ __forceinline__ void fill_rows(const DiffArgs &p, int first, int pair, int row0, int rows, float x, float lse) {
    for (int c = threadIdx.x; c < rows * (WIDE / 4); c += THREADS) {
        const int r = c / (WIDE / 4), d = c % (WIDE / 4) * 4;
        store4<TYPE>(p, first, pair, row0 + r, d, (float4v){x, x, x, x});
        if (d == 0) store_lse(p, first, pair, 0, row0 + r, lse, 1.0f), store_lse(p, first, pair, 1, row0 + r, lse, 1.0f);
    }
}

// ---- few query rows ----
//
// The work is cut as agft_kv_attend cuts it, a pair of heads in the place of a head:
// units of 64 tokens of one request, for one pair's 16 query rows (tokens x group).
// Of a workgroup's four wavefronts two take the first map and two the second, each
// half of the tokens: a wavefront reads its own map's keys and both heads' values,
// which the other map's wavefront beside it reads at the same time (from the L1).
// Every wavefront keeps its map's maximum, sum and 16 rows of 2 dim sums; the two
// of a map join in LDS, pieces of several workgroups through memory, and the
// difference and its norm are made once, where everything has met.
//
// What follows the loop over the tokens runs once a segment, over the rows that
// there are, a thread for four numbers of a row of both maps: short code, since
// code that has not run lately comes from memory as data does.
//
// What bounds it: memory for long contexts (24 tokens over 60,000 to 131,071 tokens, 8
// heads of 128 numbers, 4.45 GB: 782 us, 5.7 TB/s), and below a chain of loads
// (requests, page, codes) and of meetings (LDS, the pieces' way through memory): one
// token over 778 tokens 12.9 us, 3 until the first codes are asked for, 4 in the loop,
// 5 from there.  More on its way does not help: a third workgroup of 128 numbers
// on a compute unit (queries in LDS, 17 registers spilled) 849 us for the long contexts,
// two steps' codes ahead (30 spilled) 813, both maps in each wavefront, a value decoded
// once, 816 (and one token 24).

// Workgroups that share the work: what the registers let run at once.
template <int DIM>
constexpr int few_groups() {
    return DIM == 64 ? 768 : 512;
}

// A workgroup takes at least few_share units (64 numbers, 4 / 6: 200 requests of 16 to
// 32 rows over up to 3,000 tokens 31.0 / 26.9 us; 128 numbers, 2 / 4 / 6: one token over
// 778 tokens 12.4 / 12.9 / 13.8, 8 tokens over 500 to 4,000 24.2 / 18.2 / 18.9).  While its
// share is at most kFewEven, rows are cut evenly if that takes no more workgroups; beyond,
// up to 64 requests are cut by what their segments cost, kSegment units beside their own
// (64 tokens over 100 to 8,192 tokens, 128 numbers: 63 us; by the units alone 77; in even
// pieces, twice as many as run at once, 72).
template <int DIM>
constexpr int few_share() {
    return DIM == 64 ? 6 : 4;
}
constexpr int kFewEven = 8;
constexpr int kSegment = 2;

template <int DIM>
struct FewLds {
    static constexpr int C = DIM / 8;              // blocks of 16 numbers of a value row
    static constexpr int ROW = 2 * DIM + 4;        // off the banks
    // the second half's sums of a map, as the lanes hold them; then the map's, by rows
    union {
        float4v half[2][C * 64];
        float rows[2][kRowTile * ROW];
    };
    float m[2][2][kRowTile], l[2][2][kRowTile], lambda[kRowTile];   // [map][half]
    EvenLds even;
    int last;
};

// A piece: both maps' sums by rows, their maxima, their sums of probabilities.
template <int DIM>
constexpr int piece_floats() {
    return 2 * kRowTile * (2 * DIM + 2);
}

// Four numbers of a row of either map, with the row's maxima and sums of probabilities.
struct Both {
    float4v o[2];
    float m[2], l[2];
};

// The row's results from both maps' sums: all threads of a row, which lie side by side.
template <int FORM, int TYPE, int DIM>
__device__ __forceinline__ void finish(const DiffArgs &p, const Segment &seg, int r, int d, const Both &b, float lambda,
                                       float4v weight) {
    constexpr float unit = 1.0f / (1 << kRaise) / (1 << lift<FORM>());
    float f[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) f[a] = b.l[a] > 0.0f || b.l[a] != b.l[a] ? unit / b.l[a] : 0.0f;
    float4v y = less(b.o[0], f[0], b.o[1] * (f[1] * lambda));
    float squares = square4(y);
#pragma unroll
    for (int s = 1; s < DIM / 2; s *= 2) squares += __shfl_xor(squares, s, 64);
    const int row = seg.row + r;
    store4<TYPE>(p, seg.first, seg.head, row, d, y * row_factor<2 * DIM>(p, squares) * weight);
    if (d == 0) {
#pragma unroll
        for (int a = 0; a < 2; ++a) store_lse(p, seg.first, seg.head, a, row, b.m[a], b.l[a]);
    }
}

template <int DIM>
__device__ __forceinline__ void put_piece(float *to, int r, int d, const Both &b) {
    constexpr int WIDE = 2 * DIM, MAP = kRowTile * WIDE;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        put2(to + a * MAP + r * WIDE + d, b.o[a][0], b.o[a][1]);
        put2(to + a * MAP + r * WIDE + d + 2, b.o[a][2], b.o[a][3]);
        if (d == 0) put(to + 2 * MAP + a * kRowTile + r, b.m[a]), put(to + 2 * MAP + (2 + a) * kRowTile + r, b.l[a]);
    }
}

// Joins the pieces of the same 16 rows.  into: where the joined piece goes, or NULL:
// it is the rows' result.  (into is the first of them; a row is one wavefront's.)
template <int FORM, int TYPE, int DIM, typename F>
__device__ __forceinline__ void join_pieces(const DiffArgs &p, F piece, int pieces, float *into, const Segment &seg,
                                            const float *lambda, float4v weight) {
    constexpr int WIDE = 2 * DIM, MAP = kRowTile * WIDE;
    constexpr int AHEAD = 4;                   // pieces on their way at once, maxima and all
    for (int c = threadIdx.x; c < seg.rows * (WIDE / 4); c += 64 * kFewWaves) {
        const int r = c / (WIDE / 4), d = c % (WIDE / 4) * 4;
        Both b;
#pragma unroll
        for (int a = 0; a < 2; ++a) b.m[a] = -INFINITY, b.l[a] = 0.0f, b.o[a] = (float4v){0, 0, 0, 0};
#pragma unroll 1
        for (int w0 = 0; w0 < pieces; w0 += AHEAD) {
            float m[AHEAD][2], l[AHEAD][2];
            float2 x[AHEAD][2], y[AHEAD][2];
#pragma unroll
            for (int z = 0; z < AHEAD; ++z) {
                const float *src = piece(w0 + z < pieces ? w0 + z : w0);
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    m[z][a] = get(src + 2 * MAP + a * kRowTile + r), l[z][a] = get(src + 2 * MAP + (2 + a) * kRowTile + r);
                    x[z][a] = get2(src + a * MAP + r * WIDE + d), y[z][a] = get2(src + a * MAP + r * WIDE + d + 2);
                }
            }
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                float top = b.m[a];
#pragma unroll
                for (int z = 0; z < AHEAD; ++z) top = fmaxf(top, m[z][a]);
                const float fall = b.m[a] == -INFINITY ? 0.0f : exp2f(b.m[a] - top);
                b.m[a] = top, b.l[a] *= fall, b.o[a] *= fall;
#pragma unroll
                for (int z = 0; z < AHEAD; ++z)
                    if (w0 + z < pieces) {
                        const float f = m[z][a] == -INFINITY ? 0.0f : exp2f(m[z][a] - top);
                        b.l[a] = fmaf(l[z][a], f, b.l[a]);
                        b.o[a] += (float4v){x[z][a].x, x[z][a].y, y[z][a].x, y[z][a].y} * f;
                    }
            }
        }
        if (into == nullptr) finish<FORM, TYPE, DIM>(p, seg, r, d, b, lambda[r], weight);
        else put_piece<DIM>(into, r, d, b);
    }
}

// Where a segment costs more than its units, the work is cut by that: a lane per
// request, up to 64 of them.
struct Costs {
    int32_t tiles, units, to;   // of the lane's request: tiles of rows, units of each; the costs up to its end
    int32_t all;
};
__device__ __forceinline__ Costs costs_of(const DiffArgs &p, const Works &works) {
    const int lane = threadIdx.x & 63;
    const int few_next = __shfl_down(works.a.x, 1, 64), start_next = __shfl_down(works.a.z, 1, 64);
    const bool end = lane + 1 >= works.n;
    Costs c;
    tiles_of(p, works.a.x, works.a.z, end ? works.total.x : few_next, end ? works.total.z : start_next, c.tiles, c.units);
    if (lane >= works.n) c.tiles = 0;
    c.to = c.tiles * (c.units + kSegment) * p.heads;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int x = __shfl_up(c.to, s, 64);
        if (lane >= s) c.to += x;
    }
    c.all = __builtin_amdgcn_readlane(c.to, 63);
    return c;
}

// The segment at place x of the costs; at: its unit there, or less than 0: so far ahead of its first.
__device__ __forceinline__ Segment segment_at(const DiffArgs &p, const Works &works, const Costs &c, int32_t x) {
    const auto at = [&](int v, int k) { return __builtin_amdgcn_readlane(v, k); };
    Segment s;
    const int i = __popcll(__ballot(c.to <= x));
    if (i >= works.n) {
        s.units = 0, s.at = 0;
        return s;
    }
    const int tiles = at(c.tiles, i), one = at(c.units, i) + kSegment, rest = x - (at(c.to, i) - tiles * one * p.heads);
    const int number = rest / one, tile = number % tiles;
    const int start_next = i + 1 < works.n ? at(works.a.z, i + 1 < 64 ? i + 1 : 63) : works.total.z;
    s.request = i, s.head = number / tiles, s.row = tile * kRowTile, s.units = one - kSegment, s.at = rest - number * one - kSegment;
    s.first = at(works.a.z, i), s.granted = at(works.a.w, i), s.length = at(works.length, i);
    const int rows = (start_next - s.first) * p.group - s.row;
    s.rows = rows < kRowTile ? rows : kRowTile;
    return s;
}

// Rows of tiles that no launch makes, because a request brings more tokens than
// the caller's bound: NaN, not what the memory held.
template <int TYPE, int WIDE>
__device__ __forceinline__ void leave_nan(const DiffArgs &p, int items) {
    const int64_t all = (int64_t)items * p.heads;
    for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
        const Item item = p.items[x / p.heads];
        if (item.part > 0) continue;
        const int pair = (int)(x % p.heads), first = p.works[item.request].start, row0 = item.tile * kTileRows;
        int rows = (p.works[item.request + 1].start - first) * p.group - row0;
        if (rows > kTileRows) rows = kTileRows;
        fill_rows<TYPE, WIDE, 64 * kFewWaves>(p, first, pair, row0, rows, NAN, NAN);
    }
}

template <int FORM, int TYPE, int DIM>
__device__ __forceinline__ void attend_few(const DiffArgs &p, FewLds<DIM> &lds, int block) {
    constexpr int DG = DIM / kBlockDims, C = FewLds<DIM>::C;
    constexpr int BLK = 2;                        // blocks of 16 tokens at a time
    // Outputs of eleven bits: the probabilities' rounding, of a difference, is no less than
    // theirs, so what is left of each goes through the second product as well.
    constexpr bool FINE = TYPE == AGFT_KV_FP16;
    using H = Half<TYPE>;
    using F = Half<AGFT_KV_FP16>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15, part = wave & 1, map = wave >> 1;
    Works works(p.works, p.requests);
    if (__builtin_expect(p.alone && works.total.y > 0, 0)) leave_nan<TYPE, 2 * DIM>(p, works.total.y);
    const int32_t work = works.total.x * p.heads;
    int32_t share = (work + few_groups<DIM>() - 1) / few_groups<DIM>();
    if (share < few_share<DIM>()) share = few_share<DIM>();
    int64_t x_first = (int64_t)block * share;
    int32_t x1 = x_first + share < work ? (int32_t)x_first + share : work;
    Piece cut;
    Costs costs;
    bool even = false, by_cost = false;
    if (share <= kFewEven) {
        if (works.n <= 64)
            even = piece_of(p, works, share, few_groups<DIM>(), block, &cut) ||
                   piece_of(p, works, share + 2, few_groups<DIM>(), block, &cut);
        else if (works.n <= kEvenRequests)
            even = piece_of(p, works, share, few_groups<DIM>(), block, lds.even, &cut);
    }
    if (even) {
        x_first = cut.first, x1 = cut.last;
    } else if (works.n <= 64 && work < 1 << 28) {
        by_cost = true;
        costs = costs_of(p, works);
        share = (costs.all + few_groups<DIM>() - 1) / few_groups<DIM>();
        x_first = (int64_t)block * share;
        x1 = x_first + share < costs.all ? (int32_t)x_first + share : costs.all;
    }
    if (x_first >= x1) return;
    const int64_t side = (int64_t)p.page * DIM, page_bytes = (int64_t)p.heads * 4 * side;
    const float scale2 = p.scale * kLog2e;
    int32_t x = (int32_t)x_first;
    if (even) works.look_at(cut.request);
    else if (!by_cost) works.look(x / p.heads);
    while (x < x1) {
        Segment seg;
        if (by_cost) {
            seg = segment_at(p, works, costs, x);
            if (seg.at < 0) {
                x -= seg.at;
                seg.at = 0;
                if (x >= x1) break;
            }
        } else {
            seg = segment_of(p, works, x);
        }
        if (seg.units <= 0) break;
        const int i = seg.request, pair = seg.head, units = seg.units, u0 = seg.at, row0 = seg.row, rows = seg.rows;
        const int first = seg.first;
        const int count = units - u0 < x1 - x ? units - u0 : x1 - x;
        x += count;
        const int granted = seg.granted, len = seg.length;
        if (granted <= 0) {
            // no slots, no keys
            fill_rows<TYPE, 2 * DIM, 64 * kFewWaves>(p, first, pair, row0, rows, 0.0f, -INFINITY);
            continue;
        }
        // right operand of the scores: row n's numbers 64 dg + 16 g + 8 e.. + 7
        typename H::x8 q[DG * 2];
        const bool row_here = n < rows;
        const float lambda = lambda_of(p, first, pair, row_here ? row0 + n : row0);
        {
            const int tk = (row0 + n) / p.group, hq = (2 * pair + map) * p.group + (row0 + n) % p.group;
            const char *src = p.q + ((int64_t)(first + tk) * p.q_token + hq * p.q_head) * 2;
#pragma unroll
            for (int c = 0; c < DG * 2; ++c) {
                uint4v v = {0, 0, 0, 0};
                if (row_here) v = *reinterpret_cast<const uint4v *>(src + ((c >> 1) * kBlockDims + 16 * g + 8 * (c & 1)) * 2);
                q[c] = __builtin_bit_cast(typename H::x8, v);
            }
        }
        int limit = row_here ? len - granted + (row0 + n) / p.group + 1 : len;   // keys that row n sees
        int least = len - granted + row0 / p.group + 1;                          // keys that every row sees
        const int blocks = (len + kBlockTokens - 1) / kBlockTokens;
        const char *codes = p.codes + (int64_t)pair * 4 * side;
        const int sub_mask = (p.page >> 4) - 1;

        float m = -INFINITY, l = 0.0f;
        float4v o[C];
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = (float4v){0, 0, 0, 0};

        // this wavefront's blocks of the segment: a half, two of each unit
        static_assert(kUnit == 4 * kBlockTokens, "a unit gives either half two blocks");
        const int b_first = u0 * 4 + 2 * count * part;
        const int b_last = b_first + 2 * count < blocks ? b_first + 2 * count : blocks;
        limit = limit < b_last * kBlockTokens ? limit : b_last * kBlockTokens;
        least = least < b_last * kBlockTokens ? least : b_last * kBlockTokens;
        for (int b0 = b_first; b0 < b_last; b0 += 64) {
            // a lane per block: its page, this map's keys' exponent, the values' larger one and
            // what either head's codes are taken by
            int id, exps;
            {
                int b = b0 + lane;
                if (b >= blocks) b = blocks - 1;
                uint32_t z = (uint32_t)p.table[(int64_t)i * p.row_pages + ((b << 4) >> p.shift)];
                if (z >= (uint32_t)p.pages) z = (uint32_t)p.pages - 1;
                id = (int)z;
                const int4 e = *reinterpret_cast<const int4 *>(p.exps + ((int64_t)id * p.heads + pair) * 4);
                // (exponents lie in -127..127)
                exps = ((map == 0 ? e.x : e.z) & 255) | (e.y & 255) << 8 | (e.w & 255) << 16;
            }
            const int b1 = b0 + 64 < b_last ? b0 + 64 : b_last;
            const auto block_at = [&](int b) {
                const int bb = b >= b_last ? b_last - 1 : b;
                return codes + (int64_t)__builtin_amdgcn_readlane(id, bb - b0) * page_bytes + (bb & sub_mask) * (16 * DIM) + lane * 16;
            };
            const auto fetch_keys = [&](int b, uint4v (*dst)[DG]) {
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    const char *src = block_at(b + s) + map * 2 * side;
#pragma unroll
                    for (int dg = 0; dg < DG; ++dg) dst[s][dg] = *reinterpret_cast<const uint4v *>(src + dg * kBlockBytes);
                }
            };
            const auto fetch_values = [&](int b, uint4v (*dst)[2 * DG]) {
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    const char *src = block_at(b + s) + side;
#pragma unroll
                    for (int dg = 0; dg < 2 * DG; ++dg)
                        dst[s][dg] = *reinterpret_cast<const uint4v *>(src + (dg / DG) * 2 * side + (dg % DG) * kBlockBytes);
                }
            };
            // codes are asked for as soon as their registers are free: the next
            // keys after the scores, the next values after the sums
            uint4v kc[BLK][DG], vc[BLK][2 * DG];
            fetch_keys(b0, kc);
            fetch_values(b0, vc);
            for (int b = b0; b < b1; b += BLK) {
                float4v t[BLK];
                float back[BLK], by[BLK][2];
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    float4v acc = {0, 0, 0, 0};
#pragma unroll
                    for (int dg = 0; dg < DG; ++dg) {
                        acc = H::mfma(H::template decode<FORM>(kc[s][dg][0], kc[s][dg][1]), q[2 * dg], acc);
                        acc = H::mfma(H::template decode<FORM>(kc[s][dg][2], kc[s][dg][3]), q[2 * dg + 1], acc);
                    }
                    int bb = b + s;
                    if (bb >= b_last) bb = b_last - 1;
                    const int e = __builtin_amdgcn_readlane(exps, bb - b0);
                    const int bek = (int8_t)e, ev0 = (int8_t)(e >> 8), ev1 = (int8_t)(e >> 16), bev = ev0 > ev1 ? ev0 : ev1;
                    by[s][0] = value_scale<FORM>(ev0, bev), by[s][1] = value_scale<FORM>(ev1, bev);
                    const float ks = scale2 * pow2(bek);
                    back[s] = pow2(-bev);
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[s][j] = fmaf(acc[j], ks, (float)bev);
                }
                if (b + BLK < b1) fetch_keys(b + BLK, kc);
                if ((b + BLK) * kBlockTokens > least) {
#pragma unroll
                    for (int s = 0; s < BLK; ++s) {
                        const int key = (b + s) * kBlockTokens + 4 * g;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (key + j >= limit) t[s][j] = -INFINITY;
                        // codes past the request's tokens may be anything, NaN too
                        const int valid = len - key;
                        const uint32_t keep = valid >= 4 ? ~0u : valid <= 0 ? 0u : (1u << (8 * valid)) - 1u;
#pragma unroll
                        for (int dg = 0; dg < 2 * DG; ++dg) vc[s][dg] &= keep;
                    }
                }
                float top = t[0][0];
#pragma unroll
                for (int s = 0; s < BLK; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, t[s][j]);
                top = across_max(top);
                if (__any(top > m)) {
                    const float m1 = fmaxf(m, top);
                    float fall = m == -INFINITY ? 0.0f : exp2f(m - m1);
                    m = m1;
                    asm volatile("" : "+v"(fall));
                    l *= fall;
#pragma unroll
                    for (int c = 0; c < C; ++c) o[c] *= fall;
                }
                const float off = m == -INFINITY ? 0.0f : m;
                fp16x8 pr, rest;
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    float4v e;
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(t[s][j] - off);
                    l = fmaf((e[0] + e[1]) + (e[2] + e[3]), back[s], l);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x = e[j] * pow2(kRaise);
                        pr[4 * s + j] = (_Float16)x;
                        if constexpr (FINE) rest[4 * s + j] = (_Float16)(x - (float)pr[4 * s + j]);
                    }
                }
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const fp16x8 w = decode_scaled<FORM>(vc[0][c >> 2][c & 3], vc[1][c >> 2][c & 3], by[0][c / (C / 2)],
                                                         by[1][c / (C / 2)]);
                    o[c] = F::mfma(w, pr, o[c]);
                    if constexpr (FINE) o[c] = F::mfma(w, rest, o[c]);
                }
                if (b + BLK < b1) fetch_values(b + BLK, vc);
            }
        }
        // (a thread's four numbers of a row are the same of every row)
        const float4v weight = weight_at(p, (int)threadIdx.x % (DIM / 2) * 4);
        // the two wavefronts of a map meet, and leave its sums by rows
        l = across_sum(l);
        if (g == 0) lds.m[map][part][n] = m, lds.l[map][part][n] = l;
        if (part == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c) lds.half[map][c * 64 + lane] = o[c];
        }
        if (wave == 0 && g == 0) lds.lambda[n] = lambda;
        __syncthreads();
        if (part == 0) {
            const float m1 = lds.m[map][1][n], both = fmaxf(m, m1);
            const float f0 = m == -INFINITY ? 0.0f : exp2f(m - both), f1 = m1 == -INFINITY ? 0.0f : exp2f(m1 - both);
#pragma unroll
            for (int c = 0; c < C; ++c) o[c] = o[c] * f0 + lds.half[map][c * 64 + lane] * f1;
            if (g == 0) lds.l[map][0][n] = fmaf(l, f0, lds.l[map][1][n] * f1), lds.m[map][0][n] = both;
        }
        __syncthreads();
        if (part == 0 && row_here) {
#pragma unroll
            for (int c = 0; c < C; ++c) *reinterpret_cast<float4v *>(&lds.rows[map][n * FewLds<DIM>::ROW + 16 * c + 4 * g]) = o[c];
        }
        __syncthreads();
        const bool whole = count == units;
        float *to = p.partial + ((int64_t)block * 2 + (u0 == 0 ? 1 : 0)) * piece_floats<DIM>();
        for (int c = threadIdx.x; c < rows * (DIM / 2); c += 64 * kFewWaves) {
            const int r = c / (DIM / 2), d = c % (DIM / 2) * 4;
            Both b;
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                b.m[a] = lds.m[a][0][r], b.l[a] = lds.l[a][0][r];
                b.o[a] = *reinterpret_cast<const float4v *>(&lds.rows[a][r * FewLds<DIM>::ROW + d]);
            }
            if (whole) finish<FORM, TYPE, DIM>(p, seg, r, d, b, lds.lambda[r], weight);
            else put_piece<DIM>(to, r, d, b);
        }
        if (!whole) {
            const int32_t from = x - count - u0;                       // the place of the rows' first unit
            const int owner = even ? cut.owner : from / share;
            const int pieces = even ? cut.pieces : (from + units - 1) / share - owner + 1;
            // groups of kManyPieces first, each into its first piece's place
            const int mine = block - owner, group0 = mine / kManyPieces * kManyPieces;
            const int members = pieces - group0 < kManyPieces ? pieces - group0 : kManyPieces;
            const int groups = (pieces + kManyPieces - 1) / kManyPieces;
            // the first piece of the rows is its workgroup's second one
            const auto piece = [&](int w) {
                return p.partial + ((int64_t)(owner + w) * 2 + (w == 0 ? 1 : 0)) * piece_floats<DIM>();
            };
            int32_t *counter = p.arrived + kFewGroups + (owner + group0) * 2 + (group0 == 0 ? 1 : 0);
            // (one join in the code: of a group's pieces, then, by the last of all, of the groups')
            int parties = members, step = 1, at = group0;
            float *into = groups == 1 ? nullptr : piece(group0);
            while (last_to_arrive(counter, parties, &lds.last)) {
                join_pieces<FORM, TYPE, DIM>(p, [&](int w) { return piece(at + step * w); }, parties, into, seg, lds.lambda, weight);
                if (into == nullptr) break;
                counter = p.arrived + owner, parties = groups, step = kManyPieces, at = 0, into = nullptr;
            }
        }
        __syncthreads();
    }
}

// The lane, for what follows the loop over the tokens: nothing made from it is kept
// in registers through that loop.
__device__ __forceinline__ int lane_anew() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}

// ---- many query rows ----
//
// A tile of agft_kv_attend's plan, 128 query rows of one request, is one workgroup of
// eight wavefronts (128 numbers) or two of four (64 numbers): half of them take 32 rows'
// first map each and half their second, over the tokens 64 at a time.  The wavefronts
// fetch the tile's codes once between them, a tile ahead, and leave keys and values in
// LDS as 16 bits; each reads its map's keys there and all values.  A step makes the
// scores of the tokens that follow beside the exponentials and sums of those before
// them, 64 tokens at a time, or 32 where the registers hold no more (128 numbers: 32
// rows of 256 sums are 128 registers of 256, and two wavefronts share a SIMD).  The
// second map's sums go to the first's wavefronts through LDS at the end.
//
// The prompt (10,001 tokens, 16 query heads of 128 numbers, two maps each, int8, causal:
// 1.23 TFLOP) takes 1.21 to 1.24 ms by card, 1.0 PFLOP/s, 77 to 79% of what a large matrix
// product of the library reaches, and 1.30 called again and again without a pause (e4m3 1.17
// to 1.20 ms; 64 numbers, 0.61 TFLOP, 0.73 to 0.76 ms, half as many numbers for each
// exponential).  Of the cycles matrix instructions are busy for 45% (64 numbers 36%), vector
// ones for 46% (56%), LDS for 36% (39%), without a bank conflict; what counts is that they
// run beside one another.  What fp16 leaves of a probability is not summed here, as it is
// for few rows: it makes fp16 outputs' error 1.00 times that of 32-bit probabilities for 1.22
// to 1.39, and takes 1.73 ms for 1.20 (64 numbers 1.05 for 0.77), far more than 8-bit codes
// are worth.  Four wavefronts of 128 numbers, one on a
// SIMD, 1.89 ms; eight without the scores ahead 1.47; with three operands on their way and
// 12 registers spilled 1.38; pages and exponents in LDS instead, none spilled, 1.26, and the
// sums at a raised wave priority 1.23.  64 numbers in steps of 32 tokens 0.81 ms (0.74 on
// that card), eight wavefronts on tiles of 128 tokens the same as four on 64.
// A tile over few tokens is what comes before and after the loop: 1,024 tiles of 64
// numbers over 65 tokens 62.5 us, 51 with all that the first steps need asked for
// together and the norm's weights and lambda in LDS, 49 with results stored 16 bytes a
// lane (over 321 tokens 93, 85, 82; the prompt 1.25, 1.23, 1.22).
constexpr int kTileKeys = 64;
template <int DIM>
constexpr int tile_span() {                // tokens of a step, in 32s
    return DIM == 64 ? 2 : 1;
}
template <int DIM>
constexpr int tile_waves() {
    return DIM == 64 ? 4 : 8;
}
// Powers of two that a maximum may grow before the sums are rescaled; the
// exponential itself makes 2^kTileRaise P, as in agft_kv_attend.
constexpr int kSlack = 8;
constexpr int kTileRaise = kRaise - kSlack;

template <int DIM>
struct TileLds {
    static constexpr int HEAD = kTileKeys * DIM * 2;       // a head's keys (or values) of a tile in 16 bits
    // operands of 1 KB, 16 bytes a lane; keys: [head][32 tokens][64 numbers][32][16], values: [16 tokens][32 numbers]
    __attribute__((aligned(16))) char tile[2][2][2 * HEAD];
    float4 scale[2][16];                                   // by map, block % 16: its factor of the scores, e, 2^-e
    int2 look[tile_waves<DIM>()][2][64];                   // pages and exponents of the blocks that a wavefront fetches
    float lambda[16 * tile_waves<DIM>()], weight[2 * DIM];
    int last;
};

template <int FORM, int TYPE, int DIM>
__device__ __forceinline__ void attend_many(const DiffArgs &p, TileLds<DIM> &lds, int block) {
    constexpr int DG = DIM / kBlockDims, WIDE = 2 * DIM, WAVES = tile_waves<DIM>(), BLOCKS = kTileKeys / kBlockTokens;
    constexpr int SPAN = tile_span<DIM>(), SHIFT = 2 * SPAN;                           // of a step; blocks of it
    constexpr int GROUPS = WAVES / 2, ROWS = 32 * GROUPS, SUBS = kTileRows / ROWS;   // of 32 rows; rows; workgroups of a tile
    // heads of a block that a wavefront fetches: both, where there is a wavefront for each block
    constexpr int HEADS = BLOCKS == WAVES ? 2 : 1;
    static_assert(BLOCKS * 2 == WAVES * HEADS, "the wavefronts fetch a tile");
    using H = Half<TYPE>;
    const auto s_tile = lds.tile;
    const auto s_scale = lds.scale;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, n = lane & 31, map = wave / GROUPS, own_rows = wave % GROUPS;
    const int pair = block % p.heads, sub = block / p.heads % SUBS, place = block / p.heads / SUBS;
    const Item item = p.items[place];                      // (the list has room for every workgroup's)
    if (place >= p.works[p.requests].items) return;
    const int i = item.request;
    const int4 own = *reinterpret_cast<const int4 *>(p.works + i);
    const int len = p.works[i].length;
    const int first = own.z, granted = own.w, all_rows = (p.works[i + 1].start - first) * p.group;
    const int row0 = item.tile * kTileRows + sub * ROWS;
    const int rows = all_rows - row0 < ROWS ? all_rows - row0 : ROWS;
    if (rows <= 0) return;
    if (granted <= 0) {
        if (item.part == 0) fill_rows<TYPE, WIDE, 64 * WAVES>(p, first, pair, row0, rows, 0.0f, -INFINITY);
        return;
    }
    const int past = len - granted, at_row = 32 * own_rows;
    const bool busy = at_row < rows, row_here = at_row + n < rows;
    const int row = row_here ? row0 + at_row + n : row0 + rows - 1;
    const int limit = past + row / p.group + 1;            // keys that this lane's row sees
    const int all_tiles = (past + (row0 + rows - 1) / p.group + kTileKeys) / kTileKeys;
    const int begin = (int)((int64_t)all_tiles * item.part / item.parts);   // this part's tiles
    const int tiles = (int)((int64_t)all_tiles * (item.part + 1) / item.parts);
    int whole = (past + row0 / p.group + 1) / kTileKeys;                    // tiles that every row sees whole
    if (whole > tiles) whole = tiles;
    const int blocks = (len + kBlockTokens - 1) / kBlockTokens;

    typename H::x8 q[DG * 4];
    {
        const int tk = row / p.group, hq = (2 * pair + map) * p.group + row % p.group;
        const char *src = p.q + ((int64_t)(first + tk) * p.q_token + hq * p.q_head) * 2;
#pragma unroll
        for (int c = 0; c < DG * 4; ++c)                   // numbers 64 dg + 16 (2 c + h) + 8 e.. + 7
            q[c] = __builtin_bit_cast(typename H::x8, *reinterpret_cast<const uint4v *>(
                       src + ((c >> 2) * kBlockDims + 16 * (2 * ((c >> 1) & 1) + h) + 8 * (c & 1)) * 2));
    }
    const float scale2 = p.scale * kLog2e;
    const int64_t side = (int64_t)p.page * DIM, page_bytes = (int64_t)p.heads * 4 * side;
    // what this wavefront fetches: a block, of one head or both
    const int part = wave & (BLOCKS - 1), head = HEADS == 2 ? 0 : wave / BLOCKS;
    const char *codes = p.codes + ((int64_t)pair * 2 + head) * 2 * side;
    const int sub_mask = (p.page >> 4) - 1;

    // A step makes the scores of the tokens that follow beside the sums of those before
    // them, so its operands are the values of tile t and the keys from a step on.  A lane
    // per tile: page and exponents of this wavefront's blocks.
    struct Look {
        int id, exps;                                      // (exponents of keys and values, a byte each: they lie in -127..127)
    };
    constexpr bool KEPT = SPAN == 2;                       // in registers, where there is room; else in LDS
    int2 kept[2];
    const auto block_of = [&](int t, int side_at) {
        const int b = t * BLOCKS + part + (side_at == 0 ? SHIFT : 0);
        return b < 0 ? 0 : b >= blocks ? blocks - 1 : b;
    };
    const auto page_and_exps = [&](int b) {
        uint32_t z = (uint32_t)p.table[(int64_t)i * p.row_pages + ((b << 4) >> p.shift)];
        if (z >= (uint32_t)p.pages) z = (uint32_t)p.pages - 1;
        const int4 e = *reinterpret_cast<const int4 *>(p.exps + ((int64_t)z * p.heads + pair) * 4);
        return make_int2((int)z, (e.x & 255) | (e.y & 255) << 8 | (e.z & 255) << 16 | e.w << 24);
    };
    const auto look_up = [&](int t0) {
        const int lane = lane_anew();
        const int2 k[2] = {page_and_exps(block_of(t0 + lane, 0)), page_and_exps(block_of(t0 + lane, 1))};
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            if constexpr (KEPT) kept[a] = k[a];
            else lds.look[wave][a][lane] = k[a];
        }
    };
    // (a wavefront reads what it wrote itself)
    const auto look_at = [&](int t, int side_at) {
        if constexpr (KEPT)
            return Look{__builtin_amdgcn_readlane(kept[side_at].x, t & 63), __builtin_amdgcn_readlane(kept[side_at].y, t & 63)};
        const int2 k = lds.look[wave][side_at][t & 63];
        return Look{__builtin_amdgcn_readfirstlane(k.x), __builtin_amdgcn_readfirstlane(k.y)};
    };
    const auto block_at = [&](int t, int side_at, int id) {
        return codes + (int64_t)id * page_bytes + (block_of(t, side_at) & sub_mask) * (16 * DIM) + side_at * side;
    };
    uint4v ahead[2][HEADS][DG];                            // codes of the next step on their way
    const auto fetch = [&](int t, bool first) {
        if ((t & 63) == 0 && !first) look_up(t);
        const char *k = block_at(t, 0, look_at(t, 0).id), *v = block_at(t, 1, look_at(t, 1).id);
        const int at = lane_anew() * 16;
#pragma unroll
        for (int a = 0; a < HEADS; ++a)
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) {
                ahead[0][a][dg] = *reinterpret_cast<const uint4v *>(k + a * 2 * side + dg * kBlockBytes + at);
                ahead[1][a][dg] = *reinterpret_cast<const uint4v *>(v + a * 2 * side + dg * kBlockBytes + at);
            }
    };
    // Entry 16 g + m of the codes to the lanes that take its numbers: token m's
    // numbers 16 g.. as a row of the left operand of the scores, numbers m, 16 + m,
    // .. of tokens 4 g.. as rows of the left operand of the sums.
    // Tile t's keys and what their blocks' scores are taken by; x: the blocks' exponents.
    const auto stage_keys = [&](int t, const uint4v (*keys)[DG], int x) {
        const int buf = t & 1, lane = lane_anew(), g = lane >> 4, m16 = lane & 15;
        const int to_key = head * TileLds<DIM>::HEAD +
                           (((part >> 1) * DG * 4 + (g >> 1) * 2) * 64 + 32 * (g & 1) + 16 * (part & 1) + m16) * 16;
#pragma unroll
        for (int a = 0; a < HEADS; ++a)
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) {
                const uint4v k = keys[a][dg];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *reinterpret_cast<typename H::x8 *>(&s_tile[buf][0][to_key + a * TileLds<DIM>::HEAD + (dg * 4 + e) * 1024]) =
                        H::template decode<FORM>(k[2 * e], k[2 * e + 1]);
            }
        if (lane == 0) {
            const int e0 = (int8_t)(x >> 8), e1 = x >> 24, e = e0 > e1 ? e0 : e1;
#pragma unroll
            for (int a = 0; a < HEADS; ++a)
                s_scale[head + a][(t * BLOCKS + part + SHIFT) & 15] =
                    make_float4(scale2 * pow2(head + a == 0 ? (int8_t)x : (int8_t)(x >> 16)), (float)e, pow2(-e), 0.0f);
        }
    };
    const auto stage = [&](int t) {                        // what fetch(t) brought
        // (read by all lanes: what is made for one lane of them alone need not be there in the others)
        stage_keys(t, ahead[0], look_at(t, 0).exps);
        const int buf = t & 1, lane = lane_anew(), g = lane >> 4, m16 = lane & 15;
        const int to_value = ((part * 2 + head) * DG * 2 * 64 + 32 * (g & 1) + 16 * (g >> 1) + m16) * 16;
        if ((t * BLOCKS + part + 1) * kBlockTokens > len) {
            // codes past the request's tokens may be anything, NaN too
            const int valid = len - (t * kTileKeys + 16 * part + 4 * g);
            const uint32_t keep = valid >= 4 ? ~0u : valid <= 0 ? 0u : (1u << (8 * valid)) - 1u;
#pragma unroll
            for (int a = 0; a < HEADS; ++a)
#pragma unroll
                for (int dg = 0; dg < DG; ++dg) ahead[1][a][dg] &= keep;
        }
        const int ve = look_at(t, 1).exps;
        const int ev0 = (int8_t)(ve >> 8), ev1 = ve >> 24, ev = ev0 > ev1 ? ev0 : ev1;
#pragma unroll
        for (int a = 0; a < HEADS; ++a) {
            const float up = value_scale<FORM>(head + a == 0 ? ev0 : ev1, ev);
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) {
                // words 0, 1 (2, 3) of the entries 16 g + m and 16 (g + 2) + m come
                // together in the lower (upper) half: rows m (16 + m) of two operands
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const auto w = __builtin_amdgcn_permlane32_swap(ahead[1][a][dg][z], ahead[1][a][dg][2 + z], false, false);
                    *reinterpret_cast<fp16x8 *>(&s_tile[buf][1][to_value + ((a * DG + dg) * 2 + z) * 1024]) =
                        decode_scaled<FORM>(w[0], w[1], up, up);
                }
            }
        }
    };

    float m = -INFINITY, l = 0.0f;
    float16v o[DG * 4];
#pragma unroll
    for (int c = 0; c < DG * 4; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = 0.0f;

    constexpr int N = DG * 4;                              // instructions of 32 tokens' scores; their sums are 4 N
    const auto key_at = [&](int buf, int c) {
        return *reinterpret_cast<const uint4v *>(&s_tile[buf][0][map * TileLds<DIM>::HEAD + (c * 64 + lane) * 16]);
    };
    float16v s[SPAN];                                      // scores of the tokens whose turn is next
    // The tokens of a step: number `which` of tile t's.  MASK: some row may not see all of them.
    const auto step = [&](int t, auto which, auto mask) {
        constexpr bool MASK = mask();
        constexpr int AT = which() * SPAN;                 // in 32 tokens of the tile
        const int buf = t & 1;
        // Matrix instructions in the order of their operands in LDS, each of which is read
        // AHEAD instructions before its use: the next scores', then these tokens' sums'.
        constexpr int SCORES = SPAN * N, ALL = 3 * SCORES, AHEAD = SPAN == 2 ? 4 : 2;
        // scores beside the search for the maximum; exponentials beside the others (the rest: beside the sums)
        constexpr int EARLY = SPAN == 2 ? 0 : 3, BESIDE = SPAN == 2 ? 32 : 8;
        const auto operand = [&](int c) {
            return c < SCORES ? key_at(buf, (AT + c % SPAN) * N + c / SPAN)
                              : *reinterpret_cast<const uint4v *>(&s_tile[buf][1][((AT * 2 * N + c - SCORES) * 64 + lane) * 16]);
        };
        uint4v ring[AHEAD];
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) ring[c] = operand(c);
        float16v z[SPAN];
#pragma unroll
        for (int w = 0; w < SPAN; ++w)
#pragma unroll
            for (int j = 0; j < 16; ++j) z[w][j] = 0.0f;
        const auto score = [&](int c) {
            z[c % SPAN] = mfma32<TYPE>(__builtin_bit_cast(typename H::x8, ring[c % AHEAD]), q[c / SPAN], z[c % SPAN]);
            ring[c % AHEAD] = operand(c + AHEAD);
        };
        if constexpr (EARLY > 0) score(0);
        __builtin_amdgcn_sched_barrier(0);
        const float off = m == -INFINITY ? 0.0f : m - (float)kTileRaise;
        float pow_back[2 * SPAN];
#pragma unroll
        for (int b = 0; b < 2 * SPAN; ++b) {
            const float4 f = s_scale[map][(t * BLOCKS + 2 * AT + b) & 15];
            const float ev = f.y - off;
            pow_back[b] = f.z;
#pragma unroll
            for (int j = 8 * (b & 1); j < 8 * (b & 1) + 8; ++j) s[b >> 1][j] = fmaf(s[b >> 1][j], f.x, ev);
        }
        if constexpr (MASK) {
            const int sees = limit - t * kTileKeys - 32 * AT - 4 * (lane_anew() >> 5);
#pragma unroll
            for (int w = 0; w < SPAN; ++w)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (32 * w + 8 * (j >> 2) + (j & 3) >= sees) s[w][j] = -INFINITY;
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EARLY > 1) score(1);
        __builtin_amdgcn_sched_barrier(0);
        float top = s[0][0];
#pragma unroll
        for (int w = 0; w < SPAN; ++w)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[w][j]);
        top = halves_max(top);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EARLY > 2) score(2);
        __builtin_amdgcn_sched_barrier(0);
        // the maximum that the sums are relative to follows the real one at some distance
        // (a row's own: another row that grows, or is NaN and never begins, changes none of its bits)
        const bool grows = top > (float)kRaise || m == -INFINITY;
        if (__builtin_expect(__any(grows), 0)) {
            const float m1 = grows ? (fmaxf(m, off + top) - (float)kTileRaise) + (float)kTileRaise : m;
            float fall = m == -INFINITY ? 0.0f : exp2f(m - m1), shift = m1 == -INFINITY ? 0.0f : off - (m1 - (float)kTileRaise);
            m = m1;
            // (keeps the compiler from multiplying ahead of the branch, which is rarely taken)
            asm volatile("" : "+v"(fall), "+v"(shift));
            l *= fall;
#pragma unroll
            for (int c = 0; c < DG * 4; ++c) o[c] *= fall;
#pragma unroll
            for (int w = 0; w < SPAN; ++w) s[w] += shift;
        }
        fp16x8 pr[2 * SPAN];
        float sum = 0.0f;
        const auto exponential = [&](int x) {
            const float e = __builtin_amdgcn_exp2f(s[x >> 4][x & 15]);
            sum = (x & 7) == 0 ? e : sum + e;
            pr[x >> 3][x & 7] = (_Float16)e;
            if ((x & 7) == 7) l = fmaf(sum, pow_back[x >> 3], l);
        };
#pragma unroll
        for (int c = EARLY; c < SCORES; ++c) {
            score(c);
#pragma unroll
            for (int x = (c - EARLY) * BESIDE / (SCORES - EARLY); x < (c - EARLY + 1) * BESIDE / (SCORES - EARLY); ++x) exponential(x);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (SPAN == 1) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int c = SCORES; c < ALL; ++c) {
            const int b = (c - SCORES) / N, y = (c - SCORES) % N;
            o[y] = mfma32<AGFT_KV_FP16>(__builtin_bit_cast(fp16x8, ring[c % AHEAD]), pr[b], o[y]);
            if (c + AHEAD < ALL) ring[c % AHEAD] = operand(c + AHEAD);
            if (BESIDE < 16 * SPAN && b == 0) {
#pragma unroll
                for (int x = 8 + y * 8 / N; x < 8 + (y + 1) * 8 / N; ++x) exponential(x);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int w = 0; w < SPAN; ++w) s[w] = z[w];
        if constexpr (SPAN == 1) __builtin_amdgcn_s_setprio(0);
    };
    const auto steps = [&](int t, auto mask) {
        step(t, std::integral_constant<int, 0>{}, mask);
        if constexpr (SPAN == 1) step(t, std::integral_constant<int, 1>{}, mask);
    };

    {
        // The keys of the step before the first, the first step's operands, and what follows the
        // loop are asked for together.
        const int b = block_of(begin - 1, 0);
        int2 before = page_and_exps(b);
        before.x = __builtin_amdgcn_readfirstlane(before.x), before.y = __builtin_amdgcn_readfirstlane(before.y);
        look_up(begin & ~63);
        const bool has_lambda = threadIdx.x < ROWS, has_weight = threadIdx.x < WIDE / 4;
        const int row_of = (int)threadIdx.x < rows ? row0 + (int)threadIdx.x : row0 + rows - 1;
        const float lambda = has_lambda ? lambda_of(p, first, pair, row_of) : 0.0f;
        const float4v weight = has_weight ? weight_at(p, 4 * threadIdx.x) : (float4v){0, 0, 0, 0};
        uint4v keys[HEADS][DG];
        const char *k = block_at(begin - 1, 0, before.x) + lane * 16;
#pragma unroll
        for (int a = 0; a < HEADS; ++a)
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) keys[a][dg] = *reinterpret_cast<const uint4v *>(k + a * 2 * side + dg * kBlockBytes);
        fetch(begin, true);
        if (has_lambda) lds.lambda[threadIdx.x] = lambda;
        if (has_weight) *reinterpret_cast<float4v *>(&lds.weight[4 * threadIdx.x]) = weight;
        stage_keys(begin - 1, keys, before.y);
    }
    __syncthreads();
    if (busy) {                                            // the first tokens' scores: keys of the step before
#pragma unroll
        for (int w = 0; w < SPAN; ++w) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[w][j] = 0.0f;
#pragma unroll
            for (int c = 0; c < N; ++c)
                s[w] = mfma32<TYPE>(__builtin_bit_cast(typename H::x8, key_at((begin - 1) & 1, (2 - SPAN + w) * N + c)), q[c], s[w]);
        }
    }
    stage(begin);
    if (!busy)                                             // no rows of its own: only fetches
        for (int t = begin; t < tiles; ++t) {
            __syncthreads();
            if (t + 1 < tiles) fetch(t + 1, false), stage(t + 1);
        }
    int t = busy ? begin : tiles;
    for (; t < whole; ++t) {
        __syncthreads();                                   // this step's operands are in LDS, and the other buffer is read
        if (t + 1 < tiles) fetch(t + 1, false);
        steps(t, std::false_type{});
        if (t + 1 < tiles) stage(t + 1);
    }
    for (; t < tiles; ++t) {
        __syncthreads();
        if (t + 1 < tiles) fetch(t + 1, false);
        steps(t, std::true_type{});
        if (t + 1 < tiles) stage(t + 1);
    }
    l = halves_sum(l);
    // (made anew from the lane: not kept through the loop)
    const int lane1 = lane_anew(), h1 = lane1 >> 5, n1 = lane1 & 31;
    const bool row_here1 = at_row + n1 < rows;
    const int row1 = row_here1 ? row0 + at_row + n1 : row0 + rows - 1;
    // rows 8 z + 4 h1.. of O^T: numbers 64 dg + 32 (z / 2) + 16 T + ..
    const auto number = [&](int c, int z) { return 64 * (c >> 1) + 32 * (z >> 1) + 16 * (c & 1) + 8 * (z & 1) + 4 * h1; };
    if (item.parts > 1) {
        // each part leaves its sums as its lanes hold them, and the last to arrive joins them the same way
        constexpr int64_t PART = 2 * ROWS * (WIDE + 2);
        const int64_t stride = p.heads * SUBS * PART;
        const int64_t row_of = ((int64_t)(place - item.part) * p.heads + pair) * SUBS + sub;
        float *parts = p.partial + (int64_t)kFewGroups * 2 * piece_floats<DIM>() + row_of * PART;
        const int mine = wave * (32 * WIDE) + lane1 * 2, own_row = 2 * ROWS * WIDE + 32 * wave + n1;
        if (busy) {
            float *at = parts + item.part * stride;
#pragma unroll
            for (int c = 0; c < DG * 4; ++c)
#pragma unroll
                for (int z = 0; z < 8; ++z) put2(at + mine + (c * 8 + z) * 128, o[c][2 * z], o[c][2 * z + 1]);
            if (h1 == 0) put(at + own_row, m), put(at + own_row + 2 * ROWS, l);
        }
        if (!last_to_arrive(p.arrived + 3 * kFewGroups + row_of, item.parts, &lds.last)) return;
        if (busy) {
            m = -INFINITY, l = 0.0f;
            for (int w = 0; w < item.parts; ++w) m = fmaxf(m, get(parts + w * stride + own_row));
#pragma unroll
            for (int c = 0; c < DG * 4; ++c)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[c][j] = 0.0f;
            for (int w = 0; w < item.parts; ++w) {
                const float *at = parts + w * stride;
                const float mw = get(at + own_row), lw = get(at + own_row + 2 * ROWS);
                const float f = mw == -INFINITY ? 0.0f : exp2f(mw - m);
                l = fmaf(lw, f, l);
#pragma unroll
                for (int c = 0; c < DG * 4; ++c) {
                    float2 a[8];
#pragma unroll
                    for (int z = 0; z < 8; ++z) a[z] = get2(at + mine + (c * 8 + z) * 128);
#pragma unroll
                    for (int z = 0; z < 8; ++z)
                        o[c][2 * z] = fmaf(a[z].x, f, o[c][2 * z]), o[c][2 * z + 1] = fmaf(a[z].y, f, o[c][2 * z + 1]);
                }
            }
        }
    }
    // the second map's sums to the first's wavefronts, as the lanes hold them
    __syncthreads();
    float4v *other = reinterpret_cast<float4v *>(&s_tile[0][0][0]) + own_rows * (DG * 16 * 64) + lane1;
    static_assert(sizeof(lds.tile) >= GROUPS * DG * 16 * 64 * sizeof(float4v), "a map's sums fit where the tiles were");
    float f = l > 0.0f || l != l ? pow2(-lift<FORM>()) / l : 0.0f;
    if (busy && map == 1) {
        f *= lds.lambda[at_row + n1];
#pragma unroll
        for (int c = 0; c < DG * 4; ++c)
#pragma unroll
            for (int z = 0; z < 4; ++z)
                other[(c * 4 + z) * 64] = (float4v){o[c][4 * z], o[c][4 * z + 1], o[c][4 * z + 2], o[c][4 * z + 3]} * f;
    }
    __syncthreads();
    if (!row_here1) return;
    if (h1 == 0) store_lse(p, first, pair, map, row1, m, l * pow2(-kTileRaise));
    if (map == 1) return;
    float squares = 0.0f;
#pragma unroll
    for (int c = 0; c < DG * 4; ++c)
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const float4v y = less((float4v){o[c][4 * z], o[c][4 * z + 1], o[c][4 * z + 2], o[c][4 * z + 3]}, f, other[(c * 4 + z) * 64]);
            squares += square4(y);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[c][4 * z + j] = y[j];
        }
    const float by = row_factor<WIDE>(p, halves_sum(squares));
    char *to = p.out + ((first + row1 / p.group) * p.out_token + (pair * p.group + row1 % p.group) * p.out_head) * 2;
#pragma unroll
    for (int c = 0; c < DG * 4; ++c)
#pragma unroll
        for (int z = 0; z < 4; z += 2) {
            uint2 y[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4v x = (float4v){o[c][4 * (z + k)], o[c][4 * (z + k) + 1], o[c][4 * (z + k) + 2], o[c][4 * (z + k) + 3]} * by *
                                  *reinterpret_cast<const float4v *>(&lds.weight[number(c, z + k)]);
                y[k] = H::pack4(x[0], x[1], x[2], x[3]);
            }
            // numbers 0..3 and 8..11, 4..7 and 12..15 of the row's two lanes: 0..7, 8..15
            const auto lo = __builtin_amdgcn_permlane32_swap(y[0].x, y[1].x, false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(y[0].y, y[1].y, false, false);
            *reinterpret_cast<uint4v *>(to + (number(c, z) + 4 * h1) * 2) = (uint4v){lo[0], hi[0], lo[1], hi[1]};
        }
}

// ---- launches ----

template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64 * kFewWaves, few_groups<DIM>() / 256) void agft_diff_few_kernel(DiffArgs p) {
    __shared__ FewLds<DIM> lds;
    attend_few<FORM, TYPE, DIM>(p, lds, blockIdx.x);
}

// Tiles of many rows; of 64 numbers in one launch with the few ones' workgroups, which
// are as large (chunks of 256 to 1,024 tokens beside single ones: 116 us, apart 17 more).
template <int DIM>
constexpr bool one_launch() {
    return tile_waves<DIM>() == kFewWaves;
}
template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64 * tile_waves<DIM>(), 2) void agft_diff_tile_kernel(DiffArgs p) {
    if constexpr (one_launch<DIM>()) {
        __shared__ union {
            FewLds<DIM> few;
            TileLds<DIM> many;
        } lds;
        if ((int)blockIdx.x < p.few_blocks) attend_few<FORM, TYPE, DIM>(p, lds.few, blockIdx.x);
        else attend_many<FORM, TYPE, DIM>(p, lds.many, blockIdx.x - p.few_blocks);
    } else {
        __shared__ TileLds<DIM> lds;
        attend_many<FORM, TYPE, DIM>(p, lds, blockIdx.x);
    }
}

inline int diff_status(const agft_kv_config *c) {
    const int st = config_status(c);
    if (st != AGFT_OK) return st;
    return c->heads % 2 != 0 ? AGFT_E_INVAL : c->dim > 128 ? AGFT_E_UNSUPPORTED : AGFT_OK;
}

}  // namespace agft_diff_detail

using namespace agft_diff_detail;

extern "C" {

size_t agft_diff_attend_bytes(const agft_kv_config *cfg, int32_t max_tokens) {
    if (diff_status(cfg) != AGFT_OK || !tokens_ok(max_tokens)) return 0;
    // pieces of few rows, and parts of many
    const int64_t items = item_cap(cfg, max_tokens) * cfg->heads;
    const size_t parts = (size_t)(items < kTileParts ? items : kTileParts);
    const size_t piece = (size_t)(cfg->dim == 64 ? piece_floats<64>() : piece_floats<128>());
    return align_up(((size_t)kFewGroups * 2 * piece + parts * kTileRows * (2 * (size_t)cfg->dim + 2)) * sizeof(float));
}

int agft_diff_attend(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const void *d_tables,
                     size_t tables_bytes, void *d_step, size_t step_bytes, int32_t max_tokens, int32_t max_new,
                     const agft_kv_dense *q, const agft_diff_args *diff, const agft_kv_dense *out, float *d_lse,
                     float scale, void *d_work, size_t work_bytes, void *stream) {
    int st = diff_status(cfg);
    if (st != AGFT_OK) return st;
    agft_kv_tables_view tv;
    agft_kv_step_view sv;
    st = agft_kv_tables_at(cfg, const_cast<void *>(d_tables), tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_kv_step_at(cfg, max_tokens, d_step, step_bytes, &sv);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    if (!buffer_ok(d_work, work_bytes, agft_diff_attend_bytes(cfg, max_tokens))) return AGFT_E_INVAL;
    if (!dense_ok(q) || !dense_ok(out) || q->type != out->type || q->type == AGFT_KV_FP32) return AGFT_E_INVAL;
    if (!apart(out, max_tokens, (int64_t)cfg->heads / 2 * cfg->group)) return AGFT_E_INVAL;
    if (max_new < 1 || max_new > max_tokens || !std::isfinite(scale)) return AGFT_E_INVAL;
    if (reinterpret_cast<uintptr_t>(d_lse) % 4 != 0) return AGFT_E_INVAL;
    if (diff == nullptr || diff->lambda == nullptr || reinterpret_cast<uintptr_t>(diff->lambda) % 4 != 0) return AGFT_E_INVAL;
    if (diff->lambda_token < 0 || diff->lambda_head < 0 || reinterpret_cast<uintptr_t>(diff->weight) % 16 != 0) return AGFT_E_INVAL;
    if (!std::isfinite(diff->gain) || !std::isfinite(diff->eps) || diff->eps < 0) return AGFT_E_INVAL;
    const StepLayout L = step_layout(cfg, max_tokens);
    char *step = static_cast<char *>(d_step);
    DiffArgs p;
    p.codes = static_cast<const char *>(d_cache) + C.codes;
    p.exps = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_cache) + C.exps);
    p.table = tv.table;
    p.works = reinterpret_cast<const Work *>(step + L.works);
    p.items = reinterpret_cast<const Item *>(step + L.items);
    p.arrived = reinterpret_cast<int32_t *>(step + L.arrived);
    p.partial = static_cast<float *>(d_work);
    p.q = static_cast<const char *>(q->data), p.out = static_cast<char *>(out->data), p.lse = d_lse;
    p.q_token = q->token_stride, p.q_head = q->head_stride;
    p.out_token = out->token_stride, p.out_head = out->head_stride;
    p.scale = scale;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages;
    p.page = cfg->page, p.shift = log2_of(cfg->page), p.heads = cfg->heads / 2, p.group = cfg->group;
    p.lambda = diff->lambda, p.lambda_token = diff->lambda_token, p.lambda_head = diff->lambda_head;
    p.weight = diff->weight, p.eps = diff->eps, p.gain = diff->gain;
    const int64_t tile_groups = item_cap(cfg, max_tokens) * p.heads;
    if (tile_groups > (INT32_MAX - kFewGroups) / 2) return AGFT_E_INVAL;
    const auto go = [&](auto form, auto type, auto dim) {
        const hipStream_t hs = static_cast<hipStream_t>(stream);
        const int64_t rows = (int64_t)max_new * cfg->group;
        const bool beside = one_launch<dim()>() && rows > kMidRows;
        p.alone = rows <= kFewRows;
        p.few_blocks = beside ? few_groups<dim()>() : 0;
        if (!beside) {
            agft_diff_few_kernel<form(), type(), dim()><<<few_groups<dim()>(), 64 * kFewWaves, 0, hs>>>(p);
            const int code = launched();
            if (code != AGFT_OK || rows <= kFewRows) return code;
        }
        constexpr int waves = tile_waves<dim()>(), subs = 8 / waves;     // workgroups of a tile
        agft_diff_tile_kernel<form(), type(), dim()><<<(unsigned)(p.few_blocks + tile_groups * subs), 64 * waves, 0, hs>>>(p);
        return launched();
    };
    const auto dims = [&](auto form, auto type) {
        return cfg->dim == 64 ? go(form, type, std::integral_constant<int, 64>{}) : go(form, type, std::integral_constant<int, 128>{});
    };
    const auto types = [&](auto form) {
        return q->type == AGFT_KV_BF16 ? dims(form, std::integral_constant<int, AGFT_KV_BF16>{})
                                       : dims(form, std::integral_constant<int, AGFT_KV_FP16>{});
    };
    return cfg->form == AGFT_KV_E4M3 ? types(std::integral_constant<int, AGFT_KV_E4M3>{})
                                     : types(std::integral_constant<int, AGFT_KV_INT8>{});
}

}  // extern "C"
