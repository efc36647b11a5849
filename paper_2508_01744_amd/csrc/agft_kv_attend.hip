// agft_kv_attend.hip -- attention over a serving node's 8-bit paged cache.
// agft_kv.h states the rules and the layout.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "agft_kv_attend.h"

namespace agft_kv_detail {

// ---- few query rows: shared out over the cached tokens ----
//
// The work is the list of units (64 tokens of one request, for one head's 16
// query rows) of the requests with few query rows per head, requests outermost,
// then heads, then rows; every workgroup takes an equal stretch of it, so the
// split does not depend on how the lengths are spread.  A stretch's part of one
// request's 16 rows (a segment) is cut among the wavefronts, each keeping its own
// maximum and sums, and joined in LDS; rows that several workgroups share leave
// partial sums, which the last of them to arrive joins, in the workgroups' order
// whichever it is.
//
// What bounds it: memory, once there are some hundred MB (24 tokens over 60,000 to
// 131,071 tokens, a cache of 4.45 GB: 757 us, 5.9 TB/s; reading alone reaches 7.1),
// and a chain of loads below (requests, page, exponents, codes, the pieces' way to
// the join: one token over 778 tokens 8.1 us).
//
// Scores are made transposed, S^T = K Q^T (16 tokens x 16 rows per matrix
// instruction), so that a lane holds four tokens' probabilities of one row,
// which is what the second product O^T = V^T P^T takes as its right operand:
// its left operand holds the same four tokens of a number per lane, as the
// layout stores them.  Nothing moves between lanes but the maximum.
//
// With M the running maximum of s log2(e) + ev (ev the values' exponent), P =
// 2^(s log2(e) + ev - M) lies in 0..1 whatever the pages' scales are; l sums P
// 2^-ev, and the output is O / l.  P meets the codes as 2^kRaise P in fp16.
//
// That rounding is what lets the second product run on matrix instructions: each
// P keeps eleven bits (within 2^-11 of itself), what an fp16 output does.  Below
// 2^-14 fp16 keeps fewer bits and below 2^-25 nothing, hence kRaise, which brings
// the largest near the end of its range (65,504): what lies 2^-29 below the largest
// has its eleven bits, and what is lost lies 2^-40 below (2^-25 without it: of
// tokens that a wavefront saw beside one 2^25.1 times as large, nothing was left,
// which for 131,000 of them is 0.4% of the output).  l sums the P that were not
// rounded: pages' exponents may lie so far apart that one's P vanish beside
// another's larger values, and its tokens' weights must stay in l.

// Up to kFewPieces pieces are read in one round trip, weights and all (4 / 8: one
// token over 778 tokens 10.4 / 10.7 us); more get their weights first, kAtOnce on
// their way at a time (one by one: one shared head over 131,000 tokens 44 us for
// 31); beyond kManyPieces, groups of them are joined first.
constexpr int kFewPieces = 4;
constexpr int kAtOnce = 8;
constexpr int kManyPieces = 32;
// A workgroup takes at least kFewShare units, one per wavefront (2 / 4 / 8: one
// token over 778 tokens 13.0 / 10.4 / 11.9 us, 200 requests of 16 to 64 rows over
// up to 3,000 tokens 19.7 / 21.0 / 25.6).  While its share is at most kFewEven,
// rows are cut evenly instead of the work as a whole, if that takes no more
// workgroups (those two 8.2 for 10.5 and 18.8 for 21.6, 64 tokens of 4 heads of 256
// numbers over 100 to 2,000 tokens 35.6 for 38.6); beyond, an equal stretch is
// worth more than that (up to a share of 64: 64 tokens over 100 to 8,192 tokens
// 53.7 for 52.6).
constexpr int kFewShare = 4;
constexpr int kFewEven = 8;
constexpr int kRaise = 15;
template <int DIM>
constexpr int partial_floats() {
    return kRowTile * (DIM + 2);
}

// o: the sums times 2^RAISE
template <int TYPE, int DIM, int RAISE>
__device__ __forceinline__ void store_row4(const AttendArgs &p, int first, int head, int r, int d, float4v o, float l) {
    const int t = first + r / p.group, hq = head * p.group + r % p.group;
    const float f = l > 0.0f || l != l ? pow2(-RAISE) / l : 0.0f;
    uint2 *dst = reinterpret_cast<uint2 *>(p.out + (t * p.out_token + hq * p.out_head + d) * 2);
    *dst = Half<TYPE>::pack4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
}
__device__ __forceinline__ void store_lse(const AttendArgs &p, int first, int head, int r, float m, float l) {
    if (p.lse == nullptr) return;
    const int t = first + r / p.group, hq = head * p.group + r % p.group;
    p.lse[(int64_t)t * p.heads * p.group + hq] = m == -INFINITY ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// Joins `pieces` (at most kManyPieces) of the same rows.  piece(w): where piece
// w lies.  into: where the joined piece goes, or NULL: it is the rows' result.
// weight: LDS for kRowTile * kManyPieces numbers.
template <int TYPE, int DIM, typename F>
__device__ __forceinline__ void join_pieces(const AttendArgs &p, F piece, int pieces, float *into, const Segment &seg,
                                            float *weight) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = seg.rows;
    const auto finish = [&](int r, int d, float4v o, float m, float l) {
        if (into == nullptr) {
            store_row4<TYPE, DIM, kRaise>(p, seg.first, seg.head, seg.row + r, d, o, l);
            if (d == 0) store_lse(p, seg.first, seg.head, seg.row + r, m, l);
        } else {
            put2(into + r * DIM + d, o[0], o[1]);
            put2(into + r * DIM + d + 2, o[2], o[3]);
            if (d == 0) put(into + kRowTile * DIM + r, m), put(into + kRowTile * (DIM + 1) + r, l);
        }
    };
    if (pieces <= kFewPieces && into == nullptr) {
        // one round trip (not into a piece's own place, which others still read)
        for (int c = threadIdx.x; c < rows * (DIM / 4); c += blockDim.x) {
            const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
            float m[kFewPieces], l[kFewPieces];
            float2 a[kFewPieces], b[kFewPieces];
#pragma unroll
            for (int w = 0; w < kFewPieces; ++w) {
                const float *at = piece(w < pieces ? w : 0);
                m[w] = get(at + kRowTile * DIM + r), l[w] = get(at + kRowTile * (DIM + 1) + r);
                a[w] = get2(at + r * DIM + d), b[w] = get2(at + r * DIM + d + 2);
            }
            float top = m[0], sum = 0.0f;
#pragma unroll
            for (int w = 1; w < kFewPieces; ++w) top = fmaxf(top, m[w]);
            float4v o = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kFewPieces; ++w) {
                const float f = w >= pieces || m[w] == -INFINITY ? 0.0f : exp2f(m[w] - top);
                sum = fmaf(l[w], f, sum);
                o += (float4v){a[w].x, a[w].y, b[w].x, b[w].y} * f;
            }
            finish(r, d, o, top, sum);
        }
        return;
    }
    // every piece's weight, a wavefront per row and a lane per piece, then the
    // sums, a thread per four numbers
    float *s_top = weight + kRowTile * kManyPieces, *s_sum = s_top + kRowTile;
    for (int r = wave; r < rows; r += kFewWaves) {
        const bool here = lane < pieces;
        const float *at = piece(here ? lane : 0);
        const float m = here ? get(at + kRowTile * DIM + r) : -INFINITY, l = get(at + kRowTile * (DIM + 1) + r);
        float top = m;
#pragma unroll
        for (int z = 1; z < 64; z *= 2) top = fmaxf(top, __shfl_xor(top, z, 64));
        const float f = m == -INFINITY ? 0.0f : exp2f(m - top);
        if (here) weight[r * kManyPieces + lane] = f;
        float sum = here ? l * f : 0.0f;
#pragma unroll
        for (int z = 1; z < 64; z *= 2) sum += __shfl_xor(sum, z, 64);
        if (lane == 0) s_top[r] = top, s_sum[r] = sum;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < rows * (DIM / 4); c += blockDim.x) {
        const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
        float4v o = {0, 0, 0, 0};
        for (int w0 = 0; w0 < pieces; w0 += kAtOnce) {
            float2 a[kAtOnce], b[kAtOnce];
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) {
                const float *at = piece(w0 + z < pieces ? w0 + z : w0) + r * DIM + d;
                a[z] = get2(at), b[z] = get2(at + 2);
            }
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z)
                if (w0 + z < pieces) o += (float4v){a[z].x, a[z].y, b[z].x, b[z].y} * weight[r * kManyPieces + w0 + z];
        }
        finish(r, d, o, s_top[r], s_sum[r]);
    }
}

// Workgroups that share the work: what the registers let stay on 256 compute
// units at once (128 numbers, 512 with four blocks of 16 tokens on their way in a
// wavefront / 768 with two: 64 tokens over 100 to 8,192 tokens 57 / 50 us; 256
// numbers, 512 / 768, the latter in two rounds: 39 / 49; 64 numbers, 1,024 / 2,048:
// 21.0 / 25.2).
template <int DIM>
constexpr int few_groups() {
    return DIM == 64 ? 1024 : DIM == 128 ? 768 : 512;
}

template <int DIM>
struct FewLds {
    static constexpr int ROW = DIM + 4;                   // off the banks
    // the wavefronts' sums; then a join's weights, largest maxima and sums
    __attribute__((aligned(16))) float o[kFewWaves][kRowTile * ROW];
    float m[kFewWaves][kRowTile], l[kFewWaves][kRowTile];
    EvenLds even;
    int last;
    static_assert(kFewWaves * ROW >= kManyPieces + 2, "a join's numbers fit where the sums were");
};

// Rows of tiles that no launch makes, because a request brings more tokens than
// the caller's bound: NaN, not what the memory held.
template <int TYPE, int DIM>
__device__ __forceinline__ void leave_nan(const AttendArgs &p, int items) {
    const int64_t all = (int64_t)items * p.heads;
    for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
        const Item item = p.items[x / p.heads];
        if (item.part > 0) continue;
        const int head = (int)(x % p.heads), first = p.works[item.request].start, row0 = item.tile * kTileRows;
        int rows = (p.works[item.request + 1].start - first) * p.group - row0;
        if (rows > kTileRows) rows = kTileRows;
        for (int c = threadIdx.x; c < rows * (DIM / 4); c += blockDim.x) {
            const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
            store_row4<TYPE, DIM, 0>(p, first, head, row0 + r, d, (float4v){0, 0, 0, 0}, NAN);
            if (d == 0) store_lse(p, first, head, row0 + r, 0.0f, NAN);
        }
    }
}

// BESIDE: in a launch that makes the tiles of many rows too
template <int FORM, int TYPE, int DIM, bool BESIDE>
__device__ __forceinline__ void attend_few(const AttendArgs &p, FewLds<DIM> &lds, int block) {
    constexpr int DG = DIM / kBlockDims;
    constexpr int BLK = 2;                        // blocks of 16 tokens at a time
    constexpr int ROW = FewLds<DIM>::ROW;
    using H = Half<TYPE>;
    using F = Half<AGFT_KV_FP16>;
    const auto s_o = lds.o;
    const auto s_m = lds.m, s_l = lds.l;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    Works works(p.works, p.requests);
    if constexpr (!BESIDE)
        if (__builtin_expect(p.alone && works.total.y > 0, 0)) {
            // (arguments read anew: kept for this path they cost every call 0.2 us)
            uint64_t args = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
            asm volatile("" : "+s"(args));
            leave_nan<TYPE, DIM>(*reinterpret_cast<const AttendArgs *>(args), works.total.y);
        }
    const int32_t work = works.total.x * p.heads;
    int32_t share = (work + few_groups<DIM>() - 1) / few_groups<DIM>();
    if (share < kFewShare) share = kFewShare;
    int64_t x_first = (int64_t)block * share;
    int32_t x1 = x_first + share < work ? (int32_t)x_first + share : work;
    Piece cut;
    bool even = false;
    if (share <= kFewEven) {
        if (works.n <= 64)
            even = piece_of(p, works, share, few_groups<DIM>(), block, &cut) ||
                   piece_of(p, works, share + 2, few_groups<DIM>(), block, &cut);
        else if (works.n <= kEvenRequests)
            even = piece_of(p, works, share, few_groups<DIM>(), block, lds.even, &cut);
    }
    if (even) x_first = cut.first, x1 = cut.last;
    if (x_first >= x1) return;
    const int64_t page_bytes = (int64_t)p.heads * 2 * p.page * DIM;
    const float scale2 = p.scale * kLog2e;
    int32_t x = (int32_t)x_first;
    if (even) works.look_at(cut.request);
    else works.look(x / p.heads);
    while (x < x1) {
        const Segment seg = segment_of(p, works, x);
        if (seg.units <= 0) break;
        const int i = seg.request, head = seg.head, units = seg.units, u0 = seg.at, row0 = seg.row, rows = seg.rows;
        const int first = seg.first;
        const int count = units - u0 < x1 - x ? units - u0 : x1 - x;
        x += count;
        const int granted = seg.granted, len = seg.length;
        if (granted <= 0) {
            // no slots, no keys
            for (int c = threadIdx.x; c < rows * DIM / 4; c += blockDim.x) {
                const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
                store_row4<TYPE, DIM, 0>(p, first, head, row0 + r, d, (float4v){0, 0, 0, 0}, 0.0f);
                if (d == 0) store_lse(p, first, head, row0 + r, -INFINITY, 0.0f);
            }
            continue;
        }
        // right operand of the scores: row n's numbers 64 dg + 16 g + 8 e.. + 7
        typename H::x8 q[DG * 2];
        const bool row_here = n < rows;
        {
            const int tk = (row0 + n) / p.group, hq = head * p.group + (row0 + n) % p.group;
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
        const char *codes = p.codes + (int64_t)head * 2 * p.page * DIM;
        const int sub_mask = (p.page >> 4) - 1;

        float m = -INFINITY, l = 0.0f;
        float4v o[DG * 4];
#pragma unroll
        for (int c = 0; c < DG * 4; ++c) o[c] = (float4v){0, 0, 0, 0};

        // this wavefront's blocks of the segment: a quarter (kUnit / kBlockTokens == kFewWaves)
        static_assert(kUnit == kBlockTokens * kFewWaves, "a unit gives every wavefront a block");
        const int b_first = u0 * kFewWaves + count * wave;
        const int b_last = b_first + count < blocks ? b_first + count : blocks;
        limit = limit < b_last * kBlockTokens ? limit : b_last * kBlockTokens;
        least = least < b_last * kBlockTokens ? least : b_last * kBlockTokens;
        for (int b0 = b_first; b0 < b_last; b0 += 64) {
            // a lane per block: its page and exponents
            int id;
            int2 ee;
            {
                int b = b0 + lane;
                if (b >= blocks) b = blocks - 1;
                uint32_t z = (uint32_t)p.table[(int64_t)i * p.row_pages + ((b << 4) >> p.shift)];
                if (z >= (uint32_t)p.pages) z = (uint32_t)p.pages - 1;
                id = (int)z;
                ee = *reinterpret_cast<const int2 *>(p.exps + ((int64_t)id * p.heads + head) * 2);
            }
            const int b1 = b0 + 64 < b_last ? b0 + 64 : b_last;
            const auto fetch = [&](int b, int side, uint4v (*dst)[DG]) {
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    int bb = b + s;
                    if (bb >= b_last) bb = b_last - 1;
                    const int64_t page_id = __builtin_amdgcn_readlane(id, bb - b0);
                    const char *src = codes + page_id * page_bytes + side * p.page * DIM + (bb & sub_mask) * (16 * DIM);
#pragma unroll
                    for (int dg = 0; dg < DG; ++dg)
                        dst[s][dg] = *reinterpret_cast<const uint4v *>(src + dg * kBlockBytes + lane * 16);
                }
            };
            // codes are asked for as soon as their registers are free: the next
            // keys after the scores, the next values after the sums
            uint4v kc[BLK][DG], vc[BLK][DG];
            fetch(b0, 0, kc);
            fetch(b0, 1, vc);
            for (int b = b0; b < b1; b += BLK) {
                float4v t[BLK];
                float back[BLK];
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
                    const int ek = __builtin_amdgcn_readlane(ee.x, bb - b0), ev = __builtin_amdgcn_readlane(ee.y, bb - b0);
                    const float ks = scale2 * pow2(ek);
                    back[s] = pow2(-ev);
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[s][j] = fmaf(acc[j], ks, (float)ev);
                }
                if (b + BLK < b1) fetch(b + BLK, 0, kc);
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
                        for (int dg = 0; dg < DG; ++dg) vc[s][dg] &= keep;
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
                    for (int c = 0; c < DG * 4; ++c) o[c] *= fall;
                }
                const float off = m == -INFINITY ? 0.0f : m;
                fp16x4 pr[BLK];
#pragma unroll
                for (int s = 0; s < BLK; ++s) {
                    float4v e;
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(t[s][j] - off);
                    l = fmaf((e[0] + e[1]) + (e[2] + e[3]), back[s], l);
#pragma unroll
                    for (int j = 0; j < 4; ++j) pr[s][j] = (_Float16)(e[j] * pow2(kRaise));
                }
#pragma unroll
                for (int s = 0; s < BLK; s += 2) {
                    const fp16x8 pp = __builtin_shufflevector(pr[s], pr[s + 1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int c = 0; c < DG * 4; ++c)
                        o[c] = F::mfma(F::template decode<FORM>(vc[s][c >> 2][c & 3], vc[s + 1][c >> 2][c & 3]), pp, o[c]);
                }
                if (b + BLK < b1) fetch(b + BLK, 1, vc);
            }
        }
        l = across_sum(l);
        if (row_here) {
#pragma unroll
            for (int c = 0; c < DG * 4; ++c)
                *reinterpret_cast<float4v *>(&s_o[wave][n * ROW + 16 * c + 4 * g]) = o[c];
            if (g == 0) s_m[wave][n] = m, s_l[wave][n] = l;
        }
        __syncthreads();
        const bool whole = count == units;
        const int32_t from = x - count - u0;                       // the rows' first unit
        const int owner = even ? cut.owner : from / share;
        const int pieces = even ? cut.pieces : (from + units - 1) / share - owner + 1;
        float *part = p.partial + ((int64_t)block * 2 + (u0 == 0 ? 1 : 0)) * partial_floats<DIM>();
        for (int c = threadIdx.x; c < rows * (DIM / 4); c += blockDim.x) {
            const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
            float mm = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) mm = fmaxf(mm, s_m[w][r]);
            float4v oo = {0, 0, 0, 0};
            float ll = 0.0f;
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                const float f = s_m[w][r] == -INFINITY ? 0.0f : exp2f(s_m[w][r] - mm);
                oo += *reinterpret_cast<const float4v *>(&s_o[w][r * ROW + d]) * f;
                ll = fmaf(s_l[w][r], f, ll);
            }
            if (whole) {
                store_row4<TYPE, DIM, kRaise>(p, first, head, row0 + r, d, oo, ll);
                if (d == 0) store_lse(p, first, head, row0 + r, mm, ll);
            } else {
                put2(part + r * DIM + d, oo[0], oo[1]);
                put2(part + r * DIM + d + 2, oo[2], oo[3]);
                if (d == 0) put(part + kRowTile * DIM + r, mm), put(part + kRowTile * (DIM + 1) + r, ll);
            }
        }
        if (!whole) {
            // groups of kManyPieces first, each into its first piece's place
            const int mine = block - owner, group0 = mine / kManyPieces * kManyPieces;
            const int members = pieces - group0 < kManyPieces ? pieces - group0 : kManyPieces;
            const int groups = (pieces + kManyPieces - 1) / kManyPieces;
            // the first piece of the rows is its workgroup's second one
            const auto piece = [&](int w) {
                return p.partial + ((int64_t)(owner + w) * 2 + (w == 0 ? 1 : 0)) * partial_floats<DIM>();
            };
            int32_t *counter = p.arrived + kFewGroups + (owner + group0) * 2 + (group0 == 0 ? 1 : 0);
            if (last_to_arrive(counter, members, &lds.last)) {
                float *into = groups == 1 ? nullptr : piece(group0);
                join_pieces<TYPE, DIM>(p, [&](int w) { return piece(group0 + w); }, members, into, seg, s_o[0]);
                if (groups > 1 && last_to_arrive(p.arrived + owner, groups, &lds.last))
                    join_pieces<TYPE, DIM>(p, [&](int w) { return piece(kManyPieces * w); }, groups, nullptr, seg, s_o[0]);
            }
        }
        __syncthreads();
    }
}

// ---- many query rows: tiles of 128 ----
//
// A workgroup takes 128 rows (tokens x group) of one request and head, 32 per
// wavefront, and goes over the tokens 64 at a time.  Vector instructions are what
// such a kernel runs out of before the matrix cores (a matrix instruction takes
// 15 ns of a SIMD, an exponential 4, a conversion 2), so codes are turned into 16
// bits once per workgroup: each wavefront fetches one block of 16 tokens, a tile
// ahead, and leaves its numbers in LDS as the matrix instructions (32 x 32 x 16)
// take them, 16 bytes a lane (every wavefront for itself: 2.38 ms for 2.20 on a
// prompt of 16,380 tokens).  As above, S^T = K Q^T and O^T = V^T P^T, so a row's
// probabilities stay in the lanes that made them.  The tiles of tokens that every
// row sees whole have a loop of their own, without masks.  Consecutive workgroups
// take consecutive heads, so that (with 8 heads) an XCD's L2 holds one head's
// tokens.
//
// The prompt (32 query heads, 8 key/value heads of 128 numbers, causal: 2.2 TFLOP)
// takes 2.08 to 2.23 ms on different cards, 1.0 PFLOP/s, 80% of what a large matrix
// product of the library reaches; matrix cores, LDS and vector instructions are each
// busy for about half of the cycles at a clock that their power sets.
constexpr int kTileWaves = 4;
constexpr int kTileKeys = 64;
// Powers of two that a maximum may grow before the sums are rescaled (0 / 8: the
// chunks 133 / 126 us, the prompt 2.10 / 2.06 ms).  Here the exponential itself
// makes 2^kTileRaise P, below the end of fp16's range where the maximum has grown (a
// multiplication for each P, as the few rows have it: the chunks 123 for 120 us, the
// prompt 2.15 for 2.08 ms); what is lost lies 2^-32 below the largest.  M is the
// maximum to within 2^-21, so that M - kTileRaise is exact: an exponent s log2(e) +
// ev - M + kTileRaise is then rounded once, by 2^-22 near the largest, which is a
// power of two in fp16 as before.
constexpr int kSlack = 8;
constexpr int kTileRaise = kRaise - kSlack;

template <int DIM>
struct TileLds {
    static constexpr int SIDE = kTileKeys * DIM * 2;       // a tile's keys (or values) in 16 bits
    // operands of 1 KB, 16 bytes a lane; keys: [32 tokens][64 numbers][32][16], values: [16 tokens][32 numbers]
    __attribute__((aligned(16))) char tile[2][2][SIDE];
    float4 scale[4][4];                                    // by tile % 4: a block's factor of the scores, ev, 2^-ev
    int last;
};

template <int FORM, int TYPE, int DIM>
__device__ __forceinline__ void attend_many(const AttendArgs &p, TileLds<DIM> &lds, int block) {
    constexpr int DG = DIM / kBlockDims;
    using H = Half<TYPE>;
    using F = Half<AGFT_KV_FP16>;
    const auto s_tile = lds.tile;
    const auto s_scale = lds.scale;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, n = lane & 31;
    const int head = block % p.heads, place = block / p.heads;
    if (place >= p.works[p.requests].items) return;
    const Item item = p.items[place];
    const int i = item.request;
    const int4 own = *reinterpret_cast<const int4 *>(p.works + i);
    const int len = p.works[i].length;
    const int first = own.z, granted = own.w, all_rows = (p.works[i + 1].start - first) * p.group;
    const int row0 = item.tile * kTileRows;
    const int rows = all_rows - row0 < kTileRows ? all_rows - row0 : kTileRows;
    if (rows <= 0) return;
    if (granted <= 0) {
        if (item.part > 0) return;
        for (int c = threadIdx.x; c < rows * DIM / 4; c += blockDim.x) {
            const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
            store_row4<TYPE, DIM, 0>(p, first, head, row0 + r, d, (float4v){0, 0, 0, 0}, 0.0f);
            if (d == 0) store_lse(p, first, head, row0 + r, -INFINITY, 0.0f);
        }
        return;
    }
    const int past = len - granted;
    const bool busy = 32 * wave < rows, row_here = 32 * wave + n < rows;
    const int row = row_here ? row0 + 32 * wave + n : row0 + rows - 1;
    const int limit = past + row / p.group + 1;            // keys that this lane's row sees
    const int all_tiles = (past + (row0 + rows - 1) / p.group + kTileKeys) / kTileKeys;
    const int begin = (int)((int64_t)all_tiles * item.part / item.parts);   // this part's tiles
    const int tiles = (int)((int64_t)all_tiles * (item.part + 1) / item.parts);
    int whole = (past + row0 / p.group + 1) / kTileKeys;                    // tiles that every row sees whole
    if (whole > tiles) whole = tiles;
    const int blocks = (len + kBlockTokens - 1) / kBlockTokens;

    typename H::x8 q[DG * 4];
    {
        const int tk = row / p.group, hq = head * p.group + row % p.group;
        const char *src = p.q + ((int64_t)(first + tk) * p.q_token + hq * p.q_head) * 2;
#pragma unroll
        for (int c = 0; c < DG * 4; ++c)                   // numbers 64 dg + 16 (2 c + h) + 8 e.. + 7
            q[c] = __builtin_bit_cast(typename H::x8, *reinterpret_cast<const uint4v *>(
                       src + ((c >> 2) * kBlockDims + 16 * (2 * ((c >> 1) & 1) + h) + 8 * (c & 1)) * 2));
    }
    const float scale2 = p.scale * kLog2e;
    const int64_t page_bytes = (int64_t)p.heads * 2 * p.page * DIM;
    const char *codes = p.codes + (int64_t)head * 2 * p.page * DIM;
    const int sub_mask = (p.page >> 4) - 1;

    // a lane per tile: the page and exponents of this wavefront's block of it
    int id = 0;
    int2 ee = make_int2(0, 0);
    const auto look_up = [&](int t0) {
        int b = (t0 + lane) * 4 + wave;
        if (b >= blocks) b = blocks - 1;
        uint32_t z = (uint32_t)p.table[(int64_t)i * p.row_pages + ((b << 4) >> p.shift)];
        if (z >= (uint32_t)p.pages) z = (uint32_t)p.pages - 1;
        id = (int)z;
        ee = *reinterpret_cast<const int2 *>(p.exps + ((int64_t)id * p.heads + head) * 2);
    };
    // Step t makes the scores of tile t + 1 beside the sums of tile t, so its
    // operands are the keys of one tile and the values of the one before.
    uint4v ahead[2][DG];                                   // codes of the next step on their way
    const char *values = codes;                            // this wavefront's values of the tile whose keys were last
    const auto fetch = [&](int t, bool both) {             // keys of tile t, values of tile t - 1
        if (both) {
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) ahead[1][dg] = *reinterpret_cast<const uint4v *>(values + dg * kBlockBytes);
        }
        if ((t & 63) == 0 || !both) look_up(t & ~63);
        int b = t * 4 + wave;
        if (b >= blocks) b = blocks - 1;
        const int64_t page_id = __builtin_amdgcn_readlane(id, t & 63);
        const char *src = codes + page_id * page_bytes + (b & sub_mask) * (16 * DIM) + lane * 16;
#pragma unroll
        for (int dg = 0; dg < DG; ++dg) ahead[0][dg] = *reinterpret_cast<const uint4v *>(src + dg * kBlockBytes);
        values = src + p.page * DIM;
    };
    // Entry 16 g + m of the codes to the lanes that take its numbers: token m's
    // numbers 16 g.. as a row of the left operand of the scores, numbers m, 16 + m,
    // .. of tokens 4 g.. as rows of the left operand of the sums.
    const int g = lane >> 4, m16 = lane & 15;
    const int to_key = (((wave >> 1) * DG * 4 + (g >> 1) * 2) * 64 + 32 * (g & 1) + 16 * (wave & 1) + m16) * 16;
    const int to_value = (wave * DG * 2 * 64 + 32 * (g & 1) + 16 * (g >> 1) + m16) * 16;
    const auto stage = [&](int t, bool both) {             // what fetch(t, both) brought
        const int buf = (t + 1) & 1;
#pragma unroll
        for (int dg = 0; dg < DG; ++dg) {
            const uint4v k = ahead[0][dg];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<typename H::x8 *>(&s_tile[buf][0][to_key + (dg * 4 + e) * 1024]) =
                    H::template decode<FORM>(k[2 * e], k[2 * e + 1]);
        }
        if (lane == (t & 63)) s_scale[t & 3][wave] = make_float4(scale2 * pow2(ee.x), (float)ee.y, pow2(-ee.y), 0.0f);
        if (!both) return;
        if (((t - 1) * 4 + wave + 1) * kBlockTokens > len) {
            // codes past the request's tokens may be anything, NaN too
            const int valid = len - ((t - 1) * kTileKeys + 16 * wave + 4 * g);
            const uint32_t keep = valid >= 4 ? ~0u : valid <= 0 ? 0u : (1u << (8 * valid)) - 1u;
#pragma unroll
            for (int dg = 0; dg < DG; ++dg) ahead[1][dg] &= keep;
        }
#pragma unroll
        for (int dg = 0; dg < DG; ++dg) {
            // words 0, 1 (2, 3) of the entries 16 g + m and 16 (g + 2) + m come
            // together in the lower (upper) half: rows m (16 + m) of two operands
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const auto w = __builtin_amdgcn_permlane32_swap(ahead[1][dg][z], ahead[1][dg][2 + z], false, false);
                *reinterpret_cast<fp16x8 *>(&s_tile[buf][1][to_value + (dg * 2 + z) * 1024]) =
                    F::template decode<FORM>(w[0], w[1]);
            }
        }
    };

    float m = -INFINITY, l = 0.0f;
    float16v o[DG * 2];
#pragma unroll
    for (int c = 0; c < DG * 2; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[c][j] = 0.0f;

    float16v s[2];                                         // scores of the tile whose turn is next
    const auto scores = [&](int buf, float16v *z) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int j = 0; j < 16; ++j) z[half][j] = 0.0f;
#pragma unroll
            for (int c = 0; c < DG * 4; ++c)
                z[half] = mfma32<TYPE>(*reinterpret_cast<const typename H::x8 *>(
                                           &s_tile[buf][0][((half * DG * 4 + c) * 64 + lane) * 16]), q[c], z[half]);
        }
    };
    // One step.  MASK: some row may not see all of the tile's keys.
    const auto step = [&](int t, auto mask) {
        constexpr bool MASK = mask();
        const int buf = t & 1;
        const float off = m == -INFINITY ? 0.0f : m - (float)kTileRaise;
        float pow_back[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const float4 f = s_scale[t & 3][b];
            const float ev = f.y - off;
            pow_back[b] = f.z;
#pragma unroll
            for (int j = 0; j < 8; ++j) s[b >> 1][8 * (b & 1) + j] = fmaf(s[b >> 1][8 * (b & 1) + j], f.x, ev);
        }
        if constexpr (MASK) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (t * kTileKeys + 32 * half + 8 * (j >> 2) + 4 * h + (j & 3) >= limit) s[half][j] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[half][j]);
        top = halves_max(top);
        // the maximum that the sums are relative to follows the real one at some distance
        if (__builtin_expect(__any(top > (float)kRaise || m == -INFINITY), 0)) {
            const float m1 = (fmaxf(m, off + top) - (float)kTileRaise) + (float)kTileRaise;
            float fall = m == -INFINITY ? 0.0f : exp2f(m - m1), shift = m1 == -INFINITY ? 0.0f : off - (m1 - (float)kTileRaise);
            m = m1;
            // (keeps the compiler from multiplying ahead of the branch, which is rarely taken)
            asm volatile("" : "+v"(fall), "+v"(shift));
            l *= fall;
#pragma unroll
            for (int c = 0; c < DG * 2; ++c) o[c] *= fall;
#pragma unroll
            for (int half = 0; half < 2; ++half) s[half] += shift;
        }
        // Matrix instructions in the order of their operands in LDS, each of which
        // is read AHEAD instructions before its use; the scores' instructions
        // alternate between the two halves of the tile, with this tile's
        // exponentials between them.  (Left to itself the compiler reads every
        // operand right before its use and waits for it.)
        constexpr int N = DG * 8, AHEAD = 4;               // instructions of the scores, and of the sums
        const auto operand = [&](int c) {
            return *reinterpret_cast<const uint4v *>(
                c < N ? &s_tile[buf][0][(((c & 1) * (N / 2) + (c >> 1)) * 64 + lane) * 16]
                      : &s_tile[buf][1][((c - N) * 64 + lane) * 16]);
        };
        uint4v ring[AHEAD];
        float16v z[2];
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) ring[c] = operand(c);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int j = 0; j < 16; ++j) z[half][j] = 0.0f;
        fp16x8 pr[4];
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            z[c & 1] = mfma32<TYPE>(__builtin_bit_cast(typename H::x8, ring[c % AHEAD]), q[c >> 1], z[c & 1]);
            ring[c % AHEAD] = operand(c + AHEAD);
#pragma unroll
            for (int x = c * 32 / N; x < (c + 1) * 32 / N; ++x) {
                const float e = __builtin_amdgcn_exp2f(s[x >> 4][x & 15]);
                sum = (x & 7) == 0 ? e : sum + e;
                pr[x >> 3][x & 7] = (_Float16)e;
                if ((x & 7) == 7) l = fmaf(sum, pow_back[x >> 3], l);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = N; c < 2 * N; ++c) {
            const int b = (c - N) / (DG * 2), y = (c - N) % (DG * 2);
            o[y] = mfma32<AGFT_KV_FP16>(__builtin_bit_cast(fp16x8, ring[c % AHEAD]), pr[b], o[y]);
            if (c + AHEAD < 2 * N) ring[c % AHEAD] = operand(c + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
        s[0] = z[0], s[1] = z[1];
    };

    fetch(begin, false);
    stage(begin, false);
    fetch(begin + 1, true);
    __syncthreads();
    if (busy) scores((begin + 1) & 1, s);                  // of the first tile, whose keys lie in the buffer of the step before
    stage(begin + 1, true);
    if (!busy)                                             // no rows of its own: only fetches
        for (int t = begin; t < tiles; ++t) {
            __syncthreads();
            if (t + 1 < tiles) fetch(t + 2, true), stage(t + 2, true);
        }
    int t = busy ? begin : tiles;
    for (; t < whole; ++t) {
        __syncthreads();                                   // this step's operands are in LDS, and the other buffer is read
        if (t + 1 < tiles) fetch(t + 2, true);
        step(t, std::false_type{});
        if (t + 1 < tiles) stage(t + 2, true);
    }
    for (; t < tiles; ++t) {
        __syncthreads();
        if (t + 1 < tiles) fetch(t + 2, true);
        step(t, std::true_type{});
        if (t + 1 < tiles) stage(t + 2, true);
    }
    l = halves_sum(l);
    // rows 8 z + 4 h.. of O^T: numbers 64 dg + 32 (z / 2) + 16 T + ..
    const auto number = [&](int c, int z) { return 64 * (c >> 1) + 32 * (z >> 1) + 16 * (c & 1) + 8 * (z & 1) + 4 * h; };
    if (item.parts > 1) {
        // Parts meet as the pieces of few rows do: each leaves its sums as its lanes
        // hold them, and the last to arrive joins them the same way, a lane its own
        // numbers: whole lines.  (By rows, 8 bytes of 32 rows at a time: 128 rows of
        // each of 64 requests over 4,000 tokens 129 us for 102, 64 tokens of 16 query
        // heads over 131,000 148 for 111.)
        constexpr int64_t PART = kTileRows * (DIM + 2);
        const int64_t stride = p.heads * PART;
        float *parts = p.partial + kFewGroups * 2 * partial_floats<DIM>() +
                       ((int64_t)(place - item.part) * p.heads + head) * PART;
        const int mine = wave * (32 * DIM) + lane * 2, own_row = kTileRows * DIM + 32 * wave + n;
        if (busy) {
            float *at = parts + item.part * stride;
#pragma unroll
            for (int c = 0; c < DG * 2; ++c)
#pragma unroll
                for (int z = 0; z < 8; ++z) put2(at + mine + (c * 8 + z) * 128, o[c][2 * z], o[c][2 * z + 1]);
            if (h == 0) put(at + own_row, m), put(at + own_row + kTileRows, l);
        }
        if (!last_to_arrive(p.arrived + 3 * kFewGroups + (place - item.part) * p.heads + head, item.parts, &lds.last)) return;
        if (!busy) return;
        m = -INFINITY, l = 0.0f;
        for (int w0 = 0; w0 < item.parts; w0 += kAtOnce) {
            float mw[kAtOnce];
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) mw[z] = get(parts + (w0 + z < item.parts ? w0 + z : w0) * stride + own_row);
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) m = fmaxf(m, mw[z]);
        }
#pragma unroll
        for (int c = 0; c < DG * 2; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[c][j] = 0.0f;
        for (int w = 0; w < item.parts; ++w) {
            const float *at = parts + w * stride;
            const float mw = get(at + own_row), lw = get(at + own_row + kTileRows);
            float2 a[DG * 2][8];
#pragma unroll
            for (int c = 0; c < DG * 2; ++c)
#pragma unroll
                for (int z = 0; z < 8; ++z) a[c][z] = get2(at + mine + (c * 8 + z) * 128);
            const float f = mw == -INFINITY ? 0.0f : exp2f(mw - m);
            l = fmaf(lw, f, l);
#pragma unroll
            for (int c = 0; c < DG * 2; ++c)
#pragma unroll
                for (int z = 0; z < 8; ++z)
                    o[c][2 * z] = fmaf(a[c][z].x, f, o[c][2 * z]), o[c][2 * z + 1] = fmaf(a[c][z].y, f, o[c][2 * z + 1]);
        }
    }
    if (!row_here) return;
#pragma unroll
    for (int c = 0; c < DG * 2; ++c)
#pragma unroll
        for (int z = 0; z < 4; ++z)
            store_row4<TYPE, DIM, 0>(p, first, head, row, number(c, z),
                                  (float4v){o[c][4 * z], o[c][4 * z + 1], o[c][4 * z + 2], o[c][4 * z + 3]}, l);
    if (h == 0) store_lse(p, first, head, row, m, l * pow2(-kTileRaise));
}

// ---- launches ----

template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64 * kFewWaves, few_groups<DIM>() / 256) void agft_kv_few_kernel(AttendArgs p) {
    __shared__ FewLds<DIM> lds;
    attend_few<FORM, TYPE, DIM, false>(p, lds, blockIdx.x);
}

// Tiles of many rows, in one launch with the few ones' workgroups where a request
// may have more than kMidRows (10 chunks of 256 to 1,024 tokens beside 38 single
// tokens 127 us, 137 in two launches).  Up to kMidRows the few ones come alone
// first, at their own occupancy (200 requests of 16 to 64 rows 20.4 us, 23.6 in one
// launch).
template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64 * kTileWaves, DIM > 128 ? 1 : 2) void agft_kv_tile_kernel(AttendArgs p) {
    static_assert(kFewWaves == kTileWaves, "one workgroup size");
    __shared__ union {
        FewLds<DIM> few;
        TileLds<DIM> many;
    } lds;
    if ((int)blockIdx.x < p.few_blocks) attend_few<FORM, TYPE, DIM, true>(p, lds.few, blockIdx.x);
    else attend_many<FORM, TYPE, DIM>(p, lds.many, blockIdx.x - p.few_blocks);
}

}  // namespace agft_kv_detail

using namespace agft_kv_detail;

extern "C" {

size_t agft_kv_attend_bytes(const agft_kv_config *cfg, int32_t max_tokens) {
    if (config_status(cfg) != AGFT_OK || !tokens_ok(max_tokens)) return 0;
    // pieces of few rows, and parts of many
    const int64_t items = item_cap(cfg, max_tokens) * cfg->heads;
    const size_t parts = (size_t)(items < kTileParts ? items : kTileParts);
    return align_up(((size_t)kFewGroups * 2 * kRowTile + parts * kTileRows) * (cfg->dim + 2) * sizeof(float));
}

int agft_kv_attend(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const void *d_tables,
                   size_t tables_bytes, void *d_step, size_t step_bytes, int32_t max_tokens,
                   int32_t max_new, const agft_kv_dense *q, const agft_kv_dense *out, float *d_lse, float scale,
                   void *d_work, size_t work_bytes, void *stream) {
    agft_kv_tables_view tv;
    agft_kv_step_view sv;
    int st = agft_kv_tables_at(cfg, const_cast<void *>(d_tables), tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_kv_step_at(cfg, max_tokens, d_step, step_bytes, &sv);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    if (!buffer_ok(d_work, work_bytes, agft_kv_attend_bytes(cfg, max_tokens))) return AGFT_E_INVAL;
    if (!dense_ok(q) || !dense_ok(out) || q->type != out->type || q->type == AGFT_KV_FP32) return AGFT_E_INVAL;
    if (!apart(out, max_tokens, (int64_t)cfg->heads * cfg->group)) return AGFT_E_INVAL;
    if (max_new < 1 || max_new > max_tokens || !std::isfinite(scale)) return AGFT_E_INVAL;
    if (reinterpret_cast<uintptr_t>(d_lse) % 4 != 0) return AGFT_E_INVAL;
    AttendArgs p;
    p.codes = static_cast<const char *>(d_cache) + C.codes;
    p.exps = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_cache) + C.exps);
    p.table = tv.table;
    p.works = reinterpret_cast<const Work *>(static_cast<const char *>(d_step) + step_layout(cfg, max_tokens).works);
    p.partial = static_cast<float *>(d_work);
    p.arrived = reinterpret_cast<int32_t *>(static_cast<char *>(d_step) + step_layout(cfg, max_tokens).arrived);
    p.q = static_cast<const char *>(q->data), p.out = static_cast<char *>(out->data), p.lse = d_lse;
    p.q_token = q->token_stride, p.q_head = q->head_stride;
    p.out_token = out->token_stride, p.out_head = out->head_stride;
    p.scale = scale;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages;
    p.page = cfg->page, p.shift = log2_of(cfg->page), p.heads = cfg->heads, p.group = cfg->group;
    p.items = reinterpret_cast<const Item *>(static_cast<const char *>(d_step) + step_layout(cfg, max_tokens).items);
    const int64_t tile_groups = item_cap(cfg, max_tokens) * cfg->heads;
    if (tile_groups > INT32_MAX - kFewGroups) return AGFT_E_INVAL;
    const auto go = [&](auto form, auto type, auto dim) {
        const hipStream_t hs = static_cast<hipStream_t>(stream);
        const int64_t rows = (int64_t)max_new * cfg->group;
        p.few_blocks = rows > kMidRows ? few_groups<dim()>() : 0;
        p.alone = rows <= kFewRows;
        if (rows <= kMidRows) {
            agft_kv_few_kernel<form(), type(), dim()><<<few_groups<dim()>(), 64 * kFewWaves, 0, hs>>>(p);
            const int code = launched();
            if (code != AGFT_OK || rows <= kFewRows) return code;
        }
        agft_kv_tile_kernel<form(), type(), dim()><<<(unsigned)(p.few_blocks + tile_groups), 64 * kTileWaves, 0, hs>>>(p);
        return launched();
    };
    const auto dims = [&](auto form, auto type) {
        if (cfg->dim == 64) return go(form, type, std::integral_constant<int, 64>{});
        if (cfg->dim == 128) return go(form, type, std::integral_constant<int, 128>{});
        return go(form, type, std::integral_constant<int, 256>{});
    };
    const auto types = [&](auto form) {
        return q->type == AGFT_KV_BF16 ? dims(form, std::integral_constant<int, AGFT_KV_BF16>{})
                                       : dims(form, std::integral_constant<int, AGFT_KV_FP16>{});
    };
    return cfg->form == AGFT_KV_E4M3 ? types(std::integral_constant<int, AGFT_KV_E4M3>{})
                                     : types(std::integral_constant<int, AGFT_KV_INT8>{});
}

}  // extern "C"
