// agft_kv_attend.hip -- attention over a serving node's 8-bit paged cache.
// agft_kv.h states the rules and the layout.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "agft_kv_common.h"

namespace agft_kv_detail {

struct AttendArgs {
    const char *codes;
    const int32_t *exps, *table;
    const int32_t *starts, *granted, *lengths, *work;
    const char *q;
    char *out;
    float *lse, *partial;
    int64_t q_token, q_head, out_token, out_head;   // numbers
    float scale;
    int32_t requests, row_pages, pages, page, shift, heads, group;
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
    static __device__ __forceinline__ float load(const void *p, int64_t i) {
        return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, float x) {
        static_cast<__bf16 *>(p)[i] = (__bf16)x;
    }
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
    static __device__ __forceinline__ float load(const void *p, int64_t i) {
        return (float)static_cast<const _Float16 *>(p)[i];
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, float x) {
        static_cast<_Float16 *>(p)[i] = (_Float16)x;
    }
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

// The last i in [0, n) with a[i] <= x, a[0] <= x and a ascending; the whole
// wavefront looks, 64 places at a time.
__device__ __forceinline__ int find_last(const int32_t *a, int n, int32_t x) {
    const int lane = threadIdx.x & 63;
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + 63) >> 6, k = lane * step;
        const bool below = k < len && a[lo + k] <= x;
        const int hits = __popcll(__ballot(below));
        const int skip = (hits < 1 ? 0 : hits - 1) * step;
        lo += skip;
        len = len - skip < step ? len - skip : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// max (or sum) over the lanes that share lane % 16
__device__ __forceinline__ float across_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16, 64));
    return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float across_sum(float x) {
    x += __shfl_xor(x, 16, 64);
    return x + __shfl_xor(x, 32, 64);
}

// ---- few query rows: shared out over the cached tokens ----
//
// The work is the list of units (64 tokens of one request and head) of the
// requests with at most 16 query rows, requests outermost; every workgroup
// takes an equal stretch of it, so the split does not depend on how the lengths
// are spread.  A stretch's part of one request and head (a segment) is cut among
// the wavefronts, each keeping its own maximum and sums, and joined in LDS; a
// request and head that several workgroups share leaves partial sums, joined by
// agft_kv_join_kernel in the order of the workgroups.
//
// Scores are made transposed, S^T = K Q^T (16 tokens x 16 rows per matrix
// instruction), so that a lane holds four tokens' probabilities of one row,
// which is what the second product O^T = V^T P^T takes as its right operand:
// its left operand holds the same four tokens of a number per lane, as the
// layout stores them.  Nothing moves between lanes but the maximum.
//
// With M the running maximum of s log2(e) + ev (ev the values' exponent), P =
// 2^(s log2(e) + ev - M) lies in 0..1 whatever the pages' scales are, and meets
// the codes in fp16; l sums P 2^-ev, and the output is O / l.
constexpr int kFewWaves = 4;
constexpr int kFewGroups = 512;      // workgroups that share the work
constexpr int kFewShare = 4;         // units below which a stretch is not cut
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Stretch {
    int32_t total, share;
};
__device__ __forceinline__ Stretch stretch_of(const AttendArgs &p) {
    Stretch s;
    s.total = p.work[p.requests] * p.heads;
    s.share = (s.total + kFewGroups - 1) / kFewGroups;
    if (s.share < kFewShare) s.share = kFewShare;
    return s;
}

template <int DIM>
constexpr int partial_floats() {
    return kFewRows * (DIM + 2);
}

template <int TYPE, int DIM>
__device__ __forceinline__ void store_row4(const AttendArgs &p, int first, int head, int r, int d, float4v o, float l) {
    const int t = first + r / p.group, hq = head * p.group + r % p.group;
    const float f = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    uint2 *dst = reinterpret_cast<uint2 *>(p.out + (t * p.out_token + hq * p.out_head + d) * 2);
    *dst = Half<TYPE>::pack4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
}
__device__ __forceinline__ void store_lse(const AttendArgs &p, int first, int head, int r, float m, float l) {
    if (p.lse == nullptr) return;
    const int t = first + r / p.group, hq = head * p.group + r % p.group;
    p.lse[(int64_t)t * p.heads * p.group + hq] = m == -INFINITY ? -INFINITY : (m + __log2f(l)) * kLn2;
}

template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64 * kFewWaves, 2) void agft_kv_few_kernel(AttendArgs p) {
    constexpr int DG = DIM / kBlockDims;
    constexpr int BLK = DIM > 128 || (DIM == 128 && FORM == AGFT_KV_INT8 && TYPE == AGFT_KV_BF16) ? 2 : 4;   // blocks of 16 tokens at a time
    constexpr int ROW = DIM + 4;                  // LDS row, off the banks
    using H = Half<TYPE>;
    using F = Half<AGFT_KV_FP16>;
    __shared__ float s_o[kFewWaves][kFewRows * ROW];
    __shared__ float s_m[kFewWaves][kFewRows], s_l[kFewWaves][kFewRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const Stretch st = stretch_of(p);
    const int64_t x_first = (int64_t)blockIdx.x * st.share;
    if (x_first >= st.total) return;
    const int32_t x1 = x_first + st.share < st.total ? (int32_t)x_first + st.share : st.total;
    const int64_t page_bytes = (int64_t)p.heads * 2 * p.page * DIM;
    const float scale2 = p.scale * kLog2e;
    int32_t x = (int32_t)x_first;
    while (x < x1) {
        const int i = find_last(p.work, p.requests, x / p.heads);
        const int32_t base = p.work[i], units = p.work[i + 1] - base;
        if (units <= 0) break;
        const int32_t rest = x - base * p.heads;
        const int head = rest / units, u0 = rest % units;
        const int count = units - u0 < x1 - x ? units - u0 : x1 - x;
        x += count;
        const int first = p.starts[i], rows = (p.starts[i + 1] - first) * p.group;
        const int granted = p.granted[i], len = p.lengths[i];
        if (granted <= 0) {
            // no slots, no keys
            for (int c = threadIdx.x; c < rows * DIM / 4; c += blockDim.x) {
                const int r = c / (DIM / 4), d = c % (DIM / 4) * 4;
                store_row4<TYPE, DIM>(p, first, head, r, d, (float4v){0, 0, 0, 0}, 0.0f);
                if (d == 0) store_lse(p, first, head, r, -INFINITY, 0.0f);
            }
            continue;
        }
        // right operand of the scores: row n's numbers 64 dg + 16 g + 8 e.. + 7
        typename H::x8 q[DG * 2];
        const bool row_here = n < rows;
        {
            const int tk = n / p.group, hq = head * p.group + n % p.group;
            const char *src = p.q + ((int64_t)(first + tk) * p.q_token + hq * p.q_head) * 2;
#pragma unroll
            for (int c = 0; c < DG * 2; ++c) {
                uint4v v = {0, 0, 0, 0};
                if (row_here) v = *reinterpret_cast<const uint4v *>(src + ((c >> 1) * kBlockDims + 16 * g + 8 * (c & 1)) * 2);
                q[c] = __builtin_bit_cast(typename H::x8, v);
            }
        }
        const int limit = row_here ? len - granted + n / p.group + 1 : len;     // keys that row n sees
        const int least = len - granted + 1;                                    // keys that every row sees
        const int blocks = (len + kBlockTokens - 1) / kBlockTokens;
        const char *codes = p.codes + (int64_t)head * 2 * p.page * DIM;
        const int sub_mask = (p.page >> 4) - 1;

        float m = -INFINITY, l = 0.0f;
        float4v o[DG * 4];
#pragma unroll
        for (int c = 0; c < DG * 4; ++c) o[c] = (float4v){0, 0, 0, 0};

        // this wavefront's blocks of the segment
        const int b_first = (u0 + count * wave / kFewWaves) * (kUnit / kBlockTokens);
        int b_last = (u0 + count * (wave + 1) / kFewWaves) * (kUnit / kBlockTokens);
        if (b_last > blocks) b_last = blocks;
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
                    if (bb >= blocks) bb = blocks - 1;
                    const int64_t page_id = __builtin_amdgcn_readlane(id, bb - b0);
                    const char *src = codes + page_id * page_bytes + side * p.page * DIM + (bb & sub_mask) * (16 * DIM);
#pragma unroll
                    for (int dg = 0; dg < DG; ++dg)
                        dst[s][dg] = *reinterpret_cast<const uint4v *>(src + dg * kBlockBytes + lane * 16);
                }
            };
            uint4v kc[BLK][DG], kn[BLK][DG], vc[BLK][DG];
            fetch(b0, 0, kc);
            for (int b = b0; b < b1; b += BLK) {
                fetch(b, 1, vc);
                if (b + BLK < b1) fetch(b + BLK, 0, kn);
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
                    if (bb >= blocks) bb = blocks - 1;
                    const int ek = __builtin_amdgcn_readlane(ee.x, bb - b0), ev = __builtin_amdgcn_readlane(ee.y, bb - b0);
                    const float ks = scale2 * pow2(ek);
                    back[s] = pow2(-ev);
#pragma unroll
                    for (int j = 0; j < 4; ++j) t[s][j] = fmaf(acc[j], ks, (float)ev);
                }
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
                    const float fall = m == -INFINITY ? 0.0f : exp2f(m - m1);
                    m = m1;
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
                    for (int j = 0; j < 4; ++j) pr[s][j] = (_Float16)e[j];
                }
#pragma unroll
                for (int s = 0; s < BLK; s += 2) {
                    const fp16x8 pp = __builtin_shufflevector(pr[s], pr[s + 1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int c = 0; c < DG * 4; ++c)
                        o[c] = F::mfma(F::template decode<FORM>(vc[s][c >> 2][c & 3], vc[s + 1][c >> 2][c & 3]), pp, o[c]);
                }
#pragma unroll
                for (int s = 0; s < BLK; ++s)
#pragma unroll
                    for (int dg = 0; dg < DG; ++dg) kc[s][dg] = kn[s][dg];
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
        float *part = p.partial + ((int64_t)blockIdx.x * 2 + (u0 == 0 ? 1 : 0)) * partial_floats<DIM>();
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
                store_row4<TYPE, DIM>(p, first, head, r, d, oo, ll);
                if (d == 0) store_lse(p, first, head, r, mm, ll);
            } else {
                *reinterpret_cast<float4v *>(part + r * DIM + d) = oo;
                if (d == 0) part[kFewRows * DIM + r] = mm, part[kFewRows * (DIM + 1) + r] = ll;
            }
        }
        __syncthreads();
    }
}

// Partial sums of the request and head whose first unit lies in this
// workgroup's stretch and whose last does not; a wavefront per row.
template <int TYPE, int DIM>
__global__ __launch_bounds__(256) void agft_kv_join_kernel(AttendArgs p) {
    const Stretch st = stretch_of(p);
    const int64_t x_first = (int64_t)blockIdx.x * st.share;
    if (x_first + st.share >= st.total) return;
    const int32_t x1 = (int32_t)x_first + st.share;               // the next stretch's first unit
    const int i = find_last(p.work, p.requests, (x1 - 1) / p.heads);
    const int32_t base = p.work[i], units = p.work[i + 1] - base;
    if (units <= 0) return;
    const int head = (x1 - 1 - base * p.heads) / units;
    const int32_t from = base * p.heads + head * units;
    if (from < x_first || from + units <= x1) return;
    if (p.granted[i] <= 0) return;
    const int first = p.starts[i], rows = (p.starts[i + 1] - first) * p.group;
    const int last = (from + units - 1) / st.share;               // the workgroup with the last unit
    const int lane = threadIdx.x & 63;
    const int r = blockIdx.y * 4 + (threadIdx.x >> 6);
    if (r >= rows) return;
    constexpr int PER = DIM / 4;                                  // lanes of a row
    constexpr int STEP = PER < 64 ? 64 / PER : 1;                 // pieces read at once
    const int d = lane % PER * 4, ph = lane / PER;
    const auto piece = [&](int w) {
        return p.partial + ((int64_t)w * 2 + (w == (int)blockIdx.x ? 1 : 0)) * partial_floats<DIM>();
    };
    float mm = -INFINITY, ll = 0.0f;
    float4v oo = {0, 0, 0, 0};
    for (int w = blockIdx.x + ph; w <= last; w += STEP) {
        const float *a = piece(w);
        const float m = a[kFewRows * DIM + r], l = a[kFewRows * (DIM + 1) + r];
        const float4v o = *reinterpret_cast<const float4v *>(a + r * DIM + d);
        const float m1 = fmaxf(mm, m);
        const float f0 = mm == -INFINITY ? 0.0f : exp2f(mm - m1), f1 = m == -INFINITY ? 0.0f : exp2f(m - m1);
        oo = oo * f0 + o * f1;
        ll = ll * f0 + l * f1;
        mm = m1;
    }
#pragma unroll
    for (int z = PER; z < 64; z *= 2) {
        const float m = __shfl_xor(mm, z, 64), l = __shfl_xor(ll, z, 64);
        float4v o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __shfl_xor(oo[j], z, 64);
        const float m1 = fmaxf(mm, m);
        const float f0 = mm == -INFINITY ? 0.0f : exp2f(mm - m1), f1 = m == -INFINITY ? 0.0f : exp2f(m - m1);
        // (both partners add in one order)
        const bool low = (lane & z) == 0;
        oo = low ? oo * f0 + o * f1 : o * f1 + oo * f0;
        ll = low ? ll * f0 + l * f1 : l * f1 + ll * f0;
        mm = m1;
    }
    if (ph == 0) {
        store_row4<TYPE, DIM>(p, first, head, r, d, oo, ll);
        if (d == 0) store_lse(p, first, head, r, mm, ll);
    }
}

// One wavefront per token and query head, 64 keys at a time: a lane per key for
// the scores, a lane per number for the sums.
template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(64) void agft_kv_attend_kernel(AttendArgs p) {
    __shared__ float s_q[DIM], s_p[64];
    const int lane = threadIdx.x;
    const int t = blockIdx.x, hq = blockIdx.y, head = hq / p.group;
    if (t >= p.starts[p.requests]) return;
    int lo = 0, hi = p.requests;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.starts[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int i = lo, n = p.granted[i];
    if ((p.starts[i + 1] - p.starts[i]) * p.group <= kFewRows) return;
    const int keys = n > 0 ? p.lengths[i] - n + (t - p.starts[i]) + 1 : 0;
    for (int d = lane; d < DIM; d += 64) s_q[d] = Half<TYPE>::load(p.q, t * p.q_token + hq * p.q_head + d);
    __syncthreads();
    float m = -INFINITY, l = 0.0f, acc[DIM / 64] = {};
    for (int j0 = 0; j0 < keys; j0 += 64) {
        const int j = j0 + lane;
        float s = -INFINITY;
        if (j < keys) {
            const int64_t page_id = (uint32_t)p.table[(int64_t)i * p.row_pages + (j >> p.shift)] % (uint32_t)p.pages;
            const int pos = j & (p.page - 1);
            const char *block = p.codes + (page_id * p.heads + head) * 2 * p.page * DIM + (pos >> 4) * 16 * DIM;
            float dot = 0.0f;
            for (int c = 0; c < DIM / 16; ++c) {
                const uint32_t *w = reinterpret_cast<const uint32_t *>(block + c / 4 * kBlockBytes + ((c % 4) * 16 + (pos & 15)) * 16);
                for (int b = 0; b < 4; ++b) {
                    float x[4];
                    Code<FORM>::unpack4(w[b], x);
                    for (int z = 0; z < 4; ++z) dot += x[z] * s_q[c * 16 + b * 4 + z];
                }
            }
            s = dot * p.scale * pow2(p.exps[(page_id * p.heads + head) * 2]);
        }
        float top = s;
        for (int z = 1; z < 64; z *= 2) top = fmaxf(top, __shfl_xor(top, z, 64));
        const float m1 = fmaxf(m, top), keep = expf(m - m1);
        const float w = j < keys ? expf(s - m1) : 0.0f;
        float sum = w;
        for (int z = 1; z < 64; z *= 2) sum += __shfl_xor(sum, z, 64);
        l = l * keep + sum;
        m = m1;
        s_p[lane] = w;
        __syncthreads();
        for (int dg = 0; dg < DIM / 64; ++dg) acc[dg] *= keep;
        for (int k = 0; k < 64 && j0 + k < keys; ++k) {
            const int jj = j0 + k;
            const int64_t page_id = (uint32_t)p.table[(int64_t)i * p.row_pages + (jj >> p.shift)] % (uint32_t)p.pages;
            const int pos = jj & (p.page - 1), mm = pos & 15;
            const int64_t base = (page_id * p.heads + head) * 2 + 1;
            const char *block = p.codes + base * p.page * DIM + (pos >> 4) * 16 * DIM;
            const float f = s_p[k] * pow2(p.exps[base]);
            for (int dg = 0; dg < DIM / 64; ++dg) {
                float x[4];
                Code<FORM>::unpack4((uint8_t)block[dg * kBlockBytes + ((mm >> 2) * 16 + (lane & 15)) * 16 + (lane >> 4) * 4 + (mm & 3)], x);
                acc[dg] += f * x[0];
            }
        }
        __syncthreads();
    }
    for (int dg = 0; dg < DIM / 64; ++dg)
        Half<TYPE>::store(p.out, t * p.out_token + hq * p.out_head + dg * 64 + lane, keys > 0 ? acc[dg] / l : 0.0f);
    if (p.lse != nullptr && lane == 0)
        p.lse[(int64_t)t * p.heads * p.group + hq] = keys > 0 ? m + logf(l) : -INFINITY;
}

inline int log2_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

}  // namespace agft_kv_detail

using namespace agft_kv_detail;

extern "C" {

size_t agft_kv_attend_bytes(const agft_kv_config *cfg, int32_t max_tokens) {
    if (config_status(cfg) != AGFT_OK || !tokens_ok(max_tokens)) return 0;
    return align_up((size_t)kFewGroups * 2 * kFewRows * (cfg->dim + 2) * sizeof(float));
}

int agft_kv_attend(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const void *d_tables,
                   size_t tables_bytes, const void *d_step, size_t step_bytes, int32_t max_tokens,
                   int32_t max_new, const agft_kv_dense *q, const agft_kv_dense *out, float *d_lse, float scale,
                   void *d_work, size_t work_bytes, void *stream) {
    agft_kv_tables_view tv;
    agft_kv_step_view sv;
    int st = agft_kv_tables_at(cfg, const_cast<void *>(d_tables), tables_bytes, &tv);
    if (st != AGFT_OK) return st;
    st = agft_kv_step_at(cfg, max_tokens, const_cast<void *>(d_step), step_bytes, &sv);
    if (st != AGFT_OK) return st;
    const CacheLayout C = cache_layout(cfg);
    if (!buffer_ok(d_cache, cache_bytes, C.total)) return AGFT_E_INVAL;
    if (!buffer_ok(d_work, work_bytes, agft_kv_attend_bytes(cfg, max_tokens))) return AGFT_E_INVAL;
    if (!dense_ok(q) || !dense_ok(out) || q->type != out->type || q->type == AGFT_KV_FP32) return AGFT_E_INVAL;
    if (max_new < 1 || max_new > max_tokens || !std::isfinite(scale)) return AGFT_E_INVAL;
    if (reinterpret_cast<uintptr_t>(d_lse) % 4 != 0) return AGFT_E_INVAL;
    AttendArgs p;
    p.codes = static_cast<const char *>(d_cache) + C.codes;
    p.exps = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_cache) + C.exps);
    p.table = tv.table;
    p.starts = sv.starts, p.granted = sv.granted, p.lengths = sv.lengths;
    p.work = reinterpret_cast<const int32_t *>(static_cast<const char *>(d_step) + step_layout(cfg, max_tokens).work);
    p.partial = static_cast<float *>(d_work);
    p.q = static_cast<const char *>(q->data), p.out = static_cast<char *>(out->data), p.lse = d_lse;
    p.q_token = q->token_stride, p.q_head = q->head_stride;
    p.out_token = out->token_stride, p.out_head = out->head_stride;
    p.scale = scale;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages;
    p.page = cfg->page, p.shift = log2_of(cfg->page), p.heads = cfg->heads, p.group = cfg->group;
    const dim3 grid((unsigned)max_tokens, (unsigned)(cfg->heads * cfg->group));
    const auto go = [&](auto form, auto type, auto dim) {
        const hipStream_t hs = static_cast<hipStream_t>(stream);
        agft_kv_few_kernel<form(), type(), dim()><<<kFewGroups, 64 * kFewWaves, 0, hs>>>(p);
        int code = launched();
        if (code != AGFT_OK) return code;
        agft_kv_join_kernel<type(), dim()><<<dim3(kFewGroups, kFewRows / 4), 256, 0, hs>>>(p);
        code = launched();
        if (code != AGFT_OK || (int64_t)max_new * cfg->group <= kFewRows) return code;
        agft_kv_attend_kernel<form(), type(), dim()><<<grid, 64, 0, hs>>>(p);
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
