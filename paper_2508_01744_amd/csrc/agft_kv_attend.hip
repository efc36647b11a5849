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
    const int32_t *starts, *granted, *lengths;
    const char *q;
    char *out;
    float *lse;
    int64_t q_token, q_head, out_token, out_head;   // numbers
    float scale;
    int32_t requests, row_pages, pages, page, shift, heads, group;
};

template <int TYPE>
struct Half;
template <>
struct Half<AGFT_KV_BF16> {
    static __device__ __forceinline__ float load(const void *p, int64_t i) {
        return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, float x) {
        static_cast<__bf16 *>(p)[i] = (__bf16)x;
    }
};
template <>
struct Half<AGFT_KV_FP16> {
    static __device__ __forceinline__ float load(const void *p, int64_t i) {
        return (float)static_cast<const _Float16 *>(p)[i];
    }
    static __device__ __forceinline__ void store(void *p, int64_t i, float x) {
        static_cast<_Float16 *>(p)[i] = (_Float16)x;
    }
};

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
    return config_status(cfg) == AGFT_OK && tokens_ok(max_tokens) ? kAlign : 0;
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
    p.q = static_cast<const char *>(q->data), p.out = static_cast<char *>(out->data), p.lse = d_lse;
    p.q_token = q->token_stride, p.q_head = q->head_stride;
    p.out_token = out->token_stride, p.out_head = out->head_stride;
    p.scale = scale;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages;
    p.page = cfg->page, p.shift = log2_of(cfg->page), p.heads = cfg->heads, p.group = cfg->group;
    const dim3 grid((unsigned)max_tokens, (unsigned)(cfg->heads * cfg->group));
    const auto go = [&](auto form, auto type, auto dim) {
        agft_kv_attend_kernel<form(), type(), dim()><<<grid, 64, 0, static_cast<hipStream_t>(stream)>>>(p);
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
