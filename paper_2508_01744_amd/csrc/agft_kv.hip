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
    int32_t *out_counters, *starts, *granted, *out_lengths, *work, *tiles, *need, *touched, *back, *runs;
    int64_t *slots;
    int32_t requests, row_pages, pages, page, shift, group, max_tokens;
};

__device__ __forceinline__ int32_t pages_of(int32_t n, int32_t page, int32_t shift) { return (n + page - 1) >> shift; }

// What a request asks of the window, from its own lengths alone.
struct Ask {
    int32_t past, add, held, tokens, need;
    bool ends;
};

__device__ __forceinline__ Ask ask_of(const PlanArgs &p, int32_t past, int32_t add) {
    Ask a;
    const int32_t cap = p.row_pages << p.shift;
    a.past = past < 0 ? 0 : past > cap ? cap : past;
    a.add = add;
    a.ends = add < 0;
    a.held = pages_of(a.past, p.page, p.shift);
    a.tokens = add > 0 && add <= cap - a.past ? add : 0;
    a.need = pages_of(a.past + a.tokens, p.page, p.shift) - a.held;
    return a;
}

template <typename T>
__device__ __forceinline__ T wave_inclusive(T x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const T y = __shfl_up(x, s, 64);
        if (lane >= s) x += y;
    }
    return x;
}

// Prefix sums over the requests, by one workgroup.
constexpr int kScanThreads = 1024;

__global__ __launch_bounds__(kScanThreads) void agft_kv_scan_kernel(PlanArgs p) {
    constexpr int W = kScanThreads / 64;
    __shared__ int64_t s64[2][W];
    __shared__ int32_t s32[6][W];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t head = p.counters[0], free_pages = p.counters[1];
    int64_t need0 = 0, tok0 = 0;                                        // sums of the requests before this round's
    int32_t touched0 = 0, work0 = 0, tiles0 = 0, back0 = 0, refused0 = 0, taken0 = 0;
    for (int r0 = 0; r0 < p.requests; r0 += kScanThreads) {
        const int i = r0 + threadIdx.x;
        const bool live = i < p.requests;
        const Ask a = ask_of(p, live ? p.lengths[i] : 0, live ? p.add[i] : 0);
        int64_t need = wave_inclusive((int64_t)a.need), tok = wave_inclusive((int64_t)a.tokens);
        if (lane == 63) s64[0][wave] = need, s64[1][wave] = tok;
        __syncthreads();
        int64_t need_all = 0, tok_all = 0;
        for (int w = 0; w < W; ++w) {
            if (w == wave) need += need_all, tok += tok_all;
            need_all += s64[0][w], tok_all += s64[1][w];
        }
        need += need0, tok += tok0;
        need0 += need_all, tok0 += tok_all;
        const bool ok = a.tokens > 0 && (a.need == 0 || need <= free_pages) && tok <= p.max_tokens;
        const int32_t granted = ok ? a.tokens : 0;
        const int64_t first64 = tok - a.tokens;
        const int32_t first = first64 < p.max_tokens ? (int32_t)first64 : p.max_tokens;
        const int32_t last = tok < p.max_tokens ? (int32_t)tok : p.max_tokens;
        const int32_t after = a.ends ? 0 : a.past + granted;
        // what the window's kernels have to do for it
        const int32_t rows = last - first;                              // rows of the window's tensors
        const bool few = (int64_t)rows * p.group <= kFewRows;
        int32_t v[6];
        v[0] = ok ? pages_of(after, p.page, p.shift) - (a.past >> p.shift) : 0;            // pages written to
        // units of few rows: every 16 rows read the request's tokens (one unit where there are none)
        v[1] = rows == 0 || !few ? 0
                                 : (ok ? (after + kUnit - 1) / kUnit : 1) * ((rows * p.group + kRowTile - 1) / kRowTile);
        v[2] = rows == 0 || few ? 0 : (int32_t)(((int64_t)rows * p.group + kTileRows - 1) / kTileRows);
        v[3] = a.ends ? a.held : 0;
        v[4] = live && a.add > 0 && !ok ? 1 : 0;
        v[5] = ok ? a.need : 0;
        int32_t own[6];
        for (int k = 0; k < 6; ++k) {
            own[k] = v[k];
            v[k] = wave_inclusive(v[k]);
            if (lane == 63) s32[k][wave] = v[k];
        }
        __syncthreads();
        int32_t all[6] = {};
        for (int w = 0; w < W; ++w)
            for (int k = 0; k < 6; ++k) {
                if (w == wave) v[k] += all[k];
                all[k] += s32[k][w];
            }
        if (live) {
            p.starts[i] = first;
            p.granted[i] = granted;
            p.out_lengths[i] = after;
            p.need[i] = (int32_t)(need - a.need < free_pages ? need - a.need : free_pages);
            p.touched[i] = touched0 + v[0] - own[0];
            p.work[i] = work0 + v[1] - own[1];
            p.tiles[i] = tiles0 + v[2] - own[2];
            p.back[i] = back0 + v[3] - own[3];
        }
        touched0 += all[0], work0 += all[1], tiles0 += all[2], back0 += all[3], refused0 += all[4], taken0 += all[5];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const int32_t total = tok0 < p.max_tokens ? (int32_t)tok0 : p.max_tokens;
        p.starts[p.requests] = total;
        p.touched[p.requests] = touched0;
        p.work[p.requests] = work0;
        p.tiles[p.requests] = tiles0;
        p.back[p.requests] = back0;
        p.runs[0] = touched0;
        int32_t *c = p.out_counters;
        c[0] = (int32_t)(((int64_t)head + taken0) % p.pages);
        c[1] = free_pages - taken0 + back0;
        c[2] = total;
        c[3] = refused0;
        c[4] = taken0;
        c[5] = back0;
        c[6] = c[7] = 0;
    }
}

// the last i with a[i] <= x (a[0] <= x, a ascending, n entries)
__device__ __forceinline__ int32_t last_at_most(const int32_t *a, int32_t n, int32_t x) {
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Slots, runs and new table entries by tokens; the pages that come back by pages.
__global__ __launch_bounds__(256) void agft_kv_slots_kernel(PlanArgs p) {
    const int32_t head = p.counters[0], free_pages = p.counters[1];
    const int32_t total = p.starts[p.requests];
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    for (int64_t t = id; t < p.max_tokens; t += stride) {
        int64_t slot = -1;
        if (t < total) {
            const int32_t i = last_at_most(p.starts, p.requests, (int32_t)t);
            if (p.granted[i] > 0) {
                const int32_t past = p.lengths[i], k = (int32_t)t - p.starts[i], pos = past + k;
                const int32_t n = pos >> p.shift, held = pages_of(past, p.page, p.shift), off = pos & (p.page - 1);
                int32_t id_of;
                if (n >= held) {
                    id_of = p.ring[((int64_t)head + p.need[i] + n - held) % p.pages];
                    if (off == 0) p.table[(int64_t)i * p.row_pages + n] = id_of;
                } else {
                    id_of = p.table[(int64_t)i * p.row_pages + n];
                }
                slot = ((int64_t)id_of << p.shift) + off;
                if (k == 0 || off == 0) p.runs[1 + p.touched[i] + n - (past >> p.shift)] = (int32_t)t;
            }
        }
        p.slots[t] = slot;
    }
    const int32_t gone = p.back[p.requests];
    for (int64_t g = id; g < gone; g += stride) {
        const int32_t i = last_at_most(p.back, p.requests, (int32_t)g);
        const int32_t page_id = p.table[(int64_t)i * p.row_pages + (g - p.back[i])];
        p.ring[((int64_t)head + free_pages + g) % p.pages] = page_id;
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
template <int FORM, int TYPE, int DIM>
__global__ void agft_kv_append_kernel(AppendArgs p) {
    constexpr int DG = DIM / kBlockDims;
    __shared__ float s_top[8];
    __shared__ uint32_t s_turn[8][kBlockBytes / 4];
    if ((int)blockIdx.x >= p.runs[0]) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, m = lane & 15;
    const int head = blockIdx.y, side = blockIdx.z;
    const int32_t t0 = p.runs[1 + blockIdx.x], total = p.counters[2];
    const int64_t slot0 = p.slots[t0];
    if (slot0 < 0 || slot0 >= p.pool_tokens) return;
    const int64_t page_id = slot0 >> p.shift;
    const int off = (int)(slot0 & (p.page - 1));
    // this lane's token
    const int pos = 16 * wave + m, k = pos - off;
    const bool live = k >= 0 && t0 + k < total && p.slots[t0 + k < total ? t0 + k : t0] == slot0 + k;
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
    __syncthreads();
    top = s_top[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) top = fmaxf(top, s_top[w]);
    int e = exponent<FORM>(top);
    int32_t *ep = p.exps + (page_id * p.heads + head) * 2 + side;
    int drop = 0;                              // how far the older codes' exponent rises
    if (off > 0) {
        const int old = *ep;
        if (e < old) e = old;
        drop = e - old;
    }
    __syncthreads();                           // every wavefront has read the exponent
    if (threadIdx.x == 0) *ep = e;
    const bool older = off > 16 * wave;        // tokens of earlier windows among these 16
    const bool any = __ballot(live) != 0;
    if (!any && !(older && drop > 0)) return;
    const float inv = pow2(-e), fall = drop > 126 ? 0.0f : pow2(-drop);
    uint4 *block = reinterpret_cast<uint4 *>(p.codes + ((page_id * p.heads + head) * 2 + side) * p.page * DIM) +
                   (size_t)wave * DG * 64;
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
        uint4 held = make_uint4(0, 0, 0, 0);
        if (older) {
            held = block[dg * 64 + lane];
            uint32_t h[4] = {held.x, held.y, held.z, held.w};
            if (drop > 0)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float y[4];
                    Code<FORM>::unpack4(h[j], y);
                    h[j] = Code<FORM>::pack4(y[0] * fall, y[1] * fall, y[2] * fall, y[3] * fall);
                }
            held = make_uint4(h[0], h[1], h[2], h[3]);
        }
        if (side == 0) {
            block[dg * 64 + lane] = live ? make_uint4(c[0], c[1], c[2], c[3]) : held;
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
            block[dg * 64 + lane] = make_uint4((fresh.x & mask) | (held.x & ~mask), (fresh.y & mask) | (held.y & ~mask),
                                               (fresh.z & mask) | (held.z & ~mask), (fresh.w & mask) | (held.w & ~mask));
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

// One thread per number pair (key and value) of a slot.
template <int FORM, int TYPE, int DIM>
__global__ __launch_bounds__(256) void agft_kv_export_kernel(ExportArgs p) {
    using T = typename Dense<TYPE>::type;
    const int64_t count = p.n * p.heads * DIM;
    for (int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; id < count; id += (int64_t)gridDim.x * blockDim.x) {
        const int d = (int)(id % DIM);
        const int64_t rest = id / DIM;
        const int head = (int)(rest % p.heads);
        const int64_t t = rest / p.heads;
        const int64_t slot = p.slots[t];
        const bool here = slot >= 0 && slot < p.pool_tokens;
        const int64_t page_id = here ? slot >> p.shift : 0;
        const int pos = (int)(slot & (p.page - 1)), m = pos & 15, dg = d / 64, in = d % 64;
        const int64_t base = (page_id * p.heads + head) * 2;
        const size_t at[2] = {(size_t)(((in >> 4) * 16 + m) * 16 + (in & 15)),
                              (size_t)(((m >> 2) * 16 + (in & 15)) * 16 + (in >> 4) * 4 + (m & 3))};
        for (int side = 0; side < 2; ++side) {
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (here) {
                const uint8_t c = (uint8_t)p.codes[(base + side) * p.page * DIM +
                                                   ((size_t)(pos >> 4) * (DIM / 64) + dg) * kBlockBytes + at[side]];
                Code<FORM>::unpack4(c, x);
                const int e = p.exps[base + side];
                x[0] = ldexpf(x[0], e);
            }
            static_cast<T *>(p.data[side])[t * p.token_stride[side] + head * p.head_stride[side] + d] =
                Dense<TYPE>::from(x[0]);
        }
    }
}

// ---- host side ----

inline int log2_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

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
    p.work = part(L.work), p.tiles = part(L.tiles), p.need = part(L.need), p.touched = part(L.touched);
    p.back = part(L.back), p.runs = part(L.runs), p.slots = sv.slots;
    p.requests = cfg->requests, p.row_pages = cfg->row_pages, p.pages = cfg->pages, p.page = cfg->page;
    p.shift = log2_of(cfg->page), p.group = cfg->group, p.max_tokens = max_tokens;
    hipLaunchKernelGGL(agft_kv_scan_kernel, dim3(1), dim3(kScanThreads), 0, static_cast<hipStream_t>(stream), p);
    st = launched();
    if (st != AGFT_OK) return st;
    const int64_t blocks = ((int64_t)max_tokens + 255) / 256;
    hipLaunchKernelGGL(agft_kv_slots_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0,
                       static_cast<hipStream_t>(stream), p);
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
    const int64_t blocks = (n * cfg->heads * cfg->dim + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536));
    return by_form_type_dim(cfg, k->type, [&](auto form, auto type, auto dim) {
        agft_kv_export_kernel<form(), type(), dim()><<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(p);
        return launched();
    });
}

}  // extern "C"
