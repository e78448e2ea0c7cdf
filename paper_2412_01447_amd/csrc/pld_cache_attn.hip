// pld_cache_attn.hip -- attention of a verification pass's rows over the paged
// cache, and the attention weights of chosen heads at one row (Eq. 3's artifact).
#include "pld_cache.h"

namespace pld {

struct AttnArgs {
    CacheView c;
    Rows r;
    const uint16_t *q;
    int64_t qs, qr;
    int Hq;
    float scale, cap, inv2_log2e;   // inv2_log2e = 2 log2(e) / cap
    int window;
    uint16_t *out;
    int64_t os, orow;
    float *lse;
    // the chosen heads' weights
    const int32_t *row, *heads;
    int R;
    float *attn;
    int64_t as, ar, n_keys;
};

// Element t of a head's row.
template <bool kE4m3>
__device__ __forceinline__ float cache_get(const char *row, int t) {
    if constexpr (kE4m3) {
        return __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)row)[t], 0);
    } else {
        return __uint_as_float((uint32_t)((const uint16_t *)row)[t] << 16);
    }
}

// Score of key j (on page `page`) against the query row in `q`.
template <int D, bool kE4m3>
__device__ __forceinline__ float score(const AttnArgs &a, const float *q, int page, int64_t j,
                                       int kv) {
    const char *row = a.c.k + slot_at(a.c, page, j, kv);
    float s = 0.f;
    for (int t = 0; t < D; ++t) s = fmaf(q[t], cache_get<kE4m3>(row, t), s);
    s *= a.scale;
    if (kE4m3) s *= a.c.ks[scale_at(a.c, page, j, kv)];
    return a.cap > 0.f ? soft_cap(s, a.cap, a.inv2_log2e) : s;
}

// One wave per row and head: 64 keys a round, a running maximum and sum.
template <int D, bool kE4m3>
__global__ __launch_bounds__(64) void cache_attn_kernel(AttnArgs a) {
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, lane = lane_id();
    int pos0;
    if (i >= row_count(a.r, b, pos0)) return;
    __shared__ float q[D], p[64];
    __shared__ int64_t at[64];
    const uint16_t *qp = a.q + (int64_t)b * a.qs + (int64_t)i * a.qr + (int64_t)h * D;
    for (int t = lane; t < D; t += 64) q[t] = __uint_as_float((uint32_t)qp[t] << 16);
    __syncthreads();
    const int kv = h / (a.Hq / a.c.heads);
    const int64_t pos = (int64_t)pos0 + i, cap = (int64_t)a.c.max_pages << a.c.shift;
    const int64_t lo = a.window && pos + 1 > a.window ? pos + 1 - a.window : 0;
    bool bad = pos >= cap;
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    for (int64_t j0 = lo; !bad && j0 <= pos; j0 += 64) {
        const int64_t j = j0 + lane;
        float s = -INFINITY;
        int page = 0;
        if (j <= pos) {
            page = page_of(a.c, b, j);
            if (page >= 0) s = score<D, kE4m3>(a, q, page, j, kv);
        }
        if (__any(page < 0)) {
            bad = true;
            break;
        }
        const float mn = fmaxf(m, wave_max_f32(s));
        const float e = __builtin_amdgcn_exp2f((s - mn) * kLog2E);
        const float f = __builtin_amdgcn_exp2f((m - mn) * kLog2E);
        m = mn;
        l = l * f + wave_sum_f32(e);
        p[lane] = kE4m3 && j <= pos ? e * a.c.vs[scale_at(a.c, page, j, kv)] : e;
        at[lane] = slot_at(a.c, page, j, kv);
        __syncthreads();
        const int cnt = (int)min((int64_t)64, pos + 1 - j0);
        for (int u = 0; u < D / 64; ++u) {
            float s2 = o[u] * f;
            for (int x = 0; x < cnt; ++x)
                s2 = fmaf(p[x], cache_get<kE4m3>(a.c.v + at[x], lane + 64 * u), s2);
            o[u] = s2;
        }
        __syncthreads();
    }
    const float nan = __uint_as_float(0x7fc00000u);
    uint16_t *out = a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)h * D;
    for (int u = 0; u < D / 64; ++u)
        out[lane + 64 * u] = (uint16_t)pack_bf16(bad ? nan : o[u] / l, 0.f);
    if (a.lse && lane == 0)
        a.lse[((int64_t)b * a.r.n + i) * a.Hq + h] = bad ? nan : m + logf(l);
}

// One thread per key and chosen head.
template <int D, bool kE4m3>
__global__ __launch_bounds__(256) void cache_attn_rows_kernel(AttnArgs a) {
    const int r = blockIdx.y, b = blockIdx.z, T = a.r.lens[b], i = a.row[b];
    if (T < 1 || i < 0 || i >= a.r.n) return;
    const int64_t pos = (int64_t)T - 1 + i, end = min(pos + 1, a.n_keys);
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j - threadIdx.x >= end) return;
    __shared__ float q[D];
    const int h = a.heads[r];
    const bool known = h >= 0 && h < a.Hq;
    if (known) {
        const uint16_t *qp = a.q + (int64_t)b * a.qs + (int64_t)i * a.qr + (int64_t)h * D;
        for (int t = threadIdx.x; t < D; t += 256) q[t] = __uint_as_float((uint32_t)qp[t] << 16);
    }
    __syncthreads();
    if (j >= end) return;
    float w = __uint_as_float(0x7fc00000u);
    if (known) {
        const int page = page_of(a.c, b, j);
        if (a.window && j <= pos - a.window)
            w = 0.f;
        else if (page >= 0)
            w = __builtin_amdgcn_exp2f((score<D, kE4m3>(a, q, page, j, h / (a.Hq / a.c.heads)) -
                                        a.lse[((int64_t)b * a.r.n + i) * a.Hq + h]) *
                                       kLog2E);
    }
    a.attn[(int64_t)b * a.as + (int64_t)r * a.ar + j] = w;
}

static int prep_attn(const pld_cache *cache, bool needs_v, const uint16_t *q, int64_t qs,
                     int64_t qr, const int32_t *lens, const int32_t *draft_len, int B, int n,
                     int Hq, float scale, float softcap, int window, AttnArgs &a) {
    a = AttnArgs{};
    int rc = prep_cache(cache, needs_v, a.c);
    if (rc == PLD_OK) rc = check_batch(cache, lens, B, n, Hq);
    if (rc == PLD_OK) rc = check_rows(q, qs, qr, B, n, (int64_t)Hq * cache->head_dim);
    if (rc != PLD_OK) return rc;
    if (!(scale > 0.f) || !isfinite(scale) || !(softcap >= 0.f) || !isfinite(softcap) || window < 0)
        return PLD_ERR_INVALID;
    a.r = Rows{lens, draft_len, B, n};
    a.q = q, a.qs = qs, a.qr = qr;
    a.Hq = Hq;
    a.scale = scale, a.cap = softcap;
    a.inv2_log2e = softcap > 0.f ? 2.f * kLog2E / softcap : 0.f;
    a.window = window;
    return PLD_OK;
}

}  // namespace pld

using namespace pld;

extern "C" size_t pld_cache_attn_workspace_bytes(int B, int n, int Hq, int heads, int head_dim) {
    if (B < 1 || B > 65535 || n < 1 || n > PLD_MAX_CACHE_ROWS || heads < 1 || heads > 1024 ||
        Hq < 1 || Hq > 4096 || Hq % heads ||
        (head_dim != 64 && head_dim != 128 && head_dim != 256))
        return 0;
    return 256;
}

extern "C" int pld_cache_attn(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                              int64_t q_row_stride, const int32_t *lens, const int32_t *draft_len,
                              int B, int n, int Hq, float scale, float softcap, int window,
                              uint16_t *out, int64_t o_seq_stride, int64_t o_row_stride,
                              float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    AttnArgs a;
    int rc = prep_attn(cache, true, q, q_seq_stride, q_row_stride, lens, draft_len, B, n, Hq,
                       scale, softcap, window, a);
    if (rc != PLD_OK) return rc;
    const int D = cache->head_dim;
    rc = check_rows(out, o_seq_stride, o_row_stride, B, n, (int64_t)Hq * D);
    if (rc != PLD_OK) return rc;
    if ((uintptr_t)lse % 4) return PLD_ERR_ALIGN;
    if (!workspace || (uintptr_t)workspace % 16 ||
        workspace_bytes < pld_cache_attn_workspace_bytes(B, n, Hq, cache->heads, D))
        return PLD_ERR_WORKSPACE;
    a.out = out, a.os = o_seq_stride, a.orow = o_row_stride;
    a.lse = lse;
    const dim3 grid((unsigned)Hq, (unsigned)n, (unsigned)B);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(64), 0, (hipStream_t)stream, a);
    };
    const bool q8 = cache->dtype == PLD_E4M3;
    if (D == 64)
        q8 ? go(cache_attn_kernel<64, true>) : go(cache_attn_kernel<64, false>);
    else if (D == 128)
        q8 ? go(cache_attn_kernel<128, true>) : go(cache_attn_kernel<128, false>);
    else
        q8 ? go(cache_attn_kernel<256, true>) : go(cache_attn_kernel<256, false>);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}

extern "C" int pld_cache_attn_rows(const pld_cache *cache, const uint16_t *q,
                                   int64_t q_seq_stride, int64_t q_row_stride, const int32_t *lens,
                                   const int32_t *row, const int32_t *heads, int R,
                                   const float *lse, int B, int n, int Hq, float scale,
                                   float softcap, int window, float *attn, int64_t a_seq_stride,
                                   int64_t a_row_stride, int64_t n_keys, void *stream) {
    AttnArgs a;
    int rc = prep_attn(cache, false, q, q_seq_stride, q_row_stride, lens, nullptr, B, n, Hq, scale,
                       softcap, window, a);
    if (rc != PLD_OK) return rc;
    if (!row || !heads || !lse || !attn || R < 1 || R > 65535 || n_keys < 1)
        return PLD_ERR_INVALID;
    if ((B > 1 && a_seq_stride < n_keys) || (R > 1 && a_row_stride < n_keys))
        return PLD_ERR_INVALID;
    if ((uintptr_t)lse % 4 || (uintptr_t)attn % 4) return PLD_ERR_ALIGN;
    a.row = row, a.heads = heads, a.R = R;
    a.lse = const_cast<float *>(lse);
    a.attn = attn, a.as = a_seq_stride, a.ar = a_row_stride, a.n_keys = n_keys;
    // positions past the table have no page: more keys than it holds (and a page's
    // worth, for rows past its end) are of no use
    const int64_t keys = n_keys < kMaxTokStride ? n_keys : kMaxTokStride;
    const dim3 grid((unsigned)((keys + 255) / 256), (unsigned)R, (unsigned)B);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, a);
    };
    const bool q8 = cache->dtype == PLD_E4M3;
    if (cache->head_dim == 64)
        q8 ? go(cache_attn_rows_kernel<64, true>) : go(cache_attn_rows_kernel<64, false>);
    else if (cache->head_dim == 128)
        q8 ? go(cache_attn_rows_kernel<128, true>) : go(cache_attn_rows_kernel<128, false>);
    else
        q8 ? go(cache_attn_rows_kernel<256, true>) : go(cache_attn_rows_kernel<256, false>);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
