// pld_cache.h -- what the paged cache's kernels share: the device's view of a
// cache, which rows exist and where a position's slot is, and the host checks.
#pragma once

#include <math.h>
#include <stdint.h>

#include "pld_device.h"
#include "pld_model.h"

namespace pld {

constexpr float kE4m3Max = 448.f;
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct CacheView {
    char *k, *v;
    float *ks, *vs;                // scales, or null
    int64_t page, slot, head;      // strides in bytes
    int64_t spage;                 // scale stride of a page
    const int32_t *table;
    int64_t table_stride;
    int num_pages, shift, max_pages, heads;   // page_size = 1 << shift
};

// The rows of a batch: row i of sequence b is at position lens[b]-1+i.
struct Rows {
    const int32_t *lens, *draft_len;
    int B, n;
};

// How many rows sequence b has, and the first one's position.
__device__ __forceinline__ int row_count(const Rows &r, int b, int &pos0) {
    const int T = r.lens[b], L = r.draft_len ? r.draft_len[b] : r.n - 1;
    pos0 = T - 1;
    return T >= 1 && L >= 0 && L < r.n ? L + 1 : 0;
}

// The page of position pos (< 2^32), or -1 for a bad one.
__device__ __forceinline__ int page_of(const CacheView &c, int b, int64_t pos) {
    const int64_t i = pos >> c.shift;
    if (i >= c.max_pages) return -1;
    const int page = c.table[(int64_t)b * c.table_stride + i];
    return (uint32_t)page < (uint32_t)c.num_pages ? page : -1;
}

// Host checks of a cache (needs_v: the call uses the values).
inline int prep_cache(const pld_cache *c, bool needs_v, CacheView &o) {
    if (!c || !c->k || !c->table || (needs_v && !c->v)) return PLD_ERR_INVALID;
    if (c->dtype != PLD_BF16 && c->dtype != PLD_E4M3) return PLD_ERR_INVALID;
    const bool q8 = c->dtype == PLD_E4M3;
    if (q8 && (!c->k_scale || (needs_v && !c->v_scale))) return PLD_ERR_INVALID;
    if (!q8 && (c->k_scale || c->v_scale)) return PLD_ERR_INVALID;
    if (c->num_pages < 1 || c->max_pages < 1 || c->heads < 1 || c->heads > 1024)
        return PLD_ERR_INVALID;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return PLD_ERR_INVALID;
    const int ps = c->page_size;
    if (ps < 16 || ps > 4096 || (ps & (ps - 1))) return PLD_ERR_INVALID;
    if ((int64_t)c->max_pages * ps > kMaxTokStride || c->table_stride < c->max_pages)
        return PLD_ERR_INVALID;
    // (strides of a single page or head are never used)
    const int64_t page = c->num_pages > 1 ? c->page_stride : c->head_dim;
    const int64_t head = c->heads > 1 ? c->head_stride : c->head_dim;
    const int64_t spage = c->num_pages > 1 ? c->scale_page_stride : (int64_t)c->heads * ps;
    if (c->slot_stride < c->head_dim || head < c->head_dim || page < c->head_dim)
        return PLD_ERR_INVALID;
    // a tile's offsets, and a page's stride in 16 bytes, are 32-bit
    if (c->slot_stride > 1 << 24 || page > (int64_t)1 << 34) return PLD_ERR_INVALID;
    const int64_t esz = q8 ? 1 : 2;
    if ((uintptr_t)c->k % 16 || (needs_v && (uintptr_t)c->v % 16) || (uintptr_t)c->table % 4 ||
        page * esz % 16 || c->slot_stride * esz % 16 || head * esz % 16)
        return PLD_ERR_ALIGN;
    if (q8) {
        if (spage < (int64_t)c->heads * ps || spage > (int64_t)1 << 31) return PLD_ERR_INVALID;
        if ((uintptr_t)c->k_scale % 16 || (needs_v && (uintptr_t)c->v_scale % 16) ||
            spage % 4)
            return PLD_ERR_ALIGN;
    }
    o = CacheView{};
    o.k = (char *)c->k;
    o.v = (char *)c->v;
    o.ks = c->k_scale;
    o.vs = c->v_scale;
    o.page = page * esz;
    o.slot = c->slot_stride * esz;
    o.head = head * esz;
    o.spage = spage;
    o.table = c->table;
    o.table_stride = c->table_stride;
    o.num_pages = c->num_pages;
    o.shift = __builtin_ctz((unsigned)ps);
    o.max_pages = c->max_pages;
    o.heads = c->heads;
    return PLD_OK;
}

// A bf16 operand [B][n][heads][head_dim] with strides of sequences and rows, in
// either order (the stride of a single sequence or row is never used).
inline int check_rows(const void *p, int64_t seq, int64_t row, int B, int n, int64_t width) {
    if (!p || (B > 1 && seq < width) || (n > 1 && row < width)) return PLD_ERR_INVALID;
    if ((uintptr_t)p % 16 || (B > 1 && seq % 8) || (n > 1 && row % 8)) return PLD_ERR_ALIGN;
    return PLD_OK;
}

inline int check_batch(const pld_cache *c, const int32_t *lens, int B, int n, int Hq) {
    if (!lens || B < 1 || B > 65535 || n < 1 || n > PLD_MAX_CACHE_ROWS) return PLD_ERR_INVALID;
    if (Hq < 1 || Hq > 4096 || Hq % c->heads) return PLD_ERR_INVALID;
    return PLD_OK;
}

// A head's row in the cache, in bytes.
__device__ __forceinline__ int64_t slot_at(const CacheView &c, int page, int64_t pos, int head) {
    return (int64_t)page * c.page + (pos & ((1 << c.shift) - 1)) * c.slot + (int64_t)head * c.head;
}
__device__ __forceinline__ int64_t scale_at(const CacheView &c, int page, int64_t pos, int head) {
    return (int64_t)page * c.spage + ((int64_t)head << c.shift) + (pos & ((1 << c.shift) - 1));
}

// Two fp32 values rounded to nearest (ties to even) as bf16, and four as e4m3.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const bf16x2_t v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// cap * tanh(y), y = x / cap, to some ten 2^-24 of itself.  Below |y| = 0.35, x times a
// polynomial in y^2 (tanh(y) / y, fitted for the smallest relative error: 2^-24.5).
__device__ __forceinline__ float soft_cap_near(float x, float inv2_log2e) {
    constexpr float s = 0.25f * kLn2 * kLn2;   // y^2 = s w^2
    constexpr float c1 = -0.33332663f * s, c2 = 0.13299825f * s * s, c3 = -0.0491485f * s * s * s;
    const float w = x * inv2_log2e, u = w * w;
    return x * fmaf(u, fmaf(u, fmaf(u, c3, c2), c1), 1.f);
}
// Anywhere: from |x| = cap_near on as cap times 1 - 2 / (1 + e^(2|y|)), whose error of a few 2^-24
// of the cap is no more than that of the result; nearer to 0 the difference would cancel.  (The
// same comparison as before a branch on many scores: a score's bits go by it alone.)
constexpr float kCapNear = 0.347f;   // cap_near, of the cap
__device__ __forceinline__ float soft_cap(float x, float cap, float cap_x2, float cap_near, float inv2_log2e) {
    const float e = __builtin_amdgcn_exp2f(fabsf(x) * inv2_log2e);   // e^(2|y|)
    const float far = cap - cap_x2 * __builtin_amdgcn_rcpf(e + 1.f);
    return fabsf(x) >= cap_near ? copysignf(far, x) : soft_cap_near(x, inv2_log2e);
}

}  // namespace pld
