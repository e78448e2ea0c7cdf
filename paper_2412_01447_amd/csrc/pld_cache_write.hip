// pld_cache_write.hip -- a layer's new rows join its paged cache: per-head norms
// and position rotation of queries and keys, quantisation, the page slots.
#include "pld_cache.h"

namespace pld {

struct WriteArgs {
    CacheView c;
    Rows r;
    const uint16_t *q, *k, *v;
    int64_t qs, qr, ks, kr, vs, vr;
    const uint16_t *qw, *kw;
    float eps;
    const float *rope;
    int64_t rope_stride;
    int n_pos, rot, Hq;
    uint16_t *out;
    int64_t os, orow;
};

// Sum and maximum over a group of G consecutive lanes (8, 16 or 32), the same
// bits in each of them.
template <int kCtrl>
__device__ __forceinline__ float moved(float v) {
    return __int_as_float(dpp_move<kCtrl, 0xf>(__float_as_int(v)));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    v += moved<kDppQuadSwap1>(v);
    v += moved<kDppQuadSwap2>(v);
    v += moved<kDppHalfMirror>(v);
    if (G > 8) v += moved<kDppMirror>(v);
    if (G > 16) v += __shfl_xor(v, 16);
    return v;
}
template <int G>
__device__ __forceinline__ float group_max(float v) {
    v = fmaxf(v, moved<kDppQuadSwap1>(v));
    v = fmaxf(v, moved<kDppQuadSwap2>(v));
    v = fmaxf(v, moved<kDppHalfMirror>(v));
    if (G > 8) v = fmaxf(v, moved<kDppMirror>(v));
    if (G > 16) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

// D / 8 lanes a head's row, each holding two runs of four elements, t0 and t1:
// with pairs of halves the runs are each other's partners (t1 = t0 + rot/2), so
// a rotation needs no other lane; elsewhere they are neighbours.  Bound by memory: 4 x 2048
// rows of 32 + 2 x 8 heads of 128 (202 MB) in 41 us, 4.9 TB/s, what a large copy reaches (4.83);
// up to 17 rows of 64 + 2 x 8 heads in each of 64 sequences, into e4m3 (36 MB), in 11 us, the vector
// instructions of norms and quotients included.  One head a lane group: with four, and their
// loads together, the waves are too few (41 and 13.5 us, and 3.9 instead of 2.6 us for a
// single row).  Blocks of one kind of head each would have less to select, but are a third
// more, and the launch of blocks takes as long as the memory (52 us instead of 41).
template <int D, bool kHalves, bool kE4m3>
__global__ __launch_bounds__(256) void cache_write_kernel(WriteArgs a) {
    constexpr int G = D / 8;
    const int i = blockIdx.y, b = blockIdx.z;
    int pos0;
    if (i >= row_count(a.r, b, pos0)) return;
    const int item = (int)(blockIdx.x * blockDim.x + threadIdx.x) / G;
    const int c = (int)threadIdx.x % G;
    const int Hkv = a.c.heads;
    if (item >= a.Hq + 2 * Hkv) return;
    const int kind = item < a.Hq ? 0 : item < a.Hq + Hkv ? 1 : 2;   // query, key, value
    const int head = kind == 0 ? item : item - a.Hq - (kind == 2 ? Hkv : 0);

    const int64_t pos = (int64_t)pos0 + i;
    const bool turned = a.rope && kind != 2;
    const int page = page_of(a.c, b, pos);
    const bool ok = page >= 0 && (!a.rope || pos < a.n_pos);
    const int rot = turned ? a.rot : 0;
    const bool mine = 8 * c < rot;   // this lane's runs are rotated
    int t0 = 8 * c, t1 = 8 * c + 4;
    if (kHalves && mine) {
        t0 = 4 * c;
        t1 = rot / 2 + 4 * c;
    }
    const uint16_t *src = kind == 0   ? a.q + (int64_t)b * a.qs + (int64_t)i * a.qr
                          : kind == 1 ? a.k + (int64_t)b * a.ks + (int64_t)i * a.kr
                                      : a.v + (int64_t)b * a.vs + (int64_t)i * a.vr;
    src += (int64_t)head * D;
    float x[8];
    auto get = [](const uint16_t *p, float *o) {
        const uint2 w = *reinterpret_cast<const uint2 *>(p);
        o[0] = bf16_lo(w.x), o[1] = bf16_hi(w.x), o[2] = bf16_lo(w.y), o[3] = bf16_hi(w.y);
    };
    get(src + t0, x);
    get(src + t1, x + 4);

    const uint16_t *w = kind == 0 ? a.qw : kind == 1 ? a.kw : nullptr;
    if (w) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
        const float inv = 1.f / sqrtf(group_sum<G>(s) / (float)D + a.eps);
        float g[8];
        get(w + t0, g);
        get(w + t1, g + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
    }
    if (mine && ok) {
        const float *row = a.rope + pos * a.rope_stride + 4 * c;
        const float4 co = *reinterpret_cast<const float4 *>(row);
        const float4 si = *reinterpret_cast<const float4 *>(row + rot / 2);
        const float cs[4] = {co.x, co.y, co.z, co.w}, sn[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float &p = kHalves ? x[e] : x[2 * e];
            float &r = kHalves ? x[e + 4] : x[2 * e + 1];
            const float np = p * cs[e] - r * sn[e], nr = r * cs[e] + p * sn[e];
            p = np;
            r = nr;
        }
    }
    auto put = [](uint16_t *p, const float *o) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
    };
    if (kind == 0) {
        if (!ok)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(0x7fc00000u);
        uint16_t *dst = a.out + (int64_t)b * a.os + (int64_t)i * a.orow + (int64_t)head * D;
        put(dst + t0, x);
        put(dst + t1, x + 4);
        return;
    }
    if (!ok) return;
    char *dst = (kind == 1 ? a.c.k : a.c.v) + slot_at(a.c, page, pos, head);
    if constexpr (kE4m3) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));
        // a scale of at least the smallest normal number, so that the division stays finite
        const float scale = fmaxf(group_max<G>(m) / kE4m3Max, 1.17549435e-38f);
        // a quotient from the reciprocal, with what it leaves over put right: one that is rounded
        // otherwise than x / scale differs from it by 2^-24, before the rounding to 2^-4
        const float inv = 1.f / scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = x[e] * inv;
            x[e] = fmaf(fmaf(-y, scale, x[e]), inv, y);
        }
        *reinterpret_cast<uint32_t *>(dst + t0) = pack_e4m3(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint32_t *>(dst + t1) = pack_e4m3(x[4], x[5], x[6], x[7]);
        if (c == 0) (kind == 1 ? a.c.ks : a.c.vs)[scale_at(a.c, page, pos, head)] = scale;
    } else {
        put(reinterpret_cast<uint16_t *>(dst) + t0, x);
        put(reinterpret_cast<uint16_t *>(dst) + t1, x + 4);
    }
}

template <int D>
static void launch_write(const WriteArgs &a, bool halves, bool e4m3, hipStream_t s) {
    const int items = a.Hq + 2 * a.c.heads;
    const dim3 grid((unsigned)((items * (D / 8) + 255) / 256), (unsigned)a.r.n, (unsigned)a.r.B);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
    if (halves)
        e4m3 ? go(cache_write_kernel<D, true, true>) : go(cache_write_kernel<D, true, false>);
    else
        e4m3 ? go(cache_write_kernel<D, false, true>) : go(cache_write_kernel<D, false, false>);
}

}  // namespace pld

using namespace pld;

extern "C" int pld_model_version(void) { return PLD_MODEL_ABI_VERSION; }

extern "C" int pld_cache_write(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                               int64_t q_row_stride, const uint16_t *k, int64_t k_seq_stride,
                               int64_t k_row_stride, const uint16_t *v, int64_t v_seq_stride,
                               int64_t v_row_stride, const uint16_t *q_norm,
                               const uint16_t *k_norm, float eps, const float *rope,
                               int64_t rope_stride, int n_pos, int rot_dim, int rope_pairs,
                               const int32_t *lens, const int32_t *draft_len, int B, int n, int Hq,
                               uint16_t *q_out, int64_t o_seq_stride, int64_t o_row_stride,
                               void *stream) {
    WriteArgs a{};
    int rc = prep_cache(cache, true, a.c);
    if (rc == PLD_OK) rc = check_batch(cache, lens, B, n, Hq);
    if (rc != PLD_OK) return rc;
    const int64_t D = cache->head_dim, qw = Hq * D, kw = cache->heads * D;
    if ((rc = check_rows(q, q_seq_stride, q_row_stride, B, n, qw)) != PLD_OK ||
        (rc = check_rows(k, k_seq_stride, k_row_stride, B, n, kw)) != PLD_OK ||
        (rc = check_rows(v, v_seq_stride, v_row_stride, B, n, kw)) != PLD_OK ||
        (rc = check_rows(q_out, o_seq_stride, o_row_stride, B, n, qw)) != PLD_OK)
        return rc;
    if (q_out == q && ((B > 1 && o_seq_stride != q_seq_stride) || (n > 1 && o_row_stride != q_row_stride)))
        return PLD_ERR_INVALID;
    if (!(eps >= 0.f) || !isfinite(eps)) return PLD_ERR_INVALID;
    if ((uintptr_t)q_norm % 16 || (uintptr_t)k_norm % 16) return PLD_ERR_ALIGN;
    if (rope_pairs != PLD_ROPE_HALVES && rope_pairs != PLD_ROPE_NEIGHBOURS) return PLD_ERR_INVALID;
    if (rope) {
        if (n_pos < 1 || rot_dim < 8 || rot_dim > D || rot_dim % 8 || rope_stride < rot_dim)
            return PLD_ERR_INVALID;
        if ((uintptr_t)rope % 16 || rope_stride % 4) return PLD_ERR_ALIGN;
    }
    a.r = Rows{lens, draft_len, B, n};
    a.q = q, a.qs = q_seq_stride, a.qr = q_row_stride;
    a.k = k, a.ks = k_seq_stride, a.kr = k_row_stride;
    a.v = v, a.vs = v_seq_stride, a.vr = v_row_stride;
    a.qw = q_norm, a.kw = k_norm, a.eps = eps;
    a.rope = rope, a.rope_stride = rope_stride, a.n_pos = n_pos, a.rot = rope ? rot_dim : 0;
    a.Hq = Hq;
    a.out = q_out, a.os = o_seq_stride, a.orow = o_row_stride;
    const bool halves = rope_pairs == PLD_ROPE_HALVES, e4m3 = cache->dtype == PLD_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (D == 64)
        launch_write<64>(a, halves, e4m3, s);
    else if (D == 128)
        launch_write<128>(a, halves, e4m3, s);
    else
        launch_write<256>(a, halves, e4m3, s);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
