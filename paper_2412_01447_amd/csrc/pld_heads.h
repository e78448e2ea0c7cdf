// pld_heads.h -- what the cache's writes share: reductions over the lanes of a head's row and
// the row's elements as they are loaded, normed, turned and stored.
#pragma once

#include "pld_cache.h"

namespace pld {

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

// Four bf16 elements as fp32, and back.
__device__ __forceinline__ void get4(const uint16_t *p, float *o) {
    const uint2 w = *reinterpret_cast<const uint2 *>(p);
    o[0] = bf16_lo(w.x), o[1] = bf16_hi(w.x), o[2] = bf16_lo(w.y), o[3] = bf16_hi(w.y);
}
__device__ __forceinline__ void put4(uint16_t *p, const float *o) {
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
}

// A lane's eight elements x, in two runs of four at t0 and t1, of a head's row of D.
template <int D>
__device__ __forceinline__ void norm_row(float (&x)[8], const uint16_t *w, int t0, int t1, float eps) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], x[e], s);
    const float inv = 1.f / sqrtf(group_sum<D / 8>(s) / (float)D + eps);
    float g[8];
    get4(w + t0, g);
    get4(w + t1, g + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
}
template <bool kHalves>
__device__ __forceinline__ void turn_row(float (&x)[8], const float (&cs)[4], const float (&sn)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float &p = kHalves ? x[e] : x[2 * e];
        float &r = kHalves ? x[e + 4] : x[2 * e + 1];
        // (as fused multiply-adds of one order, so that both writes give the same bits)
        const float np = fmaf(p, cs[e], -(r * sn[e])), nr = fmaf(p, sn[e], r * cs[e]);
        p = np;
        r = nr;
    }
}
// The row into its slot at dst (e4m3: the scale to *scale_at, by the lane of `first`).
template <int D, bool kE4m3>
__device__ __forceinline__ void store_row(float (&x)[8], char *dst, int t0, int t1, float *scale_to, bool first) {
    if constexpr (kE4m3) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));
        // a scale of at least the smallest normal number, so that the division stays finite
        const float scale = fmaxf(group_max<D / 8>(m) / kE4m3Max, 1.17549435e-38f);
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
        if (first) *scale_to = scale;
    } else {
        put4(reinterpret_cast<uint16_t *>(dst) + t0, x);
        put4(reinterpret_cast<uint16_t *>(dst) + t1, x + 4);
    }
}

}  // namespace pld
