// pld_write_packed.hip -- packed rows join a layer's paged cache: pld_cache_write with the
// sequences' rows one behind the other and positions on several axes.
#include "pld_heads.h"
#include "pld_packed.h"

namespace pld {

struct PackedWriteArgs {
    CacheView c;
    Packed p;
    const int32_t *first;
    const uint16_t *q, *k, *v;
    int64_t qr, kr, vr;
    const uint16_t *qw, *kw;
    float eps;
    const float *rope;
    int64_t rope_stride;
    int n_pos, rot, Hq;
    const int32_t *pos, *pair_axis;   // or null
    int64_t axis_stride;
    int axes;
    uint16_t *out, *k_out;
    int64_t orow, korow;
};

// D / 8 lanes a head's row, as in cache_write_kernel, whose elements a lane has; kPer heads of a row in
// turn, which share the row's place and its angles.  Groups of heads of all rows are in one order, so that rows
// of few heads fill a block too.  Memory bounds many rows (17206 of 32 + 2 x 8 heads into e4m3: 104 us, 4.1 TB/s,
// 85% of a copy's rate), the search of the row's sequence, its page and its angles, one after the other, few
// (3.8 us).
template <int D, bool kHalves, bool kE4m3, int kPer>
__global__ __launch_bounds__(256) void cache_write_packed_kernel(PackedWriteArgs a) {
    constexpr int G = D / 8, kGroups = 256 / G;   // groups of heads of a block
    const int Hkv = a.c.heads, items = a.Hq + 2 * Hkv, groups = (items + kPer - 1) / kPer;
    const int64_t x0 = wide_block() * kGroups, row0 = quotient(x0, groups);
    if (row0 >= a.p.N) return;
    const uint32_t x = (uint32_t)(x0 - row0 * groups) + threadIdx.x / G;
    const int over = (int)(x / (uint32_t)groups), item0 = ((int)x - over * groups) * kPer;
    // (a row past the end is the last one again, and is not written)
    const bool past = row0 + over >= a.p.N;
    const int row = past ? a.p.N - 1 : (int)row0 + over;
    const int c = (int)threadIdx.x % G;
    auto kind_of = [&](int item) { return item < a.Hq ? 0 : item < a.Hq + Hkv ? 1 : 2; };   // query, key, value
    auto head_of = [&](int item, int kind) { return kind == 0 ? item : item - a.Hq - (kind == 2 ? Hkv : 0); };

    const bool mine = 8 * c < a.rot;   // this lane's runs are rotated
    const int near = kHalves && mine ? 4 * c : 8 * c, far = kHalves && mine ? a.rot / 2 + 4 * c : 8 * c + 4;
    uint2 in[kPer][2];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int item = min(item0 + j, items - 1), kind = kind_of(item);
        const uint16_t *src = kind == 0 ? a.q + row * a.qr : kind == 1 ? a.k + row * a.kr : a.v + row * a.vr;
        src += (int64_t)head_of(item, kind) * D;
        in[j][0] = *reinterpret_cast<const uint2 *>(src + (kind == 2 ? 8 * c : near));
        in[j][1] = *reinterpret_cast<const uint2 *>(src + (kind == 2 ? 8 * c + 4 : far));
    }
    // each axis' position of the row, and the axes of the lane's four pairs
    int at[PLD_MAX_AXES];
    int4 axis = make_int4(0, 0, 0, 0);
    if (a.pos) {
#pragma unroll
        for (int j = 0; j < PLD_MAX_AXES; ++j) at[j] = j < a.axes ? a.pos[j * a.axis_stride + row] : 0;
        if (a.pair_axis && mine) axis = *reinterpret_cast<const int4 *>(a.pair_axis + 4 * c);
    }
    const Span s = spans_of(a.p, row);
    if (s.b < 0 || past) return;
    const int64_t slot = (int64_t)a.first[s.b] + row - s.begin;
    const int page = slot >= 0 ? page_of(a.c, s.b, slot) : -1;
    int64_t pos[4] = {slot, slot, slot, slot};
    if (a.pos) {
        const int by[4] = {axis.x, axis.y, axis.z, axis.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int v = at[0];
#pragma unroll
            for (int j = 1; j < PLD_MAX_AXES; ++j) v = j < a.axes && by[e] == j ? at[j] : v;
            pos[e] = v;
        }
    }
    bool bad = page < 0;
    if (mine)
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (uint64_t)pos[e] >= (uint64_t)a.n_pos;
    // of any lane of the row (lanes that have returned are not in the ballot, but no part of a row has)
    const uint64_t group = ((1ull << G) - 1) << (lane_id() / G * G);
    const bool ok = !(__ballot(bad) & group);
    float cs[4], sn[4];
    if (mine && ok && item0 < a.Hq + Hkv) {
        const float *t = a.rope + 4 * c;
        if (pos[0] == pos[1] && pos[0] == pos[2] && pos[0] == pos[3]) {
            const float4 co = *reinterpret_cast<const float4 *>(t + pos[0] * a.rope_stride);
            const float4 si = *reinterpret_cast<const float4 *>(t + pos[0] * a.rope_stride + a.rot / 2);
            cs[0] = co.x, cs[1] = co.y, cs[2] = co.z, cs[3] = co.w;
            sn[0] = si.x, sn[1] = si.y, sn[2] = si.z, sn[3] = si.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cs[e] = t[pos[e] * a.rope_stride + e];
                sn[e] = t[pos[e] * a.rope_stride + a.rot / 2 + e];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int item = item0 + j;
        if (item >= items) break;
        const int kind = kind_of(item), head = head_of(item, kind);
        const int t0 = kind == 2 ? 8 * c : near, t1 = kind == 2 ? 8 * c + 4 : far;
        float y[8] = {bf16_lo(in[j][0].x), bf16_hi(in[j][0].x), bf16_lo(in[j][0].y), bf16_hi(in[j][0].y),
                      bf16_lo(in[j][1].x), bf16_hi(in[j][1].x), bf16_lo(in[j][1].y), bf16_hi(in[j][1].y)};
        const uint16_t *w = kind == 0 ? a.qw : kind == 1 ? a.kw : nullptr;
        if (w) norm_row<D>(y, w, t0, t1, a.eps);
        if (mine && ok && kind != 2) turn_row<kHalves>(y, cs, sn);
        if (kind != 2 && (kind == 0 || a.k_out)) {
            uint16_t *dst = kind == 0 ? a.out + row * a.orow : a.k_out + row * a.korow;
            dst += (int64_t)head * D;
            if (ok) {
                put4(dst + t0, y);
                put4(dst + t1, y + 4);
            } else {
                const uint2 nan = make_uint2(0x7fc07fc0u, 0x7fc07fc0u);
                *reinterpret_cast<uint2 *>(dst + t0) = nan;
                *reinterpret_cast<uint2 *>(dst + t1) = nan;
            }
        }
        if (kind == 0 || !ok) continue;
        char *dst = (kind == 1 ? a.c.k : a.c.v) + slot_at(a.c, page, slot, head);
        float *scale_to = kE4m3 ? (kind == 1 ? a.c.ks : a.c.vs) + scale_at(a.c, page, slot, head) : nullptr;
        store_row<D, kE4m3>(y, dst, t0, t1, scale_to, c == 0);
    }
}

template <int D, int kPer>
static void launch_write_packed(const PackedWriteArgs &a, bool halves, bool e4m3, hipStream_t s) {
    const int64_t groups = (int64_t)a.p.N * ((a.Hq + 2 * a.c.heads + kPer - 1) / kPer);
    const dim3 grid = wide_grid((groups * (D / 8) + 255) / 256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
    if (halves)
        e4m3 ? go(cache_write_packed_kernel<D, true, true, kPer>) : go(cache_write_packed_kernel<D, true, false, kPer>);
    else
        e4m3 ? go(cache_write_packed_kernel<D, false, true, kPer>) : go(cache_write_packed_kernel<D, false, false, kPer>);
}
template <int D>
static void launch_write_packed(const PackedWriteArgs &a, bool halves, bool e4m3, hipStream_t s) {
    // More heads a lane group share more, and leave fewer waves (32 + 2 x 8 heads of 128 into e4m3, three axes
    // in turns; 1, 2 and 4 heads): 64 rows 4.8, 5.1 and 7.0 us, 1088 rows 12.5, 11.0 and 13.6, 17206 rows (426 MB) 163,
    // 118 and 104, of the 88 that a copy's rate allows.  Eight are no better at any size.
    const int64_t lanes = (int64_t)a.p.N * (a.Hq + 2 * a.c.heads) * (D / 8);
    if (lanes >= 4000000)
        launch_write_packed<D, 4>(a, halves, e4m3, s);
    else if (lanes >= 400000)
        launch_write_packed<D, 2>(a, halves, e4m3, s);
    else
        launch_write_packed<D, 1>(a, halves, e4m3, s);
}

}  // namespace pld

using namespace pld;

extern "C" int pld_prompt_version(void) { return PLD_PROMPT_ABI_VERSION; }

extern "C" int pld_cache_write_packed(const pld_cache *cache, const uint16_t *q, int64_t q_row_stride,
                                      const uint16_t *k, int64_t k_row_stride, const uint16_t *v,
                                      int64_t v_row_stride, const uint16_t *q_norm, const uint16_t *k_norm,
                                      float eps, const float *rope, int64_t rope_stride, int n_pos,
                                      int rot_dim, int rope_pairs, const int32_t *positions, int axes,
                                      int64_t axis_stride, const int32_t *pair_axis, const int32_t *starts,
                                      const int32_t *first, int B, int N, int Hq, uint16_t *q_out,
                                      int64_t o_row_stride, uint16_t *k_out, int64_t ko_row_stride,
                                      void *stream) {
    PackedWriteArgs a{};
    int rc = prep_cache(cache, true, a.c);
    if (rc != PLD_OK) return rc;
    if (!starts || !first || B < 1 || B > 65535 || N < 1 || N > PLD_MAX_PACKED_ROWS || Hq < 1 || Hq > 4096 ||
        Hq % cache->heads)
        return PLD_ERR_INVALID;
    const int64_t D = cache->head_dim, qw = Hq * D, kw = cache->heads * D;
    constexpr int64_t most = 1ll << 31;
    if ((rc = check_packed(q, q_row_stride, N, qw, most)) != PLD_OK ||
        (rc = check_packed(k, k_row_stride, N, kw, most)) != PLD_OK ||
        (rc = check_packed(v, v_row_stride, N, kw, most)) != PLD_OK ||
        (rc = check_packed(q_out, o_row_stride, N, qw, most)) != PLD_OK ||
        (k_out && (rc = check_packed(k_out, ko_row_stride, N, kw, most)) != PLD_OK))
        return rc;
    if (N > 1 && ((q_out == q && o_row_stride != q_row_stride) || (k_out && k_out == k && ko_row_stride != k_row_stride)))
        return PLD_ERR_INVALID;
    if (!(eps >= 0.f) || !isfinite(eps)) return PLD_ERR_INVALID;
    if ((uintptr_t)q_norm % 16 || (uintptr_t)k_norm % 16 || ((uintptr_t)starts | (uintptr_t)first) % 4) return PLD_ERR_ALIGN;
    if (rope_pairs != PLD_ROPE_HALVES && rope_pairs != PLD_ROPE_NEIGHBOURS) return PLD_ERR_INVALID;
    if (rope) {
        if (n_pos < 1 || rot_dim < 8 || rot_dim > D || rot_dim % 8 || rope_stride < rot_dim || rope_stride > most)
            return PLD_ERR_INVALID;
        if ((uintptr_t)rope % 16 || rope_stride % 4) return PLD_ERR_ALIGN;
        if (positions && (axes < 1 || axes > PLD_MAX_AXES || (axes > 1 && axis_stride < N))) return PLD_ERR_INVALID;
        if ((uintptr_t)positions % 4 || (uintptr_t)pair_axis % 16) return PLD_ERR_ALIGN;
    }
    if (q_out == k || q_out == v || (k_out && (k_out == q || k_out == v || k_out == q_out))) return PLD_ERR_INVALID;
    a.p = Packed{starts, B, N};
    a.first = first;
    a.q = q, a.qr = q_row_stride, a.k = k, a.kr = k_row_stride, a.v = v, a.vr = v_row_stride;
    a.qw = q_norm, a.kw = k_norm, a.eps = eps;
    a.rope = rope, a.rope_stride = rope_stride, a.n_pos = n_pos, a.rot = rope ? rot_dim : 0, a.Hq = Hq;
    if (rope && positions) a.pos = positions, a.pair_axis = pair_axis, a.axes = axes, a.axis_stride = axis_stride;
    a.out = q_out, a.orow = o_row_stride, a.k_out = k_out, a.korow = ko_row_stride;
    const bool halves = rope_pairs == PLD_ROPE_HALVES, e4m3 = cache->dtype == PLD_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (D == 64)
        launch_write_packed<64>(a, halves, e4m3, s);
    else if (D == 128)
        launch_write_packed<128>(a, halves, e4m3, s);
    else
        launch_write_packed<256>(a, halves, e4m3, s);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
