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
    float scale;
    // The cap in the units of the scores, twice it, the score from which on soft_cap_near will not
    // do (all 0: no cap) and soft_cap's factor: taken here they would hold vector registers all along.
    float cap, cap_x2, cap_near, inv2_log2e;
    float nat;                      // from log2 units, as the scores have them, to natural ones
    int window;
    int G, groups;                  // query heads per key head; row groups per sequence
    uint32_t page16, slot16;        // strides of a page and a slot in 16 bytes
    uint32_t spage32;               // scale stride of a page
    uint16_t *out;
    int64_t os, orow;
    float *lse;
    float *partials;
    struct Opened *opened;          // [blocks]
    // the chosen heads' weights
    const int32_t *row, *heads;
    int R;
    float *attn;
    int64_t as, ar, n_keys;
};

// ------------------------------------------------------------ matrix tiles
// Everything is computed transposed, with v_mfma_f32_16x16x32_bf16: the scores
// as K Q^T, whose result gives lane (g, c) = (lane / 16, lane % 16) the scores of
// query c and keys 4g .. 4g+3 of a 16-key tile, and the output as V^T P^T.  The
// second product sums over keys in any order, as long as both operands have the
// same one, so its slot (g, e) is key 16 (e/4) + 4g + e%4 of a 32-key chunk: the
// weights are then the second product's operand where they are, without a move
// between lanes, and a lane's eight keys of V are eight row loads.  The rows of
// V^T are dealt to the tiles so that a lane's eight loads are whole vectors
// (D / 16 elements) of a V row and one byte permute a pair of keys makes an operand.
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ bf16x8_t as_bf16x8(uint4 v) { return __builtin_bit_cast(bf16x8_t, v); }
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8_t, v); }
__device__ __forceinline__ f32x4_t mfma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Two of the four e4m3 values in v as bf16 (exact).
template <bool kHi>
__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t v) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, kHi));
}
// A value that is the same in every lane, as a scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
// Maximum over the four lanes of a query.
__device__ __forceinline__ float query_max(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float query_sum(float v) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// --------------------------------------------------------------- the work
// An item is one key head's rows of one sequence, up to 16 kMT of them (row m is
// query head m % G of row m / G), over the units of 128 keys that they see.  All
// items' units, in order of (sequence, row group, key head, unit), are dealt to the
// blocks in equal contiguous ranges, whatever the sequences' lengths; an item that
// spans blocks leaves one partial result per block, joined by a second launch.
constexpr int kUnit = 128;        // keys
// Two per CU; nothing depends on their being resident at once.  Twice as many cost a start
// and a join more than evener ends gain: 35 us become 47 (8 sequences of 4096, 11 rows), and
// 510 become 540 (4 of 131072, 33 rows).
constexpr int kAttnBlocks = 512;

struct Item {
    int b, cnt, pos0, r0, rows;   // rows: of this group
    int lo, hi;                   // keys that some row sees: [lo, hi)
    int units;                    // 0: no rows
};

__device__ __forceinline__ Item make_item(const AttnArgs &a, int e, int R, int cnt, int pos0) {
    Item it;
    it.b = a.groups == 1 ? e : e / a.groups;
    it.cnt = cnt;
    it.pos0 = pos0;
    it.r0 = (e - it.b * a.groups) * R;
    it.rows = min(it.cnt * a.G - it.r0, R);
    it.units = 0;
    if (it.rows <= 0) return it;
    const int64_t cap = (int64_t)a.c.max_pages << a.c.shift;
    const int64_t p0 = (int64_t)it.pos0 + it.r0 / a.G;
    const int64_t p1 = (int64_t)it.pos0 + (it.r0 + it.rows - 1) / a.G;
    it.lo = a.window && p0 + 1 > a.window ? (int)min(p0 + 1 - a.window, cap) : 0;
    it.hi = (int)min(p1 + 1, cap);
    // rows past the table's end have no keys here, but are written
    it.units = max(1, (it.hi + kUnit - 1) / kUnit - it.lo / kUnit);
    return it;
}

__device__ __forceinline__ Item item_of(const AttnArgs &a, int e, int R) {
    int pos0;
    const int cnt = row_count(a.r, a.groups == 1 ? e : e / a.groups, pos0);
    return make_item(a, e, R, cnt, pos0);
}

// An item that begins in a block's range and ends in a later one.
struct Opened {
    int e, kv, last, pos0;   // entry (-1: none), key head, last block, of the sequence
    int rows, b, r0, pad;    // as in Item
};
constexpr Opened kNothing = {-1, 0, 0, 0, 0, 0, 0, 0};

// The part of all units that is this block's, by each block from the lengths: there are
// as many ranges as blocks, or as units where those are fewer, so that none between
// two others is empty.
struct Range {
    int64_t x0, x1;          // [x0, x1) of all units
    int64_t per;             // units of a range; the first `longer` ranges have one more
    int longer;
    int e;                   // the entry (sequence and row group) of unit x0
    Item it;                 // that entry's
    int64_t first;           // its first unit
    __device__ __forceinline__ int block_of(int64_t x) const {
        const int64_t of_longer = (per + 1) * longer;
        return (int)(x < of_longer ? quotient(x, per + 1) : longer + quotient(x - of_longer, per));
    }
};
__device__ __forceinline__ Range block_range(const AttnArgs &a, int R, int64_t *s_w, int *s_e) {
    const int lane = lane_id(), wave = uniform((int)threadIdx.x / 64);
    const int entries = a.r.B * a.groups, per = (entries + 255) / 256;
    const int e0 = min((int)threadIdx.x * per, entries), e1 = min(e0 + per, entries);
    int64_t mine = 0;
    Item it;   // of the thread's last entry
    for (int e = e0; e < e1; ++e) {
        it = item_of(a, e, R);
        mine += it.units;
    }
    mine *= a.c.heads;
    int64_t before = wave_incl_scan(mine);
    if (lane == 63) s_w[wave] = before;
    __syncthreads();
    Range r;
    int64_t total = 0;
    before -= mine;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += s_w[w];
        total += s_w[w];
    }
    total = uniform(total);
    const int64_t ranges = min(total, (int64_t)gridDim.x), block = blockIdx.x;
    r.per = ranges ? quotient(total, ranges) : 0;
    r.longer = (int)(total - r.per * ranges);
    r.x0 = block < ranges ? r.per * block + min(block, (int64_t)r.longer) : total;
    r.x1 = block < ranges ? r.x0 + r.per + (block < r.longer) : total;
    if (before <= r.x0 && r.x0 < before + mine) {
        // the thread whose entries hold x0 steps to the one that does
        int e = e0;
        if (per > 1) it = item_of(a, e, R);
        for (int64_t u; r.x0 >= before + (u = (int64_t)it.units * a.c.heads); it = item_of(a, ++e, R)) before += u;
        s_e[0] = e;
        s_e[1] = it.cnt;
        s_e[2] = it.pos0;
        s_w[4] = before;
    }
    __syncthreads();
    if (r.x0 >= r.x1) return r;
    r.e = uniform(s_e[0]);
    r.it = make_item(a, r.e, R, uniform(s_e[1]), uniform(s_e[2]));
    r.first = uniform(s_w[4]);
    return r;
}

// Loads at a uniform address plus 32-bit offsets, a lane's and a scalar one: no vector
// arithmetic for addresses.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void *p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0x7fffffff, 0x00027000);
}
template <int kAux = 0>
__device__ __forceinline__ u32x4_t buffer_load16(__amdgpu_buffer_rsrc_t b, uint32_t off, uint32_t soff) {
    return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(b, off, soff, kAux));
}
// kAux of rows that one block reads once: without it the caches keep what nobody asks for
// again (64 sequences of 8192 tokens, 8 heads of 128 in bf16: 367 us without, 331 with it).
// Not for rows of half a 128-byte line, whose other half is the next head's, read by another
// block (32 heads of 64 in e4m3, slot by slot: 376 without and 391 with it for 16 sequences of
// 16384 in pages of 16, though 419 and 377 for 32 of 8192 in pages of 64; head by head 198 to
// 204 either way), and not in the wide form, whose keys other row groups read too (4 x 2048 rows
// over 8192 tokens: 1510 without, 1880 with it).
template <int D, bool kE4m3>
constexpr int kOnce = D * (kE4m3 ? 1 : 2) >= 128 ? 2 : 0;
template <int kBytes, int kAux = 0, int W>
__device__ __forceinline__ void buffer_load(uint32_t (&v)[W], __amdgpu_buffer_rsrc_t b, uint32_t off, uint32_t soff) {
    if constexpr (kBytes == 2) {
        v[0] = __builtin_amdgcn_raw_buffer_load_b16(b, off, soff, kAux);
    } else if constexpr (kBytes == 4) {
        v[0] = __builtin_amdgcn_raw_buffer_load_b32(b, off, soff, kAux);
    } else if constexpr (kBytes == 8) {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(b, off, soff, kAux);
        v[0] = w[0], v[1] = w[1];
    } else {
        const auto w = __builtin_amdgcn_raw_buffer_load_b128(b, off, soff, kAux);
        v[0] = w[0], v[1] = w[1], v[2] = w[2], v[3] = w[3];
    }
}

// The pages of T tiles of 16 keys: lane l stands for key l % (16 T) of those from k0 on.
// load_entry takes the table's entries (the last key's page stands in for keys past the
// end), a step ahead; take_tiles makes addresses of them.  A page that cannot be read is 0,
// with a bit in `bad` for each of its keys that the item has.
template <int T>
__device__ __forceinline__ int load_entry(const AttnArgs &a, const Item &it, int k0) {
    const int j = min(k0 + (lane_id() & (16 * T - 1)), it.hi - 1);
    return a.c.table[(int64_t)it.b * a.c.table_stride + (j >> a.c.shift)];
}
struct Tiles {
    uint64_t at;       // of the first row of this lane's tile, in 16 bytes
    int64_t scale;     // of this lane's key
    uint64_t bad;
    // Tile t's first row in bytes, from a uniform t.
    __device__ __forceinline__ int64_t row(int t) const { return (int64_t)(read(at, 16 * t) << 4); }
    __device__ __forceinline__ int64_t first_scale(int t) const { return (int64_t)read((uint64_t)scale, 16 * t); }
    __device__ __forceinline__ static uint64_t read(uint64_t v, int l) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)v, l);
    }
};
template <int T, bool kScales>
__device__ __forceinline__ Tiles take_tiles(const AttnArgs &a, const Item &it, int k0, int entry, int kv) {
    Tiles r;
    const bool ok = (uint32_t)entry < (uint32_t)a.c.num_pages;
    const uint32_t page = ok ? entry : 0, mask = (1u << a.c.shift) - 1;
    const int j = k0 + (lane_id() & (16 * T - 1));
    r.at = (uint64_t)page * a.page16 + (uint64_t)((uint32_t)j & mask & ~15u) * a.slot16;
    if constexpr (kScales) r.scale = (int64_t)((uint64_t)page * a.spage32 + (((uint32_t)kv << a.c.shift) + ((uint32_t)j & mask)));
    r.bad = __ballot(!ok && j < it.hi);
    return r;
}

// The keys of T 16-key tiles on their way to being operands.  As an operand a lane has one
// key's row in pieces of 16 bytes, g of each four; loaded like that, an instruction reads 64
// bytes of each of 16 rows, and a read of a large cache reaches 5.1 TB/s where whole rows
// side by side reach 6.3.  So rows are loaded whole, kLanes lanes each, and turned in LDS,
// in a part of a wave's own.  Piece p of key k goes to unit 16 p + (k ^ p % 16) of its
// tile: neither side meets a bank twice.
template <int D, bool kE4m3, int T>
struct KeyRows {
    static constexpr int kLanes = D * (kE4m3 ? 1 : 2) / 16;    // lanes of a row: 4 .. 32
    static constexpr int kRows = kWave / kLanes;               // rows of a load
    static constexpr int kLoads = 16 * T / kRows;
    static constexpr int kPieces = kLanes / 4;                 // operand pieces a lane
    u32x4_t r[kLoads];

    __device__ __forceinline__ static int row() { return lane_id() / kLanes; }
    __device__ __forceinline__ static int piece() { return lane_id() % kLanes; }
    // off: row() slot + 16 piece(); at(t): tile t's address
    template <int kAux, class At>
    __device__ __forceinline__ void load(uint32_t off, uint32_t slot, At at) {
        __amdgpu_buffer_rsrc_t buf;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (i * kRows % 16 == 0) buf = buffer_at(at(i * kRows / 16));
            r[i] = buffer_load16<kAux>(buf, off, i * kRows % 16 * slot);
        }
    }
    __device__ __forceinline__ static int unit(int key, int piece) { return 16 * piece + ((key ^ piece) & 15); }
    __device__ __forceinline__ void store(u32x4_t (*lds)[kPieces * kWave]) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) lds[i * kRows / 16][unit(i * kRows + row(), piece())] = r[i];
    }
    // Piece f of this lane's key of tile t: key lane % 16, bytes 64 f + 16 (lane / 16) on.
    __device__ __forceinline__ static u32x4_t read(const u32x4_t (*lds)[kPieces * kWave], int t, int f) {
        return lds[t][unit(lane_id() & 15, 4 * f + (lane_id() >> 4))];
    }
};
// Operand s of a head's row from its pieces: bf16 has one a piece, e4m3 two.
template <bool kE4m3>
__device__ __forceinline__ bf16x8_t key_operand(u32x4_t piece, int s) {
    if constexpr (kE4m3) {
        const uint32_t w0 = s & 1 ? piece.z : piece.x, w1 = s & 1 ? piece.w : piece.y;
        return as_bf16x8(u32x4_t{e4m3_bf16<false>(w0), e4m3_bf16<true>(w0), e4m3_bf16<false>(w1), e4m3_bf16<true>(w1)});
    } else {
        return as_bf16x8(piece);
    }
}

// The log sum from a maximum in the scores' log2 units and the weights' sum.
__device__ __forceinline__ float log_sum(const AttnArgs &a, float m, float l) {
    return fmaf(m, a.nat, __log2f(l) * kLn2);
}

// Where a partial result is: blocks keep one of an item that began before their
// range (slot 0) and one of an item that ends after it (slot 1).
template <int D>
__device__ __forceinline__ float *partial_at(const AttnArgs &a, int block, int slot, int R) {
    return a.partials + ((int64_t)block * 2 + slot) * R * (D + 2);
}

template <int D>
__device__ __forceinline__ void put_row(const AttnArgs &a, const Item &it, int kv, int m, int64_t &o,
                                        int64_t &l, bool &gone) {
    const int i = (it.r0 + m) / a.G, h = kv * a.G + (it.r0 + m) % a.G;
    o = (int64_t)it.b * a.os + (int64_t)i * a.orow + (int64_t)h * D;
    l = ((int64_t)it.b * a.r.n + i) * a.Hq + h;
    gone = (int64_t)it.pos0 + i >= ((int64_t)a.c.max_pages << a.c.shift);
}

// ------------------------------------------------- 32 keys against 16 queries
// A lane's products q.k: x[t][r] of key 16 t + 4 g + r.  What a query sees of the keys, where
// it may not be all of them: j0 <= j < j1 counted from x[0][0]'s key, and the keys (a bit
// each, this lane's first one lowest) that turn what sees them into NaN.
struct Seen {
    int j0, j1;
    uint32_t nan;
};
__device__ __forceinline__ void mask_scores(f32x4_t (&x)[2], const Seen &see) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * t + r;
            const float v = (see.nan >> j) & 1 ? __uint_as_float(0x7fc00000u) : x[t][r];
            x[t][r] = j >= see.j0 && j < see.j1 ? v : -INFINITY;
        }
}
__device__ __forceinline__ float max_of(const f32x4_t (&x)[2]) {
    return fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                 fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
}

// Products into scores; returns the factor that is left to their units (c1, where it is the
// same for all keys and no cap comes between): log2 units in the attention, whose weights are
// then one fused multiply-add and 2^x, natural ones for the chosen heads' weights.  ks: the keys' scales times c1.
template <bool kE4m3>
__device__ __forceinline__ float scale_scores(const AttnArgs &a, f32x4_t (&x)[2], float c1, f32x4_t ks0,
                                              f32x4_t ks1) {
    if constexpr (kE4m3) {
        x[0] *= ks0;
        x[1] *= ks1;
        c1 = 1.f;
    }
    if (a.cap > 0.f) {
        float w = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            x[t] *= c1;
#pragma unroll
            for (int r = 0; r < 4; ++r) w = fmaxf(w, fabsf(x[t][r]));
        }
        // One branch for the wave: few scores come to a third of the cap as a rule (64 x 17 rows
        // over 16384 tokens in e4m3, cap 50: 1060 us, 1300 with both forms for every score; where
        // every wave has such a score, cap 8, 1480).
        if (__any(w >= a.cap_near)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[t][r] = soft_cap(x[t][r], a.cap, a.cap_x2, a.cap_near, a.inv2_log2e);
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[t][r] = soft_cap_near(x[t][r], a.inv2_log2e);
        }
        c1 = 1.f;
    }
    return c1;
}
// Scores into weights 2^(x c - m), with the running maximum m of the query (the same in its
// four lanes) and the sum l of this lane's keys.  The maximum is raised, and output and sum
// are rescaled, only where a score of any query of the tile is kSlack above it: weights of
// up to 2^kSlack lose nothing in fp32 and bf16, and what random scores still grow by after a
// few keys seldom comes that far.
constexpr float kSlack = 8.f;
constexpr float kNoMax = -1e30f;   // of a query that has seen no key
template <int NJ>
__device__ __forceinline__ void weigh(f32x4_t (&x)[2], float c, float &m, float &l, f32x4_t (&o)[NJ]) {
    const float mx = max_of(x) * c;
    if (__any(mx > m + kSlack)) {
        const float mn = fmaxf(m, query_max(mx));
        const float f = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] *= f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[t][r] = __builtin_amdgcn_exp2f(fmaf(x[t][r], c, -m));
            l += x[t][r];
        }
}
// The weights as an operand, rounded to bf16: the matrix product takes no wider ones, and
// half a step (2^-8) of each term is no more than the output's own rounding.
__device__ __forceinline__ bf16x8_t weight_operand(const f32x4_t (&x)[2]) {
    return as_bf16x8(make_uint4(pack_bf16(x[0][0], x[0][1]), pack_bf16(x[0][2], x[0][3]),
                                pack_bf16(x[1][0], x[1][1]), pack_bf16(x[1][2], x[1][3])));
}
// Eight values of an element of two bf16 (word w of each key's) as an operand.
template <int N, int W>
__device__ __forceinline__ bf16x8_t value_operand(const uint32_t (&vp)[8][N][W], int v, int w, bool hi) {
    const uint32_t sel = hi ? 0x07060302u : 0x05040100u;
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_perm(vp[2 * i + 1][v][w], vp[2 * i][v][w], sel);
    return as_bf16x8(make_uint4(r[0], r[1], r[2], r[3]));
}

// Four waves a block, each with all of the item's rows and 32 of a unit's keys.  Bound by
// HBM where there is much to read: 64 sequences of 8192, a row of 32 query heads over 8 key
// heads of 128 in bf16 (2.15 GB): 331 us, 6.5 TB/s; in e4m3 64 of 16384: 367 us.  By the way
// of one dependent load to the next (lengths, page entries, keys, partial results) where there
// is little: 10.3 us for one row over 1024 tokens, both launches.
template <int D, bool kE4m3, int kMT>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_attn_kernel(AttnArgs a) {
    constexpr int R = 16 * kMT;
    constexpr int S = D / 32;            // products over a head's elements
    constexpr int NJ = D / 16;           // output tiles
    constexpr int NV = D > 128 ? 2 : 1;  // vector loads of a V row
    constexpr int VE = D / 16 / NV;      // their elements
    constexpr int VW = VE * (kE4m3 ? 1 : 2) / 4;       // words of a V load
    using Keys = KeyRows<D, kE4m3, 2>;
    __shared__ uint4 s_q[kMT][S][64];
    __shared__ u32x4_t s_keys[4][2][Keys::kPieces * 64];
    __shared__ float s_ml[2][4][R];
    __shared__ float s_o[4][kMT][NJ][64];
    __shared__ int64_t s_w[8];
    __shared__ int s_e[3];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int g = lane >> 4, c = lane & 15;

    const Range rg = block_range(a, R, s_w, s_e);
    int e = rg.e;
    Item it = rg.it;
    int64_t x = rg.x0, first = rg.first;    // first unit of entry e
    Opened opened = kNothing;
    const float c1 = a.scale * kLog2E;
    while (x < rg.x1) {
        const int64_t span = (int64_t)it.units * a.c.heads;
        if (x >= first + span) {
            first += span;
            it = item_of(a, ++e, R);
            continue;
        }
        const int kv = (int)quotient(x - first, it.units);
        const int u0 = (int)((x - first) - (int64_t)kv * it.units);
        const int u1 = (int)min((int64_t)it.units, u0 + (rg.x1 - x));
        x += u1 - u0;

        const int ubase = it.lo / kUnit;
        const int kbase = (ubase + u0) * kUnit + 32 * wave, kend = (ubase + u1) * kUnit;
        int entry = load_entry<2>(a, it, kbase);

        // The rows' queries, as operands in LDS (in registers they would cost a wave the
        // room for its loads): asked for here, put there once the first keys are asked for.
        constexpr int kQ = (kMT * S + 3) / 4;   // a wave's pieces
        u32x4_t qv[kQ];
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
            const int piece = min(4 * u + wave, kMT * S - 1), t = piece / S, s = piece % S;
            const int m = min(16 * t + c, it.rows - 1);
            const int i = (it.r0 + m) / a.G, h = kv * a.G + (it.r0 + m) % a.G;
            const uint16_t *qp =
                a.q + (int64_t)it.b * a.qs + (int64_t)i * a.qr + (int64_t)h * D;
            const int d = kE4m3 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            qv[u] = *reinterpret_cast<const u32x4_t *>(qp + d);
        }
        // keys that every row sees: [all_lo, all_hi)
        const int64_t pf = (int64_t)it.pos0 + it.r0 / a.G;
        const int64_t pl = (int64_t)it.pos0 + (it.r0 + it.rows - 1) / a.G;
        const int all_hi = (int)min(pf + 1, (int64_t)it.hi);
        const int all_lo = a.window && pl + 1 > a.window ? (int)min(pl + 1 - a.window, (int64_t)1 << 30) : 0;

        Keys kr;
        uint32_t vr[8][NV][VW];
        f32x4_t kf[2], vf[2];
        uint32_t bad = 0;   // the chunk's keys on bad pages

        const char *kh = a.c.k + (int64_t)kv * a.c.head, *vh = a.c.v + (int64_t)kv * a.c.head;
        const uint32_t slot = (uint32_t)a.c.slot;
        const uint32_t k_off = (uint32_t)Keys::row() * slot + 16 * Keys::piece(), v_off = 4 * (uint32_t)g * slot + c * (4 * VW);
        auto load_k = [&](const Tiles &tl) {
            kr.template load<kOnce<D, kE4m3>>(k_off, slot, [&](int t) { return kh + tl.row(t); });
            if constexpr (kE4m3)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    kf[t] = __builtin_bit_cast(f32x4_t, buffer_load16(buffer_at(a.c.ks + tl.first_scale(t)), 16 * g, 0));
        };
        auto load_v = [&](const Tiles &tl) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const auto buf = buffer_at(vh + tl.row(t));
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
                        buffer_load<4 * VW, kOnce<D, kE4m3>>(vr[4 * t + i][v], buf, v_off + v * (64 * VW), i * slot);
                if constexpr (kE4m3)
                    vf[t] = __builtin_bit_cast(f32x4_t, buffer_load16(buffer_at(a.c.vs + tl.first_scale(t)), 16 * g, 0));
            }
        };

        Tiles tl = take_tiles<2, kE4m3>(a, it, kbase, entry, kv);
        entry = load_entry<2>(a, it, kbase + kUnit);   // ahead of the loads that go by it
        load_k(tl);
        load_v(tl);
        int see_lo[kMT], see_hi[kMT];   // the keys that each lane's queries see
#pragma unroll
        for (int t = 0; t < kMT; ++t) {
            const int64_t p = (int64_t)it.pos0 + (it.r0 + min(16 * t + c, it.rows - 1)) / a.G;
            see_hi[t] = (int)min(p + 1, (int64_t)it.hi);
            see_lo[t] = a.window && p + 1 > a.window ? (int)min(p + 1 - a.window, (int64_t)1 << 30) : 0;
        }
        f32x4_t o[kMT][NJ];
        float m[kMT], l[kMT];   // log2 units; l: of this lane's keys
#pragma unroll
        for (int t = 0; t < kMT; ++t) {
            m[t] = kNoMax;
            l[t] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[t][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }

        __syncthreads();   // the item before is done with LDS
#pragma unroll
        for (int u = 0; u < kQ; ++u) {
            const int piece = min(4 * u + wave, kMT * S - 1);   // (a last piece twice is the same)
            s_q[piece / S][piece % S][lane] = __builtin_bit_cast(uint4, qv[u]);
        }
        __syncthreads();
        for (int k0 = kbase; k0 < kend; k0 += kUnit) {
            asm volatile("" ::: "memory");   // the queries are read from LDS anew
            const bool more = k0 + kUnit < kend;
            bad = (uint32_t)tl.bad;
            if (more) {
                tl = take_tiles<2, kE4m3>(a, it, k0 + kUnit, entry, kv);
                entry = load_entry<2>(a, it, k0 + 2 * kUnit);
            }
            const bool plain = k0 >= all_lo && k0 + 32 <= all_hi && bad == 0;   // every row sees every key

            kr.store(s_keys[wave]);
            f32x4_t ks[2];
            if constexpr (kE4m3) ks[0] = kf[0] * c1, ks[1] = kf[1] * c1;
            asm volatile("" ::: "memory");
            if (more) load_k(tl);
            f32x4_t x[kMT][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int n = 0; n < kMT; ++n) x[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const bf16x8_t k = key_operand<kE4m3>(Keys::read(s_keys[wave], t, kE4m3 ? s / 2 : s), s);
#pragma unroll
                    for (int n = 0; n < kMT; ++n) x[n][t] = mfma(k, as_bf16x8(s_q[n][s][lane]), x[n][t]);
                }
            }

#pragma unroll
            for (int n = 0; n < kMT; ++n) {
                const float sc = scale_scores<kE4m3>(a, x[n], c1, ks[0], ks[1]);
                const int j = k0 + 4 * g;
                if (!plain) mask_scores(x[n], Seen{see_lo[n] - j, see_hi[n] - j, bad >> (4 * g)});
                weigh<NJ>(x[n], sc, m[n], l[n], o[n]);
            }
            if constexpr (kE4m3) {
                if (!plain) {
                    // a scale that is not finite, as with the values below
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (fabsf(vf[i / 4][i % 4]) < INFINITY) continue;
                        const int j = k0 + 16 * (i / 4) + 4 * g + i % 4;
                        vf[i / 4][i % 4] = 0.f;
#pragma unroll
                        for (int n = 0; n < kMT; ++n)
                            if (j >= see_lo[n] && j < see_hi[n]) x[n][i / 4][i % 4] = __uint_as_float(0x7fc00000u);
                    }
                }
#pragma unroll
                for (int n = 0; n < kMT; ++n) {
                    x[n][0] *= vf[0];
                    x[n][1] *= vf[1];
                }
            }
            // A product by a weight of 0 would let through what is not finite in a value that
            // not every row sees.  It becomes 0, and where it was not finite, the weights of
            // the rows that do see it become NaN.  vp: V as bf16 pairs, [key][element / 2].
            auto mask_values = [&](uint32_t (&vp)[8][NV][VE / 2]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int j = k0 + 16 * (i / 4) + 4 * g + i % 4;
                    const bool any = j >= it.lo && j < it.hi, every = j >= all_lo && j < all_hi;
                    bool odd = false;
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int w = 0; w < VE / 2; ++w) {
                            const uint32_t y = vp[i][v][w];
                            odd |= (y & 0x7f80u) == 0x7f80u || (y & 0x7f800000u) == 0x7f800000u;
                        }
                    const bool row_odd = (__ballot(odd && any && !every) >> (16 * g) & 0xffff) != 0;
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int w = 0; w < VE / 2; ++w)
                            if (!any || row_odd) vp[i][v][w] = 0;
#pragma unroll
                    for (int n = 0; n < kMT; ++n)
                        if (row_odd && j >= see_lo[n] && j < see_hi[n])
                            x[n][i / 4][i % 4] = __uint_as_float(0x7fc00000u);
                    __builtin_amdgcn_sched_barrier(0);   // key by key: all at once take too many registers
                }
            };
            auto add_product = [&](const uint32_t (&vp)[8][NV][VE / 2]) {
                bf16x8_t p[kMT];
#pragma unroll
                for (int n = 0; n < kMT; ++n) p[n] = weight_operand(x[n]);
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const bf16x8_t vj = value_operand(vp, j / VE, j % VE / 2, j & 1);
#pragma unroll
                    for (int n = 0; n < kMT; ++n) o[n][j] = mfma(vj, p[n], o[n][j]);
                }
            };
            if constexpr (kE4m3) {
                uint32_t vp[8][NV][VE / 2];
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int w = 0; w < VE / 2; ++w)
                            vp[i][v][w] = w & 1 ? e4m3_bf16<true>(vr[i][v][w / 2]) : e4m3_bf16<false>(vr[i][v][w / 2]);
                if (!plain) mask_values(vp);
                add_product(vp);
            } else {
                if (!plain) mask_values(vr);
                add_product(vr);
            }
            if (more) load_v(tl);
        }

        // The four waves' results joined: a common maximum, then, for each register r of
        // the output tiles in turn, the sum by wave r (it holds whole vectors of a row).
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kMT; ++t) {
            const float lq = query_sum(l[t]);
            if (g == 0) {
                s_ml[0][wave][16 * t + c] = m[t];
                s_ml[1][wave][16 * t + c] = lq;
            }
        }
        __syncthreads();
        const bool whole = u0 == 0 && u1 == it.units;
        float *part = partial_at<D>(a, blockIdx.x, u0 == 0, R);
        float mg[kMT], lg[kMT];
#pragma unroll
        for (int t = 0; t < kMT; ++t) {
            const int r = 16 * t + c;
            mg[t] = fmaxf(fmaxf(s_ml[0][0][r], s_ml[0][1][r]), fmaxf(s_ml[0][2][r], s_ml[0][3][r]));
            lg[t] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) lg[t] += s_ml[1][w][r] * __builtin_amdgcn_exp2f(s_ml[0][w][r] - mg[t]);
            const float f = __builtin_amdgcn_exp2f(m[t] - mg[t]);
#pragma unroll
            for (int j = 0; j < NJ; ++j) o[t][j] *= f;
        }
        const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (r) __syncthreads();
#pragma unroll
            for (int t = 0; t < kMT; ++t)
#pragma unroll
                for (int j = 0; j < NJ; ++j) s_o[wave][t][j][lane] = o[t][j][r];
            __syncthreads();
            if (wave != r) continue;
#pragma unroll
            for (int t = 0; t < kMT; ++t) {
                const int row = 16 * t + c;
                if (row >= it.rows) continue;
                int64_t oat, lat;
                bool gone;
                put_row<D>(a, it, kv, row, oat, lat, gone);
                const float inv = 1.f / lg[t];
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float y[VE];
#pragma unroll
                    for (int j = 0; j < VE; ++j) {
                        const int jj = v * VE + j;
                        y[j] = (s_o[0][t][jj][lane] + s_o[1][t][jj][lane]) + (s_o[2][t][jj][lane] + s_o[3][t][jj][lane]);
                    }
                    const int d = (D / NV) * v + VE * (4 * g + r);
                    if (whole) {
                        uint32_t w[VE / 2];
#pragma unroll
                        for (int j = 0; j < VE / 2; ++j)
                            w[j] = gone ? 0x7fc07fc0u : pack_bf16(y[2 * j] * inv, y[2 * j + 1] * inv);
                        __builtin_memcpy(__builtin_assume_aligned(a.out + oat + d, 2 * VE), w, 2 * VE);
                    } else {
                        __builtin_memcpy(__builtin_assume_aligned(part + row * D + d, 16), y, 4 * VE);
                    }
                }
                if (r == 0 && g == 0) {
                    if (whole) {
                        if (a.lse) a.lse[lat] = gone ? nan : log_sum(a, mg[t], lg[t]);
                    } else {
                        part[R * D + 2 * row] = mg[t];
                        part[R * D + 2 * row + 1] = lg[t];
                    }
                }
            }
        }
        if (u0 == 0 && !whole) {
            const int64_t end = first + (int64_t)(kv + 1) * it.units;   // of the item
            opened = Opened{e, kv, rg.block_of(end - 1), it.pos0, it.rows, it.b, it.r0, 0};
        }
    }
    if (threadIdx.x == 0) a.opened[blockIdx.x] = opened;
}

// More rows: a block's waves share the keys and each has tiles of 16 rows of its own,
// wave w the tiles w, w+4, w+8.  Keys and values of 64 positions go through LDS once,
// as operands: each wave fetches a 16-key tile of K and, of 32 keys, half the elements
// of V, into registers while the block works on the 64 before, and turns them (e4m3 to
// bf16, V to pairs of keys) once for all waves on the way to LDS.  16 x 8 rows of 8 heads a key
// head over 8192 tokens: 133 us, 4.1 TB/s, of which the slowest XCD is 20 us behind the mean.
// With three tiles a wave it is the instructions: 64 x 17 such rows over 16384 tokens in
// e4m3 (144 rows a key head) take 840 us, 530 TFLOP/s, the matrix units busy for 27% of the time and
// the vector units for 46%, two waves a SIMD (512 registers hold no third) waiting for the
// rest; 4 x 33 rows of 4 heads a key head over 131072 tokens in bf16 490 to 515 us, some 560 TFLOP/s
// and 4.3 TB/s.
// (A ninth tile as two waves' work, half the keys each, took 5% longer.)
constexpr int kStep = 64;   // keys
template <int D, int kMT>
struct WideLds {
    static constexpr bool kThird = kMT > 2;             // some waves have a third tile
    u32x4_t k[2][4][D / 32][64], v[2][2][D / 16][64];   // operands of two steps
    u32x4_t q[kThird ? 3 : 1][D / 32][kThird ? 64 : 1]; // the queries of tiles 8 .. 10
    f32x4_t scale[2][2][kStep / 4];
    uint32_t odd[2][2][3];                              // [step][32 keys][half; scales]: not finite
};

// A wave's whole work on an item, with NT tiles of its own (from tile0 on, every fourth):
// a block's waves meet at the same barriers whatever their NT.
template <int D, bool kE4m3, int NT, int kMT>
__device__ __forceinline__ void wide_segment(const AttnArgs &a, WideLds<D, kMT> &lds, const Item &it, int kv,
                                             int u0, int u1, int tile0, int R) {
    constexpr int S = D / 32, NJ = D / 16, NA = NT ? NT : 1;
    constexpr int KL = kE4m3 ? S / 2 : S;           // 16-byte loads of a key's row per lane
    constexpr int VE = NJ / 2;                      // elements of a wave's V loads
    constexpr int VB = VE * (kE4m3 ? 1 : 2);        // their bytes: 2 .. 16
    constexpr int VW = (VB + 3) / 4;
    const int lane = lane_id(), wave = uniform((int)threadIdx.x / 64);
    const int g = lane >> 4, c = lane & 15;
    const float c1 = a.scale * kLog2E;
    const int kbase = (it.lo / kUnit + u0) * kUnit, kend = (it.lo / kUnit + u1) * kUnit;
    int entry = load_entry<4>(a, it, kbase);
    constexpr int kQ = NT > 2 ? 2 : NT;   // tiles whose queries stay in registers
    bf16x8_t q[NT > 2 ? 2 : NA][S];
    int see_lo[NA], see_hi[NA];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int m = min(16 * (tile0 + 4 * t) + c, it.rows - 1);
        const int i = (it.r0 + m) / a.G, h = kv * a.G + (it.r0 + m) % a.G;
        const uint16_t *qp = a.q + (int64_t)it.b * a.qs + (int64_t)i * a.qr + (int64_t)h * D;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int d = kE4m3 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            const u32x4_t v = *reinterpret_cast<const u32x4_t *>(qp + d);
            if (t < kQ) {
                q[t][s] = as_bf16x8(v);
            } else if constexpr (NT > 2) {
                if (tile0 < 3) lds.q[tile0][s][lane] = v;   // read by this wave alone
            }
        }
        const int64_t p = (int64_t)it.pos0 + i;
        see_hi[t] = (int)min(p + 1, (int64_t)it.hi);
        see_lo[t] = a.window && p + 1 > a.window ? (int)min(p + 1 - a.window, (int64_t)1 << 30) : 0;
    }
    const int64_t pf = (int64_t)it.pos0 + it.r0 / a.G;
    const int64_t pl = (int64_t)it.pos0 + (it.r0 + it.rows - 1) / a.G;
    const int all_hi = (int)min(pf + 1, (int64_t)it.hi);
    const int all_lo = a.window && pl + 1 > a.window ? (int)min(pl + 1 - a.window, (int64_t)1 << 30) : 0;

    f32x4_t o[NA][NJ];
    float m[NA], l[NA];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = kNoMax;
        l[t] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[t][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const char *kh = a.c.k + (int64_t)kv * a.c.head, *vh = a.c.v + (int64_t)kv * a.c.head;
    const uint32_t slot = (uint32_t)a.c.slot;
    const uint32_t k_off = (uint32_t)c * slot + 16 * g;
    const uint32_t v_off = 4 * (uint32_t)g * slot + (16 * (wave & 1) + c) * VB;
    u32x4_t kr[KL];
    uint32_t vr[8][1][VW];
    float sc = 0.f;
    uint64_t bad_next = 0;
    auto fetch = [&](int k0) {
        const Tiles tl = take_tiles<4, kE4m3>(a, it, k0, entry, kv);
        bad_next = tl.bad;
        entry = load_entry<4>(a, it, k0 + kStep);   // ahead of the loads that go by it
        const auto kb = buffer_at(kh + tl.row(wave));
#pragma unroll
        for (int s = 0; s < KL; ++s) kr[s] = buffer_load16(kb, k_off + 64 * s, 0);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const auto vb = buffer_at(vh + tl.row(2 * (wave >> 1) + t));
#pragma unroll
            for (int i = 0; i < 4; ++i) buffer_load<VB>(vr[4 * t + i][0], vb, v_off, i * slot);
        }
        // The keys' scales for wave 0, the values' for wave 1 (and 2 and 3, which have no use
        // for them: a branch here had the compiler wait for all loads before it).
        if constexpr (kE4m3) sc = (wave ? a.c.vs : a.c.ks)[tl.scale];
    };
    // What was fetched for the keys from k0 on, as operands in LDS.
    auto stage = [&](int k0, int buf) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if constexpr (kE4m3) {
                const uint32_t w0 = s & 1 ? kr[s / 2].z : kr[s / 2].x, w1 = s & 1 ? kr[s / 2].w : kr[s / 2].y;
                lds.k[buf][wave][s][lane] = u32x4_t{e4m3_bf16<false>(w0), e4m3_bf16<true>(w0),
                                                  e4m3_bf16<false>(w1), e4m3_bf16<true>(w1)};
            } else {
                lds.k[buf][wave][s][lane] = kr[s];
            }
        }
        uint32_t vp[8][1][VE / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int w = 0; w < VE / 2; ++w) {
                if constexpr (kE4m3)
                    vp[i][0][w] = w & 1 ? e4m3_bf16<true>(vr[i][0][w / 2]) : e4m3_bf16<false>(vr[i][0][w / 2]);
                else
                    vp[i][0][w] = vr[i][0][w];
            }
        uint32_t odd_keys = 0;
        const bool every_row = k0 >= all_lo && k0 + kStep <= all_hi;   // sees every key
        if (!every_row) {
            // values that not every row sees (see mask_values above)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int kk = 16 * (i / 4) + 4 * g + i % 4, j = k0 + 32 * (wave >> 1) + kk;
                const bool any = j >= it.lo && j < it.hi, every = j >= all_lo && j < all_hi;
                bool odd = false;
#pragma unroll
                for (int w = 0; w < VE / 2; ++w) {
                    const uint32_t y = vp[i][0][w];
                    odd |= (y & 0x7f80u) == 0x7f80u || (y & 0x7f800000u) == 0x7f800000u;
                }
                const uint64_t ball = __ballot(odd && any && !every);
                const bool row_odd = (ball >> (16 * g) & 0xffff) != 0;
#pragma unroll
                for (int gg = 0; gg < 4; ++gg)
                    if (ball >> (16 * gg) & 0xffff) odd_keys |= 1u << (16 * (i / 4) + 4 * gg + i % 4);
#pragma unroll
                for (int w = 0; w < VE / 2; ++w)
                    if (!any || row_odd) vp[i][0][w] = 0;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (lane == 0) lds.odd[buf][wave >> 1][wave & 1] = odd_keys;
#pragma unroll
        for (int j = 0; j < VE; ++j)
            lds.v[buf][wave >> 1][VE * (wave & 1) + j][lane] = __builtin_bit_cast(u32x4_t, value_operand(vp, 0, j / 2, j & 1));
        if constexpr (kE4m3) {
            if (wave == 0) sc *= c1;
            if (wave == 1) {
                // a scale that is not finite, as with the values: where every row sees its key it
                // stays, and every row's output is not finite either
                const bool odd = !every_row && !(fabsf(sc) < INFINITY);
                const uint64_t ball = __ballot(odd);
                if (odd) sc = 0.f;
                if (lane < 2) lds.odd[buf][lane][2] = (uint32_t)(ball >> (32 * lane));
            }
            if (wave < 2) reinterpret_cast<float *>(lds.scale[buf][wave])[lane] = sc;
        }
    };

    fetch(kbase);
    uint64_t bad = bad_next;
    int buf = 0;
    __syncthreads();   // the item before is done with LDS
    stage(kbase, 0);
    __syncthreads();
    for (int k0 = kbase; k0 < kend; k0 += kStep) {
        const bool more = k0 + kStep < kend;
        if (more) fetch(k0 + kStep);
        if constexpr (NT > 0) {
#pragma unroll 1
            for (int hh = 0; hh < 2; ++hh) {
                const int j0 = k0 + 32 * hh;
                asm volatile("" ::: "memory");   // operands are read from LDS anew
                const bool plain = k0 >= all_lo && k0 + kStep <= all_hi && bad == 0;
                f32x4_t sx[NT][2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) sx[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const bf16x8_t k = as_bf16x8(lds.k[buf][2 * hh + t][s][lane]);
#pragma unroll
                        for (int n = 0; n < kQ; ++n) sx[n][t] = mfma(k, q[n][s], sx[n][t]);
                        if constexpr (NT > 2) sx[2][t] = mfma(k, as_bf16x8(lds.q[tile0][s][lane]), sx[2][t]);
                    }
                }
                bf16x8_t p[NT];
                // (a value that is not finite: as if its key's page were bad)
                uint32_t nan = 0;
                if (!plain) {
                    nan = (uint32_t)(bad >> (32 * hh)) | lds.odd[buf][hh][0] | lds.odd[buf][hh][1];
                    if constexpr (kE4m3) nan |= lds.odd[buf][hh][2];
                    nan >>= 4 * g;
                }
                // the tiles' scores together: one branch for all of them, and exponentials of one
                // among sums of another
                float sc[NT];
                f32x4_t ks[2];
                if constexpr (kE4m3) ks[0] = lds.scale[buf][0][8 * hh + g], ks[1] = lds.scale[buf][0][8 * hh + 4 + g];
                bool raise = false;
                float mx[NT];
                const int j = j0 + 4 * g;
#pragma unroll
                for (int n = 0; n < NT; ++n) sc[n] = scale_scores<kE4m3>(a, sx[n], c1, ks[0], ks[1]);
                if (!plain) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) mask_scores(sx[n], Seen{see_lo[n] - j, see_hi[n] - j, nan});
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mx[n] = max_of(sx[n]) * sc[n];
                    raise |= mx[n] > m[n] + kSlack;
                }
                if (__any(raise)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float mn = fmaxf(m[n], query_max(mx[n]));
                        const float f = __builtin_amdgcn_exp2f(m[n] - mn);
                        m[n] = mn;
                        l[n] *= f;
#pragma unroll
                        for (int j = 0; j < NJ; ++j) o[n][j] *= f;
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            sx[n][t][r] = __builtin_amdgcn_exp2f(fmaf(sx[n][t][r], sc[n], -m[n]));
                            l[n] += sx[n][t][r];
                        }
                    if constexpr (kE4m3) {
                        sx[n][0] *= lds.scale[buf][1][8 * hh + g];
                        sx[n][1] *= lds.scale[buf][1][8 * hh + 4 + g];
                    }
                    p[n] = weight_operand(sx[n]);
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const bf16x8_t v = as_bf16x8(lds.v[buf][hh][j][lane]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][j] = mfma(v, p[n], o[n][j]);
                }
            }
        }
        if (more) stage(k0 + kStep, buf ^ 1);
        bad = bad_next;
        buf ^= 1;
        __syncthreads();
    }

    const bool whole = u0 == 0 && u1 == it.units;
    float *part = partial_at<D>(a, blockIdx.x, u0 == 0, R);
    const float nan = __uint_as_float(0x7fc00000u);
    int first_tile = tile0;   // (what follows is not computed ahead of the loop)
    asm volatile("" : "+s"(first_tile));
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float lg = query_sum(l[n]);
        const int row = 16 * (first_tile + 4 * n) + c;
        if (row >= it.rows) continue;
        int64_t oat, lat;
        bool gone;
        put_row<D>(a, it, kv, row, oat, lat, gone);
        const float inv = 1.f / lg;
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (D / 2) * v + VE * (4 * g + r);
                if (whole) {
                    uint32_t w[VE / 2];
#pragma unroll
                    for (int j = 0; j < VE / 2; ++j)
                        w[j] = gone ? 0x7fc07fc0u
                                    : pack_bf16(o[n][VE * v + 2 * j][r] * inv, o[n][VE * v + 2 * j + 1][r] * inv);
                    __builtin_memcpy(__builtin_assume_aligned(a.out + oat + d, 2 * VE), w, 2 * VE);
                } else {
                    float y[VE];
#pragma unroll
                    for (int j = 0; j < VE; ++j) y[j] = o[n][VE * v + j][r];
                    __builtin_memcpy(__builtin_assume_aligned(part + row * D + d, VE < 4 ? 8 : 16), y, 4 * VE);
                }
            }
        if (g == 0) {
            if (whole) {
                if (a.lse) a.lse[lat] = gone ? nan : log_sum(a, m[n], lg);
            } else {
                part[R * D + 2 * row] = m[n];
                part[R * D + 2 * row + 1] = lg;
            }
        }
    }
}

template <int D, bool kE4m3, int kMT>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void cache_attn_wide_kernel(AttnArgs a, int R) {
    __shared__ WideLds<D, kMT> lds;
    __shared__ int64_t s_w[8];
    __shared__ int s_e[3];
    const int wave = uniform((int)threadIdx.x / 64);
    const Range rg = block_range(a, R, s_w, s_e);
    int e = rg.e;
    Item it = rg.it;
    int64_t x = rg.x0, first = rg.first;
    Opened opened = kNothing;
    while (x < rg.x1) {
        const int64_t span = (int64_t)it.units * a.c.heads;
        if (x >= first + span) {
            first += span;
            it = item_of(a, ++e, R);
            continue;
        }
        const int kv = (int)quotient(x - first, it.units);
        const int u0 = (int)((x - first) - (int64_t)kv * it.units);
        const int u1 = (int)min((int64_t)it.units, u0 + (rg.x1 - x));
        x += u1 - u0;

        const int tiles = (it.rows + 15) / 16;
        // (the waves that have a tile more are others in every other block, and so on other SIMDs)
        const int tile0 = (wave + blockIdx.x) & 3;
        if (tile0 + 4 * (kMT - 1) < tiles)
            wide_segment<D, kE4m3, kMT>(a, lds, it, kv, u0, u1, tile0, R);
        else if (tile0 >= tiles)
            wide_segment<D, kE4m3, 0>(a, lds, it, kv, u0, u1, tile0, R);
        else   // (or fewer, in an item of few rows)
            wide_segment<D, kE4m3, kMT - 1>(a, lds, it, kv, u0, u1, tile0, R);
        if (u0 == 0 && u1 < it.units) {   // it ends in a later block
            const int64_t end = first + (int64_t)(kv + 1) * it.units;
            opened = Opened{e, kv, rg.block_of(end - 1), it.pos0, it.rows, it.b, it.r0, 0};
        }
    }
    if (threadIdx.x == 0) a.opened[blockIdx.x] = opened;
}

// D / 4 lanes per row of an item that spans blocks, which is found by the block that opens it:
// the parts' rows, weighed by their maxima, added up in order.  Up to eight parts are asked for
// together, and ahead of the eight before being used.  4 to 12 us, by the latency of two
// dependent loads; 18 us for 512 items of 136 rows, by the 72 MB of their parts.
template <int D>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(AttnArgs a, int R) {
    constexpr int L = D / 4, kParts = 8;
    const int row = blockIdx.y * (256 / L) + (int)threadIdx.x / L, lane = (int)threadIdx.x % L;
    // (eight neighbours change places: items of one length are opened by blocks at some even
    // distance, which would all be joined on one XCD)
    const uint32_t x = blockIdx.x;
    const int block = x < (gridDim.x & ~7u) ? (x & ~7u) | ((x - x / 8 - x / 64 - blockIdx.y) & 7) : x;
    const Opened op = a.opened[block];
    if (op.e < 0 || row >= op.rows) return;
    const int parts = op.last - block + 1;
    float ml[2][kParts][2];
    f32x4_t y[2][kParts];
    auto load = [&](int i0, int to) {
        auto some = [&](int first, int last) {
#pragma unroll
            for (int i = first; i < last; ++i) {
                const int n = min(i0 + i, parts - 1);   // (the last one again for those past the end)
                const float *p = partial_at<D>(a, block + n, n == 0, R);
                y[to][i] = *reinterpret_cast<const f32x4_t *>(p + row * D + 4 * lane);
                const float2 w = *reinterpret_cast<const float2 *>(p + R * D + 2 * row);
                ml[to][i][0] = w.x;
                ml[to][i][1] = w.y;
            }
        };
        some(0, 2);
        if (i0 + 2 < parts) some(2, 4);
        if (i0 + 4 < parts) some(4, kParts);
    };
    load(0, 0);
    float m = kNoMax, l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < parts; i0 += kParts) {
        if (i0 + kParts < parts) load(i0 + kParts, 1);
        float mx = m;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            if (i0 + i < parts) mx = fmaxf(mx, ml[0][i][0]);
        const float f = __builtin_amdgcn_exp2f(m - mx);
        m = mx;
        l *= f;
        o *= f;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            if (i0 + i >= parts) continue;
            const float w = __builtin_amdgcn_exp2f(ml[0][i][0] - m);
            l = fmaf(w, ml[0][i][1], l);
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = fmaf(w, y[0][i][k], o[k]);
        }
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            y[0][i] = y[1][i];
            ml[0][i][0] = ml[1][i][0];
            ml[0][i][1] = ml[1][i][1];
        }
    }
    Item it;
    it.b = op.b, it.r0 = op.r0, it.pos0 = op.pos0;
    int64_t oat, lat;
    bool gone;
    put_row<D>(a, it, op.kv, row, oat, lat, gone);
    const float inv = gone ? __uint_as_float(0x7fc00000u) : 1.f / l;
    *reinterpret_cast<uint2 *>(a.out + oat + 4 * lane) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    if (a.lse && lane == 0) a.lse[lat] = gone ? inv : log_sum(a, m, l);
}

// ------------------------------------------------ chosen heads at one row
// The keys of a sequence once per key head that has chosen query heads, as the first
// operand, against up to 16 of those as the second: with the log sums known a weight is
// final at once, and a lane stores its four keys of a row together.  The units of all
// (sequence, used key head) pairs are dealt to the blocks as in the attention; a block's
// four waves have 32 of a unit's keys each.  Bound by memory, keys read and weights written:
// 40 heads of 32 sequences of up to 8192 tokens (507 MB): 109 to 113 us, 4.5 to 4.6 TB/s (in e4m3,
// 280 MB, 74 us); 8 heads of one of 1024: 7.0 us.
constexpr int kRowsBlocks = 1024;   // four per CU

// kAux as above where no key head can have more than 16 chosen rows; where one has more, its keys
// are read again for each 16.  16 sequences of 8192, 8 key heads of 128 in bf16, keys not in the
// caches before, through them and past them: 16 rows a key head 81 and 76 us, 17 rows 117 and 133,
// 32 rows 146 and 148, 64 rows 269 and 301, 128 rows 514 and 703.  Which heads are chosen is known on
// the device alone: 24 spread over key heads of 24 query heads each, 3 a key head, take 64 us this
// way and would take 58 past the caches, but 24 of one key head would lose more.
template <int D, bool kE4m3, int kAux>
__global__ __launch_bounds__(256, D == 256 ? 2 : 3) void cache_attn_rows_kernel(AttnArgs a) {
    constexpr int S = D / 32;
    using Keys = KeyRows<D, kE4m3, 2>;
    __shared__ u32x4_t s_keys[4][2][Keys::kPieces * 64];
    constexpr int kHeadList = 512;   // chosen heads that are kept in LDS
    __shared__ int s_used[1024], s_heads[kHeadList], s_list[256], s_cnt[4];
    __shared__ int64_t s_w[5];
    __shared__ int s_b;
    const int lane = lane_id(), wave = uniform((int)threadIdx.x / 64), tid = threadIdx.x;
    const int g = lane >> 4, c = lane & 15;

    // A sequence's keys to write, and its units.
    auto keys_of = [&](int b) {
        const int T = a.r.lens[b], i = a.row[b];
        return T >= 1 && i >= 0 && i < a.r.n ? min((int64_t)T + i, a.n_keys) : 0;
    };
    auto units_of = [&](int b) { return (keys_of(b) + kUnit - 1) / kUnit; };
    const int per = (a.r.B + 255) / 256, b0 = min(tid * per, a.r.B), b1 = min(b0 + per, a.r.B);
    int64_t mine = 0;
    const int head0 = tid < a.R ? a.heads[tid] : -1;   // (asked for together with the lengths)
    for (int b = b0; b < b1; ++b) mine += units_of(b);

    // The key heads that are used, in order, and a place after them for chosen heads that do
    // not exist: their rows are NaN.
    for (int h = tid; h < a.c.heads; h += 256) s_used[h] = 0;
    __syncthreads();
    bool unknown = false;
    for (int r = tid; r < a.R; r += 256) {
        const int h = r == tid ? head0 : a.heads[r];
        if (r < kHeadList) s_heads[r] = h;
        if (h >= 0 && h < a.Hq)
            s_used[h / a.G] = 1;
        else
            unknown = true;
    }
    unknown = __syncthreads_or(unknown);
    if (wave == 0) {
        int n = 0;
        for (int h0 = 0; h0 < a.c.heads; h0 += 64) {
            const bool in = h0 + lane < a.c.heads && s_used[h0 + lane];
            const uint64_t m = __ballot(in);
            asm volatile("" ::: "memory");
            if (in) s_used[n + __popcll(m & lanemask_lt())] = h0 + lane;   // (never past h0)
            n += __popcll(m);
        }
        if (lane == 0) s_cnt[0] = n;
    }
    // the waves' sums go through LDS at the same barrier
    int64_t before = wave_incl_scan(mine);
    if (lane == 63) s_w[wave] = before;
    __syncthreads();
    const int used = uniform(s_cnt[0]), heads = used + unknown;

    int64_t total = 0;
    before -= mine;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += s_w[w];
        total += s_w[w];
    }
    total = uniform(total) * heads;
    before *= heads;
    mine *= heads;
    const int64_t part = quotient(total, gridDim.x), longer = total - part * gridDim.x;
    int64_t x = part * blockIdx.x + min((int64_t)blockIdx.x, longer);
    const int64_t x1 = x + part + (blockIdx.x < longer);
    if (x >= x1) return;
    if (before <= x && x < before + mine) {
        int b = b0;
        for (int64_t u; x >= before + (u = units_of(b) * heads); ++b) before += u;
        s_b = b;
        s_w[4] = before;
    }
    __syncthreads();
    int b = uniform(s_b);
    int64_t first = uniform(s_w[4]);

    const float c1 = a.scale, nan = __uint_as_float(0x7fc00000u);
    const int64_t cap = (int64_t)a.c.max_pages << a.c.shift;
    while (x < x1) {
        const int64_t units = uniform(units_of(b)), span = units * heads;
        if (x >= first + span) {
            first += span;
            ++b;
            continue;
        }
        const int ki = (int)quotient(x - first, units);
        const int u0 = (int)((x - first) - ki * units), u1 = (int)min(units, u0 + (x1 - x));
        x += u1 - u0;
        const int kv = ki < used ? uniform(s_used[ki]) : -1;
        const int row = uniform(a.row[b]);
        const int64_t pos = (int64_t)uniform(a.r.lens[b]) - 1 + row;
        const int end = (int)min(keys_of(b), (int64_t)u1 * kUnit);      // of what is written here
        const int lo = a.window && pos + 1 > a.window ? (int)min(pos + 1 - a.window, (int64_t)1 << 30) : 0;
        Item it;
        it.b = b;
        it.hi = (int)min(min(pos + 1, a.n_keys), cap);

        for (int r0 = 0; r0 < a.R; r0 += 256) {
            // the rows r of this key head among 256, in order
            const int h = r0 + tid >= a.R ? 0 : r0 + tid < kHeadList ? s_heads[r0 + tid] : a.heads[r0 + tid];
            const bool known = h >= 0 && h < a.Hq;
            const bool in = r0 + tid < a.R && (known ? h / a.G == kv : kv < 0);
            const uint64_t m = __ballot(in);
            __syncthreads();
            if (lane == 0) s_cnt[wave] = __popcll(m);
            __syncthreads();
            int to = __popcll(m & lanemask_lt()), cnt = 0;
            for (int w = 0; w < 4; ++w) {
                if (w < wave) to += s_cnt[w];
                cnt += s_cnt[w];
            }
            cnt = uniform(cnt);
            if (in) s_list[to] = r0 + tid;
            __syncthreads();

            for (int t0 = 0; t0 < cnt; t0 += 16) {
                const bool own = t0 + c < cnt;
                const int r = s_list[min(t0 + c, cnt - 1)];
                const int head = kv < 0 ? 0 : r < kHeadList ? s_heads[r] : a.heads[r];
                const uint16_t *qp = a.q + (int64_t)b * a.qs + (int64_t)row * a.qr + (int64_t)head * D;
                bf16x8_t q[S];
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const int d = kE4m3 ? 64 * (s / 2) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
                    q[s] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(qp + d));
                }
                const float lse = a.lse[((int64_t)b * a.r.n + row) * a.Hq + head];
                float *dst = a.attn + (int64_t)b * a.as + (int64_t)r * a.ar;
                const bool vec = ((uintptr_t)dst & 15) == 0;

                const char *kh = a.c.k + (int64_t)max(kv, 0) * a.c.head;
                const uint32_t slot = (uint32_t)a.c.slot, k_off = (uint32_t)Keys::row() * slot + 16 * Keys::piece();
                Keys kr;
                f32x4_t kf[2];
                auto load_k = [&](const Tiles &tl) {
                    kr.template load<kAux>(k_off, slot, [&](int t) { return kh + tl.row(t); });
                    if constexpr (kE4m3)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            kf[t] = __builtin_bit_cast(f32x4_t, buffer_load16(buffer_at(a.c.ks + tl.first_scale(t)), 16 * g, 0));
                };
                const int kbase = u0 * kUnit + 32 * wave;
                int entry = load_entry<2>(a, it, kbase);
                Tiles tl = take_tiles<2, kE4m3>(a, it, kbase, entry, max(kv, 0));
                entry = load_entry<2>(a, it, kbase + kUnit);
                // (keys before the window are written, not read)
                if (kbase < end && kbase + 32 > lo) load_k(tl);
                for (int k0 = kbase; k0 < end; k0 += kUnit) {
                    const uint32_t bad = (uint32_t)tl.bad;
                    kr.store(s_keys[wave]);
                    f32x4_t w[2], ks[2];
                    if constexpr (kE4m3) ks[0] = kf[0] * c1, ks[1] = kf[1] * c1;
                    asm volatile("" ::: "memory");
                    if (k0 + kUnit < end) {
                        tl = take_tiles<2, kE4m3>(a, it, k0 + kUnit, entry, max(kv, 0));
                        entry = load_entry<2>(a, it, k0 + 2 * kUnit);
                        if (k0 + kUnit + 32 > lo) load_k(tl);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        w[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int s = 0; s < S; ++s)
                            w[t] = mfma(key_operand<kE4m3>(Keys::read(s_keys[wave], t, kE4m3 ? s / 2 : s), s), q[s], w[t]);
                    }
                    const float sc = scale_scores<kE4m3>(a, w, c1, ks[0], ks[1]);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[t][e] = __builtin_amdgcn_exp2f(fmaf(w[t][e], sc, -lse) * kLog2E);
                    if (bad || kv < 0 || k0 < lo || k0 + 32 > it.hi) {
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int j = k0 + 16 * t + 4 * g + e;
                                if ((bad >> (16 * t + 4 * g + e)) & 1 || j >= cap) w[t][e] = nan;
                                if (j < lo) w[t][e] = 0.f;
                                if (kv < 0) w[t][e] = nan;
                            }
                    }
                    if (!own) continue;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int j = k0 + 16 * t + 4 * g;
                        if (vec && j + 4 <= end) {
                            *reinterpret_cast<f32x4_t *>(dst + j) = w[t];
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (j + e < end) dst[j + e] = w[t][e];
                        }
                    }
                }
            }
        }
    }
}

// Tiles of 16 rows per item, and row groups per sequence, from a key head's rows.
// Up to 2 tiles (1 for heads of 256) a wave has all of an item's rows; past that a wave has
// up to three tiles (two) of its own.  Eleven and not twelve: the third tiles' queries are in
// LDS, where two blocks a CU leave room for three.
struct AttnShape {
    int tiles, groups;
};
static int most_tiles(int D) { return D == 256 ? 8 : 11; }
static int64_t all_tiles(int n, int G) { return ((int64_t)n * G + 15) / 16; }
static AttnShape attn_shape(int n, int G, int D) {
    const int most = most_tiles(D);
    const int64_t tiles = all_tiles(n, G);
    AttnShape s;
    s.groups = (int)((tiles + most - 1) / most);
    s.tiles = (int)((tiles + s.groups - 1) / s.groups);
    return s;
}
static size_t partials_bytes(int tiles, int D) {
    return align_up((size_t)kAttnBlocks * 2 * 16 * tiles * (D + 2) * sizeof(float), 256);
}

template <int D, bool kE4m3>
static void launch_attn(const AttnArgs &a, const AttnShape &sh, hipStream_t s) {
    const int64_t units = (((int64_t)a.c.max_pages << a.c.shift) + kUnit - 1) / kUnit;
    const int64_t most = units * a.r.B * sh.groups * a.c.heads;
    const dim3 grid((unsigned)(most < kAttnBlocks ? most : kAttnBlocks));
    const int R = 16 * sh.tiles;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a); };
    auto go_wide = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, R); };
    if (sh.tiles == 1)
        go(cache_attn_kernel<D, kE4m3, 1>);
    else if (D < 256 && sh.tiles == 2)
        go(cache_attn_kernel<D, kE4m3, D < 256 ? 2 : 1>);
    else if (sh.tiles <= 4)
        go_wide(cache_attn_wide_kernel<D, kE4m3, 1>);
    else if (sh.tiles <= 8)
        go_wide(cache_attn_wide_kernel<D, kE4m3, 2>);
    else if constexpr (D < 256)
        go_wide(cache_attn_wide_kernel<D, kE4m3, 3>);
    hipLaunchKernelGGL(cache_attn_join_kernel<D>, dim3(grid.x, (unsigned)((R + 1024 / D - 1) / (1024 / D))), dim3(256), 0, s, a, R);
}

static int prep_attn(const pld_cache *cache, bool needs_v, const uint16_t *q, int64_t qs,
                     int64_t qr, const int32_t *lens, const int32_t *draft_len, int B, int n,
                     int Hq, float scale, float softcap, int window, float unit, AttnArgs &a) {
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
    a.scale = scale;
    a.cap = softcap * unit, a.cap_x2 = 2.f * a.cap, a.cap_near = kCapNear * a.cap;
    a.inv2_log2e = softcap > 0.f ? (float)(2. * kLog2E / a.cap) : 0.f;
    // (scale and cap times log2(e) are rounded, a relative error of every score; the way back by
    // the rounded ones takes it from the log sum, which would be off by 10^-6 at a score of 15)
    a.nat = softcap > 0.f ? (float)((double)softcap / a.cap) : (float)((double)scale / (scale * unit));
    if (!isfinite(scale * kLog2E) || !isfinite(2.f * (softcap * kLog2E)) || !isfinite(a.inv2_log2e)) return PLD_ERR_INVALID;
    a.G = Hq / cache->heads;
    a.page16 = (uint32_t)(a.c.page / 16), a.slot16 = (uint32_t)(a.c.slot / 16);
    a.spage32 = (uint32_t)a.c.spage;
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
    // (groups are even: with more rows than one group's an item may have fewer tiles than with
    // less, and a workspace for many rows has to serve few)
    const int64_t tiles = all_tiles(n, Hq / heads), most = most_tiles(head_dim);
    return partials_bytes((int)(tiles < most ? tiles : most), head_dim) + kAttnBlocks * sizeof(Opened);
}

extern "C" int pld_cache_attn(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                              int64_t q_row_stride, const int32_t *lens, const int32_t *draft_len,
                              int B, int n, int Hq, float scale, float softcap, int window,
                              uint16_t *out, int64_t o_seq_stride, int64_t o_row_stride,
                              float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    AttnArgs a;
    int rc = prep_attn(cache, true, q, q_seq_stride, q_row_stride, lens, draft_len, B, n, Hq,
                       scale, softcap, window, kLog2E, a);
    if (rc != PLD_OK) return rc;
    const int D = cache->head_dim;
    rc = check_rows(out, o_seq_stride, o_row_stride, B, n, (int64_t)Hq * D);
    if (rc != PLD_OK) return rc;
    if ((uintptr_t)lse % 4) return PLD_ERR_ALIGN;
    if (!workspace || (uintptr_t)workspace % 16 ||
        workspace_bytes < pld_cache_attn_workspace_bytes(B, n, Hq, cache->heads, D))
        return PLD_ERR_WORKSPACE;
    const AttnShape sh = attn_shape(n, a.G, D);
    if (out == q || (int64_t)B * sh.groups > INT32_MAX / 2) return PLD_ERR_INVALID;
    a.out = out, a.os = o_seq_stride, a.orow = o_row_stride;
    a.lse = lse;
    a.groups = sh.groups;
    a.partials = static_cast<float *>(workspace);
    a.opened = reinterpret_cast<Opened *>(static_cast<char *>(workspace) + partials_bytes(sh.tiles, D));
    const bool q8 = cache->dtype == PLD_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (D == 64)
        q8 ? launch_attn<64, true>(a, sh, s) : launch_attn<64, false>(a, sh, s);
    else if (D == 128)
        q8 ? launch_attn<128, true>(a, sh, s) : launch_attn<128, false>(a, sh, s);
    else
        q8 ? launch_attn<256, true>(a, sh, s) : launch_attn<256, false>(a, sh, s);
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
                       softcap, window, 1.f, a);
    if (rc != PLD_OK) return rc;
    if (!row || !heads || !lse || !attn || R < 1 || R > 65535 || n_keys < 1 ||
        n_keys > INT32_MAX - 65536)
        return PLD_ERR_INVALID;
    if ((B > 1 && a_seq_stride < n_keys) || (R > 1 && a_row_stride < n_keys))
        return PLD_ERR_INVALID;
    if ((uintptr_t)lse % 4 || (uintptr_t)attn % 4) return PLD_ERR_ALIGN;
    a.row = row, a.heads = heads, a.R = R;
    a.lse = const_cast<float *>(lse);
    a.attn = attn, a.as = a_seq_stride, a.ar = a_row_stride, a.n_keys = n_keys;
    const int64_t most = (n_keys / kUnit + 1) * B * (cache->heads + 1);   // units
    const dim3 grid((unsigned)(most < kRowsBlocks ? most : kRowsBlocks));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, a);
    };
    const bool q8 = cache->dtype == PLD_E4M3, once = a.G <= 16 || R <= 16;
    auto pick = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (q8)
            kOnce<D, true> && once ? go(cache_attn_rows_kernel<D, true, kOnce<D, true>>)
                                   : go(cache_attn_rows_kernel<D, true, 0>);
        else
            once ? go(cache_attn_rows_kernel<D, false, kOnce<D, false>>)
                 : go(cache_attn_rows_kernel<D, false, 0>);
    };
    if (cache->head_dim == 64)
        pick(std::integral_constant<int, 64>{});
    else if (cache->head_dim == 128)
        pick(std::integral_constant<int, 128>{});
    else
        pick(std::integral_constant<int, 256>{});
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
