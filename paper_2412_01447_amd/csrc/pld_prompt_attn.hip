// pld_prompt_attn.hip -- causal attention of packed prompts to themselves.
//
// One pass over the keys with the running maximum m and sum l of each row: where the maximum rises to m', sum
// and output are scaled by 2^(m - m'), and in the end the output is divided by l.  The rows of one key head,
// G query heads by rows, are one long list; a block takes 128 or 256 of them, whose queries and output stay in
// registers, and goes through the keys that any of them sees, so that each is read once for all of them.
//
// Bound by its instructions: for long prompts (32 heads over 8 of 128, 16384 rows: 1850 us, 1190 TFLOP/s) matrix
// units are busy 60% of the time and the clock gives way under the power of products, weights and LDS reads
// together (a loop of these alone, in the same proportion, comes to 1250 TFLOP/s where a library's
// product of 8192 cubed has 1394); with heads of 64, and with a cap, vector instructions (84% busy).
// 2000 rows (8 sequences, 290 us, 905) pay 14 of 64 thousand cycles a block for their queries, first keys and output,
// 300 rows (64 sequences, 133 us) 15 of 26, two blocks a CU: half of it the wait for the queries, which comes no
// shorter with whole lines through LDS or with the sequences' starts loaded before them.
#include "pld_cache.h"
#include "pld_packed.h"

namespace pld {

#define PLD_INLINE __attribute__((always_inline))   // of a lambda: its arrays are registers

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t qr, kr, vr;
    Packed p;
    int G, heads;                  // query heads per key head; key heads
    int64_t tiles;                 // of a key head's rows
    float c1;                      // products to scores in log2 units
    float cap, cap_x2, cap_near, inv2_log2e;   // as in AttnArgs
    float inv_cap;                 // from products to parts y of the cap
    float nat;                     // from log2 units to natural ones
    int window;
    uint16_t *out;
    int64_t orow;
    float *lse;
};

// ------------------------------------------------------------ matrix tiles
// Everything is computed transposed, with v_mfma_f32_32x32x16_bf16: scores as K Q^T, so that lane
// (h, c) = (lane / 32, lane % 32) has the scores of query c and of keys 8 j + 4 h + 0..3, j = 0..3, of
// a tile of 32, and the output as V^T P^T.  The second product sums over keys in any order that both
// operands share: its slot (h, e) is key 8 (e/4) + 4 h + e%4 of each 16, where the weights are already.
// Keys come from LDS by rows, values by transposing reads of four keys by sixteen elements.
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char *lds_ptr;

__device__ __forceinline__ f32x16_t mfma32(bf16x8_t a, bf16x8_t b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Maximum and sum over the two lanes of a query.
__device__ __forceinline__ float pair_max(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
// A pointer that is the same in every lane, as a scalar.
__device__ __forceinline__ const char *uniform(const char *p) {
    const uint64_t v = (uint64_t)p;
    return (const char *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                          (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
// 16 bytes a lane from base + off to LDS, lane after lane from `to` on, without a register between
// (a lane's place in LDS is fixed, so the swizzle is in the addresses it reads).  The caller waits
// (vmcnt): the compiler does not know of these loads.
template <int kAhead>   // a distance of both addresses
__device__ __forceinline__ void load_to_lds(uint32_t to, const void *base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" ::"s"(to), "v"(off), "s"(base), "n"(kAhead) : "memory");
}
// Before a barrier: what this wave loads into LDS is there, and what it reads from LDS is read, so that
// after it other waves may read the one and load over the other.
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0), in a form that the compiler counts by too
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void block_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr float kSlack = 8.f;      // as in the cache's attention
constexpr float kNoMax = -1e30f;   // of a query that has seen no key

// kWaves waves of 32 kQT rows each: a tile of the rows of one key head, row m of all being query head
// m % G of row m / G, over the keys that they see, kKeys at a time.
constexpr int kKeys = 64;
template <int D, int kQT, int kWaves>
struct PromptTile {
    static constexpr int kRows = kWaves * 32 * kQT;
    // Keys and values in LDS: units of 16 rows by four pieces of 16 bytes, what one load instruction of a
    // wave brings, piece by piece with row j of a unit's piece q at place j ^ 4 q.  Sixteen lanes that read
    // a piece of as many rows, or two pieces of four, meet no bank twice, nor do 32, and where a
    // lane reads changes from unit to unit by constants alone.
    static constexpr int kUnits = D / 32;                    // of 16 rows
    static constexpr int kGroup = kUnits * 1024;             // bytes of 16 rows
    static constexpr int kTileBytes = kKeys * D * 2;
    static constexpr int kLoads = kKeys / 16 * kUnits / kWaves;   // a wave's units of a tile, of the same rows
    static constexpr int kDT = D / 32;
    static_assert((kLoads == 1 || kLoads == 2 || kLoads == 4 || kLoads == 8) && kUnits % kLoads == 0);
};

template <int D, int kQT, int kWaves, bool kCap>
__global__ __launch_bounds__(kWaves * 64, D == 256 ? 1 : 2) void prompt_attn_kernel(PromptArgs a) {
    using T = PromptTile<D, kQT, kWaves>;
    constexpr int kDT = T::kDT, kLoads = T::kLoads;
    __shared__ __attribute__((aligned(256))) char s_k[2][T::kTileBytes], s_v[2][T::kTileBytes];
    __shared__ int s_range[kWaves][2];
    __shared__ uint32_t s_bad[2];

    // The last rows first: their tiles see the most keys.  Neighbouring blocks, which are dealt to the
    // XCDs in turn, have different key heads, so that an XCD's L2 holds what its blocks share.
    const int64_t unit = wide_block();
    if (unit >= a.tiles * a.heads) return;
    const int64_t up = quotient(unit, a.heads);
    const int kv = __builtin_amdgcn_readfirstlane((int)(unit - up * a.heads));
    const int64_t m0 = (a.tiles - 1 - up) * T::kRows;
    const int64_t first = quotient(m0, a.G);
    const int over = (int)(m0 - first * a.G);
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int h = lane >> 5;

    // ---- the rows: what each sees, [lo, hi)
    auto row_of = [&](int t, int over, int &row, int &head) PLD_INLINE {
        const uint32_t m = (uint32_t)(over + (wave * kQT + t) * 32 + (lane & 31));
        const int r = (int)(m / (uint32_t)a.G);
        row = (int)first + r;
        head = kv * a.G + (int)m - r * a.G;
    };
    int lo[kQT], hi[kQT];   // (none: 0 and 0)
    int wave_lo = INT32_MAX, wave_hi = 0, full_lo = 0, full_hi = INT32_MAX;
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        int row, head;
        row_of(t, over, row, head);
        const bool in = row < a.p.N;
        if (!in) row = a.p.N - 1;
        const Span sp = spans_of(a.p, row);
        lo[t] = hi[t] = 0;
        if (in && sp.b >= 0) {
            hi[t] = row + 1;
            lo[t] = min(max(max(sp.begin, 0), a.window ? hi[t] - a.window : 0), row);
        }
        // both grow from row to row: a wave's range is between its first and its last row that has one
        const uint32_t some = (uint32_t)__ballot(hi[t] > 0);
        if (some) {
            const int i = __builtin_ctz(some), j = 31 - __builtin_clz(some);
            wave_lo = min(wave_lo, __builtin_amdgcn_readlane(lo[t], i));
            wave_hi = max(wave_hi, __builtin_amdgcn_readlane(hi[t], j));
            full_lo = max(full_lo, __builtin_amdgcn_readlane(lo[t], j));
            full_hi = min(full_hi, __builtin_amdgcn_readlane(hi[t], i));
        }
    }
    if (lane == 0) s_range[wave][0] = wave_lo, s_range[wave][1] = wave_hi;
    __syncthreads();
    int block_lo = INT32_MAX, block_hi = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        block_lo = min(block_lo, s_range[w][0]);
        block_hi = max(block_hi, s_range[w][1]);
    }
    block_lo = __builtin_amdgcn_readfirstlane(block_lo);
    block_hi = __builtin_amdgcn_readfirstlane(block_hi);
    if (block_lo >= block_hi) return;

    // ---- loads: a wave brings kLoads units of the same 16 rows, a lane 16 bytes of one row of each
    const int unit0 = wave * kLoads;
    const int j0 = unit0 / T::kUnits * 16 + ((lane & 15) ^ (lane >> 4) * 4);
    const int64_t byte0 = unit0 % T::kUnits * 64;
    const char *kbase = (const char *)(a.k + (int64_t)kv * D) + byte0, *vbase = (const char *)(a.v + (int64_t)kv * D) + byte0;
    const uint32_t kstride = (uint32_t)(a.kr * 2), vstride = (uint32_t)(a.vr * 2), piece = (lane >> 4) * 16;
    const uint32_t koff = (uint32_t)j0 * kstride + piece, voff = (uint32_t)j0 * vstride + piece;
    const uint32_t k_lds = (uint32_t)(uintptr_t)(lds_ptr)&s_k[0][0] + unit0 * 1024;
    const uint32_t v_lds = (uint32_t)(uintptr_t)(lds_ptr)&s_v[0][0] + unit0 * 1024;
    // keys or values to a buffer: a lane's from `from` + off on
    auto fetch_at = [&](const char *from, uint32_t off, int buf, bool values) PLD_INLINE {
        const uint32_t to = (values ? v_lds : k_lds) + buf * T::kTileBytes;
        load_to_lds<0>(to, from, off);
        if constexpr (kLoads > 1) load_to_lds<64>(to + 960, from, off);
        if constexpr (kLoads > 2) load_to_lds<128>(to + 1920, from, off), load_to_lds<192>(to + 2880, from, off);
        if constexpr (kLoads > 4) {
            load_to_lds<256>(to + 3840, from, off), load_to_lds<320>(to + 4800, from, off);
            load_to_lds<384>(to + 5760, from, off), load_to_lds<448>(to + 6720, from, off);
        }
    };
    // those of the rows from k0 on, which the block has; for rows past its last that one stands in
    auto fetch = [&](int k0, int buf, bool values) PLD_INLINE {
        const uint32_t stride = values ? vstride : kstride, off = (uint32_t)min(j0, block_hi - 1 - k0) * stride + piece;
        fetch_at(uniform((values ? vbase : kbase) + (int64_t)k0 * stride), off, buf, values);
    };

    // ---- the products, of 32 keys at a time: `part` of a tile
    bf16x8_t qf[kQT][D / 16];
    f32x16_t o[kQT][kDT];
    float mx[kQT];
    double l;   // of this lane's keys; with two tiles the whole of tile h's row
    const int c16 = lane & 15, odd16 = lane >> 4 & 1;
    int kat[2], vat[2];   // of even and odd steps of 16 elements; of the first and second eight of 16 rows
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int q = odd16 * 2 + (c16 >> 1 & 1);
        kat[x] = odd16 * T::kGroup + (2 * x + h) * 256 + (c16 ^ (8 * x + 4 * h)) * 16;
        vat[x] = q * 256 + ((8 * x + 4 * h + (c16 >> 2)) ^ 4 * q) * 16 + (c16 & 1) * 8;
    }
    auto key_operand = [&](const char *buf, int part, int x) PLD_INLINE {   // elements 16 x .. of 32 keys
        return *reinterpret_cast<const bf16x8_t *>(buf + part * 2 * T::kGroup + x / 2 * 1024 + kat[x & 1]);
    };
    auto value_operand = [&](const char *buf, int x, int dt) PLD_INLINE {   // 16 keys from 16 x on
        auto read = [&](int at) PLD_INLINE {
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4_t *>(
                (lds_ptr)(buf + x * T::kGroup + dt * 1024 + at)));
        };
        const s16x4_t x0 = read(vat[0]), x1 = read(vat[1]);
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto scores = [&](const char *buf, int part, f32x16_t (&s)[kQT]) PLD_INLINE {
#pragma unroll
        for (int t = 0; t < kQT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            const bf16x8_t f = key_operand(buf, part, x);
#pragma unroll
            for (int t = 0; t < kQT; ++t) s[t] = mfma32(f, qf[t][x], s[t]);
        }
    };
    auto largest = [&](const f32x16_t &s) PLD_INLINE {
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
        return top;
    };
    const float c = kCap ? 1.f : a.c1;   // from scores as they are kept to log2 units
    // Capped scores, x tanh(y) / y with y = x / cap.  They stay products s, and where all are near
    // (soft_cap_near's) fit[], its polynomial with the scale in it, is multiplied in the weight's own fma: five
    // instructions a score and not eight.  Where one is not, all are made s - m before (`settle`), with fit and
    // base 1 and 0 for the step: either way a score's bits go by it alone.  4 x 4096 of 32 heads of 64, 464
    // to 425 us.
    float fit[4], base[kQT];
    auto set_fit = [&](bool is_near) PLD_INLINE {
        fit[0] = is_near ? a.c1 : 1.f;
        fit[1] = is_near ? a.c1 * -0.33332663f : 0.f;
        fit[2] = is_near ? a.c1 * 0.13299825f : 0.f;
        fit[3] = is_near ? a.c1 * -0.0491485f : 0.f;
    };
    auto near = [&](float s) PLD_INLINE {
        const float y = s * a.inv_cap, u = fminf(fmaxf(y * y, 0.f), 1.f);   // (of -inf as well)
        return fmaf(u, fmaf(u, fmaf(u, fit[3], fit[2]), fit[1]), fit[0]);
    };
    auto capped = [&](float s, float less) PLD_INLINE {
        const float x = s * a.c1, e = __builtin_amdgcn_exp2f(fabsf(x) * a.inv2_log2e);
        const float far = copysignf(a.cap - a.cap_x2 * __builtin_amdgcn_rcpf(e + 1.f), x) - less;
        return fabsf(x) >= a.cap_near ? far : fmaf(s, near(s), -less);
    };
    auto mask = [&](int k0, f32x16_t (&s)[kQT]) PLD_INLINE {
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            const int from = lo[t] - k0 - 4 * h, count = hi[t] - lo[t];
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = (uint32_t)(8 * (r / 4) + r % 4 - from) < (uint32_t)count ? s[t][r] : -INFINITY;
        }
    };
    // The running maximum m is raised where a score is kSlack above it: score_high says whether any row's is,
    // raise goes by each row's own scores (its bits do not go by its neighbours').
    auto score_high = [&](const float (&top)[kQT]) PLD_INLINE {
        float over = fmaf(top[0], c, -mx[0]);
#pragma unroll
        for (int t = 1; t < kQT; ++t) over = fmaxf(over, fmaf(top[t], c, -mx[t]));
        return __ballot(over > kSlack);
    };
    auto raise = [&](const float (&top)[kQT]) PLD_INLINE {
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            const float all = pair_max(top[t]), mn = fmaf(all, c, -mx[t]) > kSlack ? all * c : mx[t];   // (as score_high)
            const float f = __builtin_amdgcn_exp2f(mx[t] - mn);
            mx[t] = mn;
            if (kQT == 1 || h == t) l *= (double)f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) o[t][dt] *= f;
        }
    };
    // Capped scores: the largest, from the largest product; and the scores themselves, after raise.  Where all
    // the row's products with the keys from k0 on that it sees are -inf, they are scores of -cap and no masks.
    auto settle_top = [&](float (&top)[kQT], bool far, int k0) PLD_INLINE {
        set_fit(true);
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            const bool sees = lo[t] < k0 + 32 && hi[t] > k0;
            top[t] = far && sees ? capped(top[t], 0.f) : top[t] * near(top[t]);
        }
    };
    auto settle = [&](f32x16_t (&s)[kQT], bool far) PLD_INLINE {
#pragma unroll
        for (int t = 0; t < kQT; ++t) base[t] = far ? 0.f : mx[t];
        if (far) {
#pragma unroll
            for (int t = 0; t < kQT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = capped(s[t][r], mx[t]);
            set_fit(false);
        }
    };
    // Weights 2^(s c - m), rounded to bf16 in pairs, as the product takes them: half a step (2^-8) of
    // each term.  The sum is of the unrounded ones: a lane's sixteen of a step in fp32, the steps' in 64
    // bits.  Equal weights that are added one by one in fp32 round one way all along: 10^-4 of the sum at
    // 32768 keys, 10^-2 at 4 million, 2 10^-6 of it this way (+-0.6% of the time, most 16384 rows).
    auto weigh = [&](float s, int t) PLD_INLINE {
        return __builtin_amdgcn_exp2f(fmaf(s, kCap ? near(s) : c, kCap ? -base[t] : -mx[t]));
    };
    // the sums of a step; of two tiles, the rows' halves trade places, so that a lane has one sum and not two
    auto add_up = [&](const float (&sum)[kQT]) PLD_INLINE {
        if constexpr (kQT == 1) {
            l += (double)sum[0];
        } else {
            const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[0]), __float_as_uint(sum[1]), false, false);
            l += (double)(__uint_as_float(a[0]) + __uint_as_float(a[1]));
        }
    };
    auto begin = [&]() PLD_INLINE {
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            mx[t] = kNoMax, l = 0.;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][dt][r] = 0.f;
        }
    };
    auto seen = [&](int k0) PLD_INLINE { return k0 < wave_hi && k0 + 32 > wave_lo; };

    // ---- the keys, 32 at a time.  A step takes the weights of its scores while the products of the next
    // step's are under way, and reads values, and then the step's after it keys, from LDS for the products
    // that follow: each has a part of what the vector units and LDS do beside them, in this order.
    constexpr int kX = D / 16, kLead = kQT == 2 ? 2 : kX < 8 ? kX : 8;   // products of a kind; values are read so many ahead
    f32x16_t s0[kQT], s1[kQT];
    bf16x8_t kf[kX];                 // keys of the next scores
    float top[kQT];
    uint64_t too_high = 0;           // score_high(top)
    bool far = false;                // of capped scores: some are not near
    // from the largest products `top`, and those of either sign
    auto look = [&](const float (&most)[kQT]) PLD_INLINE {
        if constexpr (kCap) {
            float x = most[0];
#pragma unroll
            for (int t = 1; t < kQT; ++t) x = fmaxf(x, most[t]);
            far = __any(x * a.c1 >= a.cap_near);
            set_fit(true);
#pragma unroll
            for (int t = 0; t < kQT; ++t) top[t] *= near(top[t]);
        }
        too_high = score_high(top);
    };
    auto first_scores = [&](f32x16_t (&s)[kQT]) PLD_INLINE {
        float most[kQT];
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
#pragma unroll
            for (int x = 0; x < kX; ++x) s[t] = mfma32(kf[x], qf[t][x], s[t]);
            top[t] = largest(s[t]);
            most[t] = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) most[t] = fmaxf(most[t], fabsf(s[t][r]));
        }
        look(most);
    };
    auto read_keys = [&](const char *buf, int part) PLD_INLINE {
#pragma unroll
        for (int x = 0; x < kX; ++x) kf[x] = key_operand(buf, part, x);
    };
    // Weights of s times values at (vbuf, part); the next step's scores into `ahead`; keys at (kbuf, part).
    auto products = [&](const char *vbuf, const char *kbuf, int part, f32x16_t (&s)[kQT], f32x16_t (&ahead)[kQT]) PLD_INLINE {
        // A slot is a product; what goes with it is a constant of its number z.
        constexpr int kZ = kX * kQT;                       // products of scores, and as many of values
        bf16x8_t vf[kLead];
        float w0[kQT], sum[kQT];
        uint32_t w[kQT][8];
        auto weights = [&](int z) PLD_INLINE {             // in the first three quarters
#pragma unroll
            for (int e = 0; e < 16 * kQT; ++e)
                if (e * 3 * kX / 32 == z) {
                    const int r = e / kQT, t = e % kQT;
                    const float x = weigh(s[t][r], t);
                    sum[t] = r ? sum[t] + x : x;
                    if (e == 16 * kQT - 1) add_up(sum);
                    if (r % 2) w[t][r / 2] = pack_bf16(w0[t], x);
                    else w0[t] = x;
                }
        };
        auto read_value = [&](int x) PLD_INLINE { vf[x % kLead] = value_operand(vbuf, part * 2 + x / kDT, x % kDT); };
        float m[kQT], most[kQT];
        // (past the last keys: of whatever is there, and not used)
#pragma unroll
        for (int z = 0; z < kZ; ++z) {
            const int x = z / kQT, t = z % kQT;
            if (x == 0)
#pragma unroll
                for (int r = 0; r < 16; ++r) ahead[t][r] = 0.f;
            ahead[t] = mfma32(kf[x], qf[t][x], ahead[t]);
            if (t == 0 && x >= kX - kLead) read_value(x - (kX - kLead));
            weights(z);
            if (!kCap || z % 2) __builtin_amdgcn_sched_barrier(0);   // (two slots: a cap is a chain of instructions)
        }
#pragma unroll
        for (int z = 0; z < kZ; ++z) {
            const int x = z / kQT, t = z % kQT;
            const uint32_t *p = w[t] + x / kDT * 4;
            o[t][x % kDT] = mfma32(vf[x % kLead], __builtin_bit_cast(bf16x8_t, make_uint4(p[0], p[1], p[2], p[3])), o[t][x % kDT]);
            if (t == kQT - 1) {
                if (x + kLead < kX) read_value(x + kLead);
                kf[x] = key_operand(kbuf, part, x);
            }
            weights(kZ + z);
            constexpr int kFrom = kZ / 4, kEach = 16 * kQT / (kZ / 2);   // the next maximum
            if (z >= kFrom && z < kFrom + kZ / 2)
#pragma unroll
                for (int e = (z - kFrom) * kEach; e < (z - kFrom + 1) * kEach; ++e) {
                    const int u = e / 16, r = e % 16;
                    m[u] = fmaxf(r ? m[u] : -INFINITY, ahead[u][r]);
                    if (kCap) most[u] = fmaxf(r ? most[u] : 0.f, fabsf(ahead[u][r]));
                }
            if (z == kFrom + kZ / 2 - 1) {
#pragma unroll
                for (int u = 0; u < kQT; ++u) {
                    asm volatile("" : "+v"(m[u]));   // taken here, among the products, and not where it is used
                    top[u] = m[u];
                }
                look(most);
            }
            if (!kCap || z % 2) __builtin_amdgcn_sched_barrier(0);
        }
    };
    // values of keys k0 .. at (vbuf, part); keys of k0 + 64 .. at (kbuf, part)
    auto step = [&](int k0, const char *vbuf, const char *kbuf, int part, f32x16_t (&s)[kQT], f32x16_t (&ahead)[kQT]) PLD_INLINE {
        if (seen(k0)) {
            const bool masked = k0 < full_lo || k0 + 32 > full_hi;
            if (masked) mask(k0, s);
            if (masked || (kCap && far)) {
#pragma unroll
                for (int t = 0; t < kQT; ++t) top[t] = largest(s[t]);
                if (kCap) settle_top(top, far, k0);
                too_high = score_high(top);
            }
            if (too_high) raise(top);
            if (kCap) settle(s, far);
            if (kCap && far && masked) mask(k0, s);   // (once more: an infinite score is capped, and no mask)
            products(vbuf, kbuf, part, s, ahead);
        } else {
            if (seen(k0 + 32)) first_scores(ahead);
            if (seen(k0 + 64)) read_keys(kbuf, part);
        }
    };
    // K of tile i + 2 and V of i + 1 are on their way during tile i.
    auto tile = [&](int k0, auto odd) PLD_INLINE {
        constexpr int kOdd = decltype(odd)::value;
        wait_loads();
        block_barrier();   // what tile i reads is there, and all have done with tile i - 1
        if (k0 + 2 * kKeys < block_hi) fetch(k0 + 2 * kKeys, kOdd, false);
        if (k0 + kKeys < block_hi) fetch(k0 + kKeys, !kOdd, true);
        step(k0, s_v[kOdd], s_k[!kOdd], 0, s0, s1);
        step(k0 + 32, s_v[kOdd], s_k[!kOdd], 1, s1, s0);
    };
    // a tile that all rows of the wave see whole, and two more behind it
    auto whole_tile = [&](int k0, auto odd) PLD_INLINE {
        constexpr int kOdd = decltype(odd)::value;
        wait_loads();
        block_barrier();
        fetch_at(kbase + (int64_t)(k0 + 2 * kKeys) * kstride, koff, kOdd, false);
        fetch_at(vbase + (int64_t)(k0 + kKeys) * vstride, voff, !kOdd, true);
        auto whole = [&](int part, f32x16_t (&s)[kQT], f32x16_t (&ahead)[kQT]) PLD_INLINE {
            if (kCap && far) {
#pragma unroll
                for (int t = 0; t < kQT; ++t) top[t] = largest(s[t]);
                settle_top(top, true, k0 + part * 32);
                too_high = score_high(top);
            }
            if (too_high) raise(top);
            if (kCap) settle(s, far);
            products(s_v[kOdd], s_k[!kOdd], part, s, ahead);
        };
        whole(0, s0, s1);
        whole(1, s1, s0);
    };
    begin();
    fetch(block_lo, 0, false);
    // the queries, on their way with the first keys
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        int row, head;
        row_of(t, over, row, head);
        const uint4 *src = reinterpret_cast<const uint4 *>(a.q + min(row, a.p.N - 1) * a.qr + (int64_t)head * D);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[t][s] = __builtin_bit_cast(bf16x8_t, src[2 * s + h]);
    }
    wait_loads();
    block_barrier();
    if (block_lo + kKeys < block_hi) fetch(block_lo + kKeys, 1, false);
    fetch(block_lo, 0, true);
    read_keys(s_k[0], 0);
    first_scores(s0);
    read_keys(s_k[0], 1);
    for (int k0 = block_lo; k0 < block_hi; k0 += 2 * kKeys) {
        for (; k0 >= full_lo && k0 + 2 * kKeys <= full_hi && k0 + 4 * kKeys <= block_hi; k0 += 2 * kKeys) {
            whole_tile(k0, std::integral_constant<int, 0>{});
            whole_tile(k0 + kKeys, std::integral_constant<int, 1>{});
        }
        tile(k0, std::integral_constant<int, 0>{});
        if (k0 + kKeys < block_hi) tile(k0 + kKeys, std::integral_constant<int, 1>{});
    }

    // A weight of 0 times a value that is not finite reaches rows that do not see it: where the output
    // holds such a number, all is done once more, a part after the other, with those values as 0 and NaN
    // for the rows that see them.
    bool odd = false;
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        float x = 0.f;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) x = fmaf(o[t][dt][r], 0.f, x);
        odd |= lo[t] < hi[t] && (!(x == 0.f) || (!(l < (double)INFINITY) && (kQT == 1 || h == t)));
    }
    if (__syncthreads_or(odd)) {
        begin();
#pragma unroll 1
        for (int key0 = block_lo; key0 < block_hi; key0 += kKeys) {
            fetch(key0, 0, false);
            fetch(key0, 0, true);
            if (threadIdx.x < 2) s_bad[threadIdx.x] = 0;
            wait_loads();
            __syncthreads();
            for (int at = threadIdx.x; at < kKeys * D / 8; at += kWaves * 64) {
                uint16_t *e = reinterpret_cast<uint16_t *>(s_v[0] + at * 16);
                bool hit = false;
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if ((e[x] & 0x7f80) == 0x7f80) e[x] = 0, hit = true;
                const int j = at / 64 / T::kUnits * 16 + ((at & 15) ^ (at >> 4 & 3) * 4);
                if (hit) atomicOr(&s_bad[j >> 5], 1u << (j & 31));
            }
            __syncthreads();
#pragma unroll 1
            for (int part = 0; part < kKeys / 32; ++part) {
                const int k0 = key0 + part * 32;
                if (!seen(k0)) continue;
                const uint32_t bad = s_bad[part] >> 4 * h;
                scores(s_k[0], part, s0);
#pragma unroll
                for (int t = 0; t < kQT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (bad >> (8 * (r / 4) + r % 4) & 1) s0[t][r] = __uint_as_float(0x7fc00000u);
                mask(k0, s0);
#pragma unroll
                for (int t = 0; t < kQT; ++t) top[t] = largest(s0[t]);
                if (kCap) settle_top(top, true, k0);
                raise(top);
                if (kCap) settle(s0, true), mask(k0, s0);
                uint32_t w[kQT][8];
                float sum[kQT];
#pragma unroll
                for (int t = 0; t < kQT; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float w0 = weigh(s0[t][2 * i], t), w1 = weigh(s0[t][2 * i + 1], t);
                        sum[t] = (i ? sum[t] : 0.f) + w0 + w1;
                        w[t][i] = pack_bf16(w0, w1);
                    }
                add_up(sum);
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const bf16x8_t f = value_operand(s_v[0], part * 2 + x / kDT, x % kDT);
#pragma unroll
                    for (int t = 0; t < kQT; ++t) {
                        const uint32_t *p = w[t] + x / kDT * 4;
                        o[t][x % kDT] = mfma32(f, __builtin_bit_cast(bf16x8_t, make_uint4(p[0], p[1], p[2], p[3])), o[t][x % kDT]);
                    }
                }
            }
            __syncthreads();
        }
    }
    float total[kQT];
    if constexpr (kQT == 1) {
        total[0] = pair_sum((float)l);
    } else {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint((float)l), __float_as_uint((float)l), false, false);
        total[0] = __uint_as_float(a[0]), total[1] = __uint_as_float(a[1]);
    }

    // ---- out: a lane has four consecutive elements of every eight; the two lanes of a query trade
    // halves, so that each stores eight
    int over_again = over;   // (taken again, so that no register keeps rows all along)
    asm volatile("" : "+s"(over_again));
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        if (lo[t] >= hi[t]) continue;   // (both lanes of a query alike)
        int row, head;
        row_of(t, over_again, row, head);
        const float inv = 1.f / total[t];
        uint16_t *dst = a.out + row * a.orow + (int64_t)head * D;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 8) {
                uint32_t w[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) w[x] = pack_bf16(o[t][dt][r + 2 * x] * inv, o[t][dt][r + 2 * x + 1] * inv);
                const auto y0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto y1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                *reinterpret_cast<uint4 *>(dst + dt * 32 + r * 2 + h * 8) = make_uint4(y0[0], y1[0], y0[1], y1[1]);
            }
        if (a.lse && h == 0)
            a.lse[(int64_t)row * a.G * a.heads + head] = fmaf(mx[t], a.nat, __log2f(total[t]) * kLn2);
    }
}

template <int D, int kQT, int kWaves, bool kCap>
static void launch_prompt(PromptArgs &a, hipStream_t s) {
    constexpr int rows = PromptTile<D, kQT, kWaves>::kRows;
    a.tiles = ((int64_t)a.p.N * a.G + rows - 1) / rows;
    hipLaunchKernelGGL((prompt_attn_kernel<D, kQT, kWaves, kCap>), wide_grid(a.tiles * a.heads), dim3(kWaves * 64), 0, s, a);
}

}  // namespace pld

using namespace pld;

extern "C" int pld_prompt_attn(const uint16_t *q, int64_t q_row_stride, const uint16_t *k, int64_t k_row_stride,
                               const uint16_t *v, int64_t v_row_stride, const int32_t *starts, int B, int N,
                               int Hq, int heads, int head_dim, float scale, float softcap, int window,
                               uint16_t *out, int64_t o_row_stride, float *lse, void *stream) {
    if (!starts || B < 1 || B > 65535 || N < 1 || N > PLD_MAX_PACKED_ROWS || heads < 1 || heads > 1024 || Hq < 1 ||
        Hq > 4096 || Hq % heads || (head_dim != 64 && head_dim != 128 && head_dim != 256))
        return PLD_ERR_INVALID;
    if (!(scale > 0.f) || !isfinite(scale) || !(softcap >= 0.f) || !isfinite(softcap) || window < 0) return PLD_ERR_INVALID;
    const int64_t qw = (int64_t)Hq * head_dim, kw = (int64_t)heads * head_dim;
    constexpr int64_t most = 1 << 22;   // a tile's offsets are 32-bit
    int rc;
    if ((rc = check_packed(q, q_row_stride, N, qw, most)) != PLD_OK ||
        (rc = check_packed(k, k_row_stride, N, kw, most)) != PLD_OK ||
        (rc = check_packed(v, v_row_stride, N, kw, most)) != PLD_OK ||
        (rc = check_packed(out, o_row_stride, N, qw, most)) != PLD_OK)
        return rc;
    if (((uintptr_t)starts | (uintptr_t)lse) % 4) return PLD_ERR_ALIGN;
    if (out == k || out == v || (out == q && N > 1 && o_row_stride != q_row_stride)) return PLD_ERR_INVALID;
    PromptArgs a{};
    a.q = q, a.k = k, a.v = v, a.qr = N > 1 ? q_row_stride : 0, a.kr = N > 1 ? k_row_stride : 0, a.vr = N > 1 ? v_row_stride : 0;
    a.p = Packed{starts, B, N};
    a.G = Hq / heads, a.heads = heads;
    a.c1 = scale * kLog2E;
    a.cap = softcap * kLog2E, a.cap_x2 = 2.f * a.cap, a.cap_near = kCapNear * a.cap;
    a.inv_cap = softcap > 0.f ? (float)((double)scale / softcap) : 0.f;
    a.inv2_log2e = softcap > 0.f ? (float)(2. * kLog2E / a.cap) : 0.f;
    // (the way back from log2 units is by the rounded factor that led there)
    a.nat = softcap > 0.f ? (float)((double)softcap / a.cap) : (float)((double)scale / a.c1);
    if (!isfinite(a.c1) || !isfinite(a.cap_x2) || !isfinite(a.inv2_log2e)) return PLD_ERR_INVALID;
    a.window = window;
    a.out = out, a.orow = o_row_stride, a.lse = lse;
    const hipStream_t s = (hipStream_t)stream;
    // Blocks of 256 rows read keys and values half as often; blocks of 128, two a CU, wait less for each
    // other and share out evener.  32 heads over 8 of 128: one sequence of 1024 rows 29.5 and 23.1 us, of 2048
    // 53.0 and 54.5, of 16384 1927 and 2206; 64 of 300 150 and 137, 16 of 1000 193 and 198.  Heads of
    // 64, whose vector instructions bound them, gain where a wave of 64 rows reads each value once for two
    // products: 2 x 8192 538 and 597, 4 x 4096 319 and 341, one of 4096 95 and 91, 2048 39 and 32, 16 x 1000
    // 111 and 107, in a window of 1000 187 and 176.  Not with a cap, whose instructions come on top: 4 x 4096
    // 470 and 450.
    const int64_t wide = ((int64_t)N * a.G + 255) / 256 * heads;
    const bool cap = softcap > 0.f, wide128 = wide >= 256 && N >= (int64_t)B * 512;
    if (head_dim == 64 && !cap && wide >= 1024 && N >= (int64_t)B * 3000)
        launch_prompt<64, 2, 4, false>(a, s);
    else if (head_dim == 64)
        cap ? launch_prompt<64, 1, 4, true>(a, s) : launch_prompt<64, 1, 4, false>(a, s);
    else if (head_dim == 128 && wide128)
        cap ? launch_prompt<128, 1, 8, true>(a, s) : launch_prompt<128, 1, 8, false>(a, s);
    else if (head_dim == 128)
        cap ? launch_prompt<128, 1, 4, true>(a, s) : launch_prompt<128, 1, 4, false>(a, s);
    else
        cap ? launch_prompt<256, 1, 4, true>(a, s) : launch_prompt<256, 1, 4, false>(a, s);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
