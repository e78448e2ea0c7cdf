// pld_prompt_attn.hip -- causal attention of packed prompts to themselves.
#include "pld_cache.h"
#include "pld_packed.h"

namespace pld {

struct PromptArgs {
    const uint16_t *q, *k, *v;
    int64_t qr, kr, vr;
    Packed p;
    int G, heads;                  // query heads per key head; key heads
    int64_t tiles;                 // of a key head's rows
    float c1;                      // products to scores in log2 units
    float cap, cap_x2, cap_near, inv2_log2e;   // as in AttnArgs
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
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max(int v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = max(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}

// 16 bytes a lane from base + off to LDS, lane after lane from `to` on, without a register between
// (a lane's place in LDS is fixed, so the swizzle is in the addresses it reads).  The caller waits
// (vmcnt): the compiler does not know of these loads.
__device__ __forceinline__ void load_to_lds(uint32_t to, const void *base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void block_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

constexpr float kSlack = 8.f;      // as in the cache's attention
constexpr float kNoMax = -1e30f;   // of a query that has seen no key

// kWaves waves of 32 kQT rows each: a tile of the rows of one key head, row m of all being query head
// m % G of row m / G, over the keys that they see, kKeys at a time.
template <int D, int kQT, int kWaves, int kKeys, bool kCap>
struct PromptTile {
    static constexpr int kRows = kWaves * 32 * kQT;
    static constexpr int kPieces = D / 8;                    // 16-byte pieces of a key's row
    static constexpr int kTileBytes = kKeys * D * 2;
    static constexpr int kLoads = kKeys * kPieces / 64 / kWaves;   // instructions a wave for a tile's keys
    static constexpr int kKT = kKeys / 32, kDT = D / 32;
    static_assert(kLoads >= 1);

    // Piece p of key j's row is at place p ^ key_swizzle(j) of it.
    // keys: lanes read one piece of consecutive keys, 8 in 128 bytes of banks and 16 in 256;
    // values: 16 lanes read two pieces of each of four keys, 32 four.
    __device__ __forceinline__ static int key_swizzle(int j) { return D == 64 ? (j & 7) ^ (j >> 3 & 1) : j & 15; }
    __device__ __forceinline__ static int value_swizzle(int j) { return D == 64 ? (j & 3) << 1 : (j & 1) * 10 ^ (j & 2) << 1; }
};

template <int D, int kQT, int kWaves, int kKeys, bool kCap>
__global__ __launch_bounds__(kWaves * 64) void prompt_attn_kernel(PromptArgs a) {
    using T = PromptTile<D, kQT, kWaves, kKeys, kCap>;
    constexpr int kKT = T::kKT, kDT = T::kDT, kLoads = T::kLoads;
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

    // ---- the rows: what each sees, [lo, hi), and its query
    int row[kQT], head[kQT], lo[kQT], hi[kQT];
    bf16x8_t qf[kQT][D / 16];
    int wave_lo = INT32_MAX, wave_hi = 0, full_lo = 0, full_hi = INT32_MAX;
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        const uint32_t m = (uint32_t)(over + (wave * kQT + t) * 32 + (lane & 31));
        const int r = (int)(m / (uint32_t)a.G);
        row[t] = (int)first + r;
        head[t] = kv * a.G + (int)m - r * a.G;
        const bool in = row[t] < a.p.N;
        if (!in) row[t] = a.p.N - 1;
        const uint4 *src = reinterpret_cast<const uint4 *>(a.q + row[t] * a.qr + (int64_t)head[t] * D);
#pragma unroll
        for (int s = 0; s < D / 16; ++s) qf[t][s] = __builtin_bit_cast(bf16x8_t, src[2 * s + h]);
        const Span sp = spans_of(a.p, row[t]);
        lo[t] = hi[t] = 0;
        if (in && sp.b >= 0) {
            hi[t] = row[t] + 1;
            lo[t] = min(max(max(sp.begin, 0), a.window ? hi[t] - a.window : 0), row[t]);
            wave_lo = min(wave_lo, lo[t]);
            wave_hi = max(wave_hi, hi[t]);
            full_lo = max(full_lo, lo[t]);
            full_hi = min(full_hi, hi[t]);
        }
    }
    wave_lo = wave_min(wave_lo), wave_hi = wave_max(wave_hi);
    full_lo = wave_max(full_lo), full_hi = wave_min(full_hi);
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
    const int n = (block_hi - block_lo + kKeys - 1) / kKeys;   // tiles of keys

    // ---- loads: instruction i of a wave brings pieces (wave kLoads + i) 64 .. + 63 of a tile
    const uint16_t *kbase = a.k + (int64_t)kv * D, *vbase = a.v + (int64_t)kv * D;
    auto place = [&](int i, int &j, int &p) {
        const int at = (wave * kLoads + i) * 64 + lane;
        j = at / T::kPieces, p = at % T::kPieces;
    };
    uint32_t koff[kLoads], voff[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        int j, p;
        place(i, j, p);
        koff[i] = (uint32_t)j * (uint32_t)(a.kr * 2) + (p ^ T::key_swizzle(j)) * 16;
        voff[i] = (uint32_t)j * (uint32_t)(a.vr * 2) + (p ^ T::value_swizzle(j)) * 16;
    }
    const uint32_t k_lds = (uint32_t)(uintptr_t)(lds_ptr)&s_k[0][0], v_lds = (uint32_t)(uintptr_t)(lds_ptr)&s_v[0][0];
    // tile i of keys or values to its buffer; the last key stands in for those past the block's
    auto fetch = [&](int i, bool values) {
        const int k0 = block_lo + i * kKeys;
        const uint16_t *base = values ? vbase + k0 * a.vr : kbase + k0 * a.kr;
        const uint32_t to = (values ? v_lds : k_lds) + (i & 1) * T::kTileBytes + wave * kLoads * 1024;
        if (k0 + kKeys <= block_hi) {
#pragma unroll
            for (int x = 0; x < kLoads; ++x) load_to_lds(to + x * 1024, base, values ? voff[x] : koff[x]);
        } else {
            const uint32_t stride = (uint32_t)((values ? a.vr : a.kr) * 2);
#pragma unroll
            for (int x = 0; x < kLoads; ++x) {
                int j, p;
                place(x, j, p);
                const uint32_t off = values ? voff[x] : koff[x];
                load_to_lds(to + x * 1024, base, off - (uint32_t)(j - min(j, block_hi - 1 - k0)) * stride);
            }
        }
    };

    // ---- the products
    f32x16_t o[kQT][kDT];
    float mx[kQT], l[kQT];
    auto scores = [&](int i, f32x16_t (&s)[kQT][kKT]) {
        const char *buf = s_k[i & 1];
#pragma unroll
        for (int kt = 0; kt < kKT; ++kt) {
            const int j = kt * 32 + (lane & 31);
#pragma unroll
            for (int t = 0; t < kQT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][kt][r] = 0.f;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
                const auto f = *reinterpret_cast<const bf16x8_t *>(buf + j * D * 2 + ((2 * x + h) ^ T::key_swizzle(j)) * 16);
#pragma unroll
                for (int t = 0; t < kQT; ++t) s[t][kt] = mfma32(f, qf[t][x], s[t][kt]);
            }
        }
    };
    auto value_operand = [&](const char *buf, int x, int dt) {   // 16 keys from 16 x on
        const int c = lane & 15, j = 16 * x + 4 * h + (c >> 2), p = dt * 4 + (lane >> 4 & 1) * 2 + (c >> 1 & 1);
        auto read = [&](int key) {
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4_t *>(
                (lds_ptr)(buf + key * D * 2 + (p ^ T::value_swizzle(key)) * 16 + (c & 1) * 8)));
        };
        const s16x4_t x0 = read(j), x1 = read(j + 8);
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Scores of tile i into the output: weights 2^(s c - m) against the running maximum m, which is
    // raised where a score is kSlack above it.
    auto attend = [&](int i, f32x16_t (&s)[kQT][kKT], bool careful) {
        const int k0 = block_lo + i * kKeys;
        float c = a.c1;
        if constexpr (kCap) {
            float w = 0.f;
#pragma unroll
            for (int t = 0; t < kQT; ++t)
#pragma unroll
                for (int kt = 0; kt < kKT; ++kt) {
                    s[t][kt] *= c;
#pragma unroll
                    for (int r = 0; r < 16; ++r) w = fmaxf(w, fabsf(s[t][kt][r]));
                }
            const bool far = __any(w >= a.cap_near);
#pragma unroll
            for (int t = 0; t < kQT; ++t)
#pragma unroll
                for (int kt = 0; kt < kKT; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[t][kt][r] = far ? soft_cap(s[t][kt][r], a.cap, a.cap_x2, a.cap_near, a.inv2_log2e)
                                          : soft_cap_near(s[t][kt][r], a.inv2_log2e);
            c = 1.f;
        }
        if (careful) {
            const uint64_t bad = ((uint64_t)s_bad[1] << 32 | s_bad[0]) >> 4 * h;
#pragma unroll
            for (int t = 0; t < kQT; ++t)
#pragma unroll
                for (int kt = 0; kt < kKT; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (bad >> (kt * 32 + 8 * (r / 4) + r % 4) & 1) s[t][kt][r] = __uint_as_float(0x7fc00000u);
        }
        if (k0 < full_lo || k0 + kKeys > full_hi) {
#pragma unroll
            for (int t = 0; t < kQT; ++t) {
                const int from = lo[t] - k0 - 4 * h, count = hi[t] - lo[t];
#pragma unroll
                for (int kt = 0; kt < kKT; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[t][kt][r] = (uint32_t)(kt * 32 + 8 * (r / 4) + r % 4 - from) < (uint32_t)count ? s[t][kt][r] : -INFINITY;
            }
        }
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            float top = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < kKT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][kt][r]);
            top *= c;
            if (__any(top > mx[t] + kSlack)) {
                // (a row by its own scores: its bits do not go by its neighbours')
                const float all = pair_max(top), mn = all > mx[t] + kSlack ? all : mx[t];
                const float f = __builtin_amdgcn_exp2f(mx[t] - mn);
                mx[t] = mn;
                l[t] *= f;
#pragma unroll
                for (int dt = 0; dt < kDT; ++dt) o[t][dt] *= f;
            }
#pragma unroll
            for (int kt = 0; kt < kKT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[t][kt][r] = __builtin_amdgcn_exp2f(fmaf(s[t][kt][r], c, -mx[t]));
                    l[t] += s[t][kt][r];
                }
        }
        const char *buf = s_v[i & 1];
#pragma unroll
        for (int x = 0; x < kKeys / 16; ++x) {
            bf16x8_t p[kQT];   // rounded to bf16, as the product takes them: half a step (2^-8) of each term
#pragma unroll
            for (int t = 0; t < kQT; ++t) {
                const f32x16_t &w = s[t][x / 2];
                const int r = x % 2 * 8;
                p[t] = __builtin_bit_cast(bf16x8_t, make_uint4(pack_bf16(w[r], w[r + 1]), pack_bf16(w[r + 2], w[r + 3]),
                                                               pack_bf16(w[r + 4], w[r + 5]), pack_bf16(w[r + 6], w[r + 7])));
            }
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt) {
                const bf16x8_t f = value_operand(buf, x, dt);
#pragma unroll
                for (int t = 0; t < kQT; ++t) o[t][dt] = mfma32(f, p[t], o[t][dt]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // What is not finite in tile i's values becomes 0, and its keys a bit each of s_bad (the block).
    auto clean = [&](int i) {
        if (threadIdx.x < 2) s_bad[threadIdx.x] = 0;
        __syncthreads();
        char *buf = s_v[i & 1];
        for (int at = threadIdx.x; at < kKeys * T::kPieces; at += kWaves * 64) {
            uint16_t *e = reinterpret_cast<uint16_t *>(buf + at * 16);
            bool hit = false;
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if ((e[x] & 0x7f80) == 0x7f80) e[x] = 0, hit = true;
            const int j = at / T::kPieces;
            if (hit) atomicOr(&s_bad[j >> 5], 1u << (j & 31));
        }
        __syncthreads();
    };

    // ---- the keys.  A weight of 0 times a value that is not finite would reach rows that do not see it:
    // where the output holds such a number at the end, all is done once more, with those values as 0
    // and NaN for the rows that see them.
    bool careful = false;
    for (;;) {
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            mx[t] = kNoMax, l[t] = 0.f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][dt][r] = 0.f;
        }
        fetch(0, false);
        fetch(0, true);
        for (int i = 0; i < n; ++i) {
            wait_loads();
            block_barrier();   // tile i is there, and all have done with tile i - 1
            if (careful) clean(i);
            if (i + 1 < n) {
                fetch(i + 1, false);
                fetch(i + 1, true);
            }
            const int k0 = block_lo + i * kKeys;
            if (k0 < wave_hi && k0 + kKeys > wave_lo) {
                f32x16_t s[kQT][kKT];
                scores(i, s);
                attend(i, s, careful);
            }
        }
        bool odd = false;
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            l[t] = pair_sum(l[t]);
            float x = 0.f;
#pragma unroll
            for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) x = fmaf(o[t][dt][r], 0.f, x);
            odd |= !(x == 0.f) || !(l[t] < INFINITY);
        }
        if (careful || !__syncthreads_or(odd)) break;
        careful = true;
    }

    // ---- out: a lane has four consecutive elements of every eight; the two lanes of a query trade
    // halves, so that each stores eight
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
        if (lo[t] >= hi[t]) continue;   // (both lanes of a query alike)
        const float inv = 1.f / l[t];
        uint16_t *dst = a.out + row[t] * a.orow + (int64_t)head[t] * D;
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
            a.lse[(int64_t)row[t] * a.G * a.heads + head[t]] = fmaf(mx[t], a.nat, __log2f(l[t]) * kLn2);
    }
}

template <int D, int kQT, int kWaves, int kKeys>
static void launch_prompt(PromptArgs &a, hipStream_t s) {
    a.tiles = ((int64_t)a.p.N * a.G + PromptTile<D, kQT, kWaves, kKeys, false>::kRows - 1) /
              PromptTile<D, kQT, kWaves, kKeys, false>::kRows;
    const dim3 grid = wide_grid(a.tiles * a.heads);
    if (a.cap > 0.f)
        hipLaunchKernelGGL((prompt_attn_kernel<D, kQT, kWaves, kKeys, true>), grid, dim3(kWaves * 64), 0, s, a);
    else
        hipLaunchKernelGGL((prompt_attn_kernel<D, kQT, kWaves, kKeys, false>), grid, dim3(kWaves * 64), 0, s, a);
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
    a.inv2_log2e = softcap > 0.f ? (float)(2. * kLog2E / a.cap) : 0.f;
    // (the way back from log2 units is by the rounded factor that led there)
    a.nat = softcap > 0.f ? (float)((double)softcap / a.cap) : (float)((double)scale / a.c1);
    if (!isfinite(a.c1) || !isfinite(a.cap_x2) || !isfinite(a.inv2_log2e)) return PLD_ERR_INVALID;
    a.window = window;
    a.out = out, a.orow = o_row_stride, a.lse = lse;
    const hipStream_t s = (hipStream_t)stream;
    if (head_dim == 64)
        launch_prompt<64, 1, 8, 64>(a, s);
    else if (head_dim == 128)
        launch_prompt<128, 1, 8, 64>(a, s);
    else
        launch_prompt<256, 1, 4, 32>(a, s);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
