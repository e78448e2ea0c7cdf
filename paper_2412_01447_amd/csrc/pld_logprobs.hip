// pld_logprobs.hip -- log probabilities of given tokens with the entropy and the
// most likely alternatives of their rows.
#include <float.h>
#include <math.h>

#include "pld_model.h"
#include "pld_verify.h"

namespace pld {

struct LogprobArgs {
    const void *logits;
    int64_t ls, lr;
    int V, n, B;
    const int32_t *tokens, *count;
    float k;            // log2(e) / tau
    float *logprob, *entropy;
    int top;
    int32_t *top_ids;
    float *top_lp;
    int segs;           // segments per row
    int4 *opened;       // [waves]: (sequence, row, last wave, -) of a row that spans waves
    float *partials;    // [waves][2]: maximum, mass, mass times exponent, -, then `top` keys
};

// A segment of a row is 32 elements a lane, one wave's work at a time, in 16-byte vectors:
// lane l has the vectors l, l + 64, ...  The segments of all rows that exist, in order, are
// dealt to the waves in equal contiguous ranges; a row that spans waves leaves one partial
// result per wave (slot 0 of a wave: a row that began before it, slot 1: one that ends
// after it), joined by a second launch.
constexpr int kLogElems = 32;
template <int P>
constexpr int kLogLoads = kLogElems / P;
constexpr int kLogBlocks = 1024, kLogWaves = 4;   // 16 waves a CU
constexpr int kKeys = 512;                        // keys a wave keeps at most before it sorts them out
constexpr int kHits = 32;

// A mass is 2^x with x = z k - c for a c near the largest z k: one fused multiply-add whose
// only error is x's own rounding, whatever c is.  s sums 2^x, t sums 2^x x (the entropy is
// (log2 s - t / s) ln 2).  x is bounded so that -inf weighs nothing and 0 times x stays 0.
// c = kNoMass: nothing but -inf so far.
constexpr float kNoMass = -FLT_MAX;
__device__ __forceinline__ float bounded(float x) { return fmaxf(x, -1e4f); }
struct Mass {
    float c = kNoMass, s = 0.f, t = 0.f;
    // to a reference cn >= c
    __device__ __forceinline__ void raise(float cn) {
        const float d = bounded(c - cn), f = __builtin_amdgcn_exp2f(d);
        t = f * fmaf(d, s, t);
        s *= f;
        c = cn;
    }
    __device__ __forceinline__ void add(float z, float k) {
        const float x = bounded(fmaf(z, k, -c)), e = __builtin_amdgcn_exp2f(x);
        s += e;
        t = fmaf(e, x, t);
    }
};
// The reference of a largest value z (finite, also where z k is not).
__device__ __forceinline__ float reference(float z, float k) { return fminf(fmaxf(z * k, kNoMass), FLT_MAX); }

// The next float above v.
__device__ __forceinline__ float next_up(float v) {
    const uint32_t o = ord_f32(v);
    return o == 0xff800000u ? v : unord_f32(o + 1);
}

// The N best keys (value, then lowest index) of what a wave has seen, in its part of LDS:
// `cnt` keys, of which compress() leaves the best N, sorted.  Keys below `floor`, and values
// below `at`, cannot be among them.
struct Best {
    uint64_t *buf, *sorted;   // [kKeys], [PLD_MAX_TOP]
    int N, cnt;
    uint64_t floor;
    float at;
    bool full;   // N keys at or above `at` are there

    __device__ __forceinline__ void reset() {
        cnt = 0;
        full = false;
        floor = 0;
        at = -INFINITY;
    }
    // Ranks by counting: the keys are distinct.
    __device__ __forceinline__ void compress() {
        const int lane = lane_id();
        for (int i = lane; i - lane < cnt; i += kWave) {
            const uint64_t key = i < cnt ? buf[i] : 0;
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < cnt; ++j) rank += buf[j] > key;
            if (i < cnt && rank < N) sorted[rank] = key;
        }
        cnt = min(cnt, N);
        asm volatile("" ::: "memory");   // (one wave's LDS operations complete in order)
        if (lane < cnt) buf[lane] = sorted[lane];
        asm volatile("" ::: "memory");
        if (cnt == N) {
            const uint64_t last = sorted[N - 1];
            floor = max(floor, last + 1);
            at = fmaxf(at, unord_f32((uint32_t)(last >> 32)));
            full = true;
        }
    }
    __device__ __forceinline__ void append(uint64_t key, bool pred) {
        pred = pred && key >= floor;
        const uint64_t mask = __ballot(pred);
        if (mask == 0) return;
        if (pred) buf[cnt + __popcll(mask & lanemask_lt())] = key;
        cnt += __popcll(mask);
        asm volatile("" ::: "memory");
        if (cnt > kKeys - kWave) compress();
    }
    // The N-th best of the lanes' own best values (`own`, as ord_f32 has them; 0: none) is a
    // floor; where more lanes than are needed have it, the indexes (`index`, called then)
    // decide.  Of a bf16 value the upper half of ord_f32 says all.
    template <bool kBf16, class Index>
    __device__ __forceinline__ void raise_floor(uint32_t own, Index index) {
        uint32_t v = 0, w = 0;
        for (uint32_t bit = 1u << 31; bit > (kBf16 ? 0x8000u : 0u); bit >>= 1)
            if (__popcll(__ballot(own >= (v | bit))) >= N) v |= bit;
        if (v == 0) return;   // fewer than N lanes have one
        if (kBf16 && !(v >> 31)) v |= 0xffffu;
        const int need = N - __popcll(__ballot(own > v));
        if (__popcll(__ballot(own == v)) > need) {
            const uint32_t lo = own == v ? 0xffffffffu - index() : 0;
            for (uint32_t bit = 1u << 31; bit; bit >>= 1)
                if (__popcll(__ballot(lo >= (w | bit))) >= need) w |= bit;
        }
        floor = max(floor, (uint64_t)v << 32 | w);
        at = fmaxf(at, unord_f32(v));
    }
};

// What a row's results come from: its mass over all lanes or waves, and its best keys.
template <int kBf16>
__device__ __forceinline__ void put_row(const LogprobArgs &a, int b, int i, Mass w, const Best &best) {
    using E = Elem<kBf16>;
    using T = typename E::T;
    const T *z = reinterpret_cast<const T *>(a.logits) + (int64_t)b * a.ls + (int64_t)i * a.lr;
    const int lane = lane_id();
    const int64_t at = (int64_t)b * a.n + i;
    // No mass: only -inf, or logits so low (a mask of the type's lowest value) that times k
    // they overflow: then relative to their own maximum m.
    bool none = false;
    float m = 0.f;
    if (!(w.s > 0.f)) {
        m = -INFINITY;
        for (int v = lane; v < a.V; v += kWave) m = fmaxf(m, E::get(z, v));
        m = wave_max_f32(m);
        none = !(m > -INFINITY);
        w = Mass{0.f, 0.f, 0.f};
        for (int v = lane; v < a.V && !none; v += kWave) w.add(E::get(z, v) - m, a.k);
        w.s = wave_sum_f32(w.s);
        w.t = wave_sum_f32(w.t);
    }
    const float log2_s = __builtin_amdgcn_logf(w.s);
    auto logprob = [&](float x) { return none ? -INFINITY : (fmaf(x - m, a.k, -w.c) - log2_s) * 0.6931471805599453f; };
    if (lane == 0) {
        const int tok = a.tokens[at];
        a.logprob[at] = tok >= 0 && tok < a.V ? logprob(E::get(z, tok)) : __uint_as_float(0x7fc00000u);
        if (a.entropy) a.entropy[at] = none ? 0.f : fmaxf((log2_s - w.t / w.s) * 0.6931471805599453f, 0.f);
    }
    if (lane < a.top) {
        const bool have = lane < best.cnt;
        const uint64_t key = have ? best.buf[lane] : 0;
        a.top_ids[at * a.top + lane] = have ? (int)argmax_key_index(key) : -1;
        a.top_lp[at * a.top + lane] = have ? logprob(unord_f32((uint32_t)(key >> 32))) : -INFINITY;
    }
}

// (whole 16-byte vectors)
__host__ __device__ inline int part_floats(int top) { return 4 + 4 * ((top + 1) / 2); }
__device__ __forceinline__ float *partial_at(const LogprobArgs &a, int wave, int slot) {
    return a.partials + ((int64_t)wave * 2 + slot) * part_floats(a.top);
}

__device__ __forceinline__ int rows_of(const LogprobArgs &a, int b) {
    const int c = a.count ? a.count[b] : a.n;
    return c < 0 || c > a.n ? 0 : c;
}

// A vector's elements back together (exact).
__device__ __forceinline__ uint4 pack(const float (&z)[4]) {
    return make_uint4(__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3]));
}
__device__ __forceinline__ uint4 pack(const float (&z)[8]) {
    auto two = [&](int i) { return __float_as_uint(z[i]) >> 16 | __float_as_uint(z[i + 1]); };
    return make_uint4(two(0), two(2), two(4), two(6));
}

template <int kBf16, bool kTop>
__global__ __launch_bounds__(kLogWaves * 64, 4) void token_logprobs_kernel(LogprobArgs a) {
    using E = Elem<kBf16>;
    using T = typename E::T;
    constexpr int P = E::kPerVec;
    constexpr uint32_t kNegInf2 = kBf16 ? 0xff80ff80u : 0xff800000u;
    constexpr int L = kLogLoads<P>, kVecs = L * kWave;
    __shared__ uint64_t s_keys[kTop ? kLogWaves : 1][kTop ? kKeys + PLD_MAX_TOP : 1];
    __shared__ uint4 s_hits[kTop ? kLogWaves : 1][kTop ? kHits : 1][L];
    __shared__ int64_t s_w[kLogWaves], s_first[kLogWaves];
    __shared__ int s_b[kLogWaves];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);

    // The waves' ranges: rows before each thread's own sequences.
    const int per = (a.B + 255) / 256, b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += rows_of(a, b);
    int64_t before = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int64_t x = __shfl_up(before, o);
        if (lane >= o) before += x;
    }
    if (lane == 63) s_w[wave] = before;
    __syncthreads();
    int64_t rows = 0;
    before -= mine;
    for (int w = 0; w < kLogWaves; ++w) {
        if (w < wave) before += s_w[w];
        rows += s_w[w];
    }
    // as many ranges as waves, or as segments where there are fewer: none between two is empty
    const int64_t total = rows * a.segs, ranges = min(total, (int64_t)gridDim.x * kLogWaves);
    for (int w = 0; w < kLogWaves; ++w) {
        const int64_t id = (int64_t)blockIdx.x * kLogWaves + w;
        if (id >= ranges) break;
        const int64_t r0 = total * id / ranges / a.segs;   // the row of its first segment
        if (before <= r0 && r0 < before + mine) {
            int64_t f = before;
            int b = b0;
            for (int c; r0 >= f + (c = rows_of(a, b)); ++b) f += c;
            s_b[w] = b;
            s_first[w] = f;
        }
    }
    __syncthreads();
    const int id = (int)blockIdx.x * kLogWaves + wave;
    int4 opened = make_int4(-1, 0, 0, 0);
    if (id >= ranges) {
        if (lane == 0) a.opened[id] = opened;
        return;
    }
    int64_t x = total * id / ranges;
    const int64_t x1 = total * (id + 1) / ranges;
    int b = __builtin_amdgcn_readfirstlane(s_b[wave]), cnt = rows_of(a, b);
    int i = (int)(x / a.segs - s_first[wave]), g = (int)(x % a.segs);
    Best best{s_keys[kTop ? wave : 0], s_keys[kTop ? wave : 0] + (kTop ? kKeys : 0), a.top, 0, 0, -INFINITY, false};

    while (x < x1) {
        const RowView<T, P> rv = row_view<T, P>(a.logits, a.ls, a.lr, b, i, a.V);
        const int g0 = g, g1 = (int)min((int64_t)a.segs, g + (x1 - x));
        Mass w;
        best.reset();
        uint4 r[L];
        auto load = [&](int seg) {
            const int64_t v0 = (int64_t)seg * kVecs + lane;
#pragma unroll
            for (int u = 0; u < L; ++u) {
                r[u] = make_uint4(kNegInf2, kNegInf2, kNegInf2, kNegInf2);
                if (v0 + u * kWave < rv.nvec) r[u] = ld_stream(rv.vec + v0 + u * kWave);
            }
        };
        load(g);
        for (; g < g1; ++g) {
            const int64_t v0 = (int64_t)g * kVecs + lane;
            const bool head = g == 0 && lane < rv.head;
            const bool tail = g == a.segs - 1 && rv.body_end + lane < a.V;
            const float zh = head ? E::get(rv.row, lane) : -INFINITY;
            const float zt = tail ? E::get(rv.row, rv.body_end + lane) : -INFINITY;
            float z[L][P], top = fmaxf(zh, zt);
#pragma unroll
            for (int u = 0; u < L; ++u) {
                E::unpack(r[u], z[u]);
#pragma unroll
                for (int e = 0; e < P; ++e) top = fmaxf(top, z[u][e]);
            }
            if (g + 1 < g1) load(g + 1);   // under this segment's work
            w.raise(fmaxf(w.c, reference(top, a.k)));
            w.add(zh, a.k);
            w.add(zt, a.k);
#pragma unroll
            for (int u = 0; u < L; ++u)
#pragma unroll
                for (int e = 0; e < P; ++e) w.add(z[u][e], a.k);
            if constexpr (kTop) {
                // Values from `gate` on are looked at.  With N keys already, a later equal
                // value loses to them; before that, the lanes' own maxima give a floor.
                const bool boot = !best.full;
                if (boot)
                    best.raise_floor<kBf16>(head || tail || v0 < rv.nvec ? ord_f32(top) : 0, [&] {
                        // this lane's lowest index of `top`
                        uint32_t idx = 0xffffffffu;
                        if (zt == top && tail) idx = (uint32_t)(rv.body_end + lane);
#pragma unroll
                        for (int u = L - 1; u >= 0; --u) {
                            const bool in = v0 + u * kWave < rv.nvec;
#pragma unroll
                            for (int e = P - 1; e >= 0; --e)
                                if (in && z[u][e] == top) idx = (uint32_t)(rv.head + (v0 + u * kWave) * P + e);
                        }
                        if (zh == top && head) idx = (uint32_t)lane;
                        return idx;
                    });
                const float gate = boot ? best.at : next_up(best.at);
                uint64_t hits = __ballot(top >= gate);
                if (hits) {
                    best.append(argmax_key(zh, (uint32_t)lane), head && zh >= gate);
                    // The lanes with such values put their vectors into LDS, kHits at a time,
                    // and the wave reads a lane's elements side by side.
                    while (hits) {
                        const int slot = __popcll(hits & lanemask_lt());
                        if (((hits >> lane) & 1) && slot < kHits) {
#pragma unroll
                            for (int u = 0; u < L; ++u) s_hits[wave][slot][u] = pack(z[u]);
                        }
                        asm volatile("" ::: "memory");
                        // two lanes' elements side by side
                        const int e = lane & (kLogElems - 1), half = lane / kLogElems;
                        constexpr int kAhead = kBf16 ? 2 : 1;
                        for (int h = 0; hits && h < kHits; h += 2 * kAhead) {
                            float y[kAhead];
#pragma unroll
                            for (int q = 0; q < kAhead; ++q)
                                y[q] = E::get(reinterpret_cast<const T *>(s_hits[wave][h + 2 * q + half]), e);
#pragma unroll
                            for (int q = 0; q < kAhead; ++q) {
                                if (hits == 0) break;
                                const int l0 = __ffsll((unsigned long long)hits) - 1;
                                hits &= hits - 1;
                                const int l1 = __ffsll((unsigned long long)hits) - 1;   // -1: none
                                hits &= hits - 1;
                                const int from = half ? l1 : l0;
                                const int64_t vi = (int64_t)g * kVecs + from + (e / P) * kWave;
                                best.append(argmax_key(y[q], (uint32_t)(rv.head + vi * P + e % P)),
                                            from >= 0 && vi < rv.nvec && y[q] >= gate);
                            }
                        }
                        asm volatile("" ::: "memory");
                    }
                    best.append(argmax_key(zt, (uint32_t)(rv.body_end + lane)), tail && zt >= gate);
                    if (boot || best.cnt > 2 * kWave) best.compress();
                }
            }
        }
        if constexpr (kTop) best.compress();
        x += g1 - g0;
        // the lanes' masses to a common maximum
        w.raise(wave_max_f32(w.c));
        w.s = wave_sum_f32(w.s);
        w.t = wave_sum_f32(w.t);
        if (g0 == 0 && g1 == a.segs) {
            put_row<kBf16>(a, b, i, w, best);
        } else {
            float *part = partial_at(a, id, g0 == 0);
            if (lane == 0) *reinterpret_cast<float4 *>(part) = make_float4(w.c, w.s, w.t, 0.f);
            if (kTop && lane < a.top) reinterpret_cast<uint64_t *>(part + 4)[lane] = lane < best.cnt ? best.buf[lane] : 0;
            if (g0 == 0) {
                const int64_t end = x + (a.segs - g1);   // of the row
                opened = make_int4(b, i, (int)((end * ranges - 1) / total), 0);
            }
        }
        g = 0;
        if (x < x1 && ++i >= cnt) {
            i = 0;
            do cnt = rows_of(a, ++b);
            while (cnt == 0);
        }
    }
    if (lane == 0) a.opened[id] = opened;
}

// A wave per row that spans waves, in the order of the waves that open one.
template <int kBf16, bool kTop>
__global__ __launch_bounds__(kLogWaves * 64) void token_logprobs_join_kernel(LogprobArgs a) {
    __shared__ uint64_t s_keys[kTop ? kLogWaves : 1][kTop ? kKeys + PLD_MAX_TOP : 1];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int id = (int)blockIdx.x * kLogWaves + wave;
    const int4 row = a.opened[id];
    if (row.x < 0) return;
    const int parts = row.z - id + 1;
    auto part = [&](int p) { return partial_at(a, id + p, p == 0); };
    Mass w;
    for (int p = lane; p < parts; p += 64) {
        const float4 v = *reinterpret_cast<const float4 *>(part(p));
        Mass o;
        o.c = v.x, o.s = v.y, o.t = v.z;
        const float cn = fmaxf(w.c, o.c);
        w.raise(cn);
        o.raise(cn);
        w.s += o.s;
        w.t += o.t;
    }
    w.raise(wave_max_f32(w.c));
    w.s = wave_sum_f32(w.s);
    w.t = wave_sum_f32(w.t);
    Best best{s_keys[kTop ? wave : 0], s_keys[kTop ? wave : 0] + (kTop ? kKeys : 0), a.top, 0, 0, -INFINITY, false};
    if constexpr (kTop) {
        best.reset();
        // sorted lists: 64 of them at a time, to the depth at which none has a key in reach
        for (int p0 = 0; p0 < parts; p0 += 64) {
            const bool in = p0 + lane < parts;
            const uint64_t *list = reinterpret_cast<const uint64_t *>(part(in ? p0 + lane : 0) + 4);
            constexpr int kAhead = 4;
            for (int k0 = 0; k0 < a.top; k0 += kAhead) {
                uint64_t key[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) key[k] = in && k0 + k < a.top ? list[k0 + k] : 0;
                if (k0 == 0 && !best.full)
                    best.raise_floor<false>((uint32_t)(key[0] >> 32), [&] { return argmax_key_index(key[0]); });
                bool any = false;
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    any = __any(key[k] != 0 && key[k] >= best.floor);
                    if (any) best.append(key[k], key[k] != 0);
                }
                if (!any) break;
            }
            best.compress();
        }
    }
    put_row<kBf16>(a, row.x, row.y, w, best);
}

static int log_segs(int V) {
    const int64_t per = kLogElems * kWave;
    return (int)((V + per - 1) / per);
}
static int log_blocks(int B, int n, int segs) {
    const int64_t waves = (int64_t)B * n * segs, blocks = (waves + kLogWaves - 1) / kLogWaves;
    return (int)(blocks < kLogBlocks ? blocks : kLogBlocks);
}

}  // namespace pld

using namespace pld;

extern "C" size_t pld_token_logprobs_workspace_bytes(int B, int n, int V, int dtype, int top) {
    if (B < 1 || B > 65535 || n < 1 || n > 65535 || V < 1 || (dtype != PLD_F32 && dtype != PLD_BF16) ||
        top < 0 || top > PLD_MAX_TOP)
        return 0;
    const size_t waves = (size_t)log_blocks(B, n, log_segs(V)) * kLogWaves;
    return waves * (sizeof(int4) + 2 * (size_t)part_floats(top) * sizeof(float));
}

extern "C" int pld_token_logprobs(const void *logits, int dtype, int64_t l_seq_stride,
                                  int64_t l_row_stride, int V, int n, const int32_t *tokens,
                                  const int32_t *count, int B, double temperature, float *logprob,
                                  float *entropy, int top, int32_t *top_ids, float *top_logprobs,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    if (!logits || !tokens || !logprob) return PLD_ERR_INVALID;
    const size_t need = pld_token_logprobs_workspace_bytes(B, n, V, dtype, top);
    if (need == 0 || (top > 0 && (!top_ids || !top_logprobs))) return PLD_ERR_INVALID;
    if ((n > 1 && l_row_stride < V) || (B > 1 && l_seq_stride < V)) return PLD_ERR_INVALID;
    if (!(temperature > 0.0) || !(temperature <= DBL_MAX)) return PLD_ERR_INVALID;
    const double k = 1.4426950408889634 / temperature;
    if (!(k <= FLT_MAX)) return PLD_ERR_INVALID;
    if ((uintptr_t)logits % (dtype == PLD_F32 ? 4 : 2)) return PLD_ERR_ALIGN;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need) return PLD_ERR_WORKSPACE;
    LogprobArgs a{};
    a.logits = logits, a.ls = l_seq_stride, a.lr = l_row_stride;
    a.V = V, a.n = n, a.B = B;
    a.tokens = tokens, a.count = count;
    a.k = (float)k;
    a.logprob = logprob, a.entropy = entropy;
    a.top = top, a.top_ids = top_ids, a.top_lp = top_logprobs;
    a.segs = log_segs(V);
    const int blocks = log_blocks(B, n, a.segs);
    a.opened = static_cast<int4 *>(workspace);
    a.partials = reinterpret_cast<float *>(a.opened + (size_t)blocks * kLogWaves);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kLogWaves * 64), 0, (hipStream_t)stream, a);
    };
    auto both = [&](auto bf16) {
        constexpr int kBf16 = decltype(bf16)::value;
        if (top > 0) {
            go(token_logprobs_kernel<kBf16, true>);
            go(token_logprobs_join_kernel<kBf16, true>);
        } else {
            go(token_logprobs_kernel<kBf16, false>);
            go(token_logprobs_join_kernel<kBf16, false>);
        }
    };
    if (dtype == PLD_F32)
        both(std::integral_constant<int, 0>{});
    else
        both(std::integral_constant<int, 1>{});
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
