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
    int2 *parts;        // [B][n]: first and last wave of a row; (0, -1): one wave has it whole
    float4 *masses;     // [waves][2]: reference, mass, mass times exponent of a wave's part of a row
    float4 *whole;      // [B][n]: the same of a row that one wave has whole
    void *maxima;       // [B][n][segs][64], the logits' type: each lane's largest value of a segment
};

// A segment of a row is 32 elements a lane, one wave's work at a time, in 16-byte vectors: lane
// l has the vectors l, l + 64, ...  The segments of all rows that exist, in order, are dealt to
// the waves in equal contiguous ranges.  A wave sums up the masses of its part of a row (slot
// 0: a row that began before it, slot 1: one that begins in it and ends after it, at most one
// each; rows that do both in it have a place of their own, since of those there are several to
// a wave where there are more rows than waves) and, where alternatives are asked for, keeps
// each lane's largest value of a segment: 1/32 of the logits, which tell a second launch, a
// wave per row, where the row's best elements are. (Kept by the first pass itself, the best
// twenty cost as much as the pass: 95 us, and 46 without them, for 64 x 17 rows of 128256 in
// bf16.)  Where 920 of these rows exist (236 MB) the pass takes 48 us, 4.9 TB/s: the card's
// reads would take 33 us, and so would an element's exponential and the six or seven other
// vector instructions.  The second launch takes 12 us with 20 alternatives.
constexpr int kLogElems = 32;
template <int P>
constexpr int kLogLoads = kLogElems / P;
constexpr int kLogBlocks = 1024, kLogWaves = 4;   // 16 waves a CU
constexpr int kKeys = 256;                        // keys a wave keeps at most before it sorts them out
constexpr int kGroups = 256;                      // (segment, lane) groups of elements to look at

// A mass is 2^x with x = z k - c for c the largest z k, rounded: one fused multiply-add whose
// only error is x's own rounding.  Up to |c| = 2^24 that c is rounded by at most 1/2, and all of
// the row's x with it; past that x would leave the range of 2^x, and the row is summed up again
// relative to its largest z, by the finishing launch.  s sums 2^x, t sums 2^x x (the entropy is
// (log2 s - t / s) ln 2).  x is bounded so that -inf weighs nothing and 0 times x stays 0.
// c = kNoMass: nothing but -inf so far.
constexpr float kNoMass = -FLT_MAX, kMostReference = 0x1p24f;
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
    // all lanes' masses together, in every lane
    __device__ __forceinline__ void join_lanes() {
        raise(wave_max_f32(c));
        s = wave_sum_f32(s);
        t = wave_sum_f32(t);
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
    int N, cnt = 0;
    uint64_t floor = 0;
    float at = -INFINITY;
    bool full = false;        // N keys at or above `at` are there

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
    // As append(), for up to kEach keys a lane (key(e) where `mask` has bit e): in one go
    // where there is room, which there is but for rows of many equal values.
    template <int kEach, class Key>
    __device__ __forceinline__ void append_some(uint32_t mask, Key key) {
        int total;
        int to = cnt + wave_excl_scan(__popc(mask), total);
        if (total == 0) return;
        if (cnt + total <= kKeys) {
            cnt += total;
            for (; mask; mask &= mask - 1) buf[to++] = key(__ffs(mask) - 1);
            asm volatile("" ::: "memory");
            if (cnt > kKeys - kWave) compress();
        } else {
            for (int e = 0; e < kEach; ++e) append(key(e), (mask >> e) & 1);
        }
    }
    // The N-th best of the lanes' own best values (`own`, kOwn a lane, as ord_f32 has them; 0:
    // none) is a floor of the values.  Of a bf16 value the upper half of ord_f32 says all.
    template <bool kBf16, int kOwn>
    __device__ __forceinline__ void raise_floor(const uint32_t (&own)[kOwn]) {
        uint32_t v = 0;
        for (uint32_t bit = 1u << 31; bit > (kBf16 ? 0x8000u : 0u); bit >>= 1) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) n += __popcll(__ballot(own[i] >= (v | bit)));
            if (n >= N) v |= bit;
        }
        if (v == 0) return;   // there are fewer than N
        if (kBf16 && !(v >> 31)) v |= 0xffffu;
        floor = max(floor, (uint64_t)v << 32);
        at = fmaxf(at, unord_f32(v));
    }
};

__device__ __forceinline__ int rows_of(const LogprobArgs &a, int b) {
    const int c = a.count ? a.count[b] : a.n;
    return c < 0 || c > a.n ? 0 : c;
}

template <int kBf16, bool kTop>
__global__ __launch_bounds__(kLogWaves * 64, 4) void token_logprobs_kernel(LogprobArgs a) {
    using E = Elem<kBf16>;
    using T = typename E::T;
    constexpr int P = E::kPerVec;
    constexpr uint32_t kNegInf2 = kBf16 ? 0xff80ff80u : 0xff800000u;
    constexpr int L = kLogLoads<P>, kVecs = L * kWave;
    __shared__ int64_t s_w[kLogWaves], s_first[kLogWaves];
    __shared__ int s_b[kLogWaves];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);

    // The waves' ranges: rows before each thread's own sequences.
    const int per = (a.B + 255) / 256, b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += rows_of(a, b);
    int64_t before = wave_incl_scan(mine);
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
    const int64_t share = ranges ? quotient(total, ranges) : 0, longer = total - share * ranges;
    auto start = [&](int64_t id) { return share * id + min(id, longer); };
    auto range_of = [&](int64_t x) {
        const int64_t of_longer = (share + 1) * longer;
        return (int)(x < of_longer ? quotient(x, share + 1) : longer + quotient(x - of_longer, share));
    };
    for (int w = 0; w < kLogWaves; ++w) {
        const int64_t id = (int64_t)blockIdx.x * kLogWaves + w;
        if (id >= ranges) break;
        const int64_t r0 = quotient(start(id), a.segs);   // the row of its first segment
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
    if (id >= ranges) return;
    int64_t x = start(id);
    const int64_t x1 = start(id + 1);
    int b = __builtin_amdgcn_readfirstlane(s_b[wave]), cnt = rows_of(a, b);
    const int64_t x_row = quotient(x, a.segs);
    int i = (int)(x_row - s_first[wave]), g = (int)(x - x_row * a.segs);

    while (x < x1) {
        const RowView<T, P> rv = row_view<T, P>(a.logits, a.ls, a.lr, b, i, a.V);
        const int64_t row = (int64_t)b * a.n + i;
        const int g0 = g, g1 = (int)min((int64_t)a.segs, g + (x1 - x));
        Mass w;
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
            // elements before the first whole vector, or after the last one
            float zh = -INFINITY, zt = -INFINITY;
            const bool ends = (g == 0 && rv.head) || (g == a.segs - 1 && rv.body_end < a.V);
            if (ends) {
                if (g == 0 && lane < rv.head) zh = E::get(rv.row, lane);
                if (g == a.segs - 1 && rv.body_end + lane < a.V) zt = E::get(rv.row, rv.body_end + lane);
            }
            float z[L][P], top = fmaxf(zh, zt);
#pragma unroll
            for (int u = 0; u < L; ++u) {
                E::unpack(r[u], z[u]);
#pragma unroll
                for (int e = 0; e < P; ++e) top = fmaxf(top, z[u][e]);
            }
            if (g + 1 < g1) load(g + 1);   // under this segment's work
            if constexpr (kTop) {
                const int64_t at = (row * a.segs + g) * kWave + lane;
                if constexpr (kBf16)
                    static_cast<uint16_t *>(a.maxima)[at] = (uint16_t)(__float_as_uint(top) >> 16);
                else
                    static_cast<float *>(a.maxima)[at] = top;
            }
            w.raise(fmaxf(w.c, reference(top, a.k)));
            if (ends) {
                w.add(zh, a.k);
                w.add(zt, a.k);
            }
#pragma unroll
            for (int u = 0; u < L; ++u)
#pragma unroll
                for (int e = 0; e < P; ++e) w.add(z[u][e], a.k);
        }
        x += g1 - g0;
        w.join_lanes();
        if (lane == 0) {
            const bool begins = g0 == 0, whole = begins && g1 == a.segs;
            (whole ? a.whole[row] : a.masses[(int64_t)id * 2 + begins]) = make_float4(w.c, w.s, w.t, 0.f);
            if (begins) a.parts[row] = whole ? make_int2(0, -1) : make_int2(id, range_of(x + (a.segs - g1) - 1));
        }
        g = 0;
        if (x < x1 && ++i >= cnt) {
            i = 0;
            do cnt = rows_of(a, ++b);
            while (cnt == 0);
        }
    }
}

// A wave per row: the masses of its parts joined, and its best elements.
template <int kBf16, bool kTop>
__global__ __launch_bounds__(kLogWaves * 64) void token_logprobs_finish_kernel(LogprobArgs a) {
    using E = Elem<kBf16>;
    using T = typename E::T;
    constexpr int P = E::kPerVec, L = kLogLoads<P>, kVecs = L * kWave;
    __shared__ uint64_t s_keys[kTop ? kLogWaves : 1][kTop ? kKeys + PLD_MAX_TOP : 1];
    __shared__ int s_groups[kTop ? kLogWaves : 1][kTop ? kGroups : 1];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int b = blockIdx.y, i = (int)blockIdx.x * kLogWaves + wave;
    if (i >= a.n) return;
    // What does not go by the count is asked for together with it, whether the row exists or
    // not: a wave has little else to do than to wait.
    const int64_t row = (int64_t)b * a.n + i;
    const int cnt = rows_of(a, b);
    const int2 part = a.parts[row];
    const float4 whole = a.whole[row];
    const int tok = a.tokens[row];
    constexpr int kChunk = 8;   // vectors a lane: a bf16 row of up to 131072 at once
    const uint4 *maxima = reinterpret_cast<const uint4 *>(static_cast<const T *>(a.maxima) + row * a.segs * kWave);
    const int vecs = a.segs * (kWave / P);
    uint4 mv[kChunk];
    auto load = [&](int v0) {
#pragma unroll
        for (int q = 0; q < kChunk; ++q) mv[q] = maxima[min(v0 + q * kWave + lane, vecs - 1)];
    };
    // Each lane's largest of the maxima, of each fourth element; the top-th largest of the lanes',
    // or for many alternatives of all 256, is a floor.
    float own[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if constexpr (kTop) {
        for (int v0 = 0; v0 < vecs; v0 += kChunk * kWave) {
            load(v0);
            // (no other lane's vector in place of an absent one: the floor counts lanes)
#pragma unroll
            for (int q = 0; q < kChunk; ++q) {
                float y[P];
                E::unpack(mv[q], y);
                if (v0 + q * kWave + lane < vecs)
#pragma unroll
                    for (int e = 0; e < P; ++e) own[e % 4] = fmaxf(own[e % 4], y[e]);
            }
        }
    }
    if (i >= cnt) return;
    const RowView<T, P> rv = row_view<T, P>(a.logits, a.ls, a.lr, b, i, a.V);
    const float z_tok = E::get(rv.row, tok >= 0 && tok < a.V ? tok : 0);
    Mass w;
    if (part.y < 0 && lane == 0) w.c = whole.x, w.s = whole.y, w.t = whole.z;
    for (int p = part.x + lane; p <= part.y; p += kWave) {
        const float4 v = a.masses[(int64_t)p * 2 + (p == part.x)];
        Mass o;
        o.c = v.x, o.s = v.y, o.t = v.z;
        const float cn = fmaxf(w.c, o.c);
        w.raise(cn);
        o.raise(cn);
        w.s += o.s;
        w.t += o.t;
    }

    Best best{s_keys[kTop ? wave : 0], s_keys[kTop ? wave : 0] + (kTop ? kKeys : 0), a.top};
    if constexpr (kTop) {
        // (of 64 values the 64th best is so low that some 260 groups of a row reach it, of 256 some 80:
        // one row of 160000 in fp32 with 64 alternatives takes 22 us by them and took 65)
        if (a.top > 32) {
            uint32_t four[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) four[i] = lane < vecs ? ord_f32(own[i]) : 0;
            best.raise_floor<kBf16>(four);
        } else {
            const float most = fmaxf(fmaxf(own[0], own[1]), fmaxf(own[2], own[3]));
            const uint32_t one[1] = {lane < vecs ? ord_f32(most) : 0};
            best.raise_floor<kBf16>(one);
        }

        // The groups of a list of (segment, lane), L lanes each: a vector a lane.
        int *groups = s_groups[wave];
        int listed = 0;
        auto look = [&] {
            asm volatile("" ::: "memory");
            constexpr int kEach = kWave / L, kRounds = 4;   // groups a round, rounds in flight
            for (int q0 = 0; q0 < listed; q0 += kEach * kRounds) {
            uint4 vec[kRounds];
            int at_group[kRounds];
#pragma unroll
            for (int t = 0; t < kRounds; ++t) {
                at_group[t] = groups[min(q0 + t * kEach + lane / L, listed - 1)];
                const int64_t vi = (int64_t)(at_group[t] / kWave) * kVecs + at_group[t] % kWave + lane % L * kWave;
                vec[t] = rv.nvec ? rv.vec[min(vi, (int64_t)rv.nvec - 1)] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int t = 0; t < kRounds; ++t) {
                const int q = q0 + t * kEach + lane / L, u = lane % L;
                if (q0 + t * kEach >= listed) continue;
                const int seg = at_group[t] / kWave, l = at_group[t] % kWave;
                const int64_t vi = (int64_t)seg * kVecs + l + u * kWave;
                float z[P];
                E::unpack(vec[t], z);
                uint32_t mask = 0;
                auto key = [&](int e) {
                    float y = z[0];
#pragma unroll
                    for (int f = 1; f < P; ++f) y = e == f ? z[f] : y;
                    return argmax_key(y, (uint32_t)(rv.head + vi * P + e));
                };
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (z[e] >= best.at && argmax_key(z[e], (uint32_t)(rv.head + vi * P + e)) >= best.floor) mask |= 1u << e;
                best.append_some<P>(q < listed && vi < rv.nvec ? mask : 0, key);
                const bool first = q < listed && u == 0;
                if (rv.head) {
                    const bool h = first && seg == 0 && l < rv.head;
                    best.append(argmax_key(h ? E::get(rv.row, l) : 0.f, (uint32_t)l), h);
                }
                if (rv.body_end < a.V) {
                    const bool t = first && seg == a.segs - 1 && rv.body_end + l < a.V;
                    best.append(argmax_key(t ? E::get(rv.row, rv.body_end + l) : 0.f, (uint32_t)(rv.body_end + l)), t);
                }
            }
            }
            listed = 0;
            best.compress();
            asm volatile("" ::: "memory");
        };
        // All of the row's groups from the floor on at once, where they are few.
        bool done = true;
        for (int v0 = 0; v0 < vecs && done; v0 += kChunk * kWave) {
            if (vecs > kChunk * kWave) load(v0);   // (else they are still there)
            uint64_t mask = 0;
#pragma unroll
            for (int q = 0; q < kChunk; ++q) {
                float y[P];
                E::unpack(mv[q], y);
#pragma unroll
                for (int e = 0; e < P; ++e)
                    mask |= (uint64_t)(v0 + q * kWave + lane < vecs && y[e] >= best.at) << (q * P + e);
            }
            int more, to = listed + wave_excl_scan(__popcll(mask), more);
            done = listed + more <= kGroups;
            listed = done ? listed + more : 0;
            if (done)
                for (; mask; mask &= mask - 1) {
                    const int bit = __ffsll((unsigned long long)mask) - 1;
                    groups[to++] = (v0 + bit / P * kWave + lane) * P + bit % P;
                }
        }
        // Else in order of the vectors, that is of the segments: once there are `top` keys, an
        // equal value of a later segment loses to them, and only larger ones are of interest.
        // (64 vectors are whole segments.)
        float gate = best.at;
        for (int v0 = 0; v0 < vecs && !done; v0 += kWave) {
            const int v = v0 + lane;
            float y[P];
            E::unpack(maxima[min(v, vecs - 1)], y);
            for (int e = 0; e < P; ++e) {
                const uint64_t hits = __ballot(v < vecs && y[0] >= gate);
                if (hits) {
                    if ((hits >> lane) & 1) groups[listed + __popcll(hits & lanemask_lt())] = v * P + e;
                    listed += __popcll(hits);
                }
                // all that is listed, where no more has room or where these segments end
                if (listed > kGroups - kWave || (e == P - 1 && listed >= kWave / L)) look();
#pragma unroll
                for (int f = 0; f + 1 < P; ++f) y[f] = y[f + 1];
            }
            if (best.full && listed == 0) gate = next_up(best.at);
        }
        if (listed) look();
    }

    w.join_lanes();
    // A reference past kMostReference: a small temperature, a row of -inf only, or of logits so
    // low (a mask of the type's lowest value) that times k they overflow.  Then relative to the
    // largest logit m, by this wave alone.
    bool none = false;
    float m = 0.f;
    if (!(fabsf(w.c) <= kMostReference)) {
        auto each = [&](auto f) {
#pragma unroll 4
            for (int v = lane; v < rv.nvec; v += kWave) {
                float z[P];
                E::unpack(rv.vec[v], z);
#pragma unroll
                for (int e = 0; e < P; ++e) f(z[e]);
            }
            if (lane < rv.head) f(E::get(rv.row, lane));
            if (rv.body_end + lane < a.V) f(E::get(rv.row, rv.body_end + lane));
        };
        m = -INFINITY;
        each([&](float z) { m = fmaxf(m, z); });
        m = wave_max_f32(m);
        none = !(m > -INFINITY);
        w = Mass{0.f, 0.f, 0.f};
        if (!none) each([&](float z) { w.add(z - m, a.k); });
        w.s = wave_sum_f32(w.s);
        w.t = wave_sum_f32(w.t);
    }
    const float log2_s = __builtin_amdgcn_logf(w.s);
    // (-inf times a k that is 0 in fp32, of a temperature past 2^149, would be NaN)
    auto logprob = [&](float x) { return none || x == -INFINITY ? -INFINITY : (fmaf(x - m, a.k, -w.c) - log2_s) * 0.6931471805599453f; };
    if (lane == 0) {
        a.logprob[row] = tok >= 0 && tok < a.V ? logprob(z_tok) : __uint_as_float(0x7fc00000u);
        if (a.entropy) a.entropy[row] = none ? 0.f : fmaxf((log2_s - w.t / w.s) * 0.6931471805599453f, 0.f);
    }
    if (kTop && lane < a.top) {
        const bool have = lane < best.cnt;
        const uint64_t key = have ? best.buf[lane] : 0;
        a.top_ids[row * a.top + lane] = have ? (int)argmax_key_index(key) : -1;
        a.top_lp[row * a.top + lane] = have ? logprob(unord_f32((uint32_t)(key >> 32))) : -INFINITY;
    }
}

static int log_segs(int V) { return (int)((V + (int64_t)kLogElems * kWave - 1) / (kLogElems * kWave)); }
static int log_blocks(int B, int n, int segs) {
    const int64_t waves = (int64_t)B * n * segs, blocks = (waves + kLogWaves - 1) / kLogWaves;
    return (int)(blocks < kLogBlocks ? blocks : kLogBlocks);
}
static size_t log_masses_bytes(int B, int n, int segs) {
    return (size_t)log_blocks(B, n, segs) * kLogWaves * 2 * sizeof(float4);
}
static size_t log_whole_bytes(int B, int n) { return (size_t)B * n * sizeof(float4); }
static size_t log_parts_bytes(int B, int n) { return align_up((size_t)B * n * sizeof(int2), 256); }

}  // namespace pld

using namespace pld;

extern "C" size_t pld_token_logprobs_workspace_bytes(int B, int n, int V, int dtype, int top) {
    if (B < 1 || B > 65535 || n < 1 || n > 65535 || V < 1 || (dtype != PLD_F32 && dtype != PLD_BF16) ||
        top < 0 || top > PLD_MAX_TOP)
        return 0;
    const int segs = log_segs(V);
    const size_t maxima = top ? (size_t)B * n * segs * kWave * (dtype == PLD_F32 ? 4 : 2) : 0;
    return log_masses_bytes(B, n, segs) + log_whole_bytes(B, n) + log_parts_bytes(B, n) + maxima;
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
    char *ws = static_cast<char *>(workspace);
    a.masses = reinterpret_cast<float4 *>(ws);
    ws += log_masses_bytes(B, n, a.segs);
    a.whole = reinterpret_cast<float4 *>(ws);
    ws += log_whole_bytes(B, n);
    a.parts = reinterpret_cast<int2 *>(ws);
    a.maxima = ws + log_parts_bytes(B, n);
    const dim3 block(kLogWaves * 64), grid((unsigned)log_blocks(B, n, a.segs));
    const dim3 finish((unsigned)((n + kLogWaves - 1) / kLogWaves), (unsigned)B);
    const hipStream_t st = (hipStream_t)stream;
    auto both = [&](auto bf16) {
        constexpr int kBf16 = decltype(bf16)::value;
        if (top > 0) {
            hipLaunchKernelGGL((token_logprobs_kernel<kBf16, true>), grid, block, 0, st, a);
            hipLaunchKernelGGL((token_logprobs_finish_kernel<kBf16, true>), finish, block, 0, st, a);
        } else {
            hipLaunchKernelGGL((token_logprobs_kernel<kBf16, false>), grid, block, 0, st, a);
            hipLaunchKernelGGL((token_logprobs_finish_kernel<kBf16, false>), finish, block, 0, st, a);
        }
    };
    if (dtype == PLD_F32)
        both(std::integral_constant<int, 0>{});
    else
        both(std::integral_constant<int, 1>{});
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
