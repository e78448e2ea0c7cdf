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
    float k, inv_tau;   // log2(e) / tau, 1 / tau
    float *logprob, *entropy;
    int top;
    int32_t *top_ids;
    float *top_lp;
};

// One block per row: the maximum, then the sums relative to it, then one search
// per alternative.
template <int kBf16>
__global__ __launch_bounds__(256) void token_logprobs_kernel(LogprobArgs a) {
    using E = Elem<kBf16>;
    using T = typename E::T;
    const int i = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int cnt = a.count ? a.count[b] : a.n;
    if (cnt > a.n || i >= cnt) return;
    const T *z = reinterpret_cast<const T *>(a.logits) + (int64_t)b * a.ls + (int64_t)i * a.lr;
    __shared__ float fs[2][4];
    __shared__ uint64_t us[4];
    float m = -INFINITY;
    for (int v = tid; v < a.V; v += 256) m = fmaxf(m, E::get(z, v));
    m = wave_max_f32(m);
    if (lane_id() == 0) fs[0][tid / 64] = m;
    __syncthreads();
    m = fmaxf(fmaxf(fs[0][0], fs[0][1]), fmaxf(fs[0][2], fs[0][3]));
    __syncthreads();
    const bool none = !(m > -INFINITY);
    float s = 0.f, t = 0.f;
    for (int v = tid; v < a.V && !none; v += 256) {
        const float x = fmaxf((E::get(z, v) - m) * a.k, -1e4f), e = __builtin_amdgcn_exp2f(x);
        s += e;
        t = fmaf(e, x, t);
    }
    s = wave_sum_f32(s);
    t = wave_sum_f32(t);
    if (lane_id() == 0) fs[0][tid / 64] = s, fs[1][tid / 64] = t;
    __syncthreads();
    s = (fs[0][0] + fs[0][1]) + (fs[0][2] + fs[0][3]);
    t = (fs[1][0] + fs[1][1]) + (fs[1][2] + fs[1][3]);
    const float log_s = logf(s);
    const int64_t at = (int64_t)b * a.n + i;
    auto logprob = [&](float x) { return none ? -INFINITY : (x - m) * a.inv_tau - log_s; };
    if (tid == 0) {
        const int tok = a.tokens[at];
        a.logprob[at] = tok >= 0 && tok < a.V ? logprob(E::get(z, tok)) : __uint_as_float(0x7fc00000u);
        if (a.entropy) a.entropy[at] = none ? 0.f : fmaxf(log_s - t * 0.6931471805599453f / s, 0.f);
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        uint64_t best = 0;
        for (int v = tid; v < a.V; v += 256) {
            const uint64_t key = argmax_key(E::get(z, v), (uint32_t)v);
            if (key < last && key > best) best = key;
        }
        best = wave_max_u64(best);
        if (lane_id() == 0) us[tid / 64] = best;
        __syncthreads();
        best = max(max(us[0], us[1]), max(us[2], us[3]));
        __syncthreads();
        last = best;
        if (tid == 0) {
            const bool have = k < a.V;
            a.top_ids[at * a.top + k] = have ? (int)argmax_key_index(best) : -1;
            a.top_lp[at * a.top + k] = have ? logprob(unord_f32((uint32_t)(best >> 32))) : -INFINITY;
        }
    }
}

}  // namespace pld

using namespace pld;

extern "C" size_t pld_token_logprobs_workspace_bytes(int B, int n, int V, int dtype, int top) {
    if (B < 1 || B > 65535 || n < 1 || n > 65535 || V < 1 || (dtype != PLD_F32 && dtype != PLD_BF16) ||
        top < 0 || top > PLD_MAX_TOP)
        return 0;
    return 256;
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
    a.k = (float)k, a.inv_tau = (float)(1.0 / temperature);
    a.logprob = logprob, a.entropy = entropy;
    a.top = top, a.top_ids = top_ids, a.top_lp = top_logprobs;
    const dim3 grid((unsigned)n, (unsigned)B);
    if (dtype == PLD_F32)
        hipLaunchKernelGGL(token_logprobs_kernel<0>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(token_logprobs_kernel<1>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}
