// pld_packed.h -- packed rows of several sequences: which sequence a row belongs to.
#pragma once

#include "pld_device.h"
#include "pld_prompt.h"

namespace pld {

struct Packed {
    const int32_t *starts;   // [B + 1]
    int B, N;
};

// The sequence of a row (the same in every lane), by a search of 64 places at a time: up to 63
// sequences take one load.  b < 0: none, for the rows of [begin, end) alike.
struct Span {
    int b, begin, end;
};
__device__ __forceinline__ Span span_of(const Packed &p, int row) {
    const int lane = lane_id();
    int lo = 0, hi = p.B + 1;   // how many starts are <= row: in [lo, hi]
    while (hi - lo > kWave) {
        const int step = (hi - lo + kWave - 1) / kWave, i = lo + (lane + 1) * step - 1;
        const int v = i < hi ? p.starts[i] : INT32_MAX;
        lo += __popcll(__ballot(v <= row)) * step;
        hi = min(hi, lo + step);
        lo = min(lo, hi);
    }
    const int v = lo + lane < hi ? p.starts[lo + lane] : INT32_MAX;
    const int c = __popcll(__ballot(v <= row)), n = lo + c;
    Span s;
    s.b = n >= 1 && n <= p.B ? n - 1 : -1;
    // the neighbours of the place that was found, of the same load as a rule
    s.begin = n == 0 ? INT32_MIN : c > 0 ? __builtin_amdgcn_readlane(v, c - 1) : p.starts[n - 1];
    s.end = n > p.B ? INT32_MAX : lo + c < hi ? __builtin_amdgcn_readlane(v, c & (kWave - 1)) : p.starts[n];
    return s;
}
// The same for each lane's own row: a search for each sequence that the wave's rows belong to.
__device__ __forceinline__ Span spans_of(const Packed &p, int row) {
    Span mine{-1, 0, 0};
    uint64_t open = __ballot(1);
    while (open) {
        const int r = __builtin_amdgcn_readlane(row, __builtin_ctzll(open));
        const Span s = span_of(p, r);
        const bool in = row == r || (row >= s.begin && row < s.end);
        if (in && (open >> lane_id() & 1)) mine = s;
        open &= ~__ballot(in);
    }
    return mine;
}

// A bf16 operand [N][heads][head_dim] with a stride of rows.
inline int check_packed(const void *p, int64_t row, int N, int64_t width, int64_t most) {
    if (!p || (N > 1 && (row < width || row > most))) return PLD_ERR_INVALID;
    if ((uintptr_t)p % 16 || (N > 1 && row % 8)) return PLD_ERR_ALIGN;
    return PLD_OK;
}

// Blocks in two dimensions: a dimension's threads are counted in 32 bits.
inline dim3 wide_grid(int64_t blocks) {
    const int64_t x = blocks < 65536 ? blocks : 65536;
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t wide_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace pld
