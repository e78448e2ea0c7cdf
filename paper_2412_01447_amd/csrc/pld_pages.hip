// pld_pages.hip -- the pages of a pool of caches: taking, freeing, forking,
// compacting and copying them.
//
// Integers first, in the order that the results ask for: lacking pages are counted a wave a sequence, a sum over
// the sequences says which of the free pages, ranked by a sum over the references, each gets.  One block does
// that (6 us, of loads that wait for each other); the copies of pages' contents follow in a
// launch over the whole card, which memory bounds (8.5 GB in 1670 us, 5.1 TB/s, a large copy's rate), with
// the integers that they do not wait for.
#include "pld_cache.h"
#include "pld_prompt.h"

namespace pld {

struct Pool {
    int32_t *table;
    int64_t stride;
    int32_t *refs;
    int seqs, max_pages, num_pages, shift;   // page_size = 1 << shift
};

// The integers' block: 1024 threads, kRun pages of the references each.
constexpr int kPoolThreads = 1024, kPoolWaves = kPoolThreads / kWave;
constexpr int kRun = 16, kSpan = kPoolThreads * kRun;   // pages of one step: 16384
// One block goes through a call's sequences, a wave each, and gives out the pages in the same launch, up to as
// many as it has waves: a take of one and of 16 sequences 3.6 us, 8.4 with launches of their own, of 16 with 16384
// entries each 10.4 and 12.6.  A fork changes every entry, and so up to this many of all sequences: one of 4096 11.8 and
// 12.4 us, 16 of 64 12.8 and 12.9, but 16 of 1024 15.6 and 13.2, of 4096 31 and 17.
constexpr int64_t kOneBlock = 1 << 12;

struct PoolWork {                // the workspace, in this order
    int32_t *head;               // [16]: pages in use, moves
    int32_t *lacks, *from, *slots;   // [count]: pages wanted (-1: refused); of the tail; to copy
    int32_t *offs;               // [count]: place of the first page in `list`, -1: none
    int32_t *spans;              // [spans]: pages in use of each
    int32_t *list;               // [num_pages]: free pages in order; compact: a code for each page
    int32_t *hole, *high;        // [num_pages / 2 + 1]
};
inline size_t pool_work(const pld_pool &p, int count, char *base, PoolWork &w) {
    size_t at = 0;
    auto take = [&](int32_t *&ptr, size_t n) {
        ptr = reinterpret_cast<int32_t *>(base + at);
        at = align_up(at + n * 4, 64);
    };
    take(w.head, 16);
    take(w.lacks, count), take(w.from, count), take(w.slots, count), take(w.offs, count);
    take(w.spans, (p.num_pages + kSpan - 1) / kSpan);
    take(w.list, p.num_pages);
    take(w.hole, p.num_pages / 2 + 1), take(w.high, p.num_pages / 2 + 1);
    return at;
}

struct EditArgs {
    Pool p;
    PoolWork w;
    const int32_t *seq, *src;    // seq: of a fork, the new sequences
    const int32_t *lens;         // need or lens
    int count;
    int32_t *status;
};

__device__ __forceinline__ bool is_page(const Pool &p, int x) { return (uint32_t)x < (uint32_t)p.num_pages; }
__device__ __forceinline__ int32_t *entries_of(const Pool &p, int seq) { return p.table + (int64_t)seq * p.stride; }

// What other waves of the block wrote to global memory before (atomics included) is read after.
__device__ __forceinline__ void block_sync() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}

// Table entries that a wave takes at a time, eight a lane: their loads are under way together.  A fork of one sequence
// of 16384 entries, with a page taken, 83 us with one a lane by one wave, 22 with eight a lane by 32 waves.
constexpr int kRow = 8, kEntries = kWave * kRow;
// Those of a sequence from p0 on, below end; behind it: page 0.
__device__ __forceinline__ void load_entries(const int32_t *e, int p0, int end, int (&v)[kRow]) {
#pragma unroll
    for (int k = 0; k < kRow; ++k) {
        const int p = p0 + k * kWave + lane_id();
        v[k] = p < end ? e[p] : 0;
    }
}

// Whether `seq` is named by any entry of `by` but the i-th (a wave).
__device__ __forceinline__ bool named_by(const int32_t *by, int count, int seq, int i) {
    bool hit = false;
    for (int j = lane_id(); j < count; j += kWave) hit |= by[j] == seq && j != i;
    return __any(hit);
}

// take, entry i (a wave): how many pages the sequence lacks.
__device__ __forceinline__ void count_lacking(const EditArgs &a, int i) {
    const int s = a.seq[i], need = max(a.lens[i], 0);
    const int64_t pages = ((int64_t)need + (1 << a.p.shift) - 1) >> a.p.shift;
    int n = -1;
    if ((uint32_t)s < (uint32_t)a.p.seqs && pages <= a.p.max_pages && !named_by(a.seq, a.count, s, i)) {
        const int32_t *e = entries_of(a.p, s);
        n = 0;
        for (int p0 = 0; p0 < (int)pages; p0 += kEntries) {
            int v[kRow];
            load_entries(e, p0, (int)pages, v);
#pragma unroll
            for (int k = 0; k < kRow; ++k) n += !is_page(a.p, v[k]);
        }
        n = wave_sum_i32(n);
    }
    if (lane_id() == 0) a.w.lacks[i] = n;
}

// fork, entry i (a wave, one of `parts`): what the sequence had is given back, whole pages are shared.
__device__ __forceinline__ void share(const EditArgs &a, int i, int part, int parts) {
    const int s = a.src[i], d = a.seq[i], T = a.lens[i], last = T > 0 ? (T - 1) >> a.p.shift : -1;
    const bool ok = (uint32_t)s < (uint32_t)a.p.seqs && (uint32_t)d < (uint32_t)a.p.seqs && T >= 0 &&
                    last < a.p.max_pages && !named_by(a.seq, a.count, d, i) &&
                    !named_by(a.src, a.count, d, -1);
    const int tail = ok && T > 0 ? entries_of(a.p, s)[last] : -1;
    if (!ok || (T > 0 && !is_page(a.p, tail))) {
        if (part == 0 && lane_id() == 0) a.w.lacks[i] = -1;
        return;
    }
    const int32_t *from = entries_of(a.p, s);
    int32_t *e = entries_of(a.p, d);
    for (int p0 = part * kEntries; p0 < a.p.max_pages; p0 += parts * kEntries) {
        int old[kRow], x[kRow];
        load_entries(e, p0, a.p.max_pages, old);
        load_entries(from, p0, max(last, 0), x);
#pragma unroll
        for (int k = 0; k < kRow; ++k) {
            const int p = p0 + k * kWave + lane_id();
            if (p >= a.p.max_pages) break;
            if (p >= last || !is_page(a.p, x[k])) x[k] = -1;
            if (is_page(a.p, old[k])) atomicSub(a.p.refs + old[k], 1);
            if (x[k] >= 0) atomicAdd(a.p.refs + x[k], 1);
            if (x[k] != old[k]) e[p] = x[k];
        }
    }
    if (part == 0 && lane_id() == 0) {
        a.w.lacks[i] = T > 0;
        a.w.from[i] = tail;
        a.w.slots[i] = T > 0 ? ((T - 1) & ((1 << a.p.shift) - 1)) + 1 : 0;
    }
}

// Exclusive sum over the block's threads; every thread gets the total.
template <class T>
__device__ __forceinline__ T block_excl_scan(T v, T &total, T *s_w) {
    const int wave = (int)threadIdx.x / kWave;
    T before;
    if constexpr (sizeof(T) == 8) {
        const T upto = wave_incl_scan(v);
        if (lane_id() == kWave - 1) s_w[wave] = upto;
        before = upto - v;
    } else {
        T of_wave;
        before = wave_excl_scan(v, of_wave);
        if (lane_id() == 0) s_w[wave] = of_wave;
    }
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < kPoolWaves; ++w) {
        before += w < wave ? s_w[w] : 0;
        total += s_w[w];
    }
    __syncthreads();
    return before;
}

// Which of a thread's run of pages are in use: a bit each (none past the end).
__device__ __forceinline__ uint32_t used_bits(const Pool &p, int x0) {
    uint32_t bits = 0;
    if (x0 + kRun <= p.num_pages) {
        int4 v[kRun / 4];
#pragma unroll
        for (int k = 0; k < kRun / 4; ++k) v[k] = reinterpret_cast<const int4 *>(p.refs + x0)[k];
#pragma unroll
        for (int k = 0; k < kRun / 4; ++k)
            bits |= (uint32_t)((v[k].x > 0) | (v[k].y > 0) << 1 | (v[k].z > 0) << 2 | (v[k].w > 0) << 3) << (4 * k);
    } else {
#pragma unroll
        for (int k = 0; k < kRun; ++k)
            if (x0 + k < p.num_pages) bits |= (uint32_t)(p.refs[x0 + k] > 0) << k;
    }
    return bits;
}

// The pages that entries lack, lowest first, into `list`; each entry's place in it, and status
// (a block).
template <bool kFork>
__device__ __forceinline__ void give_out(const EditArgs &a) {
    __shared__ int s_w[kPoolWaves], s_served;
    __shared__ int64_t s_wide[kPoolWaves];
    const int per = (a.count + kPoolThreads - 1) / kPoolThreads;
    const int i0 = min((int)threadIdx.x * per, a.count), i1 = min(i0 + per, a.count);
    int64_t mine = 0, wanted;   // (a sequence may lack 2^26 pages)
    for (int i = i0; i < i1; ++i) mine += max(a.w.lacks[i], 0);
    int64_t at = block_excl_scan(mine, wanted, s_wide);
    const int total = (int)min(wanted, (int64_t)a.p.num_pages);
    int found = 0;
    if (threadIdx.x == 0) s_served = 0;
    for (int x = 0; x < a.p.num_pages && found < total; x += kSpan) {
        const int x0 = x + (int)threadIdx.x * kRun;
        uint32_t bits = x0 < a.p.num_pages ? used_bits(a.p, x0) : 0;
        const int n = min(kRun, a.p.num_pages - x0);
        bits = n > 0 ? ~bits & ((1u << n) - 1) : 0;
        int here, k = found + block_excl_scan((int)__popc(bits), here, s_w);
        for (; bits && k < total; bits &= bits - 1, ++k) a.w.list[k] = x0 + __builtin_ctz(bits);
        found += here;
    }
    found = min(found, total);
    int served = 0;
    for (int i = i0; i < i1; ++i) {
        const int n = a.w.lacks[i];
        const bool ok = n <= 0 || at + n <= found;
        a.w.offs[i] = n > 0 && ok ? (int)at : -1;
        a.status[i] = n < 0 ? -1 : ok ? 0 : kFork ? -2 : n;
        if (n > 0) at += n;
        if (n > 0 && ok) served = (int)at;
    }
    if (served) atomicMax(&s_served, served);
    block_sync();   // (the list, too)
    for (int k = threadIdx.x; k < s_served; k += kPoolThreads) a.p.refs[a.w.list[k]] = 1;
}

// take, entry i (a wave): its pages into the table.
__device__ __forceinline__ void fill(const EditArgs &a, int i) {
    int at = a.w.offs[i];
    if (at < 0) return;
    int32_t *e = entries_of(a.p, a.seq[i]);
    const int pages = (int)(((int64_t)a.lens[i] + (1 << a.p.shift) - 1) >> a.p.shift);
    for (int p0 = 0; p0 < pages; p0 += kEntries) {
        int v[kRow];
        load_entries(e, p0, pages, v);
#pragma unroll
        for (int k = 0; k < kRow; ++k) {
            const bool lacks = !is_page(a.p, v[k]);
            const uint64_t all = __ballot(lacks);
            if (lacks) e[p0 + k * kWave + lane_id()] = a.w.list[at + __popcll(all & lanemask_lt())];
            at += __popcll(all);
        }
    }
}

// fork, entry i (a wave): the page of the last token; where none was left, the shared ones go back.
__device__ __forceinline__ void finish_fork(const EditArgs &a, int i) {
    if (a.w.lacks[i] <= 0) return;
    const int last = (a.lens[i] - 1) >> a.p.shift, at = a.w.offs[i];
    int32_t *e = entries_of(a.p, a.seq[i]);
    if (at >= 0) {
        if (lane_id() == 0) e[last] = a.w.list[at];
        return;
    }
    for (int p = lane_id(); p < last; p += kWave) {
        const int x = e[p];
        if (is_page(a.p, x)) atomicSub(a.p.refs + x, 1);
        e[p] = -1;
    }
}

// A wave a sequence; of a fork, gridDim.y of them.
template <bool kFork>
__global__ __launch_bounds__(256) void pages_edit_kernel(EditArgs a) {
    const int i = (int)(blockIdx.x * 4 + threadIdx.x / kWave);
    if (i >= a.count) return;
    kFork ? share(a, i, blockIdx.y, gridDim.y) : count_lacking(a, i);
}
// One block: with kEdit the sequences' part too, a wave each, or of forks as many as there are.
template <bool kFork, bool kEdit>
__global__ __launch_bounds__(kPoolThreads) void pages_give_kernel(EditArgs a) {
    const int wave = (int)threadIdx.x / kWave;
    if constexpr (kEdit) {
        const int parts = kFork ? min(kPoolWaves / a.count, (a.p.max_pages + kEntries - 1) / kEntries) : 1;
        const int part = wave / a.count;
        if (part < parts) kFork ? share(a, wave - part * a.count, part, parts) : count_lacking(a, wave);
        block_sync();
        // references change by atomics, at the L2: what this CU's own cache holds of them is old
        if constexpr (kFork) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    }
    give_out<kFork>(a);
    if constexpr (!kFork && kEdit) {
        block_sync();
        if (wave < a.count) fill(a, wave);
    }
}
__global__ __launch_bounds__(256) void pages_fill_kernel(EditArgs a) {
    const int i = (int)(blockIdx.x * 4 + threadIdx.x / kWave);
    if (i < a.count) fill(a, i);
}

// Entries are exchanged, so that one that two name is given back once.  A thread an entry, for up to 16384 of a sequence:
// four took 2 to 3 us more (1024 entries taken and given back, 11.3 us).
__global__ __launch_bounds__(256) void pages_free_kernel(Pool p, const int32_t *seq, const int32_t *keep) {
    const int s = seq[blockIdx.x];
    if ((uint32_t)s >= (uint32_t)p.seqs) return;
    const int64_t kept = keep ? max(keep[blockIdx.x], 0) : 0;
    const int first = (int)min((kept + (1 << p.shift) - 1) >> p.shift, (int64_t)p.max_pages);
    int32_t *e = entries_of(p, s);
    const int step = (int)(gridDim.y * blockDim.x);
    for (int x = first + (int)(blockIdx.y * blockDim.x + threadIdx.x); x < p.max_pages; x += step) {
        if (e[x] == -1) continue;
        const int old = atomicExch(e + x, -1);
        if (is_page(p, old)) atomicSub(p.refs + old, 1);
    }
}

// ---------------------------------------------------------------- compacting
// With n pages in use and r(x) of them below x, the free pages below n are holes x - r(x),
// in order, and the used ones from n on are numbered from the end, n - 1 - r(x): no block has
// to know how many there are.  codes: a used page below n itself, -1 a free one, and
// num_pages + its number one that moves.
__global__ __launch_bounds__(kPoolThreads) void pages_span_kernel(Pool p, PoolWork w) {
    __shared__ int s_w[kPoolWaves];
    const int x0 = (int)(blockIdx.x * kPoolThreads + threadIdx.x) * kRun;
    int total;
    block_excl_scan(x0 < p.num_pages ? (int)__popc(used_bits(p, x0)) : 0, total, s_w);
    if (threadIdx.x == 0) w.spans[blockIdx.x] = total;
}
__global__ __launch_bounds__(kPoolThreads) void pages_rank_kernel(Pool p, PoolWork w) {
    __shared__ int s_w[kPoolWaves];
    int n = 0, before = 0;
    if (gridDim.x > 1) {   // (at most 1024 spans)
        const int mine = threadIdx.x < gridDim.x ? w.spans[threadIdx.x] : 0;
        block_excl_scan(mine, n, s_w);
        block_excl_scan(threadIdx.x < blockIdx.x ? mine : 0, before, s_w);
    }
    const int x0 = (int)(blockIdx.x * kPoolThreads + threadIdx.x) * kRun;
    const uint32_t bits = x0 < p.num_pages ? used_bits(p, x0) : 0;
    int here;
    int r = before + block_excl_scan((int)__popc(bits), here, s_w);
    if (gridDim.x == 1) n = here;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        w.head[0] = n;
        if (n == p.num_pages) w.head[1] = 0;
    }
#pragma unroll 1
    for (int k = 0; k < kRun && x0 + k < p.num_pages; ++k) {
        const int x = x0 + k;
        const bool used = (bits >> k) & 1;
        if (x == n) w.head[1] = n - r;   // moves
        w.list[x] = !used ? -1 : x < n ? x : p.num_pages + (n - 1 - r);
        if (!used && x < n) w.hole[x - r] = x;
        if (used && x >= n) w.high[n - 1 - r] = x;
        r += used;
    }
}

struct CompactArgs {
    Pool p;
    PoolWork w;
    int32_t *map, *used, *table_out, *refs_out;
    int64_t out_stride;
};
__device__ __forceinline__ void finish_compact(const CompactArgs &a, int64_t thread, int64_t threads) {
    const int n = a.w.head[0], moves = a.w.head[1], P = a.p.num_pages;
    auto moved = [&](int code) { return code < P ? code : a.w.hole[moves - 1 - (code - P)]; };
    if (thread == 0) a.used[0] = n;
    for (int64_t x = thread; x < P; x += threads) {
        const int code = a.w.list[x];
        a.map[x] = moved(code);
        // holes and what moves into them are written in pairs below
        if (code >= 0 ? code < P : x >= n) a.refs_out[x] = code >= 0 ? a.p.refs[x] : 0;
    }
    for (int64_t h = thread; h < moves; h += threads) {
        const int x = a.w.high[moves - 1 - h], refs = a.p.refs[x];
        a.refs_out[a.w.hole[h]] = refs;
        a.refs_out[x] = 0;
    }
    const int64_t entries = (int64_t)a.p.seqs * a.p.max_pages;
    for (int64_t i = thread; i < entries; i += threads) {
        const int64_t s = quotient(i, a.p.max_pages), e = i - s * a.p.max_pages;
        const int x = a.p.table[s * a.p.stride + e];
        a.table_out[s * a.out_stride + e] = is_page(a.p, x) ? moved(a.w.list[x]) : x;
    }
}

// ------------------------------------------------------------------- copying
constexpr int kCopyLayers = 32;   // of a launch: the pointers are kernel arguments
struct CopyLayer {
    const char *k, *v;
    const float *ks, *vs;
    char *to_k, *to_v;
    float *to_ks, *to_vs;
};
struct Strides {
    int64_t page, slot, head, spage;   // bytes; floats
};
struct CopyArgs {
    CopyLayer layer[kCopyLayers];
    Strides from, to;
    int layers, num_from, num_to;
    int shift, heads;        // page_size = 1 << shift
    int row;                 // log2 of a head's row in 16 bytes
    int chunks;              // of a page's keys or values
    bool by_head;            // rows in order of head, else of slot
    bool linear;             // a page is one run of bytes in that order, on both sides
    bool q8;
    // the pages: of a copy
    const int32_t *src, *dst, *slots;
    int count;
};
enum { kPairs, kForks, kMoves };

// A block's part of a copy: 32 KB of a page's keys or values, or its scales.  Bound by memory; read and
// written past the caches where each page is read once (kOnce): what a compaction moves (32 sequences, 8
// layers in e4m3, 2.7 GB) 550 us without and 504 with it; forks read a prompt's page several times, 64 us
// without and 80 with it (56 of 8 prompts, 16 layers).  With 16 KB a part 595 us, with 64 KB 555.
constexpr int kCopyThreads = 256, kCopyEach = 8, kCopyPieces = kCopyThreads * kCopyEach;
template <bool kOnce>
__device__ __forceinline__ u32x4_t load16(const void *p) {
    const u32x4_t *q = reinterpret_cast<const u32x4_t *>(p);
    return kOnce ? __builtin_nontemporal_load(q) : *q;
}
template <bool kOnce>
__device__ __forceinline__ void store16(void *p, u32x4_t v) {
    u32x4_t *q = reinterpret_cast<u32x4_t *>(p);
    if (kOnce) __builtin_nontemporal_store(v, q);
    else *q = v;
}
template <bool kOnce>
__device__ __forceinline__ void copy_part(const CopyArgs &a, int layer, bool value, int chunk, int src, int dst, int slots) {
    const CopyLayer &l = a.layer[layer];
    if (chunk == a.chunks) {
        const float *f = (value ? l.vs : l.ks) + (int64_t)src * a.from.spage;
        float *t = (value ? l.to_vs : l.to_ks) + (int64_t)dst * a.to.spage;
        const int all = a.heads << a.shift, mask = (1 << a.shift) - 1;
        for (int i = threadIdx.x; i < all; i += kCopyThreads)
            if ((i & mask) < slots) t[i] = f[i];
        return;
    }
    const char *f = (value ? l.v : l.k) + (int64_t)src * a.from.page;
    char *t = (value ? l.to_v : l.to_k) + (int64_t)dst * a.to.page;
    const int pieces = slots * a.heads << a.row, first = chunk * kCopyPieces + (int)threadIdx.x;
    if (chunk * kCopyPieces >= pieces) return;
    u32x4_t v[kCopyEach];
    // (past the end: the last piece again, which is not stored)
    if (a.linear && (!a.by_head || slots == 1 << a.shift)) {
#pragma unroll
        for (int k = 0; k < kCopyEach; ++k) v[k] = load16<kOnce>(f + (int64_t)min(first + k * kCopyThreads, pieces - 1) * 16);
#pragma unroll
        for (int k = 0; k < kCopyEach; ++k)
            if (first + k * kCopyThreads < pieces) store16<kOnce>(t + (int64_t)(first + k * kCopyThreads) * 16, v[k]);
        return;
    }
    int64_t to[kCopyEach];
#pragma unroll
    for (int k = 0; k < kCopyEach; ++k) {
        const int i = min(first + k * kCopyThreads, pieces - 1);
        const int r = i >> a.row, inner = a.by_head ? slots : a.heads, q = r / inner, m = r - q * inner;
        const int64_t slot = a.by_head ? m : q, head = a.by_head ? q : m, piece = (i - (r << a.row)) * 16;
        v[k] = load16<kOnce>(f + slot * a.from.slot + head * a.from.head + piece);
        to[k] = slot * a.to.slot + head * a.to.head + piece;
    }
#pragma unroll
    for (int k = 0; k < kCopyEach; ++k)
        if (first + k * kCopyThreads < pieces) store16<kOnce>(t + to[k], v[k]);
}

// Parts are dealt to the grid's blocks in turn, in order of (page, layer, keys or values, chunk).
// A call's integers that the copy does not wait for are done by its last blocks (`ints` of them).
template <int kMode>
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(CopyArgs a, EditArgs e, CompactArgs c, int ints) {
    const int copiers = (int)gridDim.x - ints, block = (int)blockIdx.x;
    if (block >= copiers) {
        const int at = block - copiers;
        if constexpr (kMode == kForks) {
            for (int i = at * 4 + (int)threadIdx.x / kWave; i < e.count; i += ints * 4) finish_fork(e, i);
        } else if constexpr (kMode == kMoves) {
            finish_compact(c, (int64_t)at * kCopyThreads + threadIdx.x, (int64_t)ints * kCopyThreads);
        }
        return;
    }
    const int per = (a.chunks + a.q8) * 2, of_page = per * a.layers;
    const int count = kMode == kMoves ? c.w.head[1] : a.count;
    const int64_t parts = (int64_t)count * of_page;
    for (int64_t i = block; i < parts; i += copiers) {
        const int m = (int)quotient(i, of_page);
        const int rest = (int)(i - (int64_t)m * of_page), layer = rest / per, part = rest - layer * per;
        const bool value = part >= a.chunks + a.q8;
        const int chunk = value ? part - a.chunks - a.q8 : part;
        int src, dst, slots = 1 << a.shift;
        if constexpr (kMode == kForks) {
            const int at = e.w.offs[m];
            if (at < 0) continue;
            src = e.w.from[m], dst = e.w.list[at], slots = e.w.slots[m];
        } else if constexpr (kMode == kMoves) {
            src = c.w.high[count - 1 - m], dst = c.w.hole[m];
        } else {
            src = a.src[m], dst = a.dst[m];
            if ((uint32_t)src >= (uint32_t)a.num_from || (uint32_t)dst >= (uint32_t)a.num_to) continue;
            if (a.slots && (uint32_t)a.slots[m] < (uint32_t)slots) slots = a.slots[m];
        }
        copy_part<kMode != kForks>(a, layer, value, chunk, src, dst, slots);
    }
}

// ---------------------------------------------------------------- host checks
static int check_pool(const pld_pool *p, Pool &o) {
    if (!p || !p->table || !p->refs) return PLD_ERR_INVALID;
    const int ps = p->page_size;
    if (ps < 16 || ps > 4096 || (ps & (ps - 1))) return PLD_ERR_INVALID;
    if (p->seqs < 1 || p->seqs > 1 << 20 || p->num_pages < 1 || p->num_pages > PLD_MAX_PAGES || p->max_pages < 1 ||
        (int64_t)p->max_pages * ps > kMaxTokStride || p->table_stride < p->max_pages || p->table_stride > kMaxTokStride)
        return PLD_ERR_INVALID;
    if ((uintptr_t)p->table % 4 || (uintptr_t)p->refs % 16) return PLD_ERR_ALIGN;
    o = Pool{p->table, p->table_stride, p->refs, p->seqs, p->max_pages, p->num_pages, __builtin_ctz((unsigned)ps)};
    return PLD_OK;
}

// The caches of one side: each right by itself and alike in all but its pointers.
static int check_layers(const pld_cache *c, int n, Strides &s) {
    for (int i = 0; i < n; ++i) {
        pld_cache one = c[i];
        const pld_cache &first = c[0];
        if (one.dtype != first.dtype || one.scale_page_stride != first.scale_page_stride || one.page_stride != first.page_stride ||
            one.slot_stride != first.slot_stride || one.head_stride != first.head_stride || one.num_pages != first.num_pages ||
            one.page_size != first.page_size || one.heads != first.heads || one.head_dim != first.head_dim)
            return PLD_ERR_INVALID;
        const int32_t none = 0;   // the table is not used here
        one.table = &none;
        one.table_stride = one.max_pages = 1;
        CacheView v;
        if (const int rc = prep_cache(&one, true, v); rc != PLD_OK) return rc;
        s = Strides{v.page, v.slot, v.head, v.spage};
    }
    return PLD_OK;
}

static void fill_geometry(CopyArgs &a, const pld_cache &f, const pld_cache &t) {
    const int64_t row = f.head_dim * (f.dtype == PLD_E4M3 ? 1 : 2);   // bytes
    a.num_from = f.num_pages, a.num_to = t.num_pages;
    a.shift = __builtin_ctz((unsigned)f.page_size), a.heads = f.heads;
    a.row = __builtin_ctz((unsigned)(row / 16));
    a.chunks = (int)((((int64_t)f.heads << a.shift << a.row) + kCopyPieces - 1) / kCopyPieces);
    a.q8 = f.dtype == PLD_E4M3;
    a.by_head = f.heads > 1 && a.from.slot < a.from.head;
    auto run = [&](const Strides &s) {
        return a.by_head ? s.slot == row && s.head == row << a.shift : s.slot == row * f.heads && (f.heads == 1 || s.head == row);
    };
    a.linear = run(a.from) && run(a.to);
}
static void fill_layers(CopyArgs &a, const pld_cache *f, const pld_cache *t, int first, int n) {
    a.layers = n;
    for (int i = 0; i < n; ++i) {
        const pld_cache &x = f[first + i], &y = t[first + i];
        a.layer[i] = CopyLayer{(const char *)x.k, (const char *)x.v, x.k_scale, x.v_scale, (char *)y.k, (char *)y.v, y.k_scale, y.v_scale};
    }
}

// Past the caches two blocks a CU, 64 KB of its loads under way, are best (2.7 GB moved in 504 us, 514 with
// four and 522 with eight), through them eight.
template <int kMode>
static int launch_copy(CopyArgs &a, const EditArgs &e, const CompactArgs &c, const pld_cache *f, const pld_cache *t,
                       int n_layers, int64_t most, int ints, hipStream_t s) {
    constexpr int kCopyBlocks = kMode == kForks ? 2048 : 512;
    if (n_layers) fill_geometry(a, f[0], t[0]);
    for (int first = 0; first < n_layers || first == 0; first += kCopyLayers) {
        const int n = n_layers - first < kCopyLayers ? n_layers - first : kCopyLayers;
        if (n > 0) fill_layers(a, f, t, first, n);
        else a.layers = 0;
        const int64_t parts = n > 0 ? most * (a.chunks + a.q8) * 2 * n : 0;
        const int copiers = (int)(parts < kCopyBlocks ? parts : kCopyBlocks);
        if (copiers + ints == 0) break;
        if (!copiers) a.count = 0;
        hipLaunchKernelGGL(pages_copy_kernel<kMode>, dim3(copiers + ints), dim3(kCopyThreads), 0, s, a, e, c, ints);
        ints = 0;
    }
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}

static int check_work(const pld_pool *p, int count, void *ws, size_t bytes, PoolWork &w) {
    if (!ws || (uintptr_t)ws % 16 || bytes < pool_work(*p, count, (char *)ws, w)) return PLD_ERR_WORKSPACE;
    return PLD_OK;
}

// The launches before a copy or a filling: two, or one (kOneBlock).
template <bool kFork>
static bool launch_edit(const EditArgs &a, hipStream_t s) {
    const bool one = a.count <= kPoolWaves && (!kFork || (int64_t)a.count * a.p.max_pages <= kOneBlock);
    const int parts = kFork ? std::min((a.p.max_pages + kEntries - 1) / kEntries, 64) : 1;
    if (!one)
        hipLaunchKernelGGL(pages_edit_kernel<kFork>, dim3((a.count + 3) / 4, parts), dim3(256), 0, s, a);
    if (one)
        hipLaunchKernelGGL((pages_give_kernel<kFork, true>), dim3(1), dim3(kPoolThreads), 0, s, a);
    else
        hipLaunchKernelGGL((pages_give_kernel<kFork, false>), dim3(1), dim3(kPoolThreads), 0, s, a);
    return one;
}

}  // namespace pld

using namespace pld;

extern "C" size_t pld_pages_workspace_bytes(const pld_pool *pool, int count) {
    Pool p;
    PoolWork w;
    if (check_pool(pool, p) == PLD_ERR_INVALID || count < 1 || count > PLD_MAX_PAGE_ENTRIES) return 0;
    return pool_work(*pool, count, nullptr, w);
}

extern "C" int pld_pages_take(const pld_pool *pool, const int32_t *seq, const int32_t *need, int count,
                              int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    EditArgs a{};
    if (const int rc = check_pool(pool, a.p); rc != PLD_OK) return rc;
    if (!seq || !need || !status || count < 1 || count > PLD_MAX_PAGE_ENTRIES) return PLD_ERR_INVALID;
    if (((uintptr_t)seq | (uintptr_t)need | (uintptr_t)status) % 4) return PLD_ERR_ALIGN;
    if (const int rc = check_work(pool, count, workspace, workspace_bytes, a.w); rc != PLD_OK) return rc;
    a.seq = seq, a.lens = need, a.count = count, a.status = status;
    const hipStream_t s = (hipStream_t)stream;
    if (!launch_edit<false>(a, s))
        hipLaunchKernelGGL(pages_fill_kernel, dim3((count + 3) / 4), dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}

extern "C" int pld_pages_free(const pld_pool *pool, const int32_t *seq, const int32_t *keep, int count, void *stream) {
    Pool p;
    if (const int rc = check_pool(pool, p); rc != PLD_OK) return rc;
    if (!seq || count < 1 || count > PLD_MAX_PAGE_ENTRIES) return PLD_ERR_INVALID;
    if (((uintptr_t)seq | (uintptr_t)keep) % 4) return PLD_ERR_ALIGN;
    const int parts = (p.max_pages + 255) / 256;
    hipLaunchKernelGGL(pages_free_kernel, dim3(count, parts < 64 ? parts : 64), dim3(256), 0, (hipStream_t)stream, p, seq, keep);
    return hipGetLastError() == hipSuccess ? PLD_OK : PLD_ERR_LAUNCH;
}

extern "C" int pld_pages_fork(const pld_pool *pool, const pld_cache *layers, int n_layers, const int32_t *src,
                              const int32_t *dst, const int32_t *lens, int count, int32_t *status,
                              void *workspace, size_t workspace_bytes, void *stream) {
    EditArgs e{};
    CopyArgs a{};
    int rc = check_pool(pool, e.p);
    if (rc != PLD_OK) return rc;
    if (!src || !dst || !lens || !status || count < 1 || count > PLD_MAX_PAGE_ENTRIES || n_layers < 0 ||
        n_layers > PLD_MAX_LAYERS || (n_layers && !layers))
        return PLD_ERR_INVALID;
    if ((rc = check_layers(layers, n_layers, a.from)) != PLD_OK) return rc;
    if (n_layers && (layers[0].num_pages != pool->num_pages || layers[0].page_size != pool->page_size)) return PLD_ERR_INVALID;
    if (((uintptr_t)src | (uintptr_t)dst | (uintptr_t)lens | (uintptr_t)status) % 4) return PLD_ERR_ALIGN;
    if ((rc = check_work(pool, count, workspace, workspace_bytes, e.w)) != PLD_OK) return rc;
    a.to = a.from;
    a.count = count;
    e.src = src, e.seq = dst, e.lens = lens, e.count = count, e.status = status;
    const hipStream_t s = (hipStream_t)stream;
    launch_edit<true>(e, s);
    return launch_copy<kForks>(a, e, CompactArgs{}, layers, layers, n_layers, count, (count + 3) / 4, s);
}

extern "C" int pld_pages_compact(const pld_pool *pool, const pld_cache *layers, int n_layers, int32_t *map,
                                 int32_t *used, int32_t *table_out, int64_t table_out_stride,
                                 int32_t *refs_out, void *workspace, size_t workspace_bytes, void *stream) {
    CompactArgs c{};
    CopyArgs a{};
    int rc = check_pool(pool, c.p);
    if (rc != PLD_OK) return rc;
    if (!map || !used || !table_out || !refs_out || n_layers < 0 || n_layers > PLD_MAX_LAYERS || (n_layers && !layers) ||
        (table_out_stride < pool->max_pages && pool->seqs > 1) || table_out_stride > kMaxTokStride ||
        (table_out == pool->table && pool->seqs > 1 && table_out_stride != pool->table_stride))
        return PLD_ERR_INVALID;
    if ((rc = check_layers(layers, n_layers, a.from)) != PLD_OK) return rc;
    if (n_layers && (layers[0].num_pages != pool->num_pages || layers[0].page_size != pool->page_size)) return PLD_ERR_INVALID;
    if (((uintptr_t)map | (uintptr_t)used | (uintptr_t)table_out | (uintptr_t)refs_out) % 4) return PLD_ERR_ALIGN;
    if ((rc = check_work(pool, 1, workspace, workspace_bytes, c.w)) != PLD_OK) return rc;
    a.to = a.from;
    c.map = map, c.used = used, c.table_out = table_out, c.refs_out = refs_out;
    c.out_stride = pool->seqs > 1 ? table_out_stride : 0;
    const hipStream_t s = (hipStream_t)stream;
    const int spans = (pool->num_pages + kSpan - 1) / kSpan;
    if (spans > 1) hipLaunchKernelGGL(pages_span_kernel, dim3(spans), dim3(kPoolThreads), 0, s, c.p, c.w);
    hipLaunchKernelGGL(pages_rank_kernel, dim3(spans), dim3(kPoolThreads), 0, s, c.p, c.w);
    const int64_t elements = (int64_t)pool->seqs * pool->max_pages + pool->num_pages;
    const int64_t ints = (elements + 4 * kCopyThreads - 1) / (4 * kCopyThreads);
    return launch_copy<kMoves>(a, EditArgs{}, c, layers, layers, n_layers, pool->num_pages / 2, (int)(ints < 512 ? ints : 512), s);
}

extern "C" int pld_pages_copy(const pld_cache *from, const pld_cache *to, int n_layers, const int32_t *src,
                              const int32_t *dst, const int32_t *slots, int count, void *stream) {
    CopyArgs a{};
    if (!from || !to || n_layers < 1 || n_layers > PLD_MAX_LAYERS || !src || !dst || count < 1 || count > PLD_MAX_PAGES)
        return PLD_ERR_INVALID;
    int rc = check_layers(from, n_layers, a.from);
    if (rc == PLD_OK) rc = check_layers(to, n_layers, a.to);
    if (rc != PLD_OK) return rc;
    if (from->dtype != to->dtype || from->page_size != to->page_size || from->heads != to->heads || from->head_dim != to->head_dim)
        return PLD_ERR_INVALID;
    if (((uintptr_t)src | (uintptr_t)dst | (uintptr_t)slots) % 4) return PLD_ERR_ALIGN;
    a.src = src, a.dst = dst, a.slots = slots, a.count = count;
    return launch_copy<kPairs>(a, EditArgs{}, CompactArgs{}, from, to, n_layers, count, 0, (hipStream_t)stream);
}
