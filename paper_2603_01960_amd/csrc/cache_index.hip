// Index tensors of a serving step, built on the GPU: ancestor masks of trees of drafted tokens, and the pages, slots and
// positions of the tokens that a step appends to a cache.  See include/tiled_sdpa.h for the contract of the entry points.
//
// Both are a few kilobytes of work and bound by latency: one launch each, no atomics, no workspace, nothing that depends on
// which workgroup runs first.  Kernel / whole call, us: masks of 1 tree of 15 tokens 1.8 / 4.8, of 64 trees of 255 3.7 / 4.8; steps
// of 1 entry and token 2.8 / 4.5 to 5.3, of 256 entries of up to 60 tokens 4.1 / 4.6 to 5.3 (an empty kernel's call: 3.7 to 4.5).
// A step's sums are every workgroup's own, so that its time grows with the square of the entries: 16 tokens each, all appended /
// 64 tokens at most, a quarter of the entries giving a page up to the others, a call in us: 32 entries 3.8 / 7.3, 256 3.9 / 7.9, 1024
// 6.5 / 12, 4096 25 / 66, 8192 102 / 374.  (The pages handed over cost a sum over the threads one by one, and a search per page.)
#include "tiled_sdpa.h"

#include <cstdint>
#include <limits>

#include "sdpa_fwd_launch.h"

namespace tsdpa {

// Ancestors by pointer jumping: after r rounds a node knows its nearest 2^r ancestors (itself included) and the one after
// them, so that a round's OR of that one's set doubles what it knows; log2(T) rounds whatever the shape of the tree, fewer
// where it is shallow.  One workgroup per entry and word of the mask (64 nodes), one thread per node: the rounds on one word
// do not need the others', so wide trees repeat the jumps instead of keeping T x T bits in the LDS.
// A parent is followed only if it comes before its node; every chain thus ends, whatever the array holds.
constexpr int kMostNodes = 1024;
__global__ void __launch_bounds__(kMostNodes)
tree_mask_kernel(const int *__restrict__ parents, unsigned long long *__restrict__ mask, int *__restrict__ depths, int T, int words)
{
#if defined(__HIP_DEVICE_COMPILE__)
    // (two of each: a round writes what the next but one overwrites, so that one barrier per round is enough; and three flags: the one
    // that a round clears for the next was last read in front of the barrier before)
    __shared__ unsigned long long set_sh[2][kMostNodes];
    __shared__ int chain_sh[2][kMostNodes], more_sh[3];
    const int entry = blockIdx.x, word = blockIdx.y, node = threadIdx.x;
    // steps to the ancestor that the node has reached, and that ancestor + 1 (0: it has reached a root) in the low half
    int chain = 0;
    unsigned long long set = 0;
    if (node < T) {
        const int p = parents[(size_t)entry * T + node];
        if (p >= 0 && p < node) chain = 1 << 16 | (p + 1);
        if (node >> 6 == word) set = 1ull << (node & 63);
    }
    if (node < 3) more_sh[node] = 0;
    __syncthreads();
    for (int round = 0, flag = 0;; round ^= 1) {
        const int next = flag == 2 ? 0 : flag + 1;
        set_sh[round][node] = set;
        chain_sh[round][node] = chain;
        if ((chain & 0xffff) != 0) more_sh[flag] = 1;
        if (node == 0) more_sh[next] = 0;
        __syncthreads();
        if (more_sh[flag] == 0) break;             // (the same in every thread; the ancestors reached fall in every round)
        const int at = (chain & 0xffff) - 1;
        if (at >= 0) {
            set |= set_sh[round][at];
            chain = (chain & ~0xffff) + chain_sh[round][at];
        }
        flag = next;
    }
    const int steps = chain >> 16;
    if (node >= T) return;
    mask[((size_t)entry * T + node) * words + word] = set;
    if (word == 0 && depths != nullptr) depths[(size_t)entry * T + node] = steps;
#endif
}

constexpr int kStepThreads = 256, kStepTokens = 1024, kMostEntries = 8192;

struct StepArgs {
    const int *lens, *counts, *depths;
    int *table, *free_pages;                       // NULL: a dense cache, entry b in rows b * block_rows ...
    const int *pool;
    int *new_lens, *slots, *positions, *new_pool;
    int B, S, max_blocks, block_rows, pool_size;
    Divisor by_rows;
};

__device__ __forceinline__ int step_divide(int n, const Divisor &d) { return (int)(__umulhi(2u * (unsigned)n, d.mul) >> d.shift); }

// What an entry's request amounts to.
struct StepEntry {
    int len, next, held, need;                     // rows and pages before and after
    bool sound;                                    // the numbers can be a cache's
    int over;                                      // pages (dense: rows) past the end of the entry's place
};
__device__ __forceinline__ StepEntry step_entry(const StepArgs &a, int b)
{
    StepEntry e;
    const int len = a.lens[b], count = a.counts[b];
    const long long most = (long long)a.max_blocks * a.block_rows, next = (long long)len + count;
    e.sound = len >= 0 && len <= most && next >= 0 && count <= a.S;
    e.len = e.sound ? len : 0;
    e.next = e.len;
    e.over = 0;
    if (e.sound && next > most) {
        // (next <= 2^31 - 1 + S, held in 64 bits; the sum over the entries in 32: it is a number of pages to wait for, not an index)
        const long long over = a.table ? (next - most + a.block_rows - 1) / a.block_rows : next - most;
        e.over = (int)(over < (1 << 16) ? over : 1 << 16);
        e.next = (int)most;                        // (what is missing is counted up to the end from the pool, from there on as past it)
    } else if (e.sound) {
        e.next = (int)next;
    }
    // (rows up to a whole page: below 2^31, see the entry point's checks)
    e.held = a.table ? step_divide(e.len + a.block_rows - 1, a.by_rows) : 0;
    e.need = a.table ? step_divide(e.next + a.block_rows - 1, a.by_rows) : 0;
    return e;
}

// The sums over the workgroup of N values per thread, in every thread.
template <int N> __device__ __forceinline__ void step_sums(int (&x)[N], int *sh)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) x[i] += __shfl_xor(x[i], w, 64);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh[(threadIdx.x >> 6) * N + i] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = 0;
#pragma unroll
        for (int w = 0; w < kStepThreads / 64; ++w) x[i] += sh[w * N + i];
    }
}

// One workgroup per entry and 1024 of its tokens.  Where an entry's pages come from depends on the entries before it: every
// workgroup sums over all of them by itself (a few loads per thread), so that none waits for another and one launch does.
// Nothing that one workgroup reads is written by another: the table's columns up to `held` and the pool's pages below its
// count are only read, those from there on only written, and a page that one entry gives up goes straight to the entry that
// needs one (found in the table, whose columns past `need` a shrinking entry keeps).
__global__ void __launch_bounds__(kStepThreads) cache_step_kernel(StepArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ int released_sh[];           // [B]: pages given up by the entries up to and with this one
    __shared__ int sums_sh[kStepThreads / 64 * 6], scan_sh[kStepThreads];
    const int b = blockIdx.x, tid = threadIdx.x;
    // pages taken and given up in all, and by the entries before this one; pages past the ends; entries that are no cache's
    int sum[6] = {};
    for (int i = tid; i < a.B; i += kStepThreads) {
        const StepEntry e = step_entry(a, i);
        const int grow = e.need > e.held ? e.need - e.held : 0, drop = e.held > e.need ? e.held - e.need : 0;
        sum[0] += grow;
        sum[1] += drop;
        if (i < b) {
            sum[2] += grow;
            sum[3] += drop;
        }
        sum[4] += e.over;
        sum[5] += e.sound ? 0 : 1;
    }
    step_sums(sum, sums_sh);
    const int taken = sum[0], dropped = sum[1];
    const int have = a.table ? a.pool[0] : 0;
    const bool sound = sum[5] == 0 && have >= 0 && have <= a.pool_size && (dropped <= taken || have + (long long)(dropped - taken) <= a.pool_size);
    const int lack = taken - dropped > have ? taken - dropped - have : 0;
    const bool go = sound && lack == 0 && sum[4] == 0;
    if (b == 0 && blockIdx.y == 0 && tid == 0) {
        a.new_pool[0] = go ? have + dropped - taken : have;
        a.new_pool[1] = go ? 0 : sound ? lack + sum[4] : -1;
    }
    if (b >= a.B) return;                          // (no entries: only the pool's state is handed on)
    const StepEntry own = step_entry(a, b);
    const int len = a.lens[b], next = go ? own.next : len;
    const int grow = go && own.need > own.held ? own.need - own.held : 0, drop = go && own.held > own.need ? own.held - own.need : 0;
    int *const row_of_table = a.table + (a.table ? (size_t)b * a.max_blocks : 0);
    // the x-th page that is taken: the x-th that is given up, then the pool's from its end
    const int first = sum[2];
    const bool handed = grow > 0 && first < dropped;
    if (handed) {
        const int per = (a.B + kStepThreads - 1) / kStepThreads, lo = tid * per, hi = lo + per < a.B ? lo + per : a.B;
        int mine = 0;
        for (int i = lo; i < hi; ++i) {
            const StepEntry e = step_entry(a, i);
            mine += e.held > e.need ? e.held - e.need : 0;
            released_sh[i] = mine;
        }
        scan_sh[tid] = mine;
        __syncthreads();
        int before = 0;
        for (int t = 0; t < tid; ++t) before += scan_sh[t];
        for (int i = lo; i < hi; ++i) released_sh[i] += before;
        __syncthreads();
    }
    auto new_page = [&](int i) {
        const int x = first + i;
        if (x >= dropped) return a.free_pages[have - 1 - (x - dropped)];
        int lo = 0, hi = a.B - 1;                  // the first entry with more than x pages given up with it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (released_sh[mid] > x) hi = mid; else lo = mid + 1;
        }
        const StepEntry e = step_entry(a, lo);
        return a.table[(size_t)lo * a.max_blocks + e.held - (released_sh[lo] - x)];
    };
    if (blockIdx.y == 0) {
        if (tid == 0) a.new_lens[b] = next;
        for (int i = tid; i < grow; i += kStepThreads) row_of_table[own.held + i] = new_page(i);
        // what no entry needs goes on the pool, the first of them on top: appending as much again takes the same pages
        for (int i = tid; i < drop; i += kStepThreads) {
            const int x = sum[3] + i;
            if (x >= taken) a.free_pages[have + dropped - 1 - x] = row_of_table[own.need + i];
        }
    }
    const int i1 = (blockIdx.y + 1) * kStepTokens < a.S ? (blockIdx.y + 1) * kStepTokens : a.S;
    for (int i = blockIdx.y * kStepTokens + tid; i < i1; i += kStepThreads) {
        const int row = next - a.S + i;
        int slot = -1, position = 0;
        if (go && row >= len) {
            const int block = a.table ? step_divide(row, a.by_rows) : 0;
            const int page = !a.table ? b : block < own.held ? row_of_table[block] : new_page(block - own.held);
            slot = page * a.block_rows + row - block * a.block_rows;
            position = a.depths ? next - a.S + a.depths[(size_t)b * a.S + i] : row;
        }
        a.slots[(size_t)b * a.S + i] = slot;
        a.positions[(size_t)b * a.S + i] = position;
    }
#endif
}

}  // namespace tsdpa

extern "C" {

int tiled_sdpa_tree_mask(const int *parents, long long *mask, int *depths, int B, int T, void *stream)
{
    if (B < 0 || T < 0 || T > tsdpa::kMostNodes) return TSDPA_ERR_BAD_SHAPE;
    if ((int64_t)B * T == 0) return TSDPA_OK;
    if (!parents || !mask) return TSDPA_ERR_NULL_PTR;
    if ((((uintptr_t)parents | (uintptr_t)depths) & 3u) != 0 || ((uintptr_t)mask & 7u) != 0) return TSDPA_ERR_MISALIGNED;
    const int words = (T + 63) / 64;
    hipLaunchKernelGGL(tsdpa::tree_mask_kernel, dim3((unsigned)B, (unsigned)words), dim3((unsigned)words * 64), 0, (hipStream_t)stream,
                       parents, (unsigned long long *)mask, depths, T, words);
    return hipGetLastError() == hipSuccess ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

int tiled_sdpa_cache_step(const int *kv_lens, const int *counts, const int *depths, int *block_table, int *free_pages, const int *pool,
                          int *new_lens, int *slots, int *positions, int *new_pool,
                          int B, int S, int max_blocks, int block_rows, int pool_size, void *stream)
{
    if (B < 0 || B > tsdpa::kMostEntries || S < 0 || block_rows < 1 || max_blocks < 0 || pool_size < 0) return TSDPA_ERR_BAD_SHAPE;
    if (!block_table) max_blocks = 1;
    // rows of an entry, rounded up to whole pages, pages of all entries, slots, and the grid are 32-bit numbers
    const int64_t most = std::numeric_limits<int>::max();
    const int64_t pages = block_table ? (int64_t)pool_size : (int64_t)B;
    if (((int64_t)max_blocks + 1) * block_rows > most || (int64_t)B * max_blocks > most || pages * block_rows > most || (int64_t)B * S > most ||
        (int64_t)S + (int64_t)max_blocks * block_rows > most || S > 65535 * tsdpa::kStepTokens)
        return TSDPA_ERR_BAD_SHAPE;
    if (!new_pool || (B > 0 && (!kv_lens || !counts || !new_lens)) || ((int64_t)B * S > 0 && (!slots || !positions)) ||
        (block_table && (!free_pages || !pool)))
        return TSDPA_ERR_NULL_PTR;
    const uintptr_t bits = (uintptr_t)kv_lens | (uintptr_t)counts | (uintptr_t)depths | (uintptr_t)block_table | (uintptr_t)free_pages |
                           (uintptr_t)pool | (uintptr_t)new_lens | (uintptr_t)slots | (uintptr_t)positions | (uintptr_t)new_pool;
    if ((bits & 3u) != 0) return TSDPA_ERR_MISALIGNED;
    tsdpa::StepArgs a{kv_lens, counts, depths, block_table, free_pages, pool, new_lens, slots, positions, new_pool,
                      B, S, max_blocks, block_rows, pool_size, tsdpa::divisor((uint32_t)block_rows)};
    const unsigned chunks = S > tsdpa::kStepTokens ? (unsigned)((S + tsdpa::kStepTokens - 1) / tsdpa::kStepTokens) : 1u;
    hipLaunchKernelGGL(tsdpa::cache_step_kernel, dim3(B > 0 ? (unsigned)B : 1u, chunks), dim3(tsdpa::kStepThreads),
                       block_table ? (size_t)B * sizeof(int) : 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

}  // extern "C"
