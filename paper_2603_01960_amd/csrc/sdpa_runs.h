// The end of a decoding step whose keys are cut into runs: one state (o, m, l of Eqs. 2-4) per run and row in the workspace, combined by
// the workgroup of the head that is done last.
#pragma once
#include "sdpa_fwd_kernel.h"

namespace tsdpa {

// The runs' states are combined by whichever workgroup of the head is last to be done with its own, in run order
// whoever that is.  A workgroup writes its state, waits for the writes, marks it done, and looks at all the marks of its
// head: the last one finds them all; should two find them all, both write the same result.  Marks need no memory of
// their own and no cleared memory: they stand in the head's part of o, which nothing else uses before the result
// overwrites it, and a mark is the ticket of this very call, a 64-bit number that no other call has (the output of an
// earlier replay of the same graph, or whatever else o held, equals it with probability 2^-64).
// States and marks are written and read at agent scope, access by access: past the L2s, of which every XCD has its
// own.  (With plain accesses and release / acquire fences every workgroup writes back and invalidates its XCD's
// whole L2: 256 workgroups took 36 us instead of 15.)
struct RunPair { float x, y; };
__device__ __forceinline__ void put_pair(float *at, float x, float y)
{
    const unsigned long long both = ((unsigned long long)__builtin_bit_cast(uint32_t, y) << 32) | __builtin_bit_cast(uint32_t, x);
    __hip_atomic_store((unsigned long long *)at, both, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ RunPair get_pair(const float *at)
{
    const unsigned long long both = __hip_atomic_load((unsigned long long *)at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t lo = (uint32_t)both, hi = (uint32_t)(both >> 32);
    return RunPair{__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}

// Run sp of `splits` of this head is done (its state put into ws: o as float [heads][splits][S][D], then (m, l) [heads][splits][S][2]).
template <typename T, int D, int NW>
__device__ __forceinline__ void finish_runs(T *o, float *lse, const float *ws, lds_ptr lds, int head, int sp, int S, int heads, int splits,
                                            unsigned long long ticket, int tid, int wave, int lane)
{
#if defined(__HIP_DEVICE_COMPILE__)
    unsigned long long *marks = (unsigned long long *)(o + (size_t)head * S * D);
    TSDPA_WAIT_VMCNT0();
    __syncthreads();
    typedef TSDPA_LDS float *lds_f;
    const lds_f wgt = (lds_f)lds;
    if (wave == 0) {
        if (lane == 0) (void)__hip_atomic_exchange(marks + sp, ticket, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        TSDPA_WAIT_VMCNT0();
        bool done = true;
#pragma unroll
        for (int i = 0; i < 128; i += 64)
            if (i + lane < splits) done &= __hip_atomic_load(marks + i + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == ticket;
        const bool all = __builtin_amdgcn_ballot_w64(!done) == 0;
        if (lane == 0) wgt[0] = all ? 1.f : 0.f;
    }
    __syncthreads();
    const bool last = wgt[0] != 0.f;
    __syncthreads();
    if (!last) return;
    // weights of the runs per row, then the weighted sum of their o: [splits][S] weights in the LDS
    const float *po = ws + (size_t)head * splits * S * D;
    const float *pml = ws + (size_t)heads * splits * S * D + (size_t)head * splits * S * 2;
    // one wavefront per row, a lane per run (and another 64 runs on)
    for (int row = wave; row < S; row += NW) {
        RunPair st[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            st[i] = RunPair{-INFINITY, 0.f};
            if (lane + i * 64 < splits) st[i] = get_pair(pml + ((lane + i * 64) * S + row) * 2);
        }
        float M = fmaxf(st[0].x, st[1].x);
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) M = fmaxf(M, __shfl_xor(M, w, 64));
        float L = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float w = st[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[i].x - M);
            // (a run without keys, l = 0, has left its o unwritten: marked by a negative weight; a row of NaN scores has l = NaN)
            if (lane + i * 64 < splits) wgt[(lane + i * 64) * S + row] = st[i].y == 0.f ? -1.f : w;
            L += w * st[i].y;
        }
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) L += __shfl_xor(L, w, 64);
        if (lane == 0) {
            wgt[splits * S + row] = M == -INFINITY ? 0.f : 1.f / L;      // (a row that no key reaches: O = 0, LSE = -inf)
            if (lse != nullptr)
                lse[(size_t)head * S + row] = L != 0.f ? (M + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f : -INFINITY;
        }
    }
    __syncthreads();
    // Eight runs' loads in flight; the last batch, if it is not full, loads its first run again.  What bounds this part is the
    // number of round trips past the L2, so a thread has two columns where that takes all of them in one pass, and else four.
    // (The whole call in us, remainder run by run and two columns at all times -> this: 8 heads, one row of D = 64 in 7 runs 9.2 ->
    // 7.6, in 12 8.2 -> 7.4, in 8 or 16 level; 8 rows of D = 160 in 7 runs 14.7 -> 12.1; 30 heads, 4 rows of D = 128 in 7
    // 13.3 -> 12.0.  Four columns at all times cost 0.4 to 1 us at 8 and 16 runs, and several threads per four columns, which
    // share the runs, 0.3 us more up to 16.)
    auto combine = [&](auto pairs) {
        constexpr int P = pairs;
        for (int x = tid; x < S * (D / 2 / P); x += NW * 64) {
            const int row = x / (D / 2 / P);
            float sum[2 * P] = {};
            auto batch = [&](int s0, auto whole) {
                RunPair part[8][P];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float *at = po + (size_t)(whole || s0 + i < splits ? s0 + i : s0) * S * D + (size_t)x * (2 * P);
#pragma unroll
                    for (int p = 0; p < P; ++p) part[i][p] = get_pair(at + 2 * p);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!whole && s0 + i >= splits) break;
                    const float w = wgt[(s0 + i) * S + row];
                    if (!(w < 0.f)) {
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            sum[2 * p] += w * part[i][p].x;
                            sum[2 * p + 1] += w * part[i][p].y;
                        }
                    }
                }
            };
            int s0 = 0;
            for (; s0 + 8 <= splits; s0 += 8) batch(s0, std::true_type{});
            if (s0 < splits) batch(s0, std::false_type{});
            const float inv = wgt[splits * S + row];
            typedef T Out __attribute__((ext_vector_type(2 * P)));
            Out out;
#pragma unroll
            for (int c = 0; c < 2 * P; ++c) out[c] = (T)(sum[c] * inv);
            *(Out *)(o + (size_t)head * S * D + (size_t)x * (2 * P)) = out;
        }
    };
    if (S * (D / 2) <= NW * 64) combine(std::integral_constant<int, 1>{});
    else combine(std::integral_constant<int, 2>{});
#endif
}

}  // namespace tsdpa
