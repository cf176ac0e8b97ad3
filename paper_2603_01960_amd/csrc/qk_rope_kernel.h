// Queries and keys on their way from the projection to attention: RMS norm of each head's row, the weight of each column,
// and the rotation by the token's position, in one pass that also turns [B, S, H, D] into attention's [B, H, S, D] or writes
// keys and values into a cache.
//
//     y = x * r * w,  r = (mean(x^2) + eps)^(-1/2);   pair (a, b) of columns:  (y_a cos - y_b sin, y_b cos + y_a sin),
//     angle = position * inv_freq of the pair.
//
// Backward, g = the rotation back of the gradient:  dw = sum over the rows of g * x * r,
//     dx = r * (g * w - x * r * mean(g * w * x * r)).
//
// All of it is bound by memory (a row is read once and written once; 30 to 100 operations per 4 bytes), so the kernels are
// built for wide loads, many of them in flight, and whole lines written:
//   * a lane holds two 16-byte pieces of a row, which between them hold both columns of each of its pairs (columns i and i +
//     rot / 2 as pairs: pieces rot / 16 apart; neighbouring columns: any two), so that nothing but the sum of squares
//     crosses lanes.  D / 16 lanes make a row (of 4, 8, 8 or 16 that a row gets, so that the sum is DPP steps);
//   * a wavefront stays with one token and goes through its heads, so that the angles are computed once for all of them:
//     in 64 bits up to whole turns (a position of 2^31 has no fraction left in 32), then sine and cosine of the rest;
//   * all rows of a batch of heads are requested before the first is used.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sdpa_fwd_launch.h"

namespace tsdpa {

struct RopeRows {                                  // [B, S, heads, D], strides in elements
    const void *data;
    long long batch, row, head;
};

struct RopeArgs {
    RopeRows x[3];                                 // q, k, and in the cache form v
    RopeRows grad[2];                              // backward: where dq and dk go (as x)
    const void *dy[2];                             // backward: gradients of the results, [B, heads, S, D]
    const void *weight[2];                         // NULL: no norm
    int weight32;                                  // weights in FP32 (else in the rows' type)
    const int *positions;                          // [axis][batch][S] by the strides below
    long long pos_batch, pos_axis;
    const float *inv_freq;                         // [rot / 2]
    const int *axes;                               // NULL, or the axis of each pair
    int n_axes;
    int B, S, heads[3], rot, interleaved;
    float eps;
    void *out[3];                                  // q [B, H, S, D]; k the same or the cache; v's cache
    const int *slots;                              // cache form: [B, S]
    int cache_rows, block_rows;                    // rows of all pages (slots past it go nowhere), rows of a page
    Divisor by_rows, by_s, by_spans;
    int spans, units;                              // wavefronts per token; row groups of a token
    float *partial;                                // backward: [workgroups][2][D], sums of the weights' gradients
    int waves;                                     // backward: wavefronts of the launch
    hipStream_t stream;
};

template <int D> struct RopeGeom {
    static constexpr int LANES = D == 64 ? 4 : D == 160 ? 16 : 8;        // lanes of a row, of which D / 16 hold something
    static constexpr int ROWS = 64 / LANES;                              // rows of a wavefront at a time
};

int launch_rope_f16(int D, bool cache, const RopeArgs &a);
int launch_rope_bf16(int D, bool cache, const RopeArgs &a);
int launch_rope_bwd_f16(int D, const RopeArgs &a);
int launch_rope_bwd_bf16(int D, const RopeArgs &a);

// Backward: workgroups of the launch (each leaves one row of partial sums), of four wavefronts.
constexpr int kRopeBwdMost = 1024;
inline int rope_bwd_groups(long long tokens)
{
    const long long n = (tokens + 3) / 4;
    return (int)(n < 1 ? 1 : n < kRopeBwdMost ? n : kRopeBwdMost);
}

#if defined(__HIP_DEVICE_COMPILE__)
typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int rope_divide(int n, const Divisor &d) { return (int)(__umulhi(2u * (unsigned)n, d.mul) >> d.shift); }

// x + x of the lane that `ctrl` pairs it with
template <int CTRL> __device__ __forceinline__ float rope_dpp_add(float x)
{
    const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
    return x + __builtin_bit_cast(float, y);
}
// the sum over the lanes of a row, in each of them
template <int LANES> __device__ __forceinline__ float rope_row_sum(float x)
{
    x = rope_dpp_add<0xB1>(x);                     // lane ^ 1
    x = rope_dpp_add<0x4E>(x);                     // lane ^ 2
    if constexpr (LANES >= 8) x = rope_dpp_add<0x141>(x);       // mirrored within 8 lanes
    if constexpr (LANES >= 16) x = rope_dpp_add<0x140>(x);      // ... within 16
    return x;
}

template <typename T> struct RopePiece {           // 16 bytes: 8 values
    typedef T vec8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ void read(float (&x)[8], rope_u32x4 raw)
    {
        const vec8 v = __builtin_bit_cast(vec8, raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
    // the one rounding of a result
    static __device__ __forceinline__ rope_u32x4 write(const float (&x)[8])
    {
        vec8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)x[i];
        return __builtin_bit_cast(rope_u32x4, v);
    }
};

// What a lane has of every row, and how its pairs turn.
template <int D> struct RopeLane {
    int row, col[2];                               // row within the wavefront's; first columns of the two pieces
    bool active;
    float c[8], s[8];                              // pair i: half apart, columns col[0] + i and col[1] + i; neighbours: 2 i, 2 i + 1 of
                                                   // the first piece for i < 4, of the second from there on
    __device__ __forceinline__ RopeLane(const RopeArgs &a, int lane)
    {
        using G = RopeGeom<D>;
        row = lane / G::LANES;
        const int j = lane % G::LANES, turning = a.rot / 16;
        active = j < D / 16;
        // lanes past the rotated columns take two pieces in a row
        col[0] = j < turning ? j * 8 : j * 16;
        col[1] = j < turning ? (j + turning) * 8 : j * 16 + 8;
    }
    __device__ __forceinline__ void turn(const RopeArgs &a, int b, int s_)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = 1.f;
            s[i] = 0.f;
        }
        if (!active || col[0] >= a.rot) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = !a.interleaved ? col[0] + i : i < 4 ? col[0] / 2 + i : col[1] / 2 + i - 4;
            int axis = 0;
            if (a.axes != nullptr) {
                axis = a.axes[pair];
                axis = axis < 0 ? 0 : axis < a.n_axes ? axis : a.n_axes - 1;
            }
            const int position = a.positions[(long long)axis * a.pos_axis + (long long)b * a.pos_batch + s_];
            double turns = (double)position * (double)a.inv_freq[pair] * 0.15915494309189533577;
            turns -= __builtin_rint(turns);
            sincospif(2.f * (float)turns, &s[i], &c[i]);
        }
    }
    // rotates the pairs of a row's two pieces, by the angle or (BACK) back
    template <bool BACK> __device__ __forceinline__ void rotate(float (&x)[8], float (&y)[8], int interleaved) const
    {
        auto pair = [&](float &p, float &q, int i) __attribute__((always_inline)) {
            const float sin = BACK ? -s[i] : s[i], p0 = p;
            p = __builtin_fmaf(p0, c[i], -q * sin);
            q = __builtin_fmaf(q, c[i], p0 * sin);
        };
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pair(x[2 * i], x[2 * i + 1], i);
                pair(y[2 * i], y[2 * i + 1], i + 4);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) pair(x[i], y[i], i);
        }
    }
    // the weights of its columns (1 without a norm)
    template <typename T> __device__ __forceinline__ void weights(float (&w)[2][8], const void *at, int weight32) const
    {
        typedef float f4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[p][i] = 1.f;
            if (at == nullptr || !active) continue;
            if (weight32) {
                const f4 lo = ((const f4 *)at)[col[p] / 4], hi = ((const f4 *)at)[col[p] / 4 + 1];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[p][i] = i < 4 ? lo[i & 3] : hi[i & 3];
            } else {
                RopePiece<T>::read(w[p], ((const rope_u32x4 *)at)[col[p] / 8]);
            }
        }
    }
};
#endif

// Rows of a wavefront's heads at a time (rows that are requested together)
constexpr int kRopeBatch = 4;

template <typename T, int D, bool CACHE> __global__ void __launch_bounds__(256) rope_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePiece<T>;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int token = rope_divide(wave, a.by_spans), span = wave - token * a.spans;
    if (token >= a.B * a.S) return;
    const int b = rope_divide(token, a.by_s), s = token - b * a.S;
    RopeLane<D> me(a, lane);
    long long cache_row = -1;                      // the slot's row for head 0
    if constexpr (CACHE) {
        const int slot = __builtin_amdgcn_readfirstlane(a.slots[token]);
        if (slot >= 0 && slot < a.cache_rows) {
            const int page = rope_divide(slot, a.by_rows);
            cache_row = (long long)page * a.heads[1] * a.block_rows + (slot - page * a.block_rows);
        }
    }
    const int groups_q = (a.heads[0] + G::ROWS - 1) / G::ROWS, groups_k = (a.heads[1] + G::ROWS - 1) / G::ROWS;
    // the tensor (q, k, v) and head of a row group, and whether this lane has something of it
    struct Unit { int which, head; bool mine; };
    auto unit_at = [&](int unit) __attribute__((always_inline)) {
        const int which = unit < groups_q ? 0 : unit < groups_q + groups_k ? 1 : 2;
        const int head = (unit - (which == 0 ? 0 : which == 1 ? groups_q : groups_q + groups_k)) * G::ROWS + me.row;
        const bool wanted = unit < a.units && !(CACHE && which > 0 && cache_row < 0);
        return Unit{which, head, wanted && me.active && head < (which == 0 ? a.heads[0] : a.heads[1])};
    };
    rope_u32x4 raw[kRopeBatch][2];
    auto request = [&](int first) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            const Unit at = unit_at(first + u * a.spans);
            raw[u][0] = raw[u][1] = rope_u32x4{0, 0, 0, 0};
            if (!at.mine) continue;
            const RopeRows &in = a.x[at.which];
            const T *from = (const T *)in.data + (long long)b * in.batch + (long long)s * in.row + (long long)at.head * in.head;
            raw[u][0] = *(const rope_u32x4 *)(from + me.col[0]);
            raw[u][1] = *(const rope_u32x4 *)(from + me.col[1]);
        }
    };
    request(span);
    me.turn(a, b, s);
    float w[2][2][8];
    me.template weights<T>(w[0], a.weight[0], a.weight32);
    me.template weights<T>(w[1], a.weight[1], a.weight32);
    for (int first = span; first < a.units; first += kRopeBatch * a.spans) {
        if (first != span) request(first);
#pragma unroll
        for (int u = 0; u < kRopeBatch; ++u) {
            const Unit at = unit_at(first + u * a.spans);
            if (at.which < 2) {
                float x[8], y[8];
                P::read(x, raw[u][0]);
                P::read(y, raw[u][1]);
                if ((at.which == 0 ? a.weight[0] : a.weight[1]) != nullptr) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
                    const float r = 1.f / __builtin_sqrtf(rope_row_sum<G::LANES>(sum) * (1.f / D) + a.eps);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] *= r * (at.which == 0 ? w[0][0][i] : w[1][0][i]);
                        y[i] *= r * (at.which == 0 ? w[0][1][i] : w[1][1][i]);
                    }
                }
                me.template rotate<false>(x, y, a.interleaved);
                raw[u][0] = P::write(x);
                raw[u][1] = P::write(y);
            }
            if (!at.mine) continue;
            T *to = (T *)a.out[at.which];
            if (CACHE && at.which > 0) to += (cache_row + (long long)at.head * a.block_rows) * D;
            else to += (((long long)b * a.heads[at.which] + at.head) * a.S + s) * D;
            *(rope_u32x4 *)(to + me.col[0]) = raw[u][0];
            *(rope_u32x4 *)(to + me.col[1]) = raw[u][1];
        }
    }
#endif
}

// Backward.  A wavefront takes every `waves`-th token and keeps the sums of its columns' weight gradients in registers; a
// workgroup's are added in the LDS, in a fixed order, and written to its row of partial sums.
template <typename T, int D> __global__ void __launch_bounds__(256) rope_bwd_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePiece<T>;
    __shared__ float sums_sh[4][2][D];
    const int lane = threadIdx.x & 63, wave_in = threadIdx.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + wave_in);
    RopeLane<D> me(a, lane);
    float w[2][2][8], dw[2][2][8];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        me.template weights<T>(w[which], a.weight[which], a.weight32);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[which][p][i] = 0.f;
    }
    for (int token = wave; token < a.B * a.S; token += a.waves) {
        const int b = rope_divide(token, a.by_s), s = token - b * a.S;
        me.turn(a, b, s);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const bool norm = a.weight[which] != nullptr;
            const RopeRows &in = a.x[which], &to = a.grad[which];
            for (int h0 = 0; h0 < a.heads[which]; h0 += G::ROWS) {
                const int head = h0 + me.row;
                const bool mine = me.active && head < a.heads[which];
                rope_u32x4 raw[4] = {};
                if (mine) {
                    const T *dy = (const T *)a.dy[which] + (((long long)b * a.heads[which] + head) * a.S + s) * D;
                    raw[0] = *(const rope_u32x4 *)(dy + me.col[0]);
                    raw[1] = *(const rope_u32x4 *)(dy + me.col[1]);
                    if (norm) {
                        const T *from = (const T *)in.data + (long long)b * in.batch + (long long)s * in.row + (long long)head * in.head;
                        raw[2] = *(const rope_u32x4 *)(from + me.col[0]);
                        raw[3] = *(const rope_u32x4 *)(from + me.col[1]);
                    }
                }
                float g[8], h[8];
                P::read(g, raw[0]);
                P::read(h, raw[1]);
                me.template rotate<true>(g, h, a.interleaved);
                if (norm) {
                    float x[8], y[8], sum = 0.f, dot = 0.f;
                    P::read(x, raw[2]);
                    P::read(y, raw[3]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
                    const float r = 1.f / __builtin_sqrtf(rope_row_sum<G::LANES>(sum) * (1.f / D) + a.eps);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] *= r;
                        y[i] *= r;
                        dw[which][0][i] += g[i] * x[i];
                        dw[which][1][i] += h[i] * y[i];
                        g[i] *= w[which][0][i];
                        h[i] *= w[which][1][i];
                        dot += g[i] * x[i] + h[i] * y[i];
                    }
                    const float mean = rope_row_sum<G::LANES>(dot) * (1.f / D);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        g[i] = r * (g[i] - x[i] * mean);
                        h[i] = r * (h[i] - y[i] * mean);
                    }
                }
                if (!mine) continue;
                T *at = (T *)to.data + (long long)b * to.batch + (long long)s * to.row + (long long)head * to.head;
                *(rope_u32x4 *)(at + me.col[0]) = P::write(g);
                *(rope_u32x4 *)(at + me.col[1]) = P::write(h);
            }
        }
    }
    if (a.weight[0] == nullptr && a.weight[1] == nullptr) return;
    // over the wavefront's rows (lanes a row's length apart), then over the wavefronts
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = dw[which][p][i];
#pragma unroll
                for (int d = G::LANES; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
                if (me.row == 0 && me.active) sums_sh[wave_in][which][me.col[p] + i] = x;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += 256) {
        const float *at = &sums_sh[0][0][0] + i;
        a.partial[(size_t)blockIdx.x * 2 * D + i] = (at[0] + at[2 * D]) + (at[4 * D] + at[6 * D]);
    }
#endif
}

// The weights' gradients: rows of partial sums added up, one workgroup per four columns.
template <typename T> __global__ void __launch_bounds__(256) rope_bwd_sum_kernel(const float *__restrict__ partial, int groups, int D, void *dq, void *dk, int weight32)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef float f4 __attribute__((ext_vector_type(4)));
    __shared__ f4 sums_sh[4];
    f4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int r = threadIdx.x; r < groups; r += 256) sum += *(const f4 *)(partial + (size_t)r * 2 * D + blockIdx.x * 4);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum[c] += __shfl_xor(sum[c], d, 64);
    if ((threadIdx.x & 63) == 0) sums_sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x >= 4) return;
    const float x = (sums_sh[0][threadIdx.x] + sums_sh[1][threadIdx.x]) + (sums_sh[2][threadIdx.x] + sums_sh[3][threadIdx.x]);
    const int col = blockIdx.x * 4 + threadIdx.x;
    void *to = col < D ? dq : dk;
    if (to == nullptr) return;
    if (weight32) ((float *)to)[col % D] = x;
    else ((T *)to)[col % D] = (T)x;
#endif
}

template <typename T, int D> int launch_rope_dim(bool cache, const RopeArgs &a0)
{
    RopeArgs a = a0;
    using G = RopeGeom<D>;
    a.units = 0;
    for (int i = 0; i < (cache ? 3 : 2); ++i) a.units += (a.heads[i] + G::ROWS - 1) / G::ROWS;
    const long long tokens = (long long)a.B * a.S;
    // a wavefront for all heads of a token, or several where the tokens are few
    a.spans = 1;
    while (a.spans < a.units && tokens * a.spans < 2048) ++a.spans;
    a.by_spans = divisor((uint32_t)a.spans);
    const unsigned grid = (unsigned)((tokens * a.spans + 3) / 4);
    if (cache) hipLaunchKernelGGL((rope_kernel<T, D, true>), dim3(grid), dim3(256), 0, a.stream, a);
    else hipLaunchKernelGGL((rope_kernel<T, D, false>), dim3(grid), dim3(256), 0, a.stream, a);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_rope_bwd_dim(const RopeArgs &a0, void *dqw, void *dkw)
{
    RopeArgs a = a0;
    const int groups = rope_bwd_groups((long long)a.B * a.S);
    a.waves = groups * 4;
    hipLaunchKernelGGL((rope_bwd_kernel<T, D>), dim3((unsigned)groups), dim3(256), 0, a.stream, a);
    const int err = (int)hipGetLastError();
    if (err != 0 || (a.weight[0] == nullptr && a.weight[1] == nullptr)) return err;
    hipLaunchKernelGGL((rope_bwd_sum_kernel<T>), dim3(2 * D / 4), dim3(256), 0, a.stream, (const float *)a.partial, groups, D, dqw, dkw, a.weight32);
    return (int)hipGetLastError();
}

template <typename T> int launch_rope(int D, bool cache, const RopeArgs &a)
{
    switch (D) {
        case 64: return launch_rope_dim<T, 64>(cache, a);
        case 96: return launch_rope_dim<T, 96>(cache, a);
        case 128: return launch_rope_dim<T, 128>(cache, a);
        default: return launch_rope_dim<T, 160>(cache, a);
    }
}

template <typename T> int launch_rope_bwd(int D, const RopeArgs &a)
{
    switch (D) {
        case 64: return launch_rope_bwd_dim<T, 64>(a, a.out[0], a.out[1]);
        case 96: return launch_rope_bwd_dim<T, 96>(a, a.out[0], a.out[1]);
        case 128: return launch_rope_bwd_dim<T, 128>(a, a.out[0], a.out[1]);
        default: return launch_rope_bwd_dim<T, 160>(a, a.out[0], a.out[1]);
    }
}

}  // namespace tsdpa
