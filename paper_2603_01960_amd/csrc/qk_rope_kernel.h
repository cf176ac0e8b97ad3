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
    int spans, units_per_span;                     // parts of a token that a wavefront each takes; their row groups
    int waves;                                     // wavefronts of the launch
    // backward, for q and k: workgroups (those of q first), parts of a token that a wavefront each takes, heads of a part
    int bwd_groups[2], bwd_spans[2], bwd_heads[2];
    Divisor bwd_by_spans[2];
    float *partial;                                // backward: [workgroups][D], sums of a weight's gradient
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

#ifndef ROPE_BOCC
#define ROPE_BATCH 2
#define ROPE_OCC 4
#define ROPE_BBATCH 1
#define ROPE_BOCC 4
#endif
// Backward: most workgroups of a launch (as many as the GPU holds); each leaves a row of partial sums.
constexpr int kRopeBwdMost = ROPE_BOCC * 256;

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

// The two pieces of a row as 16 FP32 values, x and y: pair i is (x[i], y[i]).  Half a rotation apart that is what the pieces are; of
// neighbouring columns (INTER) x takes the even ones of both pieces and y the odd ones.
template <typename T, bool INTER> struct RopePairs {
    typedef T vec8 __attribute__((ext_vector_type(8)));
    static constexpr uint32_t LOW = 0x05040100u, HIGH = 0x07060302u;     // halves of two words, by v_perm
    static __device__ __forceinline__ void read(float (&x)[8], float (&y)[8], const rope_u32x4 (&raw)[2])
    {
        rope_u32x4 p[2] = {raw[0], raw[1]};
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = raw[i >> 1][(i & 1) * 2], hi = raw[i >> 1][(i & 1) * 2 + 1];
                p[0][i] = __builtin_amdgcn_perm(hi, lo, LOW);
                p[1][i] = __builtin_amdgcn_perm(hi, lo, HIGH);
            }
        }
        const vec8 u = __builtin_bit_cast(vec8, p[0]), v = __builtin_bit_cast(vec8, p[1]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = (float)u[i];
            y[i] = (float)v[i];
        }
    }
    // the one rounding of a result
    static __device__ __forceinline__ void write(rope_u32x4 (&raw)[2], const float (&x)[8], const float (&y)[8])
    {
        vec8 u, v;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = (T)x[i];
            v[i] = (T)y[i];
        }
        const rope_u32x4 p[2] = {__builtin_bit_cast(rope_u32x4, u), __builtin_bit_cast(rope_u32x4, v)};
        raw[0] = p[0];
        raw[1] = p[1];
        if constexpr (INTER) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                raw[i >> 1][(i & 1) * 2] = __builtin_amdgcn_perm(p[1][i], p[0][i], LOW);
                raw[i >> 1][(i & 1) * 2 + 1] = __builtin_amdgcn_perm(p[1][i], p[0][i], HIGH);
            }
        }
    }
};

// What a lane has of every row.
template <int D, bool INTER> struct RopeLane {
    int row, col[2];                               // row within the wavefront's; first columns of the two pieces
    bool active;                                   // the lane has something of the row
    int first;                                     // its first pair, of the D / 2 that the lanes of a row have
    __device__ __forceinline__ RopeLane(int rot, int lane)
    {
        using G = RopeGeom<D>;
        row = lane / G::LANES;
        const int own = lane % G::LANES, j = own < D / 16 ? own : D / 16 - 1;
        active = own < D / 16;
        first = j * 8;
        col[0] = columns(rot, j, 0);
        col[1] = columns(rot, j, 1);
    }
    // first column of piece p of the j-th lane of a row; lanes past the rotated columns take two pieces in a row
    static __device__ __forceinline__ int columns(int rot, int j, int p)
    {
        const int turning = rot / 16;
        return j < turning ? (j + (p ? turning : 0)) * 8 : j * 16 + p * 8;
    }
    // the column of x[i] (p = 0) or y[i], from the first columns of the pieces
    static __device__ __forceinline__ int column(int c0, int c1, int p, int i) { return !INTER ? (p ? c1 : c0) + i : (i < 4 ? c0 + 2 * i : c1 + 2 * i - 8) + p; }
    __device__ __forceinline__ float row_sum(float x) const { return rope_row_sum<RopeGeom<D>::LANES>(RopeGeom<D>::LANES * 16 == D || active ? x : 0.f); }
    // 1 / sqrt(mean of squares + eps) of the row
    __device__ __forceinline__ float scale(const float (&x)[8], const float (&y)[8], float eps) const
    {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(y[i], y[i], __builtin_fmaf(x[i], x[i], sum));
        return __builtin_amdgcn_rsqf(row_sum(sum) * (1.f / D) + eps);
    }
};

// The angles of a token's pairs: computed once per wavefront, a lane a pair, and handed to the lanes that need them through the LDS
// (a wavefront's own part, whose accesses are in order).  Tables of D / 2 values, V of them per token: cosine and sine of each pair,
// or (forward) both times the weights of its two columns, for q and for k.
template <typename T, int D, bool INTER, int V> struct RopeTable {
    static constexpr int EACH = (D / 2 + 63) / 64;       // pairs of a lane
    double step[EACH];                             // turns per position
    int axis[EACH];
    float w[EACH][2][2];                           // weights of q and k for the pair's columns
    float *mine;
    __device__ __forceinline__ RopeTable(const RopeArgs &a, int lane, float *wave_sh) : mine(wave_sh + lane)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int slot = lane + e * 64 < D / 2 ? lane + e * 64 : D / 2 - 1, j = slot / 8, i = slot % 8;
            const int c0 = RopeLane<D, INTER>::columns(a.rot, j, 0), c1 = RopeLane<D, INTER>::columns(a.rot, j, 1);
            const int pair = !INTER ? c0 + i : i < 4 ? c0 / 2 + i : c1 / 2 + i - 4;
            const bool turns = j < a.rot / 16;
            step[e] = turns ? (double)a.inv_freq[pair] * 0.15915494309189533577 : 0.0;
            int x = turns && a.axes != nullptr ? a.axes[pair] : 0;
            axis[e] = x < 0 ? 0 : x < a.n_axes ? x : a.n_axes - 1;
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int col = RopeLane<D, INTER>::column(c0, c1, p, i);
                    w[e][which][p] = a.weight[which] == nullptr ? 1.f : a.weight32 ? ((const float *)a.weight[which])[col] : (float)((const T *)a.weight[which])[col];
                }
        }
    }
    // v_sin and v_cos take whole turns: off by at most 2^-22.9 over one
    __device__ __forceinline__ void fill(const RopeArgs &a, int b, int s) const
    {
        const int *at = a.positions + ((long long)b * a.pos_batch + s);
        const int position = a.rot > 0 ? *at : 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const double p = a.axes == nullptr || a.rot == 0 ? (double)position : (double)at[(long long)axis[e] * a.pos_axis], x = p * step[e];
            const float t = (float)(x - __builtin_rint(x)), c = __builtin_amdgcn_cosf(t), sn = __builtin_amdgcn_sinf(t);
            if ((D / 2) % 64 != 0 && (int)(threadIdx.x & 63) + e * 64 >= D / 2) continue;
            float *to = mine + e * 64;
            if constexpr (V == 2) {
                to[0] = c;
                to[D / 2] = sn;
            } else {
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    to[(which * 4 + 0) * (D / 2)] = w[e][which][0] * c;
                    to[(which * 4 + 1) * (D / 2)] = w[e][which][0] * sn;
                    to[(which * 4 + 2) * (D / 2)] = w[e][which][1] * c;
                    to[(which * 4 + 3) * (D / 2)] = w[e][which][1] * sn;
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
};
__device__ __forceinline__ void rope_table_read(float (&x)[8], const float *at)
{
    typedef float f4 __attribute__((ext_vector_type(4)));
    const f4 lo = *(const f4 *)at, hi = *(const f4 *)(at + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < 4 ? lo[i & 3] : hi[i & 3];
}

// A lane's two pieces of a row group, at base + scalar offset; lanes without one keep what is in the registers, which nothing uses.
template <typename T> struct RopePointers {
    const T *at[2];
    __device__ __forceinline__ RopePointers(const void *base, long long row, const int (&col)[2])
    {
        at[0] = (const T *)base + row + col[0];
        at[1] = (const T *)base + row + col[1];
    }
    __device__ __forceinline__ void load(rope_u32x4 (&raw)[2], long long offset, bool mine) const
    {
        asm("" : "=v"(raw[0]), "=v"(raw[1]));
        if (!mine) return;
        raw[0] = *(const rope_u32x4 *)(at[0] + offset);
        raw[1] = *(const rope_u32x4 *)(at[1] + offset);
    }
    __device__ __forceinline__ void store(const rope_u32x4 (&raw)[2], long long offset) const
    {
        *(rope_u32x4 *)(at[0] + offset) = raw[0];
        *(rope_u32x4 *)(at[1] + offset) = raw[1];
    }
};
#endif

// Row groups (of RopeGeom::ROWS heads) whose rows are requested together.
constexpr int kRopeBatch = ROPE_BATCH, kRopeWaves = ROPE_OCC * 1024;

template <typename T, int D, bool CACHE, bool INTER> __global__ void __launch_bounds__(256, ROPE_OCC) rope_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePairs<T, INTER>;
    __shared__ __attribute__((aligned(16))) float table_sh[4][8 * (D / 2)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int items = a.B * a.S * a.spans;
    if (wave >= items) return;
    const RopeLane<D, INTER> me(a.rot, lane);
    float *const table = table_sh[threadIdx.x >> 6];
    const RopeTable<T, D, INTER, 8> pairs(a, lane, table);
    for (int item = wave; item < items; item += a.waves) {
        const int token = rope_divide(item, a.by_spans), span = item - token * a.spans;
        const int b = rope_divide(token, a.by_s), s = token - b * a.S;
        long long cache_row = -1;                  // the slot's row for head 0
        if constexpr (CACHE) {
            const int slot = __builtin_amdgcn_readfirstlane(a.slots[token]);
            if (slot >= 0 && slot < a.cache_rows) {
                const int page = rope_divide(slot, a.by_rows);
                cache_row = (long long)page * a.heads[1] * a.block_rows + (slot - page * a.block_rows);
            }
        }
        pairs.fill(a, b, s);
        int unit0 = 0;                             // first row group of the tensor
#pragma unroll
        for (int which = 0; which < (CACHE ? 3 : 2); ++which) {
            const int heads = a.heads[which], groups = (heads + G::ROWS - 1) / G::ROWS;
            // this span's row groups of the tensor
            int g0 = span * a.units_per_span - unit0, g1 = g0 + a.units_per_span;
            unit0 += groups;
            g0 = g0 > 0 ? g0 : 0;
            g1 = g1 < groups ? g1 : groups;
            if (g0 >= g1 || (CACHE && which > 0 && cache_row < 0)) continue;
            const bool norm = which < 2 && a.weight[which & 1] != nullptr;
            // rows are x_a (w_a cos), x_b (w_b sin) and so on, times the row's 1 / root
            float cx[8], sx[8], cy[8], sy[8];
            if (which < 2) {
                const float *at = table + which * 4 * (D / 2) + me.first;
                rope_table_read(cx, at);
                rope_table_read(sx, at + D / 2);
                rope_table_read(cy, at + 2 * (D / 2));
                rope_table_read(sy, at + 3 * (D / 2));
            }
            const RopeRows &in = a.x[which];
            const RopePointers<T> from((const T *)in.data + (long long)b * in.batch + (long long)s * in.row, me.row * in.head, me.col);
            const bool cached = CACHE && which > 0;
            const long long to_head = (long long)(cached ? a.block_rows : a.S) * D;
            const RopePointers<T> to((const T *)a.out[which] + (cached ? cache_row * D : ((long long)b * heads * a.S + s) * D), me.row * to_head, me.col);
            for (int g = g0; g < g1; g += kRopeBatch) {
                rope_u32x4 raw[kRopeBatch][2];
#pragma unroll
                for (int u = 0; u < kRopeBatch; ++u)
                    if (u == 0 || g + u < g1) from.load(raw[u], (long long)(g + u) * G::ROWS * in.head, (g + u) * G::ROWS + me.row < heads);
#pragma unroll
                for (int u = 0; u < kRopeBatch; ++u) {
                    if (u > 0 && g + u >= g1) continue;
                    if (which < 2) {
                        float x[8], y[8], r = 1.f;
                        P::read(x, y, raw[u]);
                        if (norm) r = me.scale(x, y, a.eps);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float x0 = x[i], y0 = y[i];
                            x[i] = r * __builtin_fmaf(x0, cx[i], -(y0 * sy[i]));
                            y[i] = r * __builtin_fmaf(y0, cy[i], x0 * sx[i]);
                        }
                        P::write(raw[u], x, y);
                    }
                    if (me.active && (g + u) * G::ROWS + me.row < heads) to.store(raw[u], (long long)(g + u) * G::ROWS * to_head);
                }
            }
        }
    }
#endif
}

// Backward.  A workgroup has one of the two tensors: its wavefronts take every so manieth token (or part of one) and keep the sums of
// their columns' weight gradients in registers; the workgroup's are added in the LDS, in a fixed order, and written to its row of
// partial sums.
constexpr int kRopeBwdBatch = ROPE_BBATCH;
template <typename T, int D, bool INTER> __global__ void __launch_bounds__(256, ROPE_BOCC) rope_bwd_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePairs<T, INTER>;
    __shared__ __attribute__((aligned(16))) float table_sh[4][2 * (D / 2)], weight_sh[2][D / 2];
    __shared__ float sums_sh[4][D];
    const int lane = threadIdx.x & 63, wave_in = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_k = (int)blockIdx.x >= a.bwd_groups[0];
    const int groups = is_k ? a.bwd_groups[1] : a.bwd_groups[0], wave = (blockIdx.x - (is_k ? a.bwd_groups[0] : 0)) * 4 + wave_in;
    const int heads = is_k ? a.heads[1] : a.heads[0], spans = is_k ? a.bwd_spans[1] : a.bwd_spans[0], part = is_k ? a.bwd_heads[1] : a.bwd_heads[0];
    const Divisor by_spans = is_k ? a.bwd_by_spans[1] : a.bwd_by_spans[0];
    const RopeRows in = is_k ? a.x[1] : a.x[0], out = is_k ? a.grad[1] : a.grad[0];
    const T *const grads = (const T *)(is_k ? a.dy[1] : a.dy[0]);
    const bool norm = (is_k ? a.weight[1] : a.weight[0]) != nullptr;
    const long long dy_head = (long long)a.S * D;
    const RopeLane<D, INTER> me(a.rot, lane);
    float *const table = table_sh[wave_in];
    const RopeTable<T, D, INTER, 2> pairs(a, lane, table);
    if (wave_in == 0)
#pragma unroll
        for (int e = 0; e < pairs.EACH; ++e)
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (lane + e * 64 < D / 2) weight_sh[p][lane + e * 64] = is_k ? pairs.w[e][1][p] : pairs.w[e][0][p];
    __syncthreads();
    float wx[8], wy[8], dwx[8], dwy[8];
    rope_table_read(wx, weight_sh[0] + me.first);
    rope_table_read(wy, weight_sh[1] + me.first);
#pragma unroll
    for (int i = 0; i < 8; ++i) dwx[i] = dwy[i] = 0.f;
    const int items = a.B * a.S * spans;
    for (int item = wave; item < items; item += groups * 4) {
        const int token = rope_divide(item, by_spans), b = rope_divide(token, a.by_s), s = token - b * a.S;
        const int first = (item - token * spans) * part, last = first + part < heads ? first + part : heads;
        const RopePointers<T> dy(grads + ((long long)b * heads * a.S + s) * D, me.row * dy_head, me.col);
        const RopePointers<T> from((const T *)in.data + (long long)b * in.batch + (long long)s * in.row, me.row * in.head, me.col);
        const RopePointers<T> to((const T *)out.data + (long long)b * out.batch + (long long)s * out.row, me.row * out.head, me.col);
        pairs.fill(a, b, s);
        float c[8], sn[8];
        rope_table_read(c, table + me.first);
        rope_table_read(sn, table + D / 2 + me.first);
        for (int h0 = first; h0 < last; h0 += kRopeBwdBatch * G::ROWS) {
            rope_u32x4 draw[kRopeBwdBatch][2], raw[kRopeBwdBatch][2];
#pragma unroll
            for (int u = 0; u < kRopeBwdBatch; ++u) {
                const int h1 = h0 + u * G::ROWS;
                if (u > 0 && h1 >= last) continue;
                dy.load(draw[u], h1 * dy_head, h1 + me.row < last);
                from.load(raw[u], h1 * in.head, norm && h1 + me.row < last);
            }
#pragma unroll
            for (int u = 0; u < kRopeBwdBatch; ++u) {
                const int h1 = h0 + u * G::ROWS;
                if (u > 0 && h1 >= last) continue;
                const bool mine = me.active && h1 + me.row < last;
                float g[8], h[8];
                P::read(g, h, draw[u]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {              // rotated back
                    const float g0 = g[i];
                    g[i] = __builtin_fmaf(g0, c[i], h[i] * sn[i]);
                    h[i] = __builtin_fmaf(h[i], c[i], -(g0 * sn[i]));
                }
                if (norm) {
                    float x[8], y[8], dot = 0.f;
                    P::read(x, y, raw[u]);
                    const float r = me.scale(x, y, a.eps);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float gx = g[i] * x[i], hy = h[i] * y[i];
                        if (mine) {                // (rows and columns that are not this lane's add nothing)
                            dwx[i] = __builtin_fmaf(r, gx, dwx[i]);
                            dwy[i] = __builtin_fmaf(r, hy, dwy[i]);
                        }
                        dot = __builtin_fmaf(wx[i], gx, __builtin_fmaf(wy[i], hy, dot));
                    }
                    const float back = r * r * (me.row_sum(dot) * (1.f / D));
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        g[i] = r * __builtin_fmaf(-back, x[i], wx[i] * g[i]);
                        h[i] = r * __builtin_fmaf(-back, y[i], wy[i] * h[i]);
                    }
                }
                P::write(draw[u], g, h);
                if (mine) to.store(draw[u], h1 * out.head);
            }
        }
    }
    if (!norm) return;
    // over the wavefront's rows (lanes a row's length apart), then over the wavefronts
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x = p == 0 ? dwx[i] : dwy[i];
#pragma unroll
            for (int d = G::LANES; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
            if (me.row == 0 && me.active) sums_sh[wave_in][me.column(me.col[0], me.col[1], p, i)] = x;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += 256)
        a.partial[(size_t)blockIdx.x * D + i] = (sums_sh[0][i] + sums_sh[1][i]) + (sums_sh[2][i] + sums_sh[3][i]);
#endif
}

// The weights' gradients: a tensor's rows of partial sums added up, one workgroup per four columns (grid.y: q, k).
template <typename T> __global__ void __launch_bounds__(256)
rope_bwd_sum_kernel(const float *__restrict__ partial, int groups_q, int groups_k, int D, void *dq, void *dk, int weight32)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef float f4 __attribute__((ext_vector_type(4)));
    __shared__ f4 sums_sh[4];
    void *const to = blockIdx.y == 0 ? dq : dk;
    if (to == nullptr) return;
    const int first = blockIdx.y == 0 ? 0 : groups_q, last = blockIdx.y == 0 ? groups_q : groups_q + groups_k;
    f4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int r = first + threadIdx.x; r < last; r += 256) sum += *(const f4 *)(partial + (size_t)r * D + blockIdx.x * 4);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum[c] += __shfl_xor(sum[c], d, 64);
    if ((threadIdx.x & 63) == 0) sums_sh[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x >= 4) return;
    const float x = (sums_sh[0][threadIdx.x] + sums_sh[1][threadIdx.x]) + (sums_sh[2][threadIdx.x] + sums_sh[3][threadIdx.x]);
    const int col = blockIdx.x * 4 + threadIdx.x;
    if (weight32) ((float *)to)[col] = x;
    else ((T *)to)[col] = (T)x;
#endif
}

template <typename T, int D> int launch_rope_dim(bool cache, const RopeArgs &a0)
{
    RopeArgs a = a0;
    using G = RopeGeom<D>;
    int units = 0;
    for (int i = 0; i < (cache ? 3 : 2); ++i) units += (a.heads[i] + G::ROWS - 1) / G::ROWS;
    const long long tokens = (long long)a.B * a.S;
    // a wavefront for all heads of a token, or several where the tokens are few
    const int most = kRopeWaves;
    const long long want = most / tokens;
    a.units_per_span = want >= units ? 1 : want <= 1 ? units : (int)((units + want - 1) / want);
    a.spans = (units + a.units_per_span - 1) / a.units_per_span;
    a.by_spans = divisor((uint32_t)a.spans);
    const long long items = tokens * a.spans;
    const unsigned grid = (unsigned)(((items < most ? items : most) + 3) / 4);
    a.waves = (int)grid * 4;
    const auto kernel = cache ? (a.interleaved ? rope_kernel<T, D, true, true> : rope_kernel<T, D, true, false>)
                              : (a.interleaved ? rope_kernel<T, D, false, true> : rope_kernel<T, D, false, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, a.stream, a);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_rope_bwd_dim(const RopeArgs &a0, void *dqw, void *dkw)
{
    RopeArgs a = a0;
    using G = RopeGeom<D>;
    // A wavefront for all heads of a token, or several where the tokens are few; and workgroups for as many, up to what the GPU holds, which
    // the tensors share as they share the rows.
    const long long tokens = (long long)a.B * a.S;
    long long wanted[2];
    int units[2];
    for (int i = 0; i < 2; ++i) {
        units[i] = (a.heads[i] + G::ROWS - 1) / G::ROWS;
        long long spans = tokens > 0 ? kRopeBwdMost * 2 / tokens : 1;
        spans = spans < 1 ? 1 : spans > units[i] ? (units[i] > 0 ? units[i] : 1) : spans;
        const int per = (int)((units[i] + spans - 1) / spans);
        a.bwd_heads[i] = per * G::ROWS;
        a.bwd_spans[i] = per > 0 ? (units[i] + per - 1) / per : 0;
        a.bwd_by_spans[i] = divisor((uint32_t)(a.bwd_spans[i] > 0 ? a.bwd_spans[i] : 1));
        wanted[i] = (tokens * a.bwd_spans[i] + 3) / 4;
    }
    if (wanted[0] + wanted[1] <= kRopeBwdMost) {
        a.bwd_groups[0] = (int)wanted[0];
        a.bwd_groups[1] = (int)wanted[1];
    } else {
        long long share = (long long)kRopeBwdMost * units[0] / (units[0] + units[1]);
        if (share < 1 && units[0] > 0) share = 1;
        if (share >= kRopeBwdMost && units[1] > 0) share = kRopeBwdMost - 1;
        a.bwd_groups[0] = (int)(share < wanted[0] ? share : wanted[0]);
        a.bwd_groups[1] = (int)(kRopeBwdMost - share < wanted[1] ? kRopeBwdMost - share : wanted[1]);
    }
    const int groups = a.bwd_groups[0] + a.bwd_groups[1];
    int err = 0;
    if (groups > 0) {
        hipLaunchKernelGGL((a.interleaved ? rope_bwd_kernel<T, D, true> : rope_bwd_kernel<T, D, false>), dim3((unsigned)groups), dim3(256), 0, a.stream, a);
        err = (int)hipGetLastError();
    }
    if (err != 0 || (dqw == nullptr && dkw == nullptr)) return err;
    hipLaunchKernelGGL((rope_bwd_sum_kernel<T>), dim3(D / 4, 2), dim3(256), 0, a.stream, (const float *)a.partial, a.bwd_groups[0], a.bwd_groups[1], D, dqw,
                       dkw, a.weight32);
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
