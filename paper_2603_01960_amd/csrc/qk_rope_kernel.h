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
//     crosses lanes.  D / 16 lanes make a row;
//   * a wavefront stays with one token and goes through its heads, so that the angles are computed once for all of them:
//     in 64 bits up to whole turns (a position of 2^31 has no fraction left in 32), then sine and cosine of the rest;
//   * the next row group's loads are on their way while one is worked on.
// Kernels, us and TB/s of what they have to read and write, on three sets of tensors in turn (in brackets a copy of as many bytes, likewise):
// forward B=2 S=8192 H=32+8 D=128 BF16 64, 5.3 (5.3); B=64 S=197 H=12+12 D=64 FP16 15, 5.0 (6.7); into a cache B=4 S=512 H=32+8 D=128 BF16
// 10, 4.9 (6.3), one token of it 3.2; backward of the first 90, 5.6 (5.3), and 4.6 for the weights' sums, B=4 S=2048 H=16+4 D=160 FP16 35, 4.5
// (5.1).
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
    Divisor by_rows, by_s;
    // of q, and of k (and v): parts of a token that a wavefront each takes, heads of a part; backward: workgroups (those of q first)
    int spans[2], part[2];
    Divisor by_spans[2];
    int groups[2];
    int waves;                                     // forward: wavefronts of the launch
    float *partial;                                // backward: [workgroups][D], sums of a weight's gradient
    hipStream_t stream;
};

template <int D> struct RopeGeom {
    static constexpr int LANES = D / 16;           // lanes of a row
    static constexpr int ROWS = 64 / LANES;        // rows of a wavefront at a time: 16, 10, 8 and 6 (the last 4 lanes are idle at D = 96, 160)
};

int launch_rope_f16(int D, bool cache, const RopeArgs &a);
int launch_rope_bf16(int D, bool cache, const RopeArgs &a);
int launch_rope_bwd_f16(int D, const RopeArgs &a);
int launch_rope_bwd_bf16(int D, const RopeArgs &a);

// Wavefronts per SIMD that the kernels are built for, and launches of no more: they are persistent.  One row group at a time and one
// on its way needs few registers.  (us, forward at 4 / 5 / 6 wavefronts: B=2 S=8192 H=32+8 D=128 BF16 64.1 / 63.7 / 63.5, B=64 S=197
// H=12+12 D=64 FP16 16.4 / 15.8 / 16.2, B=4 S=512 of the first into a cache 9.9 at each; backward at 2 / 3 / 4: 92.4 / 97.7 / 96.8, B=4 S=2048
// H=16+4 D=160 FP16 37.5 / 37.9 / 44.5: more rows of partial sums, and no registers to spare.  Two row groups at a time, at an earlier step:
// forward 63.5 -> 65.1, backward 93.0 -> 98.8.)
constexpr int kRopeWaves = 5 * 1024, kRopeBwdMost = 2 * 256;   // wavefronts; workgroups, each of which leaves a row of partial sums

#if defined(__HIP_DEVICE_COMPILE__)
typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int rope_divide(int n, const Divisor &d) { return (int)(__umulhi(2u * (unsigned)n, d.mul) >> d.shift); }

// x + x of the lane that `ctrl` pairs it with
template <int CTRL> __device__ __forceinline__ float rope_dpp_add(float x)
{
    const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
    return x + __builtin_bit_cast(float, y);
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
    bool active;                                   // the lane has a row
    bool turns;                                    // its columns are rotated: all of them or none
    int first;                                     // its first pair, of the D / 2 that the lanes of a row have
    int other[4];                                  // D = 96, 160: lanes that row_sum takes (times 4)
    __device__ __forceinline__ RopeLane(int rot, int lane)
    {
        using G = RopeGeom<D>;
        row = lane / G::LANES;
        const int j = lane % G::LANES;
        active = row < G::ROWS;
        turns = j < rot / 16;
        first = j * 8;
        constexpr int H = G::LANES / 2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int distance = i == 0 ? H : i == 1 ? 1 : i == 2 ? 2 : H - 1;
            other[i] = (lane - j + (j + distance) % G::LANES) * 4;
        }
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
    static __device__ __forceinline__ float from(float x, int lane4) { return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(lane4, __builtin_bit_cast(int, x))); }
    // The sum over the lanes of a row, in each of them.  A row of 4 or 8 lanes: DPP steps.  Of 6 or 10: the two lanes half a row apart, then
    // H = 3 or 5 such pairs, one after another (the lanes add them in different orders, which may differ in the last bit).
    __device__ __forceinline__ float row_sum(float x) const
    {
        if constexpr (RopeGeom<D>::LANES == 4 || RopeGeom<D>::LANES == 8) {
            x = rope_dpp_add<0xB1>(x);             // lane ^ 1
            x = rope_dpp_add<0x4E>(x);             // lane ^ 2
            if constexpr (RopeGeom<D>::LANES == 8) x = rope_dpp_add<0x141>(x);       // mirrored within 8 lanes
            return x;
        } else {
            const float pair = x + from(x, other[0]);
            const float two = pair + from(pair, other[1]);
            if constexpr (RopeGeom<D>::LANES == 6) return two + from(pair, other[2]);
            const float four = two + from(two, other[2]);
            return four + from(pair, other[3]);
        }
    }
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
// (a wavefront's own part, whose accesses are in order).  Tables of D / 2 values: cosine and sine of each pair, or (FOLD) both times the
// weights of its two columns.
template <typename T, int D, bool INTER> struct RopeTable {
    static constexpr int EACH = (D / 2 + 63) / 64;       // pairs of a lane
    double step[EACH];                             // turns per position
    float freq[EACH];
    int which[EACH];                               // its axis
    long long axis[EACH];                          // where that one's positions begin
    int column[EACH][2];
    float *mine;
    // Requests what the lane needs of the arguments' arrays.  Nothing here waits for a load, nor does request: their latencies, and in the
    // forward kernel those of the first positions and rows, pass at the same time.  (One after another: B=4 S=512 H=32+8 D=128 BF16 into a cache
    // 10.8 us instead of 9.9, B=4 S=2048 H=16+4 D=160 FP16 backward 37.7 / 37.4.  The backward's first rows requested before the
    // others have arrived: 39.9.)
    __device__ __forceinline__ RopeTable(const RopeArgs &a, int lane, float *wave_sh) : mine(wave_sh + lane)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int slot = lane + e * 64 < D / 2 ? lane + e * 64 : D / 2 - 1, j = slot / 8, i = slot % 8;
            const int c0 = RopeLane<D, INTER>::columns(a.rot, j, 0), c1 = RopeLane<D, INTER>::columns(a.rot, j, 1);
            const int pair = !INTER ? c0 + i : i < 4 ? c0 / 2 + i : c1 / 2 + i - 4;
            const bool turns = j < a.rot / 16;
            freq[e] = 0.f;
            if (turns) freq[e] = a.inv_freq[pair];
            which[e] = 0;
            if (a.axes != nullptr && turns) which[e] = a.axes[pair];
#pragma unroll
            for (int p = 0; p < 2; ++p) column[e][p] = RopeLane<D, INTER>::column(c0, c1, p, i);
        }
    }
    // Where the positions are; the frequencies.
    __device__ __forceinline__ void locate(const RopeArgs &a)
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            axis[e] = 0;
            if (a.axes == nullptr) continue;
            asm volatile("" : "+v"(which[e]));
            axis[e] = (which[e] < 0 ? 0 : which[e] < a.n_axes ? which[e] : a.n_axes - 1) * a.pos_axis;
        }
    }
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            asm volatile("" : "+v"(freq[e]));          // (not where it is loaded)
            step[e] = (double)freq[e] * 0.15915494309189533577;
            asm volatile("" : "+v"(step[e]));          // (nor in the loop, which would wait for its own loads too)
        }
    }
    // whether the lane has an e-th pair
    __device__ __forceinline__ bool has(int e) const { return (D / 2) % 64 == 0 || (int)(threadIdx.x & 63) + e * 64 < D / 2; }
    __device__ __forceinline__ void positions(const RopeArgs &a, int b, int s, int (&to)[EACH]) const
    {
        const int *at = a.positions + ((long long)b * a.pos_batch + s);
#pragma unroll
        for (int e = 0; e < EACH; ++e) to[e] = a.rot > 0 ? at[axis[e]] : 0;
    }
    template <bool FOLD> __device__ __forceinline__ void fill(const int (&position)[EACH], const float (&w)[EACH][2]) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const double x = (double)position[e] * step[e];
            // v_sin and v_cos take whole turns: off by at most 2^-22.9 over one
            const float t = (float)(x - __builtin_rint(x)), c = __builtin_amdgcn_cosf(t), sn = __builtin_amdgcn_sinf(t);
            if (!has(e)) continue;
            float *to = mine + e * 64;
            if constexpr (FOLD) {
                to[0] = w[e][0] * c;
                to[D / 2] = w[e][0] * sn;
                to[2 * (D / 2)] = w[e][1] * c;
                to[3 * (D / 2)] = w[e][1] * sn;
            } else {
                to[0] = c;
                to[D / 2] = sn;
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    // The weights of its pairs' columns: the words that hold them (16-bit ones two by two, whatever the type one load), and the values (1
    // without a norm).
    __device__ __forceinline__ void request(const void *at, int weight32, uint32_t (&words)[EACH][2]) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
#pragma unroll
            for (int p = 0; p < 2; ++p) words[e][p] = 0;
        if (at == nullptr) return;
#pragma unroll
        for (int e = 0; e < EACH; ++e)
#pragma unroll
            for (int p = 0; p < 2; ++p) words[e][p] = ((const uint32_t *)at)[weight32 ? column[e][p] : column[e][p] >> 1];
    }
    __device__ __forceinline__ void weights(const void *at, int weight32, uint32_t (&words)[EACH][2], float (&w)[EACH][2]) const
    {
#pragma unroll
        for (int e = 0; e < EACH; ++e)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                asm volatile("" : "+v"(words[e][p]));
                const float own = (float)__builtin_bit_cast(T, (uint16_t)(words[e][p] >> (column[e][p] & 1) * 16));
                w[e][p] = at == nullptr ? 1.f : weight32 ? __builtin_bit_cast(float, words[e][p]) : own;
                asm volatile("" : "+v"(w[e][p]));
            }
    }
};
__device__ __forceinline__ void rope_table_read(float (&x)[8], const float *at)
{
    typedef float f4 __attribute__((ext_vector_type(4)));
    const f4 lo = *(const f4 *)at, hi = *(const f4 *)(at + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < 4 ? lo[i & 3] : hi[i & 3];
}

// A lane's two pieces of a row group; lanes without one keep what is in the registers, which nothing uses.  STREAM: past the caches.
template <bool STREAM, typename T> __device__ __forceinline__ void rope_load(rope_u32x4 (&raw)[2], const T *at, const int (&col)[2], bool mine)
{
    asm("" : "=v"(raw[0]), "=v"(raw[1]));
    if (!mine) return;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const rope_u32x4 *from = (const rope_u32x4 *)(at + col[p]);
        if constexpr (STREAM) raw[p] = __builtin_nontemporal_load(from);
        else raw[p] = *from;
    }
}
template <bool STREAM, typename T> __device__ __forceinline__ void rope_store(const rope_u32x4 (&raw)[2], T *at, const int (&col)[2])
{
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        rope_u32x4 *to = (rope_u32x4 *)(at + col[p]);
        if constexpr (STREAM) __builtin_nontemporal_store(raw[p], to);
        else *to = raw[p];
    }
}
#endif

// An item is a tensor's heads of one token, or some of them; first those of q, then of k, then of v.  While one row group (of
// RopeGeom::ROWS heads) is worked on, the next one's loads are on their way, the next item's first one among them.
template <typename T, int D, bool CACHE, bool INTER, bool STREAM> __global__ void __launch_bounds__(256, 5) rope_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePairs<T, INTER>;
    using Table = RopeTable<T, D, INTER>;
    __shared__ __attribute__((aligned(16))) float table_sh[4][4 * (D / 2)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int tokens = a.B * a.S;
    const int items_q = tokens * a.spans[0], items_qk = items_q + tokens * a.spans[1], items = items_qk + (CACHE ? tokens * a.spans[1] : 0);
    if (wave >= items) return;
    const RopeLane<D, INTER> me(a.rot, lane);
    float *const table = table_sh[threadIdx.x >> 6];

    struct Item { int which, b, s, token, first, last; };      // (first and last head)
    auto item_at = [&](int i) __attribute__((always_inline)) {
        Item x;
        x.which = i < items_q ? 0 : !CACHE || i < items_qk ? 1 : 2;
        const int n = i - (x.which == 0 ? 0 : x.which == 1 ? items_q : items_qk);
        x.token = x.which == 0 ? rope_divide(n, a.by_spans[0]) : rope_divide(n, a.by_spans[1]);
        const int part = x.which == 0 ? a.part[0] : a.part[1], heads = x.which == 0 ? a.heads[0] : a.heads[1];
        x.first = (n - x.token * (x.which == 0 ? a.spans[0] : a.spans[1])) * part;
        x.last = x.first + part < heads ? x.first + part : heads;
        x.b = rope_divide(x.token, a.by_s);
        x.s = x.token - x.b * a.S;
        return x;
    };
    auto load = [&](const Item &x, int h0, rope_u32x4 (&raw)[2]) __attribute__((always_inline)) {
        const RopeRows in = x.which == 0 ? a.x[0] : !CACHE || x.which == 1 ? a.x[1] : a.x[2];
        const T *from = (const T *)in.data + (long long)x.b * in.batch + (long long)x.s * in.row + h0 * in.head;
        rope_load<STREAM>(raw, from + me.row * in.head, me.col, me.active && h0 + me.row < x.last);
    };

    // (two sets of registers that take turns: a copy from one to the other would wait for the loads)
    struct Rows { rope_u32x4 raw[2]; int position[Table::EACH]; };
    Item cur = item_at(wave);
    int next_item = wave + a.waves, h0 = cur.first;
    bool fresh = true;
    Rows one, two;
    Table pairs(a, lane, table);
    uint32_t words[2][Table::EACH][2];
    float weights[2][Table::EACH][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) pairs.request(a.weight[i], a.weight32, words[i]);
    pairs.locate(a);
    pairs.positions(a, cur.b, cur.s, one.position);
    load(cur, h0, one.raw);
    pairs.finish();
#pragma unroll
    for (int i = 0; i < 2; ++i) pairs.weights(a.weight[i], a.weight32, words[i], weights[i]);
    // works on `now` and requests the next row group into `then`; false after the last
    auto turn = [&](Rows &now, Rows &then) __attribute__((always_inline)) {
        Item next = cur;
        int next_h0 = h0 + G::ROWS;
        const bool steps = next_h0 >= cur.last, more = !steps || next_item < items;
        if (steps && more) {
            next = item_at(next_item);
            next_h0 = next.first;
            next_item += a.waves;
            pairs.positions(a, next.b, next.s, then.position);
        }
        if (more) load(next, next_h0, then.raw);
        if (fresh && (!CACHE || cur.which < 2)) {
            if (cur.which == 0) pairs.template fill<true>(now.position, weights[0]);
            else pairs.template fill<true>(now.position, weights[1]);
        }
        const int heads = cur.which == 0 ? a.heads[0] : a.heads[1];
        T *to;
        long long to_head = (long long)a.S * D;
        bool written = true;
        if (CACHE && cur.which > 0) {
            const int slot = __builtin_amdgcn_readfirstlane(a.slots[cur.token]);
            written = slot >= 0 && slot < a.cache_rows;
            const int page = rope_divide(written ? slot : 0, a.by_rows);
            to_head = (long long)a.block_rows * D;
            to = (T *)(cur.which == 1 ? a.out[1] : a.out[2]) + ((long long)page * heads * a.block_rows + (slot - page * a.block_rows)) * D;
        } else {
            to = (T *)(cur.which == 0 ? a.out[0] : a.out[1]) + ((long long)cur.b * heads * a.S + cur.s) * D;
        }
        to += h0 * to_head;
        // rows are x_a (w_a cos), x_b (w_b sin) and so on, times the row's 1 / root
        float cx[8], sx[8], cy[8], sy[8];
        const bool norm = (cur.which == 0 ? a.weight[0] : a.weight[1]) != nullptr, copy = CACHE && cur.which == 2;
        if (!copy) {
            const float *at = table + me.first;
            rope_table_read(cx, at);
            rope_table_read(sx, at + D / 2);
            rope_table_read(cy, at + 2 * (D / 2));
            rope_table_read(sy, at + 3 * (D / 2));
        }
        if (!copy) {
            float x[8], y[8], r = 1.f;
            P::read(x, y, now.raw);
            if (norm) r = me.scale(x, y, a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x0 = x[i], y0 = y[i];
                // (a sine of 0 would do for finite values only: columns that are not rotated have nothing of each other's)
                const float from_y = me.turns ? y0 * sy[i] : 0.f, from_x = me.turns ? x0 * sx[i] : 0.f;
                x[i] = r * __builtin_fmaf(x0, cx[i], -from_y);
                y[i] = r * __builtin_fmaf(y0, cy[i], from_x);
            }
            P::write(now.raw, x, y);
        }
        if (written && me.active && h0 + me.row < cur.last) rope_store<STREAM>(now.raw, to + me.row * to_head, me.col);
        fresh = steps;
        cur = next;
        h0 = next_h0;
        return more;
    };
    while (turn(one, two) && turn(two, one)) {}
#endif
}

// Backward.  A workgroup has one of the two tensors: its wavefronts take every so manieth token (or part of one) and keep the sums of
// their columns' weight gradients in registers; the workgroup's are added in the LDS, in a fixed order, and written to its row of
// partial sums.  The loads run ahead as in the forward kernel.
template <typename T, int D, bool INTER, bool STREAM> __global__ void __launch_bounds__(256, 2) rope_bwd_kernel(RopeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using G = RopeGeom<D>;
    using P = RopePairs<T, INTER>;
    using Table = RopeTable<T, D, INTER>;
    __shared__ __attribute__((aligned(16))) float table_sh[4][2 * (D / 2)], weight_sh[2][D / 2];
    __shared__ float sums_sh[4 * G::ROWS][D];
    const int lane = threadIdx.x & 63, wave_in = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_k = (int)blockIdx.x >= a.groups[0];
    const int groups = is_k ? a.groups[1] : a.groups[0], wave = (blockIdx.x - (is_k ? a.groups[0] : 0)) * 4 + wave_in;
    const int heads = is_k ? a.heads[1] : a.heads[0], spans = is_k ? a.spans[1] : a.spans[0], part = is_k ? a.part[1] : a.part[0];
    const Divisor by_spans = is_k ? a.by_spans[1] : a.by_spans[0];
    const RopeRows in = is_k ? a.x[1] : a.x[0], out = is_k ? a.grad[1] : a.grad[0];
    const T *const grads = (const T *)(is_k ? a.dy[1] : a.dy[0]);
    const void *const weight = is_k ? a.weight[1] : a.weight[0];
    const bool norm = weight != nullptr;
    const long long dy_head = (long long)a.S * D;
    const RopeLane<D, INTER> me(a.rot, lane);
    float *const table = table_sh[wave_in];
    const int items = a.B * a.S * spans;

    struct Item { int b, s, first, last; };
    auto item_at = [&](int i) __attribute__((always_inline)) {
        Item x;
        const int token = rope_divide(i, by_spans);
        x.b = rope_divide(token, a.by_s);
        x.s = token - x.b * a.S;
        x.first = (i - token * spans) * part;
        x.last = x.first + part < heads ? x.first + part : heads;
        return x;
    };
    auto load = [&](const Item &x, int h0, rope_u32x4 (&draw)[2], rope_u32x4 (&raw)[2]) __attribute__((always_inline)) {
        const T *dy = grads + ((long long)x.b * heads * a.S + x.s) * D + h0 * dy_head;
        const T *from = (const T *)in.data + (long long)x.b * in.batch + (long long)x.s * in.row + h0 * in.head;
        const bool mine = me.active && h0 + me.row < x.last;
        rope_load<STREAM>(draw, dy + me.row * dy_head, me.col, mine);
        rope_load<STREAM>(raw, from + me.row * in.head, me.col, norm && mine);
    };
    struct Rows { rope_u32x4 draw[2], raw[2]; int position[Table::EACH]; };
    Item cur{};
    int next_item = wave + groups * 4, h0 = 0;
    bool fresh = true;
    Rows one, two;
    Table pairs(a, lane, table);
    uint32_t words[Table::EACH][2];
    float w[Table::EACH][2];
    pairs.request(weight, a.weight32, words);
    pairs.locate(a);
    pairs.finish();
    pairs.weights(weight, a.weight32, words, w);
    if (wave_in == 0)
#pragma unroll
        for (int e = 0; e < Table::EACH; ++e)
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (pairs.has(e)) weight_sh[p][lane + e * 64] = w[e][p];
    __syncthreads();
    float wx[8], wy[8], dwx[8], dwy[8];
    rope_table_read(wx, weight_sh[0] + me.first);
    rope_table_read(wy, weight_sh[1] + me.first);
#pragma unroll
    for (int i = 0; i < 8; ++i) dwx[i] = dwy[i] = 0.f;
    auto turn = [&](Rows &now, Rows &then) __attribute__((always_inline)) {
        Item next = cur;
        int next_h0 = h0 + G::ROWS;
        const bool steps = next_h0 >= cur.last, more = !steps || next_item < items;
        if (steps && more) {
            next = item_at(next_item);
            next_h0 = next.first;
            next_item += groups * 4;
            pairs.positions(a, next.b, next.s, then.position);
        }
        if (more) load(next, next_h0, then.draw, then.raw);
        if (fresh) pairs.template fill<false>(now.position, w);
        float c[8], sn[8];
        rope_table_read(c, table + me.first);
        rope_table_read(sn, table + D / 2 + me.first);
        T *to = (T *)out.data + (long long)cur.b * out.batch + (long long)cur.s * out.row + h0 * out.head;
        const bool mine = me.active && h0 + me.row < cur.last;
        float g[8], h[8];
        P::read(g, h, now.draw);
#pragma unroll
        for (int i = 0; i < 8; ++i) {                  // rotated back
            const float g0 = g[i], from_h = me.turns ? h[i] * sn[i] : 0.f, from_g = me.turns ? g0 * sn[i] : 0.f;
            g[i] = __builtin_fmaf(g0, c[i], from_h);
            h[i] = __builtin_fmaf(h[i], c[i], -from_g);
        }
        if (norm) {
            float x[8], y[8], dot = 0.f;
            P::read(x, y, now.raw);
            const float r = me.scale(x, y, a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gx = g[i] * x[i], hy = h[i] * y[i];
                if (mine) {                    // (rows and columns that are not this lane's add nothing)
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
        P::write(now.draw, g, h);
        if (mine) rope_store<STREAM>(now.draw, to + me.row * out.head, me.col);
        fresh = steps;
        cur = next;
        h0 = next_h0;
        return more;
    };
    if (wave < items) {
        cur = item_at(wave);
        h0 = cur.first;
        pairs.positions(a, cur.b, cur.s, one.position);
        load(cur, h0, one.draw, one.raw);
        while (turn(one, two) && turn(two, one)) {}
    }
    if (!norm) return;
    // over the rows of all wavefronts
    if (me.active)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sums_sh[wave_in * G::ROWS + me.row][me.column(me.col[0], me.col[1], 0, i)] = dwx[i];
            sums_sh[wave_in * G::ROWS + me.row][me.column(me.col[0], me.col[1], 1, i)] = dwy[i];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += 256) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 4 * G::ROWS; ++r) sum += sums_sh[r][i];
        a.partial[(size_t)blockIdx.x * D + i] = sum;
    }
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

// Whether rows go past the caches: where a call's own bytes are more than the 256 MB of the last level, so that they would only push
// each other out (and the rest).
inline bool rope_streams(long long bytes) { return bytes > (256ll << 20); }

// A wavefront for all heads of a token's q (or k, or v), or several where the tokens are few: up to `most` wavefronts in all.
template <int D> void rope_spans(RopeArgs &a, long long tokens, int most)
{
    using G = RopeGeom<D>;
    for (int i = 0; i < 2; ++i) {
        const int units = (a.heads[i] + G::ROWS - 1) / G::ROWS;
        long long spans = tokens > 0 ? most / tokens : 1;
        spans = spans < 1 ? 1 : spans > units ? (units > 0 ? units : 1) : spans;
        const int per = (int)((units + spans - 1) / spans);
        a.part[i] = per * G::ROWS;
        a.spans[i] = per > 0 ? (units + per - 1) / per : 0;
        a.by_spans[i] = divisor((uint32_t)(a.spans[i] > 0 ? a.spans[i] : 1));
    }
}

template <typename T, int D> int launch_rope_dim(bool cache, const RopeArgs &a0)
{
    RopeArgs a = a0;
    const long long tokens = (long long)a.B * a.S;
    rope_spans<D>(a, tokens, kRopeWaves);
    const long long items = tokens * (a.spans[0] + (cache ? 2 : 1) * a.spans[1]);
    const unsigned grid = (unsigned)(((items < kRopeWaves ? items : kRopeWaves) + 3) / 4);
    a.waves = (int)grid * 4;
    const bool stream = rope_streams(2 * tokens * (a.heads[0] + a.heads[1]) * D * (long long)sizeof(T));
    const auto kernel = cache ? (a.interleaved ? rope_kernel<T, D, true, true, false> : rope_kernel<T, D, true, false, false>)
                      : stream ? (a.interleaved ? rope_kernel<T, D, false, true, true> : rope_kernel<T, D, false, false, true>)
                               : (a.interleaved ? rope_kernel<T, D, false, true, false> : rope_kernel<T, D, false, false, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, a.stream, a);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_rope_bwd_dim(const RopeArgs &a0, void *dqw, void *dkw)
{
    RopeArgs a = a0;
    using G = RopeGeom<D>;
    // Workgroups for as many wavefronts, up to what the GPU holds, which the tensors share as they share the rows.
    const long long tokens = (long long)a.B * a.S;
    rope_spans<D>(a, tokens, kRopeBwdMost * 4);
    const long long wanted[2] = {(tokens * a.spans[0] + 3) / 4, (tokens * a.spans[1] + 3) / 4};
    const int units[2] = {(a.heads[0] + G::ROWS - 1) / G::ROWS, (a.heads[1] + G::ROWS - 1) / G::ROWS};
    if (wanted[0] + wanted[1] <= kRopeBwdMost) {
        a.groups[0] = (int)wanted[0];
        a.groups[1] = (int)wanted[1];
    } else {
        long long share = (long long)kRopeBwdMost * units[0] / (units[0] + units[1]);
        if (share < 1 && units[0] > 0) share = 1;
        if (share >= kRopeBwdMost && units[1] > 0) share = kRopeBwdMost - 1;
        a.groups[0] = (int)(share < wanted[0] ? share : wanted[0]);
        a.groups[1] = (int)(kRopeBwdMost - share < wanted[1] ? kRopeBwdMost - share : wanted[1]);
    }
    const int groups = a.groups[0] + a.groups[1];
    int err = 0;
    if (groups > 0) {
        const bool stream = rope_streams(3 * tokens * (a.heads[0] + a.heads[1]) * D * (long long)sizeof(T));
        const auto kernel = stream ? (a.interleaved ? rope_bwd_kernel<T, D, true, true> : rope_bwd_kernel<T, D, false, true>)
                                   : (a.interleaved ? rope_bwd_kernel<T, D, true, false> : rope_bwd_kernel<T, D, false, false>);
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(256), 0, a.stream, a);
        err = (int)hipGetLastError();
    }
    if (err != 0 || (dqw == nullptr && dkw == nullptr)) return err;
    hipLaunchKernelGGL((rope_bwd_sum_kernel<T>), dim3(D / 4, 2), dim3(256), 0, a.stream, (const float *)a.partial, a.groups[0], a.groups[1], D, dqw,
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
