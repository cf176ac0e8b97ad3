// The 8-bit cache: writing a step's tokens to it, reading rows back, and the C-ABI of these and of attention over it (kernels of the
// latter in sdpa_cache8_decode_kernel.h).  See include/tiled_sdpa.h.
#include "tiled_sdpa.h"

#include <cmath>
#include <cstdint>
#include <limits>

#include "cache8_args.h"

namespace tsdpa {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int quotient(int n, const Divisor &d) { return (int)(__umulhi(2u * (unsigned)n, d.mul) >> d.shift); }

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (e + 127) << 23); }

// 16-bit numbers: the value of one, and the codes of four of them divided by `scale`, a power of two (|x| <= 448 * scale; one rounding).
template <typename T> struct Half;
template <> struct Half<_Float16> {
    static constexpr uint32_t INF = 0x7c00u;
    static __device__ __forceinline__ float value(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (unsigned short)bits); }
    static __device__ __forceinline__ uint32_t codes(uint32_t lo, uint32_t hi, float scale)
    {
        typedef _Float16 pair __attribute__((ext_vector_type(2)));
        typedef short out __attribute__((ext_vector_type(2)));
        const out a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(out{0, 0}, __builtin_bit_cast(pair, lo), scale, false);
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(a, __builtin_bit_cast(pair, hi), scale, true));
    }
};
template <> struct Half<__bf16> {
    static constexpr uint32_t INF = 0x7f80u;
    static __device__ __forceinline__ float value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
    static __device__ __forceinline__ uint32_t codes(uint32_t lo, uint32_t hi, float scale)
    {
        typedef __bf16 pair __attribute__((ext_vector_type(2)));
        typedef short out __attribute__((ext_vector_type(2)));
        const out a = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(out{0, 0}, __builtin_bit_cast(pair, lo), scale, false);
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(a, __builtin_bit_cast(pair, hi), scale, true));
    }
};

// The least exponent E with which `largest` (not negative) is at most the largest code, 448 = 1.75 * 2^8, times 2^E.
__device__ __forceinline__ int exponent_for(float largest)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, largest);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < -kScaleMost ? -kScaleMost : (e < kScaleMost ? e : kScaleMost);
}

// One wavefront: the new rows of one block of 32 rows of one head of K or V, a block being what shares a scale.  It holds them in registers
// between their largest magnitude and their codes, so that they are read once; the block's older rows are read only if the scale grows.
//
// Bound by memory where there is much to write (4 entries of up to 2048 tokens, 8 heads, D = 128, BF16: 37.8 MB in 8.5 us, a copy's rate at that size 5.0 ... 6.3
// TB/s), and else by the launch and a chain of loads, lengths, page, rows (one token: 3.3 us of the GPU, 4.4 from call to call).  One
// conversion makes two codes and divides by the scale: with it a wavefront holds its rows in 44 to 72 registers; clamping, scaling and packing value by value took
// up to 229, and is left to blocks that hold NaN, infinities or magnitudes that the largest scale does not reach.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache8_write_kernel(Cache8Args c, Cache8Rows xk, Cache8Rows xv, const int *__restrict__ kv_lens, const int *__restrict__ new_lens, int S, int capacity,
                    int windows, Divisor by_heads, Divisor by_windows, int units)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int CPR = D / 8, N = 32 * CPR / 64;  // 16-byte chunks of a row of x, and of the block per lane
    const int lane = threadIdx.x & 63;
    const int u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (u >= units) return;
    int rest = quotient(u, by_heads);
    const int h = u - rest * c.heads, tensor = rest & 1;
    rest >>= 1;
    const int b = quotient(rest, by_windows), w = rest - b * windows;
    const int now = kv_lens[b] > 0 ? kv_lens[b] : 0, next = new_lens[b] < capacity ? new_lens[b] : capacity;
    if (new_lens[b] <= 0) return;
    const int before = new_lens[b] - S;            // row of token 0
    const int lo = now > before ? now : before;
    if (lo >= next) return;
    const int block0 = lo & ~(kScaleRows - 1);
    if ((unsigned)w * kScaleRows >= (unsigned)(next - block0)) return;
    const int row0 = block0 + w * kScaleRows;
    const int first = lo > row0 ? lo : row0, end = next - row0 < kScaleRows ? next : row0 + kScaleRows;
    const int held = (now < first ? now : first) - row0;         // rows of the block that the entry has already (if > 0)
    int page = b, row = row0;
    if (c.block_table != nullptr) {
        const int shift = __builtin_ctz(c.block_rows);
        page = c.block_table[(size_t)b * c.max_blocks + (row0 >> shift)];
        if ((unsigned)page >= (unsigned)c.pages) return;          // (no memory of the cache's)
        row = row0 & (c.block_rows - 1);
    }
    const size_t head = (size_t)page * c.heads + h;
    unsigned char *codes = (unsigned char *)(tensor ? c.data[1] : c.data[0]) + (head * c.block_rows + row) * D;
    unsigned char *scale = (tensor ? c.scales[1] : c.scales[0]) + head * c.blocks + row / kScaleRows;
    const Cache8Rows x = tensor ? xv : xk;
    const T *from = (const T *)x.data + b * x.batch + h * x.head;

    u32x4 in[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int p = j * 64 + lane, r = row0 + p / CPR;
        in[j] = u32x4{0u, 0u, 0u, 0u};
        if (r >= first && r < end) in[j] = *(const u32x4 *)(from + (long long)(r - before) * x.row + p % CPR * 8);
    }
    const int was = held > 0 ? (int)*scale : 0;
    u16x2 most = {0, 0};
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t size = in[j][i] & 0x7fff7fffu;
            most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, size));
        }
    int largest = lanes_max(most[0] > most[1] ? most[0] : most[1]);
    const bool finite = largest < (int)Half<T>::INF;
    if (!finite) {                                // the largest of those that are
        int own = 0;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int size = (int)(in[j][i >> 1] >> (i & 1) * 16 & 0x7fffu);
                own = size < (int)Half<T>::INF && size > own ? size : own;
            }
        largest = lanes_max(own);
    }
    int e = exponent_for(Half<T>::value((uint32_t)largest));
    int old = was - kScaleBias;
    old = old < -kScaleMost ? -kScaleMost : (old < kScaleMost ? old : kScaleMost);
    if (held > 0 && old > e) e = old;
    if (held > 0 && e > old) {
        // the rows that are there already keep their values: code * 2^(old - e), rounded (exact but below the normal codes)
        const float move = power_of_two(old - e);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int p = j * 64 + lane;
            if (p / (D / 16) >= held) continue;
            u32x4 *at = (u32x4 *)(codes + p * 16);
            u32x4 y = *at;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], false), z = __builtin_amdgcn_cvt_pk_f32_fp8(y[i], true);
                int out = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * move, a[1] * move, 0, false);
                y[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[0] * move, z[1] * move, out, true);
            }
            *at = y;
        }
    }
    // new rows: x * 2^-e, at most 448 unless e is the largest exponent there is, to the nearest code, of two the even one
    const float down = power_of_two(e);
    if (finite && e < kScaleMost) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int p = j * 64 + lane, r = row0 + p / CPR;
            if (r < first || r >= end) continue;
            *(u32x2 *)(codes + p * 8) = u32x2{Half<T>::codes(in[j][0], in[j][1], down), Half<T>::codes(in[j][2], in[j][3], down)};
        }
    } else {
        // value by value: NaN for what is no finite number, the largest code for what is beyond it
#pragma unroll 1
        for (int j = 0; j < N; ++j) {
            const int p = j * 64 + lane, r = row0 + p / CPR;
            if (r < first || r >= end) continue;
            const T *at = from + (long long)(r - before) * x.row + p % CPR * 8;
            for (int i = 0; i < 8; ++i) {
                const uint32_t bits = ((const unsigned short *)at)[i];
                const float y = fminf(fmaxf(Half<T>::value(bits) * power_of_two(-e), -448.f), 448.f);
                codes[p * 8 + i] = (bits & 0x7fffu) < Half<T>::INF ? (unsigned char)__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false) : (unsigned char)0x7f;
            }
        }
    }
    if (lane == 0) *scale = (unsigned char)(e + kScaleBias);
#endif
}

// One thread: eight columns of one token, in one head of K and V.  Bound by memory (2 entries of 16384 rows, 8 heads, D = 128: 201 MB, a third of it
// read, in 42 us from call to call, 35.6 of the GPU), and for few rows by the launch and two loads, one behind the other (256 rows 2.7 us of the GPU).
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache8_read_kernel(Cache8Args c, const int *__restrict__ slots, T *__restrict__ k_out, T *__restrict__ v_out, int n, int tokens, Divisor by_n, Divisor by_rows)
{
#if defined(__HIP_DEVICE_COMPILE__)
    typedef T vec8 __attribute__((ext_vector_type(8)));
    constexpr int CPR = D / 8;
    const int x = blockIdx.x * 256 + threadIdx.x;
    const int token = x / CPR, col = x % CPR * 8;
    if (token >= tokens) return;
    const int slot = slots[token];
    const int b = quotient(token, by_n), i = token - b * n;
    const bool inside = slot >= 0 && slot < c.pages * c.block_rows;
    const int page = inside ? quotient(slot, by_rows) : 0, row = inside ? slot - page * c.block_rows : 0, h = blockIdx.y;
    const size_t head = (size_t)page * c.heads + h;
    u32x2 raw[2];
    int e[2];
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        raw[tensor] = u32x2{0u, 0u};
        e[tensor] = kScaleBias;
        if (inside) {
            raw[tensor] = *(const u32x2 *)((const unsigned char *)c.data[tensor] + (head * c.block_rows + row) * D + col);
            e[tensor] = c.scales[tensor][head * c.blocks + row / kScaleRows];
        }
    }
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        int x8 = e[tensor];
        x8 = x8 < kScaleBias - kScaleMost ? kScaleBias - kScaleMost : (x8 < kScaleBias + kScaleMost ? x8 : kScaleBias + kScaleMost);
        const float scale = __builtin_bit_cast(float, x8 << 23);
        vec8 out;
#pragma unroll
        for (int i4 = 0; i4 < 2; ++i4) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(raw[tensor][i4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(raw[tensor][i4], true);
            out[i4 * 4] = (T)(lo[0] * scale);
            out[i4 * 4 + 1] = (T)(lo[1] * scale);
            out[i4 * 4 + 2] = (T)(hi[0] * scale);
            out[i4 * 4 + 3] = (T)(hi[1] * scale);
        }
        *(vec8 *)((tensor ? v_out : k_out) + (((size_t)b * c.heads + h) * n + i) * D + col) = out;
    }
#endif
}

template <typename T, int D> int launch_write(const Cache8Write &x)
{
    const long long units = (long long)x.B * x.windows * x.c.heads * 2;
    hipLaunchKernelGGL((cache8_write_kernel<T, D>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, x.stream, x.c, x.x[0], x.x[1], x.kv_lens, x.new_lens, x.S,
                       x.capacity, x.windows, divisor((uint32_t)x.c.heads), divisor((uint32_t)x.windows), (int)units);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_read(const Cache8Read &x)
{
    const int tokens = x.B * x.n;
    hipLaunchKernelGGL((cache8_read_kernel<T, D>), dim3((unsigned)(((long long)tokens * (D / 8) + 255) / 256), (unsigned)x.c.heads), dim3(256), 0, x.stream, x.c,
                       x.slots, (T *)x.out[0], (T *)x.out[1], x.n, tokens, divisor((uint32_t)x.n), divisor((uint32_t)x.c.block_rows));
    return (int)hipGetLastError();
}

template <typename T> int launch_write_dim(int D, const Cache8Write &x)
{
    switch (D) {
        case 64: return launch_write<T, 64>(x);
        case 96: return launch_write<T, 96>(x);
        case 128: return launch_write<T, 128>(x);
        default: return launch_write<T, 160>(x);
    }
}

template <typename T> int launch_read_dim(int D, const Cache8Read &x)
{
    switch (D) {
        case 64: return launch_read<T, 64>(x);
        case 96: return launch_read<T, 96>(x);
        case 128: return launch_read<T, 128>(x);
        default: return launch_read<T, 160>(x);
    }
}

}  // namespace tsdpa

namespace {

constexpr int64_t kMost = std::numeric_limits<int>::max();
// Most workgroups, of 256 threads, of a launch: their threads are counted in 32 bits.
constexpr int64_t kMostGroups = (1 << 24) - 1;

bool misaligned(const void *at, uintptr_t bytes) { return ((uintptr_t)at & (bytes - 1)) != 0; }

// The cache's own numbers; capacity: rows that an entry can have.
int check_cache(const tsdpa_cache8 &c, int B, bool tables, int *capacity)
{
    if (c.D != 64 && c.D != 96 && c.D != 128 && c.D != 160) return TSDPA_ERR_UNSUPPORTED_D;
    if (B < 0 || c.pages < 0 || c.Hkv < 0 || c.block_rows < 0 || c.max_blocks < 0) return TSDPA_ERR_BAD_SHAPE;
    if ((int64_t)c.pages * c.block_rows > kMost) return TSDPA_ERR_BAD_SHAPE;
    *capacity = c.block_rows;
    if (!tables) return TSDPA_OK;
    if (c.block_table) {
        // pages of 64 << n rows, so that no tile straddles two
        if (c.block_rows < 64 || (c.block_rows & (c.block_rows - 1)) != 0 || (int64_t)c.max_blocks * c.block_rows > kMost) return TSDPA_ERR_BAD_SHAPE;
        *capacity = c.max_blocks * c.block_rows;
    } else if (c.pages != B) {
        return TSDPA_ERR_BAD_SHAPE;
    }
    return TSDPA_OK;
}

bool bad_strides(const tsdpa_rows &r, int B, int S, int heads)
{
    const struct { long long stride; int size; } d[3] = {{r.batch, B}, {r.row, S}, {r.head, heads}};
    for (const auto &x : d)
        if (x.size > 1 && (x.stride < 0 || (x.stride & 7) != 0)) return true;      // (one row has no stride)
    return false;
}

tsdpa::Cache8Args args_of(const tsdpa_cache8 &c)
{
    return tsdpa::Cache8Args{{c.k, c.v}, {c.k_scales, c.v_scales}, c.block_table, c.pages, c.Hkv, c.block_rows, tsdpa::scale_blocks(c.block_rows), c.max_blocks};
}

bool incomplete(const tsdpa_cache8 &c) { return !c.k || !c.v || !c.k_scales || !c.v_scales; }

// Which kernel: decoding up to 32 query rows per key/value head (two tiles of 16), beyond that tiles of 32 rows (sdpa_cache8_rows_kernel.h) or of 128
// (sdpa_cache8_chunk_kernel.h).  Tiles of 128 do a seventh less work per row, but have to be filled, and a wavefront of theirs passes over four times
// as many keys: tiles of 32 where those of 128 would be half empty (3.5 of them cost as much as one), and up to 2^27 scores.  Where entries have
// lengths of their own, these may be much shorter than the capacity, and unequal, both of which cost large tiles more: up to 2^28 scores, or 1024 tiles.
// (us, tiles of 32 / of 128, BF16, D = 128: 8 heads of 64 rows, 8192 keys 13.5 / 21.6; 8 of 256 rows, 2048 keys 12.0 / 22.3, 8192 keys 19.0 / 28.8, 65536 keys
// 81 / 80; 32 of 512, 2048 keys 24.6 / 38.2; 8 of 1024, 8192 keys 44 / 49, 65536 keys 284 / 259; 64 of 512, 4096 keys 80 / 81; 8 of 4096, 8192 keys 140 / 133; 8
// of 16384, 16384 keys 969 / 859; 1024 of 64, 2048 keys 122 / 160; 4 entries of 8 heads of 2000 rows, 2560 keys each 100 / 91, 1408 ... 3712 keys 100 / 103.  In
// pages, a capacity of 131072 keys: 8 heads of 256 rows, 2000 keys 16 / 28, 120000 keys 150 / 152; of 2048 rows 25 / 41, 1047 / 1002; of 4096 rows 41 / 55, 2073 / 1985; 8
// entries of 8 heads, capacity 32768: 512 rows, 800 ... 1500 keys 35 / 44, 15300 ... 16000 keys 293 / 293; 2048 rows 108 / 93, 1109 / 1054.)
// Of 17 ... 32 rows two tiles of 16 each read and convert the keys, which few heads have room for and many have not (us, 32 rows, tiles of 16 / of 32: D = 128, 8 heads of 512
// keys 7.0 / 8.0, of 8192 10.6 / 11.7, of 32768 19.0 / 18.3, 64 heads of 2048 12.9 / 15.0, of 8192 33.6 / 30.1, 256 of 2048 33.8 / 25.6; D = 64, 64 heads of 8192 28.1 / 16.9: tiles of 32
// would be right for many heads and long caches, and are not taken there yet).
enum class Form { decode, rows, chunk };
constexpr int kDecodeRows = 32;
Form form_of(int heads, int rows, int Skv, bool lengths)
{
    if (rows <= kDecodeRows) return Form::decode;
    const int64_t small = ((int64_t)rows + 31) / 32, large = ((int64_t)rows + 127) / 128;
    if (2 * small <= 7 * large || (lengths && heads * small <= 1024)) return Form::rows;
    return (int64_t)rows * Skv <= ((int64_t)1 << (lengths ? 28 : 27)) / heads ? Form::rows : Form::chunk;       // (rows * Skv < 2^61)
}

// Splits of tiles of 32 rows: the least of a model of the time.  A workgroup alone on its CU takes 1.8 + 0.0215 D ns per key, two on one CU 1.6 times as long; splits
// cost 2.5 us and, for their states, 0.08 ns per tile, run and column.  Of more than 64 tiles of entries with lengths of their own, as if these were half the capacity:
// what splits cost is then more than they gain of a short one.
// (us at 1 / 2 / 3 / 4 splits, the choice, BF16, D = 128, 8 heads: 16 tiles of 4096 keys 24.5 / 18.0 / 15.5 / 13.8, 13.2; 32 of 8192 43.1 / 28.0 / 21.9 / 19.5, 16.7; 64 of 1024 11.4 /
// 12.2 / 12.8, 11.4, of 4096 24.8 / 18.9 / 17.1 / 16.4, 15.9, of 32768 148 / 84 / 62 / 52, 48; 96 of 4096 25.5 / 20.2 / 22.2 / 21.3, 22.1; 128 of 4096 25.0 / 20.9 / 23.7, 20.7; 144 of
// 2048 16.3 / 18.8, 16.0, of 8192 42.4 / 39.2 / 34.3 / 40.3, 34.2; 192 of 8192 42.6 / 42.2 / 47.5 / 40.9, 40.9; 288 of 4096 31.2 / 38.2, 30.8, of 32768 221 / 218 / 185 / 189, 165;
// 384 of 8192 63.0 / 71.1, 71.2.)
int row_splits(int64_t tiles, int Skv, int D, bool lengths)
{
    const int keys = lengths && tiles > 64 ? Skv / 2 : Skv, most = keys / 256 < TSDPA_MAX_SPLITS ? keys / 256 : TSDPA_MAX_SPLITS;
    const float alone = (1.8e-3f + 2.15e-5f * D) * keys;
    int best = 1;
    float least = std::numeric_limits<float>::max();
    for (int n = 1; n <= (most > 1 ? most : 1) && (n == 1 || tiles * n <= 2048); ++n) {
        const int64_t groups = tiles * n, rest = groups % 512;
        const float time = alone / n * ((float)(groups / 512) * 1.6f + (rest == 0 ? 0.f : rest <= 256 ? 1.f : 1.6f)) + (n > 1 ? 2.5f + 8e-5f * D * (float)groups : 0.f);
        if (time < least) least = time, best = n;
    }
    return best;
}

// Splits along the key axis.
// Decoding: one workgroup per CU in all, of runs of at least 512 keys, or 256 while there are up to eight, which
// the kernel combines itself.  None where a pass over a head's keys takes no longer than the second look at the states.
// (us at 1 / 2 / 4 / 8 / 16 splits, BF16, D = 128, 4 rows per head: 8 heads of 1024 keys 7.8 / 8.7 / 8.0 / 8.1; of 2048
// 11.5 / 10.5 / 8.9 / 8.1 / 9.6; of 8192 33.5 / 21.8 / 14.7 / 11.1 / 10.0, 32 splits 9.6; 64 heads of 1024 keys 7.9 / 8.9 / 8.6, of 4096 18.8 / 15.7
// / 15.8 / 16.2; 90 heads of 4001, D = 96, 17.4 / 15.6 / 16.6; 32 rows per head: 8 heads of 1024 keys 10.1 / 13.0 / 12.6, of 2048 13.9 / 13.9 / 11.7, D = 64 7.3 / 9.7 / 9.4, 10.0 / 10.1
// / 9.5.)
// The bounds, at 1 / 2 / 3 / 4 splits: 40 heads of 1484 keys, D = 128 9.9 / 9.9 / 9.3 / 9.2, of 1679 10.9 / 10.8 / 10.1 / 9.2; of 1187, D = 160 10.3 / 10.9 / 10.0 / 9.9; 90 heads of 1835 keys, D = 128
// 11.9 / 12.1 / 15.5, of 2109 12.8 / 13.4; of 1468, D = 160 11.5 / 12.5, of 1687 12.6 / 14.0.  (At D = 64 they are too high: 40 heads of 2968 keys 11.6 / 10.1 / 9.0 / 8.5, 90 of 3671 14.6 / 12.3.)
// From half as many key/value heads as CUs on none either, with two exceptions where runs are long.  CUs get equal shares of the memory's rate, and one
// reaches 2.4 times that at most (58 GB/s): so 128 heads do not reach it all, and of 257 ... 448 heads those that share a CU take twice as
// long (1 / 2 / 3 splits, FP16: 128 heads of 2048 keys 13.3 / 16.4, of 4096 28.0 / 28.7, of 8192 54 / 51, in pages 60 / 54, of 16384 100 / 96, 113 / 99; 192 of 16384 133 / 145;
// 256 of 8192 95 / 98 / 98; 264 of 16384 260 / 218 / 209, of 4096 ... 16384 134 / 138 / 144; 320 of 8192 136 / 124 / 122; 384 of 16384 301 / 273 / 281, of 4096 ... 16384 208 / 195
// / 193; 512 of 16384 353 / 357 / 368).
int default_splits(Form form, int heads, int rows, int Skv, int D, bool lengths)
{
    if (form == Form::chunk) return tsdpa::row_tile_splits(heads, rows, Skv, D);
    if (form == Form::rows) return row_splits((int64_t)heads * (((int64_t)rows + 31) / 32), Skv, D, lengths);
    if (rows <= 16 ? (int64_t)Skv * D <= (heads > 64 ? 260000 : 210000) : Skv <= 1024) return 1;
    const int64_t tiles = (int64_t)heads * ((rows + 15) / 16), few = Skv / 256 < 8 ? Skv / 256 : 8, most = Skv / 512 > few ? Skv / 512 : few;
    int64_t want = tiles >= 128 ? 1 : 256 / tiles;
    if ((int64_t)Skv * D >= 1 << 20) want = tiles > 256 && tiles <= 448 ? 3 : tiles >= 128 && tiles <= 160 ? 2 : want;
    if (want > most) want = most;
    if (want < 1) want = 1;
    return (int)(want > TSDPA_MAX_SPLITS ? TSDPA_MAX_SPLITS : want);
}

int check_attention(int B, int H, int Hkv, int Sq, int Skv, int D, int dtype, unsigned flags)
{
    if (dtype != TSDPA_F16 && dtype != TSDPA_BF16) return TSDPA_ERR_BAD_DTYPE;
    if (D != 64 && D != 96 && D != 128 && D != 160) return TSDPA_ERR_UNSUPPORTED_D;
    if (B < 0 || H < 0 || Hkv < 0 || Sq < 0 || Skv < 0) return TSDPA_ERR_BAD_SHAPE;
    const int64_t bh = (int64_t)B * H;
    // (no form has more than two workgroups for each; how many runs of the keys that leaves room for is for the call to see)
    if (bh > kMost || (bh > 0 && Sq > 0 && ((int64_t)Sq + 15) / 16 > (kMostGroups - 8) / 2 / bh)) return TSDPA_ERR_BAD_SHAPE;
    // a head is addressed through 32 bits, with room for a "fetch nothing" offset above it
    if (((int64_t)Skv + 1024) * D >= ((int64_t)1 << 30)) return TSDPA_ERR_BAD_SHAPE;
    if (bh > 0 && Sq > 0 && Skv == 0) return TSDPA_ERR_BAD_SHAPE;
    if ((flags & TSDPA_FLAG_CAUSAL) && Skv < Sq) return TSDPA_ERR_BAD_SHAPE;
    if (H > 0 && (Hkv == 0 || H % Hkv != 0)) return TSDPA_ERR_BAD_SHAPE;
    if (H > 0 && (int64_t)(H / Hkv) * Sq > kMost) return TSDPA_ERR_BAD_SHAPE;
    return TSDPA_OK;
}

}  // namespace

extern "C" {

int tiled_sdpa_cache8_write(const tsdpa_cache8 *c, const tsdpa_rows *k, const tsdpa_rows *v, const int *kv_lens, const int *new_lens, int B, int S, int dtype,
                            void *stream)
{
    if (!c || !k || !v) return TSDPA_ERR_NULL_PTR;
    if (dtype != TSDPA_F16 && dtype != TSDPA_BF16) return TSDPA_ERR_BAD_DTYPE;
    int capacity;
    const int st = check_cache(*c, B, true, &capacity);
    if (st != TSDPA_OK) return st;
    if (S < 0) return TSDPA_ERR_BAD_SHAPE;
    // (S tokens of an entry touch a block more than they fill if they begin inside one; none past the capacity)
    const int64_t most = S < capacity ? S : capacity, windows = most <= 1 ? most : (most + 2 * (tsdpa::kScaleRows - 1)) / tsdpa::kScaleRows;
    const int64_t per_entry = windows * c->Hkv;
    if (B > 0 && per_entry > kMostGroups * 4 / 2 / B) return TSDPA_ERR_BAD_SHAPE;      // (four units to a workgroup)
    if (B * per_entry == 0 || c->pages == 0) return TSDPA_OK;
    if (incomplete(*c) || !k->data || !v->data || !kv_lens || !new_lens) return TSDPA_ERR_NULL_PTR;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(k->data, 16) || misaligned(v->data, 16) || misaligned(kv_lens, 4) || misaligned(new_lens, 4) ||
        misaligned(c->block_table, 4))
        return TSDPA_ERR_MISALIGNED;
    if (bad_strides(*k, B, S, c->Hkv) || bad_strides(*v, B, S, c->Hkv)) return TSDPA_ERR_BAD_STRIDE;
    tsdpa::Cache8Write x{args_of(*c), {{k->data, k->batch, k->row, k->head}, {v->data, v->batch, v->row, v->head}}, kv_lens, new_lens, B, S, capacity, (int)windows,
                         (hipStream_t)stream};
    const int err = dtype == TSDPA_F16 ? tsdpa::launch_write_dim<_Float16>(c->D, x) : tsdpa::launch_write_dim<__bf16>(c->D, x);
    return err == 0 ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

int tiled_sdpa_cache8_read(const tsdpa_cache8 *c, const int *slots, void *k_out, void *v_out, int B, int n, int dtype, void *stream)
{
    if (!c) return TSDPA_ERR_NULL_PTR;
    if (dtype != TSDPA_F16 && dtype != TSDPA_BF16) return TSDPA_ERR_BAD_DTYPE;
    int capacity;
    const int st = check_cache(*c, B, false, &capacity);
    if (st != TSDPA_OK) return st;
    if (n < 0 || (int64_t)B * n > kMost / (c->D / 8) - 256 || c->Hkv > 65535) return TSDPA_ERR_BAD_SHAPE;
    if ((int64_t)B * n == 0 || c->Hkv == 0) return TSDPA_OK;
    // (a cache without rows has no memory: every slot lies past its end)
    if (!slots || !k_out || !v_out || (capacity > 0 && c->pages > 0 && incomplete(*c))) return TSDPA_ERR_NULL_PTR;
    if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(k_out, 16) || misaligned(v_out, 16) || misaligned(slots, 4)) return TSDPA_ERR_MISALIGNED;
    tsdpa::Cache8Read x{args_of(*c), slots, {k_out, v_out}, B, n, (hipStream_t)stream};
    if (x.c.block_rows < 1) x.c.pages = 0, x.c.block_rows = 1;
    const int err = dtype == TSDPA_F16 ? tsdpa::launch_read_dim<_Float16>(c->D, x) : tsdpa::launch_read_dim<__bf16>(c->D, x);
    return err == 0 ? TSDPA_OK : TSDPA_ERR_LAUNCH;
}

int tiled_sdpa_cache8_default_splits(int B, int H, int Hkv, int Sq, int Skv, int D, int dtype, unsigned flags, int *splits)
{
    if (!splits) return TSDPA_ERR_NULL_PTR;
    const int st = check_attention(B, H, Hkv, Sq, Skv, D, dtype, flags);
    if (st != TSDPA_OK) return st;
    *splits = 1;
    if ((int64_t)B * H * Sq == 0) return TSDPA_OK;
    const int heads = B * Hkv, rows = H / Hkv * Sq;
    for (const bool lengths : {false, true}) {    // (room for either)
        const int n = default_splits(form_of(heads, rows, Skv, lengths), heads, rows, Skv, D, lengths);
        if (n > *splits) *splits = n;
    }
    return TSDPA_OK;
}

int tiled_sdpa_fwd_cache8(const tsdpa_cache8 *c, const void *q, void *o, float *lse, const int *kv_lens, int B, int H, int Sq, float scale, int dtype,
                          unsigned flags, int splits, void *workspace, unsigned long long workspace_bytes, void *stream)
{
    if (!c) return TSDPA_ERR_NULL_PTR;
    if (dtype != TSDPA_F16 && dtype != TSDPA_BF16) return TSDPA_ERR_BAD_DTYPE;
    int capacity;
    int st = check_cache(*c, B, true, &capacity);
    if (st == TSDPA_OK) st = check_attention(B, H, c->Hkv, Sq, capacity, c->D, dtype, flags);
    if (st != TSDPA_OK) return st;
    if ((int64_t)B * H * Sq == 0) return TSDPA_OK;
    if (!q || !o || incomplete(*c) || (c->block_table && !kv_lens)) return TSDPA_ERR_NULL_PTR;
    if (c->pages == 0) return TSDPA_ERR_BAD_SHAPE;
    if (misaligned(q, 16) || misaligned(o, 16) || misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(lse, 4) || misaligned(kv_lens, 4) ||
        misaligned(c->block_table, 4))
        return TSDPA_ERR_MISALIGNED;
    if (std::isnan(scale)) scale = 1.0f / std::sqrt((float)c->D);
    if (std::isinf(scale)) return TSDPA_ERR_BAD_SCALE;
    if (splits < 0 || splits > TSDPA_MAX_SPLITS) return TSDPA_ERR_BAD_SPLITS;
    const int rows = H / c->Hkv * Sq, heads = B * c->Hkv;
    const Form form = form_of(heads, rows, capacity, kv_lens != nullptr);
    if (splits == 0) {
        splits = default_splits(form, heads, rows, capacity, c->D, kv_lens != nullptr);
        // (with less memory than that takes: as many as fit)
        const unsigned long long each = tiled_sdpa_kv_workspace_bytes(B, H, Sq, c->D, 2) / 2, given = workspace ? workspace_bytes / each : 0;
        if ((unsigned long long)splits > given) splits = given > 1 ? (int)given : 1;
    }
    // (a tile of 32 or 128 rows takes the place of two of 16 or more; the padding to whole XCDs at most doubles it)
    if (splits > 1 && splits > (kMostGroups - 16) / ((int64_t)B * H * (((int64_t)Sq + 15) / 16) * 2)) return TSDPA_ERR_BAD_SPLITS;
    if (splits > 1 && (!workspace || misaligned(workspace, 16) || workspace_bytes < tiled_sdpa_kv_workspace_bytes(B, H, Sq, c->D, splits)))
        return TSDPA_ERR_WORKSPACE;
    tsdpa::Cache8Attend x{args_of(*c), {}};
    tsdpa::LaunchArgs &a = x.a;
    a.q = q;
    a.o = o;
    a.lse = lse;
    a.BH = heads;
    a.S = rows;
    a.rows_per_head = Sq;
    a.kv_lens = kv_lens;
    a.heads_per_batch = c->Hkv;
    a.batches = B;
    a.c = std::fabs(scale) * 1.44269504088896340736f;
    a.qsign = std::signbit(scale) && scale != 0.0f ? 0x80008000u : 0u;
    a.causal = (flags & TSDPA_FLAG_CAUSAL) ? 1 : 0;
    a.kv = 1;
    a.Skv = capacity;
    a.splits = splits;
    a.ws = (float *)workspace;
    a.stream = (hipStream_t)stream;
    // The decoding kernel combines the runs itself while their states are few (the conditions of the 16-bit caches' in tiled_sdpa.hip)
    if (rows <= 8 && splits > 1 && splits * rows <= 32 && splits <= rows * c->D / 4 && rows * c->D <= 1024) a.ticket = tsdpa::new_ticket();
    int err;
    if (form == Form::chunk) err = dtype == TSDPA_F16 ? tsdpa::launch_cache8_chunk_f16(c->D, x) : tsdpa::launch_cache8_chunk_bf16(c->D, x);
    else if (form == Form::rows) err = dtype == TSDPA_F16 ? tsdpa::launch_cache8_rows_f16(c->D, x) : tsdpa::launch_cache8_rows_bf16(c->D, x);
    else err = dtype == TSDPA_F16 ? tsdpa::launch_cache8_decode_f16(c->D, x) : tsdpa::launch_cache8_decode_bf16(c->D, x);
    if (err != 0) return TSDPA_ERR_LAUNCH;
    if (splits > 1 && a.ticket == 0) {
        tsdpa::merge_states(a, c->D, dtype, (int64_t)heads * rows <= 2048 && (splits > 8 || rows <= kDecodeRows));
        if (hipGetLastError() != hipSuccess) return TSDPA_ERR_LAUNCH;
    }
    return TSDPA_OK;
}

}  // extern "C"
