// The values of an 8-bit cache in the attention kernels: codes as 16-bit numbers, the scales of a tile, values that are NaN.
#pragma once
#include "cache8_args.h"
#include "sdpa_fwd_kernel.h"

namespace tsdpa {

constexpr int kTile8 = 64;                        // keys per tile: two blocks of rows that share a scale

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// Eight codes as eight 16-bit numbers (exact).
template <typename T> struct Codes;
template <> struct Codes<_Float16> {
    static __device__ __forceinline__ f16x8 wide(uint32_t lo, uint32_t hi)
    {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
        // (whole registers: put together value by value, each pair is taken apart and joined again)
        return __builtin_bit_cast(f16x8, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                                               __builtin_bit_cast(uint32_t, d)});
    }
};
template <> struct Codes<__bf16> {
    static __device__ __forceinline__ bf16x8 wide(uint32_t lo, uint32_t hi)
    {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
        return __builtin_bit_cast(bf16x8, u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                                                __builtin_bit_cast(uint32_t, d)});
    }
};

// The maximum and the sum over the four lanes (lane, lane ^ 16, ^ 32, ^ 48) that share a row, in all of them.
__device__ __forceinline__ float pair16(float x, float &other)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    other = __builtin_bit_cast(float, r1);
    return __builtin_bit_cast(float, r0);
}
__device__ __forceinline__ float quad_max(float x)
{
    float b;
    const float a = pair16(x, b);
    return pair_max(fmaxf(a, b));
}
__device__ __forceinline__ float quad_sum(float x)
{
    float b;
    const float a = pair16(x, b);
    return pair_sum(a + b);
}

// The four scale bytes of a tile: in lanes 0 and 1 of every four K's, in 2 and 3 V's (of a block past the end the last one's).  `page`: of a dense cache
// the entry.
template <bool PAGED> __device__ __forceinline__ int tile_scale_bytes(const Cache8Args &cache, int tile, int page, int h)
{
    const int lane = threadIdx.x & 63;
    const unsigned char *scales = (lane & 2) ? cache.scales[1] : cache.scales[0];
    int block = 2 * tile + (lane & 1);
    if constexpr (PAGED) block &= cache.blocks - 1;
    else block = block < cache.blocks ? block : cache.blocks - 1;
    return (int)scales[((size_t)page * cache.heads + h) * (size_t)cache.blocks + block];
}

// The weights that enter the product with V are FP16, which ends at 2^16 and has a least step of 2^-24.  So the reference m is kRoom below the greatest score plus EV
// when it is set, and stays while a lane's sum of a tile is at most 2^15: the greatest weight of a row is 2^7 or more, and what a small one loses is 2^-25, or 2^-32 of the
// greatest.  (Without that room many weights of 2^-26 would be lost from o together, though not from l: 4096 beside one key, 6e-5 of O, and all that a column has in which that
// key's value is 0.)
constexpr float kRoom = 7.f, kLazyLimit8 = 0x1p15f;

// A key counts in l by 2^(score - m), and its weight is 2^(score + EV - m), m + kRoom being the greatest score plus EV: of two keys that count alike one may have EV = 62, the
// other -62, and keys of 2^-24 of another, or many of less, still count.  So l is the sum of the weights times 2^-EV only where these are in FP32's normal range, below which
// the exponential gives 0.  Which is known by the sum of a lane's weights of a block, 8 or 16 keys: from kSmall on, what is lost is 2^-32 of that sum or less.  Below that,
// 2^-97 of the row's greatest weight, the tile's part of l is a sum of exponentials of its own, from which EV is taken before: 2^(-62 - 24) at least, with 40 powers of two
// to spare for keys that count because they are many, and 2^77 at most.  (To compare EV itself with the greatest so far in each tile took 6 % more time of large tiles at D = 64.)
constexpr float kSmallLog2 = -90.f;
constexpr uint32_t kSmall = (uint32_t)(127 + (int)kSmallLog2) << 23;

// Weights of a tile, in a lane: their sum, their part of l, and the blocks' sums.
struct TileSums {
    float p, l, block[2];
    // p above the lazy limit, inf or NaN, or a block's sum less than `least`, the bits of kSmall (or 0: of which the row sees no key).  One comparison, of the bits of numbers that
    // are not negative: what is less is 2^31 and more above, and what is not less below the limit's.
    __device__ __forceinline__ bool unusual(const uint32_t (&least)[2]) const
    {
        const uint32_t x = __builtin_bit_cast(uint32_t, block[0]) - least[0], y = __builtin_bit_cast(uint32_t, block[1]) - least[1];
        const uint32_t most = x > y ? x : y, all = __builtin_bit_cast(uint32_t, p);
        return (all > most ? all : most) > __builtin_bit_cast(uint32_t, kLazyLimit8);
    }
};

// Whether one of a lane's greatest weights of the two blocks, in powers of two, is small, and not 0 (-infinity: no key that the row sees).
__device__ __forceinline__ bool small_weights(float a, float b)
{
    const uint32_t first = __builtin_bit_cast(uint32_t, kSmallLog2) + 1, x = __builtin_bit_cast(uint32_t, a) - first, y = __builtin_bit_cast(uint32_t, b) - first;
    return (x < y ? x : y) < __builtin_bit_cast(uint32_t, -INFINITY) - first;
}

// Of a tile's two blocks: c * 2^EK, EV, 2^-EV.
struct TileScales {
    float ck[2], ev[2], ew[2];
    __device__ __forceinline__ TileScales(int x, float c)
    {
        x = x < kScaleBias - kScaleMost ? kScaleBias - kScaleMost : (x < kScaleBias + kScaleMost ? x : kScaleBias + kScaleMost);
        const float power = __builtin_bit_cast(float, x << 23) * c, e = (float)(x - kScaleBias), inverse = __builtin_bit_cast(float, (2 * kScaleBias - x) << 23);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            ck[kb] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, power), kb));
            ev[kb] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, e), 2 + kb));
            ew[kb] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, inverse), 2 + kb));
        }
    }
};

// The state (m, l, o) of a run of keys, for whoever combines runs by 2^(m - greatest m): l may be 2^62 times as large as the greatest weight, and count where that factor
// is 0.  So the reference is raised by what l has over 1, 2^62 at most, and o and l are multiplied by the result.  (A reference so large that it cannot be
// raised by so little stays as it is, and so do they.)
__device__ __forceinline__ float raise_reference(float &m, float l)
{
    const int e = (int)(__builtin_bit_cast(uint32_t, l) >> 23) - 127;
    const float old = m;
    m += (float)(e < 0 ? 0 : (e < kScaleMost ? e : kScaleMost));
    return old == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(old - m);
}

// Values that are NaN, in keys that only some rows see (the causal mask): the product with a weight of 0 would be NaN for the others.
// Eight codes: 1 (FP16) where one is NaN, and the codes without those.
struct Nan8 {
    static __device__ __forceinline__ uint32_t marks(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
    static __device__ __forceinline__ uint32_t whole(uint32_t m) { return (m >> 7) * 0xffu; }
    static __device__ __forceinline__ f16x8 ones(u32x2 x)
    {
        const uint32_t a = whole(marks(x[0])) & 0x38383838u, b = whole(marks(x[1])) & 0x38383838u;      // (0x38: the code of 1)
        return Codes<_Float16>::wide(a, b);
    }
    static __device__ __forceinline__ u32x2 without(u32x2 x) { return u32x2{x[0] & ~whole(marks(x[0])), x[1] & ~whole(marks(x[1]))}; }
};

}  // namespace tsdpa
