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

// A key counts in l by 2^(score - m), and its weight is 2^(score + EV - m), m + kRoom being the greatest score plus EV: of two keys that count alike one may have EV = 62, the other
// -62, and keys of 2^-24 of another, or many of less, still count.  So l is the sum of the weights times 2^-EV only as long as these are in FP32's normal range, below which
// the exponential gives 0: weights that count are 2^-(kFar + 24) of the greatest or more where EV is at most kFar below the greatest that the wavefront
// has met.  In tiles with a block that is further below, l is the sum of exponentials of its own, from which EV is taken before: 2^(-62 - 24) of the
// greatest weight at least, and 2^77 at most.  (2^-126 leaves 32 and 40 powers of two to keys that count only because they are many.)
constexpr int kFar = 70;

// Of a tile's two blocks: c * 2^EK, EV, 2^-EV; and in the lanes that have V's exponents whether one is far below the greatest so far (`top`, of bytes).
struct TileScales {
    float ck[2], ev[2], ew[2];
    bool far_lane;
    __device__ __forceinline__ bool far() const { return __builtin_amdgcn_ballot_w64(far_lane) != 0; }
    __device__ __forceinline__ TileScales(int x, float c, int &top)
    {
        x = x < kScaleBias - kScaleMost ? kScaleBias - kScaleMost : (x < kScaleBias + kScaleMost ? x : kScaleBias + kScaleMost);
        const int other = __builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, false);       // quad_perm: the other block's
        top = x > top ? x : top;
        top = other > top ? other : top;
        far_lane = x + ((threadIdx.x & 2) ? kFar : 1 << 16) < top;
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
