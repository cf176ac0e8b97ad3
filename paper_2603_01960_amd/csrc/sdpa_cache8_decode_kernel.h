// Attention of few query rows (16 per workgroup and up to 32, the grouped query heads' rows together) over an 8-bit cache.
//
// The values of a cache are code * 2^E, E4M3 codes, one E for each head and 32 rows of K, one of V.  With c = scale * log2(e)
//     s_j = <q, codes of key j>,   p_j = 2^(s_j * (c * 2^EK) + EV - m),   o = sum_j p_j * codes of value j,   l = sum_j p_j * 2^-EV,
// and O = o / l: the scales cost nothing per value.  EK folds into the factor of the score, EV into the exponent, so that m goes by the greatest
// score PLUS exponent seen (kRoom in sdpa_cache8_values.h): the weights that enter the products are sized by what they contribute, and the products, whose weights and
// values are both FP16 here whatever the type of q (every code is an FP16 number), keep 11 bits of the largest contributions.  l takes
// the exponent out again, in FP32, and where p_j may be none of its normal numbers before the exponential is taken (kSmall).
//
// Such a call is bound by reading the cache once.  As in sdpa_decode_kernel.h each wavefront streams tiles of its own through LDS slots
// of its own, with no barrier in the loop: one slot for K and one for V, each refilled as soon as it has been read into registers.  A
// tile is 64 keys, as many bytes as 32 keys of 16 bits, so that as many are in flight.
//
// Measured (D = 128, from call to call): 4 entries of 65536 keys, 8 heads of 4 rows, BF16, 537 MB in 96 us, 5.6 TB/s, where a stream that only reads reaches 6.1; 32
// entries of 2048 ... 8192 keys in pages, FP16, 336 MB in 69 us, for the longest of which (one workgroup per CU, 64 KB on their way) the rest waits; one
// entry of 8192 keys in 32 runs 9.3 us, of which the kernel is 7.2 (prologue and the first keys 3.5, four tiles, the states' way to memory) and their
// combination 2.1 ... 2.9.  Eight or two wavefronts per workgroup and 32 rows per wavefront (spilled) were no faster.
#pragma once
#include "sdpa_cache8_values.h"
#include "sdpa_runs.h"

namespace tsdpa {

// LDS layout of a tile: 64 rows of D bytes, unpadded; 16-byte chunks are permuted within each row (chunk c at c ^ swizzle(row)).
//   K: 16 lanes read one chunk of 16 consecutive rows.
//   V: the transposing read has 32 lanes fetch one chunk of 16 rows, 4 at a time: 0 ... 7 and 16 ... 23, or those plus 8.
// Both land on 16 different 16-byte slots of the 64 banks.  Rows of 96 and 160 bytes start on 8 different even slots, eight rows in turn: there
// the lowest bit of the chunk tells the two eights apart.
template <int D> struct Geom8 {
    static constexpr int ROW = D, CPR = D / 16;
    static constexpr int TILE = kTile8 * ROW;
    static constexpr int UNITS = TILE / 1024;     // direct-to-LDS load instructions per tile
    static constexpr int P = UNITS / 2;           // ... per 32 rows, after which the lanes' offsets repeat
    static __host__ __device__ constexpr int kx(int r) { return D == 128 ? (r >> 1) & 7 : D == 64 ? (r >> 2) & 3 : (r >> 3) & 1; }
    static __host__ __device__ constexpr int vx(int r)
    {
        return D == 128 ? ((r >> 1) & 3) | ((r >> 4) & 1) << 2 : D == 64 ? ((r >> 2) & 1) | ((r >> 4) & 1) << 1 : (r >> 4) & 1;
    }
    static constexpr int KC = D / 64;             // 16-byte pieces of K per lane and row block; D % 64 = 32: and one of 8
    static constexpr bool TAIL = D % 64 != 0;
    static constexpr int NKP = (D == 128 ? 2 : 1) + (TAIL ? 1 : 0);       // pointers of K's reads (the tail's is the last)
    static constexpr int NVP = D == 128 ? 8 : D == 64 ? 4 : 2;            // ... of V's: one per 16 columns, or per parity of these
};

// The reads of one tile and the wait for them, in one block of inline assembly each (see DecodeRead in sdpa_decode_kernel.h for why).
//   keys:   x[b][h] = 16 bytes at row block b (16 rows), y[b] = 8 bytes of the tail
//   values: x[db][kb] = transposing read of 16 columns, 32 rows
#define TSDPA_RD_K(i, a, off) "ds_read_b128 %" #i ", %" #a " offset:" #off "\n\t"
#define TSDPA_RD_K8(i, a, off) "ds_read_b64 %" #i ", %" #a " offset:" #off "\n\t"
#define TSDPA_RD_V(i, a, off) "ds_read_b64_tr_b8 %" #i ", %" #a " offset:" #off "\n\t"
#define TSDPA_RD_WAIT "s_waitcnt lgkmcnt(0)"
template <int D> struct Read8;
template <> struct Read8<64> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[4][1], u32x2 (&)[4], const uint32_t (&p)[1])
    {
        asm volatile(TSDPA_RD_K(0, 4, 0) TSDPA_RD_K(1, 4, 1024) TSDPA_RD_K(2, 4, 2048) TSDPA_RD_K(3, 4, 3 * 1024) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[1][0]), "=&v"(x[2][0]), "=&v"(x[3][0])
                     : "v"(p[0])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[4][2], const uint32_t (&p)[4])
    {
        asm volatile(TSDPA_RD_V(0, 8, 0) TSDPA_RD_V(1, 8, 2048) TSDPA_RD_V(2, 9, 0) TSDPA_RD_V(3, 9, 2048)
                     TSDPA_RD_V(4, 10, 0) TSDPA_RD_V(5, 10, 2048) TSDPA_RD_V(6, 11, 0) TSDPA_RD_V(7, 11, 2048) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3])
                     : "memory");
    }
};
template <> struct Read8<96> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[4][1], u32x2 (&y)[4], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_K(0, 8, 0) TSDPA_RD_K(1, 8, 1536) TSDPA_RD_K(2, 8, 3 * 1024) TSDPA_RD_K(3, 8, 4608)
                     TSDPA_RD_K8(4, 9, 0) TSDPA_RD_K8(5, 9, 1536) TSDPA_RD_K8(6, 9, 3 * 1024) TSDPA_RD_K8(7, 9, 4608) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[1][0]), "=&v"(x[2][0]), "=&v"(x[3][0]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[6][2], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_V(0, 12, 0) TSDPA_RD_V(1, 12, 3 * 1024) TSDPA_RD_V(2, 13, 0) TSDPA_RD_V(3, 13, 3 * 1024)
                     TSDPA_RD_V(4, 12, 32) TSDPA_RD_V(5, 12, 3104) TSDPA_RD_V(6, 13, 32) TSDPA_RD_V(7, 13, 3104)
                     TSDPA_RD_V(8, 12, 64) TSDPA_RD_V(9, 12, 3136) TSDPA_RD_V(10, 13, 64) TSDPA_RD_V(11, 13, 3136) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[4][0]), "=&v"(x[4][1]), "=&v"(x[5][0]), "=&v"(x[5][1])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
};
template <> struct Read8<128> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[4][2], u32x2 (&)[4], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_K(0, 8, 0) TSDPA_RD_K(1, 9, 0) TSDPA_RD_K(2, 8, 2048) TSDPA_RD_K(3, 9, 2048)
                     TSDPA_RD_K(4, 8, 4096) TSDPA_RD_K(5, 9, 4096) TSDPA_RD_K(6, 8, 6144) TSDPA_RD_K(7, 9, 6144) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[8][2], const uint32_t (&p)[8])
    {
        asm volatile(TSDPA_RD_V(0, 16, 0) TSDPA_RD_V(1, 16, 4096) TSDPA_RD_V(2, 17, 0) TSDPA_RD_V(3, 17, 4096)
                     TSDPA_RD_V(4, 18, 0) TSDPA_RD_V(5, 18, 4096) TSDPA_RD_V(6, 19, 0) TSDPA_RD_V(7, 19, 4096)
                     TSDPA_RD_V(8, 20, 0) TSDPA_RD_V(9, 20, 4096) TSDPA_RD_V(10, 21, 0) TSDPA_RD_V(11, 21, 4096)
                     TSDPA_RD_V(12, 22, 0) TSDPA_RD_V(13, 22, 4096) TSDPA_RD_V(14, 23, 0) TSDPA_RD_V(15, 23, 4096) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[4][0]), "=&v"(x[4][1]), "=&v"(x[5][0]), "=&v"(x[5][1]),
                       "=&v"(x[6][0]), "=&v"(x[6][1]), "=&v"(x[7][0]), "=&v"(x[7][1])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7])
                     : "memory");
    }
};
template <> struct Read8<160> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[4][2], u32x2 (&y)[4], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_K(0, 12, 0) TSDPA_RD_K(1, 12, 64) TSDPA_RD_K(2, 12, 2560) TSDPA_RD_K(3, 12, 2624)
                     TSDPA_RD_K(4, 12, 5120) TSDPA_RD_K(5, 12, 5184) TSDPA_RD_K(6, 12, 7680) TSDPA_RD_K(7, 12, 7744)
                     TSDPA_RD_K8(8, 13, 0) TSDPA_RD_K8(9, 13, 2560) TSDPA_RD_K8(10, 13, 5120) TSDPA_RD_K8(11, 13, 7680) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(y[0]), "=&v"(y[1]), "=&v"(y[2]), "=&v"(y[3])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[10][2], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_V(0, 20, 0) TSDPA_RD_V(1, 20, 5120) TSDPA_RD_V(2, 21, 0) TSDPA_RD_V(3, 21, 5120)
                     TSDPA_RD_V(4, 20, 32) TSDPA_RD_V(5, 20, 5152) TSDPA_RD_V(6, 21, 32) TSDPA_RD_V(7, 21, 5152)
                     TSDPA_RD_V(8, 20, 64) TSDPA_RD_V(9, 20, 5184) TSDPA_RD_V(10, 21, 64) TSDPA_RD_V(11, 21, 5184)
                     TSDPA_RD_V(12, 20, 96) TSDPA_RD_V(13, 20, 5216) TSDPA_RD_V(14, 21, 96) TSDPA_RD_V(15, 21, 5216)
                     TSDPA_RD_V(16, 20, 128) TSDPA_RD_V(17, 20, 5248) TSDPA_RD_V(18, 21, 128) TSDPA_RD_V(19, 21, 5248) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[4][0]), "=&v"(x[4][1]), "=&v"(x[5][0]), "=&v"(x[5][1]),
                       "=&v"(x[6][0]), "=&v"(x[6][1]), "=&v"(x[7][0]), "=&v"(x[7][1]), "=&v"(x[8][0]), "=&v"(x[8][1]),
                       "=&v"(x[9][0]), "=&v"(x[9][1])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
};
#undef TSDPA_RD_K
#undef TSDPA_RD_K8
#undef TSDPA_RD_V
#undef TSDPA_RD_WAIT

// What the launch fixes: divisors of numbers that the prologue divides by (a division by a variable is a serial chain of some thirty
// instructions; with those, and shuffles through the LDS, the prologue took 1.2 us, now 0.6).
struct Decode8Order {
    int units;                                    // (run, key/value head) pairs
    int step;                                     // heads that a run's first one is further on than the run's before
    int row_tiles;                                // workgroups of 16 query rows for each: 1 or 2
    Divisor by_heads, by_entry_heads, by_splits, by_rows;        // key/value heads in all, of an entry; runs; query positions
};

// A workgroup: NW wavefronts, one (run of keys, 16 query rows of a key/value head).  S query rows per head, of which rows_per_head (the
// query positions) belong to each query head.
template <typename T, int D, int NW, bool PAGED>
__global__ void __launch_bounds__(NW * 64, 2)
sdpa_cache8_decode_kernel(const T *__restrict__ q, T *o, float *__restrict__ lse, Cache8Args cache, int S, int heads, Decode8Order order, float c,
                          uint32_t qsign, int causal, int Skv_cap, int splits, float *ws, int rows_per_head, const int *__restrict__ kv_lens, int batches,
                          unsigned long long ticket)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using vec8 = typename Elem<T>::vec8;
    using vec4 = typename Elem<T>::vec4;
    using G = Geom8<D>;
    constexpr int KS = D / 32, DB = D / 16, NU = G::UNITS, TM = 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const lds_ptr lds = (lds_ptr)smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t = lane >> 4, l16 = lane & 15;
    // (all arguments that the prologue needs, at once)
    asm volatile("" : : "s"(q), "s"(cache.data[0]), "s"(cache.data[1]), "s"(cache.scales[0]), "s"(cache.scales[1]), "s"(cache.block_table), "s"(S), "s"(heads),
                 "s"(order.step), "s"(order.by_heads.mul), "s"(order.by_entry_heads.mul), "s"(order.by_splits.mul), "s"(Skv_cap), "s"(splits), "s"(kv_lens));

    // Run by run, each from another head on (run fastest would put the runs of one long entry next to each other: see sdpa_decode_kernel.h).  The
    // two tiles of a head's rows next to each other on one XCD, so that one of them reads the keys from its L2.
    int unit = blockIdx.x, r0 = 0;
    if (order.row_tiles == 2) {
        const int y = blockIdx.x >> 3;
        unit = (y >> 1) * 8 + (blockIdx.x & 7);
        r0 = (y & 1) * TM;
        if (unit >= order.units) return;
    }
    const int sp = divide(unit, order.by_heads);
    int head = unit - sp * heads + sp * order.step;
    if (head >= heads) head -= heads;
    const int hpb = cache.heads, b = divide(head, order.by_entry_heads), h = head - b * hpb;
    auto clamped = [&](int x) __attribute__((always_inline)) { return x < 0 ? 0 : (x < Skv_cap ? x : Skv_cap); };
    int len = Skv_cap, longest = len;             // keys of this entry, and (runs are a share of these) of the longest one
    if (kv_lens != nullptr) {
        if (splits > 1 && batches > 1 && batches <= 64) {
            const int own = clamped(lane < batches ? kv_lens[lane] : 0);
            len = __builtin_amdgcn_readlane(own, b);
            longest = lanes_max(own);
        } else {
            len = longest = clamped(kv_lens[b]);
        }
    }
    // this workgroup's run of tiles: [t0, t0 + n)
    const int nT = (len + kTile8 - 1) / kTile8;
    int run = divide((longest + kTile8 - 1) / kTile8 + splits - 1, order.by_splits);
    if (run < 2) run = 2;
    const int t0 = sp * run;
    int n = nT - t0 < run ? nT - t0 : run;
    if (n < 0) n = 0;
    const size_t states = (size_t)heads * splits * S * D;
    if (n == 0 && splits > 1) {                   // the state of no keys (o is not looked at then)
        if (tid < TM && r0 + tid < S) put_pair(ws + states + ((size_t)(head * splits + sp) * S + r0 + tid) * 2, -INFINITY, 0.f);
        if (ticket != 0) finish_runs<T, D, NW>(o, lse, ws, lds, head, sp, S, heads, splits, ticket, tid, wave, lane);
        return;
    }

    // ---- tiles: HBM -> LDS.  Wavefront w takes the tiles w, w + NW, ... of the run, entered at a tile that depends on the workgroup, and in a dense cache
    // exchanged by a number that does too (heads lie a power of two apart: in step they would keep hitting the same memory channels, and so would
    // those of them that a start of its own has brought together by chance.  The exchange, one run per head, us: 128 heads of 16384 keys, D = 128 123 -> 100,
    // 192 150 -> 133, 256 195 -> 181, 512 406 -> 353, of 20000 keys 0 ... 4 %; in pages, which lie as they come, entries of one length are level with it and
    // unequal ones 1 ... 2 % slower, 69.4 -> 70.5).
    const lds_ptr kslot = lds + wave * 2 * G::TILE, vslot = kslot + G::TILE;
    const unsigned char *kbase = (const unsigned char *)cache.data[0], *vbase = (const unsigned char *)cache.data[1];
    const size_t head_off = (size_t)head * (size_t)Skv_cap * D;
    const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(kbase + (PAGED ? 0 : head_off)), (short)0, len * G::ROW, 0x00020000);
    const auto v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + (PAGED ? 0 : head_off)), (short)0, len * G::ROW, 0x00020000);
    const int *pages = PAGED ? cache.block_table + (size_t)b * cache.max_blocks : nullptr;
    int kgoff[G::P], vgoff[G::P];
    auto offset = [&](int u, auto swizzle) __attribute__((always_inline)) {
        const int p = u * 64 + lane, r = p / G::CPR, cp = p % G::CPR;
        return r * G::ROW + ((cp ^ swizzle(r)) << 4);
    };
    const int shift = PAGED ? __builtin_ctz(cache.block_rows) : 0;
    // (a page that does not exist is none of the cache's memory: the nearest that does is read in its place)
    auto page_of = [&](int tile) __attribute__((always_inline)) {
        const int page = __builtin_amdgcn_readfirstlane(pages[(tile * kTile8) >> shift]);
        return page < 0 ? 0 : (page < cache.pages ? page : cache.pages - 1);
    };
    struct Src { decltype(k_rsrc) kr, vr; int soff; };
    auto src_of = [&](int tile, bool valid, int page) __attribute__((always_inline)) {
        if constexpr (!PAGED) return Src{k_rsrc, v_rsrc, valid ? tile * G::TILE : nT * G::TILE};
        else {
            const int row0 = tile * kTile8;
            int rows = valid ? len - row0 : 0;
            rows = rows < kTile8 ? rows : kTile8;
            const unsigned long long first = (((unsigned long long)page * hpb + h) << shift) + (row0 & ((1 << shift) - 1));
            const unsigned long long byte0 = first * (unsigned long long)G::ROW;
            const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)byte0), hi = __builtin_amdgcn_readfirstlane((unsigned)(byte0 >> 32));
            const unsigned long long at = ((unsigned long long)hi << 32) | lo;
            const int bytes = __builtin_amdgcn_readfirstlane(rows * G::ROW);
            return Src{__builtin_amdgcn_make_buffer_rsrc((void *)(kbase + at), (short)0, bytes, 0x00020000),
                       __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + at), (short)0, bytes, 0x00020000), 0};
        }
    };
    auto load_k = [&](const Src &s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(s.kr, (TSDPA_LDS void *)(kslot + u * 1024), 16, kgoff[u % G::P], s.soff + u / G::P * (32 * G::ROW), 0, 0);
    };
    auto load_v = [&](const Src &s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(s.vr, (TSDPA_LDS void *)(vslot + u * 1024), 16, vgoff[u % G::P], s.soff + u / G::P * (32 * G::ROW), 0, 0);
    };
    auto load_scale = [&](int tile, int page) __attribute__((always_inline)) { return tile_scale_bytes<PAGED>(cache, tile, PAGED ? page : b, h); };
    const int mine = (n - wave + NW - 1) / NW;       // tiles of this wavefront (n - wave > -NW)
    const int rot = n > NW ? (int)__umulhi((unsigned)blockIdx.x * 2654435761u, (unsigned)n) : 0;
    int cur = wave + rot;                         // within the run
    if (cur >= n) cur -= n;
    auto advance = [&](int x) __attribute__((always_inline)) { x += NW; return x >= n ? x - n : x; };
    const int most = n >= 256 ? 255 : 0x7fffffff >> __builtin_clz(n | 1);        // (the largest 2^i - 1 below n)
    const int mix = !PAGED && n > NW ? (int)((blockIdx.x * 2654435761u) >> 16) & most : 0;
    auto tile_of = [&](int x) __attribute__((always_inline)) { return t0 + (!PAGED && (x | most) < n ? x ^ mix : x); };

    // The first tile's K goes out before anything else is worked out, then its exponents, Q, and V, in the order in which they are needed.
    int page_next = 0, scale_next = 0;
    if constexpr (PAGED) page_next = page_of(mine > 0 ? tile_of(cur) : 0);
    const Src first = src_of(tile_of(cur), mine > 0, page_next);
#pragma unroll
    for (int u = 0; u < G::P; ++u) kgoff[u] = offset(u, G::kx);
    load_k(first);
    __builtin_amdgcn_sched_barrier(0);
    scale_next = load_scale(mine > 0 ? tile_of(cur) : 0, page_next);
    // ---- Q rows as MFMA B-operands.  The order of the products over D is free: lane t of a row takes bytes t * 16 ... of each 64 columns of K,
    // of the last 32 (D = 96, 160) t * 8 ..., and Q's columns are those.
    vec8 qf[KS];
    const int row = r0 + l16 < S ? r0 + l16 : S - 1;
    u32x4 raw[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int col = (G::TAIL && ks == KS - 1) ? ks * 32 + t * 8 : (ks >> 1) * 64 + t * 16 + (ks & 1) * 8;
        raw[ks] = *(const u32x4 *)(q + ((size_t)head * S + row) * D + col);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < G::P; ++u) vgoff[u] = offset(u, G::vx);
    load_v(first);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PAGED) page_next = page_of(mine > 1 ? tile_of(advance(cur)) : mine > 0 ? t0 : 0);
    // key j contributes to this lane's row iff j <= klim; every tile that ends behind klim_least takes the masked path
    const int klim = causal ? row - divide(row, order.by_rows) * rows_per_head + len - rows_per_head : len - 1;
    const int klim_least = causal ? len - rows_per_head : len - 1;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(vec8, raw[ks] ^ qsign);

    f32x4 oacc[DB];
    float m_ref = klim >= t0 * kTile8 ? kNoWeight : -INFINITY, l_run = 0.f;      // the lazy reference of sdpa_fwd_kernel.h, this lane's share of the normaliser
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- pointers of the reads
    uint32_t kptr[G::NKP], vptr[G::NVP];
    {
        const uint32_t row = __builtin_bit_cast(uint32_t, kslot) + l16 * G::ROW;
        kptr[0] = row + ((t ^ G::kx(l16)) << 4);
        if constexpr (D == 128) kptr[1] = row + (((4 + t) ^ G::kx(l16)) << 4);
        if constexpr (G::TAIL) kptr[G::NKP - 1] = row + (((4 * G::KC + (t >> 1)) ^ G::kx(l16)) << 4) + (t & 1) * 8;
        const int r = l16 >> 1, v_row = t * 4 + (r & 3) + (r >> 2) * 16;
#pragma unroll
        for (int i = 0; i < G::NVP; ++i)
            vptr[i] = __builtin_bit_cast(uint32_t, vslot) + v_row * G::ROW + ((i ^ G::vx(v_row)) << 4) + (l16 & 1) * 8;
    }

    f16x8 pb[2];
    // weights of one tile: their sum (what the lazy limit looks at) and their part of l
    auto exponentials = [&](const f32x4 (&s)[4], int key0, const TileScales &x8, auto mask_tag) __attribute__((always_inline)) {
        float sum[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const float off = x8.ev[kb] - m_ref;
            sum[kb] = 0.f;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb * 2 + (x >> 2)][x & 3], x8.ck[kb], off));
                if (decltype(mask_tag)::value && key0 + kb * 32 + (x >> 2) * 16 + (x & 3) > klim) p = 0.f;
                sum[kb] += p;
                pb[kb][x] = (_Float16)p;
            }
        }
        return TileSums{sum[0] + sum[1], sum[0] * x8.ew[0] + sum[1] * x8.ew[1], {sum[0], sum[1]}};
    };
    auto softmax = [&](f32x4 (&s)[4], int key0, const TileScales &x8, bool first_tile, auto mask_tag) __attribute__((always_inline)) {
        TileSums ps{INFINITY, 0.f, {0.f, 0.f}};   // (against kNoWeight any weight overflows: the first tile is not asked)
        if (!first_tile) ps = exponentials(s, key0, x8, mask_tag);
        auto least = [&](int kb) __attribute__((always_inline)) { return !decltype(mask_tag)::value || key0 + kb * 32 <= klim ? kSmall : 0u; };
        if (__builtin_amdgcn_ballot_w64(ps.unusual({least(0), least(1)})) != 0) {
            // Eq. 2 for all rows of the wavefront: the tile's maximum, new reference and the rescale of Eqs. 3-4
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < 16; ++x)
                if (!decltype(mask_tag)::value || key0 + (x >> 2) * 16 + (x & 3) <= klim) mx[x >> 3] = fmaxf(mx[x >> 3], s[x >> 2][x & 3]);
            const float most[2] = {mx[0] * x8.ck[0] + x8.ev[0], mx[1] * x8.ck[1] + x8.ev[1]}, m_tile = quad_max(fmaxf(most[0], most[1])) - kRoom;
            const bool grow = m_tile > m_ref;     // (a row without finite scores so far: -inf or NaN, left alone)
            const float half = grow ? __builtin_amdgcn_exp2f((m_ref - m_tile) * 0.5f) : 1.f, alpha = half * half;     // (l may count where alpha is 0)
            m_ref = grow ? m_tile : m_ref;
            l_run = l_run * half * half;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int e = 0; e < 4; ++e) oacc[db][e] *= alpha;
            float l = 0.f;
            const bool apart = __builtin_amdgcn_ballot_w64(small_weights(most[0] - m_ref, most[1] - m_ref)) != 0;
            if (__builtin_expect(apart, 0)) {
                float m_l = m_ref;
                asm("" : "+v"(m_l));              // (else the arguments below are kept for the exponentials that follow: 16 registers)
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x >> 2][x & 3], x8.ck[x >> 3], x8.ev[x >> 3] - m_l) - x8.ev[x >> 3]);
                    if (!decltype(mask_tag)::value || key0 + (x >> 2) * 16 + (x & 3) <= klim) l += e;
                }
            }
            ps = exponentials(s, key0, x8, mask_tag);
            if (apart) ps.l = l;
        }
        l_run += ps.l;
    };

    for (int i = 0; i < mine; ++i) {
        const int next = advance(cur), tile = tile_of(cur);
        const bool more = i + 1 < mine;
        const Src s = src_of(tile_of(next), more, page_next);
        const int page_of_next = page_next;
        if constexpr (PAGED) page_next = page_of(i + 2 < mine ? tile_of(advance(next)) : t0);
        // In flight, in this order: the tile's K, its exponents, its V.  (K has landed when at most V's loads are outstanding, V when at most
        // the next K's are.  A load of the exponents that the compiler moves makes these waits longer, never shorter.)
        u32x4 kf[4][G::KC];
        u32x2 kt[4];
        TSDPA_WAIT_VMCNT(NU);
        Read8<D>::keys(kf, kt, kptr);
        load_k(s);
        int scale_now = scale_next;
        asm volatile("" : "+v"(scale_now));       // (not looked at before: a wait for it there would be one for V)
        const TileScales scale(scale_now, c);
        f32x4 sacc[4];
#pragma unroll
        for (int blk = 0; blk < 4; ++blk) sacc[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {   // blk innermost: independent products follow one another
                vec8 a;
                if (G::TAIL && ks == KS - 1) a = Codes<T>::wide(kt[blk][0], kt[blk][1]);
                else a = Codes<T>::wide(kf[blk][ks >> 1][(ks & 1) * 2], kf[blk][ks >> 1][(ks & 1) * 2 + 1]);
                sacc[blk] = Elem16<T>::mfma(a, qf[ks], sacc[blk]);
            }
        const int key0 = tile * kTile8 + t * 4;
        const bool masked = tile * kTile8 + kTile8 - 1 > klim_least;
        if (masked) softmax(sacc, key0, scale, i == 0, std::true_type{});
        else softmax(sacc, key0, scale, i == 0, std::false_type{});
        u32x2 vf[DB][2];
        TSDPA_WAIT_VMCNT(NU);
        Read8<D>::values(vf, vptr);
        scale_next = load_scale(more ? tile_of(next) : tile, page_of_next);
        load_v(s);
        bool nan = false;
        if (masked && causal) {
            uint32_t any = 0;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) any |= Nan8::marks(vf[db][kb][0]) | Nan8::marks(vf[db][kb][1]);
            nan = __builtin_amdgcn_ballot_w64(any != 0) != 0;
        }
        if (nan) {
            // a row gets NaN if it sees one
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                f16x8 seen;
#pragma unroll
                for (int x = 0; x < 8; ++x) seen[x] = key0 + kb * 32 + (x >> 2) * 16 + (x & 3) > klim ? (_Float16)0.f : (_Float16)1.f;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const f16x8 ones = Nan8::ones(vf[db][kb]);
                    const u32x2 rest = Nan8::without(vf[db][kb]);
                    const f32x4 count = Elem16<_Float16>::mfma(ones, seen, f32x4{0.f, 0.f, 0.f, 0.f});
                    oacc[db] = Elem16<_Float16>::mfma(Codes<_Float16>::wide(rest[0], rest[1]), pb[kb], oacc[db]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[db][e] += count[e] > 0.f ? __builtin_nanf("") : 0.f;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    oacc[db] = Elem16<_Float16>::mfma(Codes<_Float16>::wide(vf[db][kb][0], vf[db][kb][1]), pb[kb], oacc[db]);
        }
        cur = next;
    }

    // ---- the wavefronts' states, over the LDS: [wave][row][D] floats, then [wave][row] (m, l)  (no load may still be on its way into it)
    float l_row = l_run;
    l_row = quad_sum(l_row);
    TSDPA_WAIT_VMCNT0();
    __syncthreads();
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    constexpr int ML = NW * TM * D * 4;
    if (r0 + l16 < S) {
#pragma unroll
        for (int db = 0; db < DB; ++db) *(TSDPA_LDS f32x4 *)(lds + ((wave * TM + l16) * D + db * 16 + t * 4) * 4) = oacc[db];
        if (t == 0) *(TSDPA_LDS f32x2 *)(lds + ML + (wave * TM + l16) * 8) = f32x2{m_ref, l_row};
    }
    __syncthreads();
    // a thread: four columns of a row
    const int rows = S - r0 < TM ? S - r0 : TM;
    for (int x = tid; x < rows * (D / 4); x += NW * 64) {
        const int r = x / (D / 4);
        f32x2 ml[NW];
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            ml[w] = *(TSDPA_LDS f32x2 *)(lds + ML + (w * TM + r) * 8);
            M = fmaxf(M, ml[w][0]);
        }
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float half = ml[w][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[w][0] - M) * 0.5f), weight = half * half;      // (2^(m - M); -inf: no key)
            L += ml[w][1] * half * half;
            const f32x4 part = *(TSDPA_LDS f32x4 *)(lds + w * (TM * D * 4) + x * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += weight * part[e];
        }
        const bool of_row = x - r * (D / 4) == 0;
        if (splits > 1) {
            float *part = ws + ((size_t)(head * splits + sp) * S + r0) * D + (size_t)x * 4;
            const float f = raise_reference(M, L);
            put_pair(part, sum[0] * f, sum[1] * f);
            put_pair(part + 2, sum[2] * f, sum[3] * f);
            if (of_row) put_pair(ws + states + ((size_t)(head * splits + sp) * S + r0 + r) * 2, M, L * f);
        } else {
            const float inv = M == -INFINITY ? 0.f : 1.f / L;     // (no key at all: O = 0, LSE = -inf)
            vec4 out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = (T)(sum[e] * inv);
            *(vec4 *)(o + ((size_t)head * S + r0) * D + (size_t)x * 4) = out;
            if (of_row && lse != nullptr) lse[(size_t)head * S + r0 + r] = L != 0.f ? (M + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f : -INFINITY;
        }
    }
    if (ticket != 0) finish_runs<T, D, NW>(o, lse, ws, lds, head, sp, S, heads, splits, ticket, tid, wave, lane);
#endif
}

template <typename T, int D, int NW, bool PAGED> int launch_cache8_decode_one(const Cache8Attend &x)
{
    auto kern = sdpa_cache8_decode_kernel<T, D, NW, PAGED>;
    constexpr int lds_bytes = NW * 2 * Geom8<D>::TILE;
    static_assert(NW * 16 * (D * 4 + 8) <= lds_bytes, "the states of all wavefronts must fit");
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes); });
    if (attr_err != hipSuccess) return (int)attr_err;
    const LaunchArgs &a = x.a;
    const int units = a.BH * a.splits, row_tiles = a.S > 16 ? 2 : 1;
    const Decode8Order order{units, a.splits > 1 ? a.BH / a.splits : 0, row_tiles, divisor((uint32_t)a.BH), divisor((uint32_t)a.heads_per_batch),
                             divisor((uint32_t)a.splits), divisor((uint32_t)a.rows_per_head)};
    hipLaunchKernelGGL(kern, dim3((unsigned)(row_tiles == 1 ? units : (units + 7) / 8 * 16)), dim3(NW * 64), lds_bytes, a.stream, (const T *)a.q, (T *)a.o, a.lse, x.c,
                       a.S, a.BH, order, a.c, a.qsign, a.causal, a.Skv, a.splits, a.ws, a.rows_per_head, a.kv_lens, a.batches, a.ticket);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_cache8_decode_dim(const Cache8Attend &x)
{
    return x.c.block_table ? launch_cache8_decode_one<T, D, 4, true>(x) : launch_cache8_decode_one<T, D, 4, false>(x);
}

template <typename T> int launch_cache8_decode(int D, const Cache8Attend &x)
{
    switch (D) {
        case 64: return launch_cache8_decode_dim<T, 64>(x);
        case 96: return launch_cache8_decode_dim<T, 96>(x);
        case 128: return launch_cache8_decode_dim<T, 128>(x);
        default: return launch_cache8_decode_dim<T, 160>(x);
    }
}

}  // namespace tsdpa
