// Attention of a block of query rows over an 8-bit cache where there are too few for sdpa_cache8_chunk_kernel.h's tiles of 128 to fill the GPU:
// prompts that are short, drafts, chunks of few sequences.
//
// A workgroup has 32 query rows of a key/value head, the same ones in all of its four wavefronts, and a run of keys; as in
// sdpa_cache8_decode_kernel.h each wavefront streams tiles of 64 keys of its own, as codes, through LDS slots of its own with no barrier in the loop, and the
// four states meet in the LDS at the end.  The products are 32 x 32 and the softmax is that of the chunks.
//
// A tile is converted by the wavefront that uses it, for 32 rows: with the softmax that is about a fifth more time on the vector units than the products take
// on the matrix units, and bounds the kernel where the GPU is full (16384 rows of 8 heads, 16384 keys, D = 128: 969 us, where tiles of 128 rows, which convert
// a quarter as often, take 859).  Where it is not full, a wavefront's number of tiles does: a quarter of what a tile of 128 rows passes over in its four (8
// heads of 64 rows, 8192 keys, D = 128, in 16 runs: 13.5 us, 21.6 in tiles of 128; a 16-bit cache 12.5).  Registers hold two workgroups per CU at D = 128
// and above; hidden keys are taken out of the scores before the softmax, which therefore is there once: with masked and unmasked forms of it
// the compiler spilled in all loops from D = 128 on.
#pragma once
#include "sdpa_cache8_values.h"

namespace tsdpa {

// LDS layout of a tile: 64 rows of D bytes, unpadded; 16-byte chunks are permuted within each row.
//   K: 16 lanes read one chunk of 16 consecutive rows (Geom8's, in sdpa_cache8_decode_kernel.h).
//   V: the transposing read has 32 lanes fetch two chunks of 8 rows, 0 ... 3 and 8 ... 11 or those plus 4: rows of a power of two put them on 16
//      different 16-byte slots of the 64 banks; in rows of 96 and 160 bytes, where the chunks of the second four rows are turned by two, 14.
template <int D> struct GeomRows {
    static constexpr int ROW = D, CPR = D / 16, TILE = kTile8 * ROW, UNITS = TILE / 1024, P = UNITS / 2;
    static constexpr int H = D / 32;              // 16-byte pieces of K per lane and 32 rows; blocks of 32 columns of V
    static constexpr int NKP = D == 128 ? 4 : D == 64 ? 2 : 1;
    static __host__ __device__ constexpr int k_at(int c, int r) { return c ^ (D == 128 ? (r >> 1) & 7 : D == 64 ? (r >> 2) & 3 : (r >> 3) & 1); }
    // where chunk c of row r stands, and which chunk stands at place c
    static __host__ __device__ constexpr int v_at(int c, int r)
    {
        if (D == 128) return c ^ ((r & 2) | (r >> 1 & 4));
        if (D == 64) return c ^ (r >> 2 & 2);
        return (c + (r >> 2 & 2)) % CPR;
    }
    static __host__ __device__ constexpr int v_of(int c, int r)
    {
        return (D & (D - 1)) == 0 ? v_at(c, r) : (c + CPR - (r >> 2 & 2)) % CPR;
    }
};

// The reads of one tile and the wait for them, in one block of inline assembly each (see DecodeRead in sdpa_decode_kernel.h for why).
//   keys:   x[nb][h] = 16 bytes of 32 rows
//   values: x[db][b] = transposing read of 32 columns, 16 rows
#define TSDPA_RD_K(i, a, off) "ds_read_b128 %" #i ", %" #a " offset:" #off "\n\t"
#define TSDPA_RD_V(i, a, off) "ds_read_b64_tr_b8 %" #i ", %" #a " offset:" #off "\n\t"
#define TSDPA_RD_WAIT "s_waitcnt lgkmcnt(0)"
template <int D> struct ReadRows;
template <> struct ReadRows<64> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[2][2], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_K(0, 4, 0) TSDPA_RD_K(1, 5, 0) TSDPA_RD_K(2, 4, 2048) TSDPA_RD_K(3, 5, 2048) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[2][4], const uint32_t (&p)[2])
    {
        asm volatile(TSDPA_RD_V(0, 8, 0) TSDPA_RD_V(1, 8, 1024) TSDPA_RD_V(2, 8, 2048) TSDPA_RD_V(3, 8, 3 * 1024)
                     TSDPA_RD_V(4, 9, 0) TSDPA_RD_V(5, 9, 1024) TSDPA_RD_V(6, 9, 2048) TSDPA_RD_V(7, 9, 3 * 1024) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]),
                       "=&v"(x[1][2]), "=&v"(x[1][3])
                     : "v"(p[0]), "v"(p[1])
                     : "memory");
    }
};
template <> struct ReadRows<96> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[2][3], const uint32_t (&p)[1])
    {
        asm volatile(TSDPA_RD_K(0, 6, 0) TSDPA_RD_K(1, 6, 32) TSDPA_RD_K(2, 6, 64) TSDPA_RD_K(3, 6, 3 * 1024)
                     TSDPA_RD_K(4, 6, 3104) TSDPA_RD_K(5, 6, 3136) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[1][2])
                     : "v"(p[0])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[3][4], const uint32_t (&p)[3])
    {
        asm volatile(TSDPA_RD_V(0, 12, 0) TSDPA_RD_V(1, 12, 1536) TSDPA_RD_V(2, 12, 3 * 1024) TSDPA_RD_V(3, 12, 4608)
                     TSDPA_RD_V(4, 13, 0) TSDPA_RD_V(5, 13, 1536) TSDPA_RD_V(6, 13, 3 * 1024) TSDPA_RD_V(7, 13, 4608)
                     TSDPA_RD_V(8, 14, 0) TSDPA_RD_V(9, 14, 1536) TSDPA_RD_V(10, 14, 3 * 1024) TSDPA_RD_V(11, 14, 4608) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]),
                       "=&v"(x[1][2]), "=&v"(x[1][3]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[2][2]), "=&v"(x[2][3])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2])
                     : "memory");
    }
};
template <> struct ReadRows<128> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[2][4], const uint32_t (&p)[4])
    {
        asm volatile(TSDPA_RD_K(0, 8, 0) TSDPA_RD_K(1, 9, 0) TSDPA_RD_K(2, 10, 0) TSDPA_RD_K(3, 11, 0)
                     TSDPA_RD_K(4, 8, 4096) TSDPA_RD_K(5, 9, 4096) TSDPA_RD_K(6, 10, 4096) TSDPA_RD_K(7, 11, 4096) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]),
                       "=&v"(x[1][2]), "=&v"(x[1][3])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[4][4], const uint32_t (&p)[4])
    {
        asm volatile(TSDPA_RD_V(0, 16, 0) TSDPA_RD_V(1, 16, 2048) TSDPA_RD_V(2, 16, 4096) TSDPA_RD_V(3, 16, 6144)
                     TSDPA_RD_V(4, 17, 0) TSDPA_RD_V(5, 17, 2048) TSDPA_RD_V(6, 17, 4096) TSDPA_RD_V(7, 17, 6144)
                     TSDPA_RD_V(8, 18, 0) TSDPA_RD_V(9, 18, 2048) TSDPA_RD_V(10, 18, 4096) TSDPA_RD_V(11, 18, 6144)
                     TSDPA_RD_V(12, 19, 0) TSDPA_RD_V(13, 19, 2048) TSDPA_RD_V(14, 19, 4096) TSDPA_RD_V(15, 19, 6144) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]),
                       "=&v"(x[1][2]), "=&v"(x[1][3]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[2][2]), "=&v"(x[2][3]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[3][2]), "=&v"(x[3][3])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3])
                     : "memory");
    }
};
template <> struct ReadRows<160> {
    static __device__ __forceinline__ void keys(u32x4 (&x)[2][5], const uint32_t (&p)[1])
    {
        asm volatile(TSDPA_RD_K(0, 10, 0) TSDPA_RD_K(1, 10, 32) TSDPA_RD_K(2, 10, 64) TSDPA_RD_K(3, 10, 96)
                     TSDPA_RD_K(4, 10, 128) TSDPA_RD_K(5, 10, 5120) TSDPA_RD_K(6, 10, 5152) TSDPA_RD_K(7, 10, 5184)
                     TSDPA_RD_K(8, 10, 5216) TSDPA_RD_K(9, 10, 5248) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[0][4]), "=&v"(x[1][0]),
                       "=&v"(x[1][1]), "=&v"(x[1][2]), "=&v"(x[1][3]), "=&v"(x[1][4])
                     : "v"(p[0])
                     : "memory");
    }
    static __device__ __forceinline__ void values(u32x2 (&x)[5][4], const uint32_t (&p)[5])
    {
        asm volatile(TSDPA_RD_V(0, 20, 0) TSDPA_RD_V(1, 20, 2560) TSDPA_RD_V(2, 20, 5120) TSDPA_RD_V(3, 20, 7680)
                     TSDPA_RD_V(4, 21, 0) TSDPA_RD_V(5, 21, 2560) TSDPA_RD_V(6, 21, 5120) TSDPA_RD_V(7, 21, 7680)
                     TSDPA_RD_V(8, 22, 0) TSDPA_RD_V(9, 22, 2560) TSDPA_RD_V(10, 22, 5120) TSDPA_RD_V(11, 22, 7680)
                     TSDPA_RD_V(12, 23, 0) TSDPA_RD_V(13, 23, 2560) TSDPA_RD_V(14, 23, 5120) TSDPA_RD_V(15, 23, 7680)
                     TSDPA_RD_V(16, 24, 0) TSDPA_RD_V(17, 24, 2560) TSDPA_RD_V(18, 24, 5120) TSDPA_RD_V(19, 24, 7680) TSDPA_RD_WAIT
                     : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[0][2]), "=&v"(x[0][3]), "=&v"(x[1][0]), "=&v"(x[1][1]),
                       "=&v"(x[1][2]), "=&v"(x[1][3]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[2][2]), "=&v"(x[2][3]),
                       "=&v"(x[3][0]), "=&v"(x[3][1]), "=&v"(x[3][2]), "=&v"(x[3][3]), "=&v"(x[4][0]), "=&v"(x[4][1]),
                       "=&v"(x[4][2]), "=&v"(x[4][3])
                     : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4])
                     : "memory");
    }
};
#undef TSDPA_RD_K
#undef TSDPA_RD_V
#undef TSDPA_RD_WAIT

// Entries of up to this number that differ in length come longest first where there are more workgroups than start at once: else a long one may be the last, and
// others wait for it.  (us, in an order of chance that is least / most in favour of it: 4 entries of 500 queries of 32 heads over 8, 1408 ... 3712 keys, D = 128,
// FP16 107.9 -> 101.7 / 100.2 -> 100.9; 16 of 64 queries, 314 ... 4000 keys, D = 64 35.0 -> 30.0 / 29.7 -> 30.0; all of 2560 keys 100.0 -> 100.9.  For 64 entries
// finding the order took as long as it gained.)
constexpr int kRanked = 16;
// Which workgroup has which tile of query rows of which unit (a head's run of keys).  A unit's tiles follow one another on one XCD, whose L2
// the keys then come from; where the units are no multiple of the 8 XCDs each is dealt to several, tile by tile, so that all have as many
// (4 heads of 64 tiles, 4096 keys, D = 128: 37.4 -> 27.4 us).
struct RowsOrder {
    int row_tiles, tiles, log2_parts;             // tiles of a unit, of one of its parts
    int ranked;                                   // entries, where they come longest first; else 0
    Divisor by_tiles, by_splits, by_entry_heads, by_rows;
};

template <typename T, int D, bool PAGED>
__global__ void __launch_bounds__(256, 2)
sdpa_cache8_rows_kernel(const T *__restrict__ q, T *__restrict__ o, float *__restrict__ lse, Cache8Args cache, int S, int units, RowsOrder order, float c,
                        uint32_t qsign, int causal, int Skv_cap, int splits, float *__restrict__ ws, int rows_per_head, const int *__restrict__ kv_lens)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using vec8 = typename Elem<T>::vec8;
    using vec4 = typename Elem<T>::vec4;
    using G = GeomRows<D>;
    constexpr int NW = 4, NB = 2, KK = D / 16, DB = D / 32, H = G::H, NU = G::UNITS, TN = kTile8, TM = 32;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const lds_ptr lds = (lds_ptr)smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 5, l32 = lane & 31;

    // (under the causal mask the last tile has the most keys: it comes first)
    const int y = blockIdx.x >> 3, yt = divide(y, order.by_tiles), part = yt * 8 + (blockIdx.x & 7);
    const int unit = part >> order.log2_parts;
    const int qt = order.row_tiles - 1 - (((y - yt * order.tiles) << order.log2_parts) + (part & ((1 << order.log2_parts) - 1)));
    if (unit >= units || qt < 0) return;
    int head = divide(unit, order.by_splits);
    const int sp = unit - head * splits, hpb = cache.heads;
    int b = divide(head, order.by_entry_heads);
    const int h = head - b * hpb;
    int len = Skv_cap;
    if (order.ranked > 0) {
        const int own = lane < order.ranked ? (kv_lens[lane] > 0 ? kv_lens[lane] : 0) : -1;
        int rank = 0;
#pragma unroll
        for (int j = 0; j < kRanked; ++j) {
            const int other = __builtin_amdgcn_readlane(own, j);
            rank += other > own || (other == own && j < lane) ? 1 : 0;
        }
        b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == b && lane < order.ranked));
        head = b * hpb + h;
        len = __builtin_amdgcn_readlane(own, b);
    } else if (kv_lens != nullptr) {
        len = kv_lens[b];
    }
    len = len < 0 ? 0 : (len < Skv_cap ? len : Skv_cap);
    // the run of tiles [t0, t0 + n) of those that the tile's last row sees
    const int Sp = rows_per_head, koff = len - Sp, r0 = qt * TM, last_row = (r0 + TM < S ? r0 + TM : S) - 1;
    const int g0 = divide(r0, order.by_rows), g1 = divide(last_row, order.by_rows);
    const int pos_lo = g0 == g1 ? r0 - g0 * Sp : 0, pos_hi = g0 == g1 ? last_row - g1 * Sp : Sp - 1;
    const int reach = pos_hi + koff;              // (below 0: no row sees a key)
    const int nT = (len + TN - 1) / TN, nTw = causal ? (reach < 0 ? 0 : reach / TN + 1) : nT;
    const int per_split = divide(nTw + splits - 1, order.by_splits), t0 = sp * per_split;
    int n = nTw - t0 < per_split ? nTw - t0 : per_split;
    if (n < 0) n = 0;
    const int klim_least = causal ? pos_lo + koff : len - 1;   // every tile that ends behind it takes the masked path

    // ---- tiles: HBM -> LDS (sdpa_cache8_decode_kernel.h)
    const lds_ptr kslot = lds + wave * 2 * G::TILE, vslot = kslot + G::TILE;
    const unsigned char *kbase = (const unsigned char *)cache.data[0], *vbase = (const unsigned char *)cache.data[1];
    const size_t head_off = PAGED ? 0 : (size_t)head * (size_t)Skv_cap * D;
    const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(kbase + head_off), (short)0, len * G::ROW, 0x00020000);
    const auto v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + head_off), (short)0, len * G::ROW, 0x00020000);
    const int *pages = PAGED ? cache.block_table + (size_t)b * cache.max_blocks : nullptr;
    const int shift = PAGED ? __builtin_ctz(cache.block_rows) : 0;
    auto page_of = [&](int tile) __attribute__((always_inline)) {
        const int page = __builtin_amdgcn_readfirstlane(pages[(tile * TN) >> shift]);
        return page < 0 ? 0 : (page < cache.pages ? page : cache.pages - 1);
    };
    struct Src { decltype(k_rsrc) kr, vr; int soff; };
    auto src_of = [&](int tile, bool valid, int page) __attribute__((always_inline)) {
        if constexpr (!PAGED) return Src{k_rsrc, v_rsrc, valid ? tile * G::TILE : nT * G::TILE};
        else {
            const int row0 = tile * TN;
            int rows = valid ? len - row0 : 0;
            rows = rows < TN ? rows : TN;
            const unsigned long long first = (((unsigned long long)page * hpb + h) << shift) + (row0 & ((1 << shift) - 1));
            const unsigned long long byte0 = first * (unsigned long long)G::ROW;
            const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)byte0), hi = __builtin_amdgcn_readfirstlane((unsigned)(byte0 >> 32));
            const unsigned long long at = ((unsigned long long)hi << 32) | lo;
            const int bytes = __builtin_amdgcn_readfirstlane(rows * G::ROW);
            return Src{__builtin_amdgcn_make_buffer_rsrc((void *)(kbase + at), (short)0, bytes, 0x00020000),
                       __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + at), (short)0, bytes, 0x00020000), 0};
        }
    };
    int kgoff[G::P], vgoff[G::P];
#pragma unroll
    for (int u = 0; u < G::P; ++u) {
        const int p = u * 64 + lane, r = p / G::CPR, cp = p % G::CPR;
        kgoff[u] = r * G::ROW + (G::k_at(cp, r) << 4);
        vgoff[u] = r * G::ROW + (G::v_of(cp, r) << 4);
    }
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
    const int mine = (n - wave + NW - 1) / NW;       // tiles of this wavefront: t0 + wave, + NW, ...
    int tile = t0 + wave;
    int page_next = 0, scale_next = 0;
    if constexpr (PAGED) page_next = page_of(mine > 0 ? tile : 0);
    const Src first = src_of(tile, mine > 0, page_next);
    load_k(first);
    __builtin_amdgcn_sched_barrier(0);
    scale_next = load_scale(mine > 0 ? tile : 0, page_next);
    // ---- Q rows as MFMA B-operands; the order of the products over D is free: lane g of a row takes bytes (2 h + g) * 16 ... of K, and Q's columns
    const int qrow = r0 + l32, qrow_c = qrow < S ? qrow : S - 1;
    u32x4 raw[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) raw[kk] = *(const u32x4 *)(q + ((size_t)head * S + qrow_c) * D + ((kk >> 1) * 2 + g) * 16 + (kk & 1) * 8);
    __builtin_amdgcn_sched_barrier(0);
    load_v(first);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PAGED) page_next = page_of(mine > 1 ? tile + NW : mine > 0 ? tile : 0);
    const int klim = causal ? qrow_c - divide(qrow_c, order.by_rows) * Sp + koff : len - 1;       // key j contributes to this lane's row iff j <= klim
    vec8 qf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = __builtin_bit_cast(vec8, raw[kk] ^ qsign);

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    float m_ref = kNoWeight, l_run = 0.f;
    uint32_t kptr[G::NKP], vptr[DB];
#pragma unroll
    for (int i = 0; i < G::NKP; ++i) kptr[i] = __builtin_bit_cast(uint32_t, kslot) + l32 * G::ROW + (G::k_at(2 * i + g, l32) << 4);
    const int l16 = lane & 15, v_row = g * 4 + (l16 >> 1 & 3) + (l16 >> 3) * 8;
#pragma unroll
    for (int db = 0; db < DB; ++db)
        vptr[db] = __builtin_bit_cast(uint32_t, vslot) + v_row * G::ROW + (G::v_at(2 * db + (lane >> 4 & 1), v_row) << 4) + (l16 & 1) * 8;

    f32x16 sacc[NB];
    f16x8 pb[NB][2];
    auto key_of = [](int nb, int i) __attribute__((always_inline)) { return nb * 32 + (i >> 2) * 8 + (i & 3); };
    auto exponentials = [&](const TileScales &x8) __attribute__((always_inline)) {
        float sum[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float off = x8.ev[nb] - m_ref;
            float part[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[nb][i], x8.ck[nb], off));
                if (i < 2) part[i] = p;
                else part[i & 1] += p;
                pb[nb][i >> 3][i & 7] = (_Float16)p;
            }
            sum[nb] = part[0] + part[1];
        }
        return TileSums{sum[0] + sum[1], sum[0] * x8.ew[0] + sum[1] * x8.ew[1], {sum[0], sum[1]}};
    };
    // (of a masked tile the scores have EV already, and x8 has none: `ev` is what it was)
    auto softmax = [&](const TileScales &x8, const float (&ev)[NB], const uint32_t (&least)[NB], bool first_tile) __attribute__((always_inline)) {
        TileSums ps{INFINITY, 0.f, {0.f, 0.f}};   // (against kNoWeight any weight overflows: the first tile is not asked)
        if (!first_tile) ps = exponentials(x8);
        if (__builtin_amdgcn_ballot_w64(ps.unusual(least)) != 0) {
            float m_tile = -INFINITY, most[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sacc[nb][i]);
                most[nb] = mx * x8.ck[nb] + x8.ev[nb];
                m_tile = fmaxf(m_tile, most[nb]);
            }
            m_tile = pair_max(m_tile) - kRoom;
            const bool grow = pair_max(ps.p <= kLazyLimit8 ? 0.f : 1.f) > 0.f && m_tile > m_ref;
            const float half = grow ? __builtin_amdgcn_exp2f((m_ref - m_tile) * 0.5f) : 1.f, alpha = half * half;     // (l may count where alpha is 0)
            m_ref = grow ? m_tile : m_ref;
            l_run = l_run * half * half;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
            float l = 0.f;
            const bool apart = __builtin_amdgcn_ballot_w64(small_weights(most[0] - m_ref, most[1] - m_ref)) != 0;
            if (__builtin_expect(apart, 0)) {
                float m_l = m_ref;
                asm("" : "+v"(m_l));              // (else the arguments below are kept for the exponentials that follow: 32 registers)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) l += __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[nb][i], x8.ck[nb], x8.ev[nb] - m_l) - ev[nb]);
            }
            ps = exponentials(x8);
            if (apart) ps.l = l;
        }
        l_run += ps.l;
    };

    for (int i = 0; i < mine; ++i) {
        const bool more = i + 1 < mine;
        const Src s = src_of(tile + NW, more, page_next);
        const int page_of_next = page_next;
        if constexpr (PAGED) page_next = page_of(i + 2 < mine ? tile + 2 * NW : t0);
        // In flight, in this order: the tile's K, its exponents, its V (the waits: see sdpa_cache8_decode_kernel.h).
        TSDPA_WAIT_VMCNT(NU);
        {
            u32x4 kf[NB][H];
            ReadRows<D>::keys(kf, kptr);
            load_k(s);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[nb][e] = 0.f;
            // (the wavefront that has products to do goes before the other one's softmax: 1 ... 4 % where the GPU is full)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    sacc[nb] = Elem<T>::mfma(Codes<T>::wide(kf[nb][kk >> 1][(kk & 1) * 2], kf[nb][kk >> 1][(kk & 1) * 2 + 1]), qf[kk], sacc[nb]);
        }
        __builtin_amdgcn_s_setprio(0);
        TileScales x8(scale_next, c);
        const bool masked = tile * TN + TN - 1 > klim_least;
        const int last = klim - (tile * TN + g * 4);          // the last of the tile's keys that this lane's row sees, from the lane's first
        const float ev[NB] = {x8.ev[0], x8.ev[1]};
        uint32_t least[NB] = {kSmall, kSmall};
        if (masked) {
            // scores as they enter the softmax, -inf for hidden keys (a factor of 0 would make them NaN)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[nb][e] = key_of(nb, e) > last ? -INFINITY : __builtin_fmaf(sacc[nb][e], x8.ck[nb], x8.ev[nb]);
                if (nb * 32 > last) least[nb] = 0u;
                x8.ck[nb] = 1.f;
                x8.ev[nb] = 0.f;
            }
        }
        softmax(x8, ev, least, i == 0);
        u32x2 vf[DB][4];
        TSDPA_WAIT_VMCNT(NU);
        ReadRows<D>::values(vf, vptr);
        scale_next = load_scale(more ? tile + NW : tile, page_of_next);
        load_v(s);
        bool nan = false;
        if (masked && causal) {
            uint32_t any = 0;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int x = 0; x < 4; ++x) any |= Nan8::marks(vf[db][x][0]) | Nan8::marks(vf[db][x][1]);
            nan = __builtin_amdgcn_ballot_w64(any != 0) != 0;
        }
        __builtin_amdgcn_sched_barrier(0);
        if (nan) {
            // values that are NaN, in keys that only some rows see: those that see one get NaN, and the tile a 0 in its place
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                u32x4 seen;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    seen[e] = (key_of(x >> 1, (x & 1) * 8 + 2 * e) > last ? 0u : 0x3c00u) | (key_of(x >> 1, (x & 1) * 8 + 2 * e + 1) > last ? 0u : 0x3c000000u);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    f32x16 count;
#pragma unroll
                    for (int e = 0; e < 16; ++e) count[e] = 0.f;
                    count = Elem<_Float16>::mfma(Nan8::ones(vf[db][x]), __builtin_bit_cast(f16x8, seen), count);
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[db][e] += count[e] > 0.f ? __builtin_nanf("") : 0.f;
                    asm volatile("" : "+v"(oacc[db]));       // (now: put off to the end, all counts are held at once)
                    vf[db][x] = Nan8::without(vf[db][x]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int db = 0; db < DB; ++db)
                oacc[db] = Elem<_Float16>::mfma(Codes<_Float16>::wide(vf[db][x][0], vf[db][x][1]), pb[x >> 1][x & 1], oacc[db]);
        __builtin_amdgcn_s_setprio(0);
        tile += NW;
    }

    // ---- the wavefronts' states, over the LDS, half of the columns at a time where the slots are too small for all: [wave][four columns][lane] and
    // [wave][row] (m, l).  A lane has one row and of each eight columns four; lanes are permuted by the columns, against bank conflicts on reading.
    // (No load may still be on its way.)
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    constexpr int PASSES = D == 160 ? 2 : 1, CH = D / 8 / PASSES, PART = CH * 1024, ML = NW * PART;
    static_assert(ML + NW * TM * 8 <= NW * 2 * G::TILE + (PASSES == 1 ? NW * TM * 8 : 0), "the states fit what the launch asks for");
    const float l_tot = pair_sum(l_run);
    TSDPA_WAIT_VMCNT0();
    const int rows = S - r0 < TM ? S - r0 : TM;
    const size_t first_row = (size_t)head * S + r0, first_state = (size_t)unit * S + r0;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        __syncthreads();
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) {
            const int at = pass * CH + ch;
            f32x4 part;
#pragma unroll
            for (int e = 0; e < 4; ++e) part[e] = oacc[at >> 2][(at & 3) * 4 + e];
            *(TSDPA_LDS f32x4 *)(lds + wave * PART + (ch * 64 + (lane ^ ((2 * ch + g) & 15))) * 16) = part;
        }
        if (g == 0) *(TSDPA_LDS f32x2 *)(lds + ML + (wave * TM + l32) * 8) = f32x2{klim >= t0 * TN ? m_ref : -INFINITY, l_tot};
        __syncthreads();
        for (int x = tid; x < rows * (2 * CH); x += NW * 64) {
            const int r = x / (2 * CH), c4 = x - r * (2 * CH), col = (pass * CH * 2 + c4) * 4;
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
                const float half = ml[w][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[w][0] - M) * 0.5f), weight = half * half;      // (-inf: no key)
                L += ml[w][1] * half * half;
                const f32x4 part = *(TSDPA_LDS f32x4 *)(lds + w * PART + ((c4 >> 1) * 64 + (((c4 & 1) * 32 + r) ^ (c4 & 15))) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += weight * part[e];
            }
            if (splits > 1) {
                const float f = raise_reference(M, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] *= f;
                *(f32x4 *)(ws + (first_state + r) * D + col) = sum;
                if (col == 0) *(f32x2 *)(ws + (size_t)units * S * D + (first_state + r) * 2) = f32x2{M, L * f};
            } else {
                const float inv = M == -INFINITY ? 0.f : 1.f / L;     // (no key at all: O = 0, LSE = -inf)
                vec4 out;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (T)(sum[e] * inv);
                *(vec4 *)(o + (first_row + r) * D + col) = out;
                if (col == 0 && lse != nullptr) lse[first_row + r] = L != 0.f ? (M + __builtin_amdgcn_logf(L)) * 0.69314718055994530942f : -INFINITY;
            }
        }
    }
#endif
}

template <typename T, int D, bool PAGED> int launch_cache8_rows_one(const Cache8Attend &x)
{
    auto kern = sdpa_cache8_rows_kernel<T, D, PAGED>;
    constexpr int lds_bytes = 4 * 2 * GeomRows<D>::TILE + (D == 160 ? 0 : 4 * 32 * 8);
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes); });
    if (attr_err != hipSuccess) return (int)attr_err;
    const LaunchArgs &a = x.a;
    const int units = a.BH * a.splits, row_tiles = (a.S + 31) / 32;
    int log2_parts = 0;
    while (log2_parts < 3 && ((units << log2_parts) & 7) != 0) ++log2_parts;
    if (row_tiles < 2 << log2_parts) log2_parts = 0;
    const int tiles = (row_tiles + (1 << log2_parts) - 1) >> log2_parts;
    const long long groups = ((((long long)units << log2_parts) + 7) / 8) * 8 * tiles;
    const int ranked = a.kv_lens && a.splits == 1 && groups > 512 && a.batches > 1 && a.batches <= kRanked ? a.batches : 0;
    const RowsOrder order{row_tiles, tiles, log2_parts, ranked, divisor((uint32_t)tiles), divisor((uint32_t)a.splits), divisor((uint32_t)a.heads_per_batch),
                          divisor((uint32_t)a.rows_per_head)};
    hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(256), lds_bytes, a.stream, (const T *)a.q, (T *)a.o, a.lse, x.c, a.S, units, order, a.c, a.qsign, a.causal,
                       a.Skv, a.splits, a.ws, a.rows_per_head, a.kv_lens);
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_cache8_rows_dim(const Cache8Attend &x)
{
    return x.c.block_table ? launch_cache8_rows_one<T, D, true>(x) : launch_cache8_rows_one<T, D, false>(x);
}

template <typename T> int launch_cache8_rows(int D, const Cache8Attend &x)
{
    switch (D) {
        case 64: return launch_cache8_rows_dim<T, 64>(x);
        case 96: return launch_cache8_rows_dim<T, 96>(x);
        case 128: return launch_cache8_rows_dim<T, 128>(x);
        default: return launch_cache8_rows_dim<T, 160>(x);
    }
}

}  // namespace tsdpa
