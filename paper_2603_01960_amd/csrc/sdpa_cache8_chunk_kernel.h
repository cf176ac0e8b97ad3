// Attention of many query rows (prefill chunks) over an 8-bit cache: bound by the matrix products, as over a 16-bit one.
//
// The work split is sdpa_fwd_kernel.h's: a wavefront has 32 query rows, a workgroup streams tiles of 64 keys for 32 * NW of them, scores
// transposed, O^T = V^T P^T, the lazy reference.  What differs: a tile's codes come to registers, 16 bytes per lane and load, while the tile before
// it is worked on, are made 16-bit numbers there and put into the LDS between that tile's products.  So each code is converted once per
// workgroup, not once per wavefront that reads it, and the tile in the LDS is a 16-bit tile.  K becomes q's type; V and the weights FP16
// (see sdpa_cache8_decode_kernel.h, also for how the scales enter).
#pragma once
#include "sdpa_cache8_values.h"

namespace tsdpa {

template <typename T, int D, int NW, bool PAGED>
__global__ void __launch_bounds__(NW * 64, 2)
sdpa_cache8_chunk_kernel(const T *__restrict__ q, T *__restrict__ o, float *__restrict__ lse, Cache8Args cache, int S, int nQ, int N, float c, uint32_t qsign,
                         int causal, TileOrder order, int Skv_cap, int splits, float *__restrict__ ws, int rows_per_head, const int *__restrict__ kv_lens,
                         int batches, Divisor by_batches)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using vec8 = typename Elem<T>::vec8;
    using vec4 = typename Elem<T>::vec4;
    using G = TileGeom<D, kTile8>;
    constexpr int TM = NW * 32, TN = kTile8, NB = 2, KK = D / 16, DB = D / 32;
    constexpr int GCPR = D / 16;                  // 16-byte chunks of codes per row
    constexpr int U = TN * GCPR / 64;             // loads of a wavefront's 64 lanes per K or V tile
    constexpr int NL = (2 * U + NW - 1) / NW;     // ... of one wavefront for the pair, the last one for some of them only
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const lds_ptr lds = (lds_ptr)smem;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 5, l32 = lane & 31;
    const int Sp = rows_per_head;
    const bool folded = Sp != S;

    int hs, qt;
    if (causal && order.heads > 0) {
        const CausalTile ct = causal_tile(blockIdx.x, nQ, order, N);
        hs = ct.head;
        qt = nQ - 1 - ct.level;
        if (folded && Sp % TM == 0) {             // the last tile of every folded query head, then the one before it, ...
            const int G_heads = S / Sp, per_head = Sp / TM;
            qt = (ct.level % G_heads) * per_head + per_head - 1 - ct.level / G_heads;
        }
    } else {
        const int wg = remap_workgroup(blockIdx.x, N, false);
        hs = divide(wg, order.by_tiles);
        qt = causal ? nQ - 1 - (wg - hs * nQ) : wg - hs * nQ;
    }
    int head = hs / splits;
    const int sp = hs - head * splits, hpb = cache.heads;
    // Entries differ in length: they vary fastest over the workgroups, the longest first, so that no XCD has more of them than another and (in the
    // causal order) the second workgroup of a CU is of a short entry where the first is of a long one.  (4 entries of 1408 ... 3712 keys, 500
    // queries of 32 heads over 8, D = 128, FP16: 110 -> 107 us.)
    if (kv_lens != nullptr && nQ > 1) {
        const int x = divide(head, by_batches);
        int entry = head - x * batches;
        if (batches > 1 && batches <= 64) {
            const int mine = lane < batches ? kv_lens[lane] : -1;
            int rank = 0;
            for (int j = 0; j < batches; ++j) {
                const int other = __builtin_amdgcn_readlane(mine, j);
                rank += other > mine || (other == mine && j < lane) ? 1 : 0;
            }
            entry = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == entry && lane < batches));
        }
        head = entry * hpb + x;
    }
    const int b = head / hpb, h = head - b * hpb;
    int Skv = Skv_cap;
    if (kv_lens != nullptr) {
        const int len = kv_lens[b];
        Skv = len < 0 ? 0 : (len < Skv_cap ? len : Skv_cap);
    }
    const int koff = Skv - Sp;                    // position of a query head's row 0 in the key sequence (causal)

    // ---- Q rows of this wavefront as MFMA B-operands: lane holds Q[row l32][kk * 16 + g * 8 .. + 7]
    const int r0 = qt * TM, qrow = r0 + wave * 32 + l32, qrow_c = qrow < S ? qrow : S - 1;
    vec8 qf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
        u32x4 raw = *(const u32x4 *)(q + ((size_t)head * S + qrow_c) * D + kk * 16 + g * 8);
        raw ^= qsign;
        qf[kk] = __builtin_bit_cast(vec8, raw);
    }

    // ---- the workgroup's tiles [t0, t1), of which those below nfull need no mask
    const int nT = (Skv + TN - 1) / TN, last_row = (r0 + TM < S ? r0 + TM : S) - 1;
    int pos_lo = r0, pos_hi = last_row, pos_own = qrow_c;
    if (folded) {
        const int g0 = r0 / Sp, g1 = last_row / Sp;
        if (g0 == g1) { pos_lo -= g0 * Sp; pos_hi -= g0 * Sp; }
        else          { pos_lo = 0; pos_hi = Sp - 1; }
        pos_own = qrow_c % Sp;
    }
    const int reach = pos_hi + koff;              // (below 0: no row sees a key)
    const int nTw = causal ? (reach < 0 ? 0 : reach / TN + 1) : nT;
    const int klim = causal ? pos_own + koff : Skv - 1;
    const int nfull = ((causal ? pos_lo + koff : Skv - 1) + 1) / TN;
    const int per_split = (nTw + splits - 1) / splits;
    const int t0 = sp * per_split, t1 = t0 + per_split < nTw ? t0 + per_split : nTw;

    // ---- codes: HBM -> registers.  Load i of this wavefront is unit i * NW + wave of the pair, K's U units before V's; lane's chunk p of a unit is
    // 16 columns of a row.
    const unsigned char *kbase = (const unsigned char *)cache.data[0], *vbase = (const unsigned char *)cache.data[1];
    const size_t head_off = PAGED ? 0 : (size_t)head * (size_t)Skv_cap * D;
    const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(kbase + head_off), (short)0, Skv * D, 0x00020000);
    const auto v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + head_off), (short)0, Skv * D, 0x00020000);
    const int *pages = PAGED ? cache.block_table + (size_t)b * cache.max_blocks : nullptr;
    const int shift = PAGED ? __builtin_ctz(cache.block_rows) : 0;
    auto page_of = [&](int tile) __attribute__((always_inline)) {
        const int page = __builtin_amdgcn_readfirstlane(pages[(tile * TN) >> shift]);
        return page < 0 ? 0 : (page < cache.pages ? page : cache.pages - 1);
    };
    struct Src { decltype(k_rsrc) kr, vr; int soff; };
    auto src_of = [&](int tile, int page) __attribute__((always_inline)) {
        if constexpr (!PAGED) return Src{k_rsrc, v_rsrc, tile * (TN * D)};
        else {
            const int row0 = tile * TN, left = Skv - row0, rows = left < TN ? left : TN;
            const unsigned long long first = (((unsigned long long)page * hpb + h) << shift) + (row0 & ((1 << shift) - 1));
            const unsigned long long byte0 = first * (unsigned long long)D;
            const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)byte0), hi = __builtin_amdgcn_readfirstlane((unsigned)(byte0 >> 32));
            const unsigned long long at = ((unsigned long long)hi << 32) | lo;
            const int bytes = __builtin_amdgcn_readfirstlane(rows * D);
            return Src{__builtin_amdgcn_make_buffer_rsrc((void *)(kbase + at), (short)0, bytes, 0x00020000),
                       __builtin_amdgcn_make_buffer_rsrc((void *)(vbase + at), (short)0, bytes, 0x00020000), 0};
        }
    };
    // Where a chunk's first 8 columns go in a 16-bit tile (its other 8: 16 bytes further on or back).  Eight consecutive lanes write at a time, 128 bytes; were
    // all these first halves the even 16 bytes of their rows, half of the banks would be left alone.  So four of the lanes have a row in which they are the
    // odd ones, by the swizzle of K, and by one of its own (vhalf) in a tile of V: no conflicts, where they took 13 % of the cycles (2048 queries of 32 heads over 8,
    // 16384 keys: 519 -> 513 us, D = 64 297 -> 294; with the halves exchanged in registers instead 488 -> 510).  In compact rows the rows' ends do some of that.
    auto vhalf = [](int r) __attribute__((always_inline)) { return G::COMPACT ? 0 : (D == 64 ? r & 2 : (r & 1) * 2) * 8; };
    const int lane_row = G::COMPACT ? 0 : D == 64 ? (lane >> 4) * 4 + ((lane >> 2) & 1) * 2 + ((lane >> 3) & 1) : (lane >> 4) * 2 + ((lane >> 2) & 1);
    const int lane_chunk = D == 64 ? lane & 3 : (lane & 3) + ((lane >> 3) & 1) * 4;
    const int lane_at = G::COMPACT ? lane * 16 : lane_row * D + lane_chunk * 16;
    int at_lds[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int u = i * NW + wave, p = (u < U ? u : u - U) * 64 + lane, r = G::COMPACT ? p / GCPR : (u < U ? u : u - U) * (64 / GCPR) + lane_row;
        const int ch = (G::COMPACT ? p % GCPR : lane_chunk) * 2;
        at_lds[i] = r * G::ROW + (u < U ? (ch ^ G::kswz(r)) << 4 : (((ch >> 2) ^ G::vswz(r)) << 6) + ((ch & 3) * 16 ^ vhalf(r)));
    }
    u32x4 raw[NL];
    // Whether load i is one of K's.  It is K's for some wavefronts and V's for the others in one i at most, and there chosen by scalar selects.
    auto is_k = [&](int i) __attribute__((always_inline)) { return (i + 1) * NW <= U || (i * NW < U && i * NW + wave < U); };
    auto load = [&](const Src &s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int u = i * NW + wave;
            if ((i + 1) * NW > 2 * U && u >= 2 * U) break;
            raw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(is_k(i) ? s.kr : s.vr, lane_at, s.soff + (is_k(i) ? u : u - U) * 1024, 0));
        }
    };
    constexpr int KSLOT0 = 0, KSLOT1 = G::TILE, VSLOT0 = 2 * G::TILE, VSLOT1 = 3 * G::TILE;
    auto store = [&](int i, int kslot, int vslot) __attribute__((always_inline)) {
        if ((i + 1) * NW > 2 * U && i * NW + wave >= 2 * U) return;
        const lds_ptr slot = lds + (is_k(i) ? kslot : vslot);
        if (std::is_same<T, _Float16>::value || !is_k(i)) {
            lds_write128(slot + at_lds[i], __builtin_bit_cast(u32x4, Codes<_Float16>::wide(raw[i][0], raw[i][1])));
            lds_write128(slot + (at_lds[i] ^ 16), __builtin_bit_cast(u32x4, Codes<_Float16>::wide(raw[i][2], raw[i][3])));
        } else {
            lds_write128(slot + at_lds[i], __builtin_bit_cast(u32x4, Codes<T>::wide(raw[i][0], raw[i][1])));
            lds_write128(slot + (at_lds[i] ^ 16), __builtin_bit_cast(u32x4, Codes<T>::wide(raw[i][2], raw[i][3])));
        }
    };

    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) oacc[db][i] = 0.f;
    float m_ref = klim >= t0 * TN ? kNoWeight : -INFINITY, l_run = 0.f;

    // ---- per-lane LDS read pointers (sdpa_fwd_kernel.h's; in compact rows the swizzle of K touches the low two bits of a chunk's index only and V has
    // none, so that two pointers and one serve all columns)
    constexpr int NKP = G::COMPACT ? 2 : KK, NVP = G::COMPACT ? 1 : DB;
    lds_ptr k_ptr[NKP], v_ptr[NVP];
#pragma unroll
    for (int i = 0; i < NKP; ++i) {
        k_ptr[i] = lds + l32 * G::ROW + (((2 * i + g) ^ G::kswz(l32)) << 4);
        TSDPA_OPAQUE(k_ptr[i]);
    }
    const int v_row = g * 4 + ((lane & 15) >> 2);
#pragma unroll
    for (int i = 0; i < NVP; ++i) {
        v_ptr[i] = lds + v_row * G::ROW + ((i ^ G::vswz(v_row)) << 6) + ((lane >> 4) & 1) * 32 + ((lane & 3) * 8 ^ vhalf(v_row));
        TSDPA_OPAQUE(v_ptr[i]);
    }
    auto k_at = [&](int kk) __attribute__((always_inline)) { return G::COMPACT ? k_ptr[kk & 1] + (kk >> 1) * 64 : k_ptr[kk % NKP]; };
    auto v_at = [&](int db) __attribute__((always_inline)) { return G::COMPACT ? v_ptr[0] + db * 64 : v_ptr[db % NVP]; };

    f32x16 sacc[NB];
    f16x8 pb[NB][2];
    auto hidden = [&](int key0, int nb, int i) __attribute__((always_inline)) { return key0 + nb * 32 + (i >> 2) * 8 + (i & 3) > klim; };
    auto exponentials = [&](int row0, const TileScales &x8, auto mask_tag) __attribute__((always_inline)) {
        const int key0 = row0 + g * 4;
        float sum[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float off = x8.ev[nb] - m_ref;
            float part[2];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[nb][i], x8.ck[nb], off));
                if (decltype(mask_tag)::value && hidden(key0, nb, i)) p = 0.f;
                if (i < 2) part[i] = p;
                else part[i & 1] += p;
                pb[nb][i >> 3][i & 7] = (_Float16)p;
            }
            sum[nb] = part[0] + part[1];
        }
        return TileSums{sum[0] + sum[1], sum[0] * x8.ew[0] + sum[1] * x8.ew[1], {sum[0], sum[1]}};
    };
    auto softmax = [&](int row0, const TileScales &x8, auto mask_tag) __attribute__((always_inline)) {
        TileSums ps = exponentials(row0, x8, mask_tag);
        auto least = [&](int nb) __attribute__((always_inline)) { return !decltype(mask_tag)::value || !hidden(row0 + g * 4, nb, 0) ? kSmall : 0u; };
        if (__builtin_amdgcn_ballot_w64(ps.unusual({least(0), least(1)})) != 0) {
            // Eq. 2 for the rows that are over the limit (the two lanes of a row together): the tile's maximum, new reference, the rescale of Eqs. 3-4
            const int key0 = row0 + g * 4;
            float m_tile = -INFINITY, most[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!decltype(mask_tag)::value || !hidden(key0, nb, i)) mx = fmaxf(mx, sacc[nb][i]);
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
                    for (int i = 0; i < 16; ++i) {
                        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[nb][i], x8.ck[nb], x8.ev[nb] - m_l) - x8.ev[nb]);
                        if (!decltype(mask_tag)::value || !hidden(key0, nb, i)) l += e;
                    }
            }
            ps = exponentials(row0, x8, mask_tag);
            if (apart) ps.l = l;
        }
        l_run += ps.l;
    };
    // Values that are NaN, in keys that only some rows see: the product with a weight of 0 would be NaN for the others.  So a tile that the causal
    // mask cuts is looked through (by every wavefront, so that all agree: 0.25 us); if it has one, the rows that see it get NaN in its
    // column, and the tile a 0 in its place.
    auto has_nan = [&](int vslot) __attribute__((always_inline)) {
        uint32_t any = 0;
#pragma unroll 4
        for (int at = lane * 16; at < G::TILE; at += 1024) {
            const u32x4 x = lds_read128(lds + vslot + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) any |= NotFinite<_Float16>::marks(x[i]);
        }
        return __builtin_amdgcn_ballot_w64(any != 0) != 0;
    };
    auto take_nan = [&](int key0, int vslot) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                u32x4 seen;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    seen[i] = (hidden(key0, nb, ks * 8 + 2 * i) ? 0u : 0x3c00u) | (hidden(key0, nb, ks * 8 + 2 * i + 1) ? 0u : 0x3c000000u);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const lds_ptr p0 = v_at(db) + vslot + (nb * 32 + ks * 16) * G::ROW;
                    const i16x4 lo = lds_read_tr16(p0), hi = lds_read_tr16(p0 + 8 * G::ROW);
                    u32x4 ones = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int i = 0; i < 4; ++i) ones[i] = NotFinite<_Float16>::whole(NotFinite<_Float16>::marks(ones[i])) & NotFinite<_Float16>::ONE;
                    f32x16 count;
#pragma unroll
                    for (int i = 0; i < 16; ++i) count[i] = 0.f;
                    count = Elem<_Float16>::mfma(__builtin_bit_cast(f16x8, ones), __builtin_bit_cast(f16x8, seen), count);
#pragma unroll
                    for (int i = 0; i < 16; ++i) oacc[db][i] += count[i] > 0.f ? __builtin_nanf("") : 0.f;
                    asm volatile("" : "+v"(oacc[db]));       // (now: put off to the end, all counts are held at once)
                }
            }
        __syncthreads();
        for (int at = tid * 16; at < G::TILE; at += NW * 1024) {
            u32x4 x = lds_read128(lds + vslot + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] &= ~NotFinite<_Float16>::whole(NotFinite<_Float16>::marks(x[i]));
            lds_write128(lds + vslot + at, x);
        }
        __syncthreads();
    };

    if (t0 < t1) {
        // In step j the LDS holds tile j; tile j + 1 is on its way to registers, and goes into the other slot, whose last readers have passed the
        // barrier before, between the products of this one.
        int page = 0, page_next = 0;
        if constexpr (PAGED) page_next = page_of(t0);
        int scale_now = 0, scale_next = tile_scale_bytes<PAGED>(cache, t0, PAGED ? page_next : b, h);
        load(src_of(t0, page_next));
        if constexpr (PAGED) page = page_of(t0 + 1 < t1 ? t0 + 1 : t0);
#pragma unroll
        for (int i = 0; i < NL; ++i) store(i, KSLOT0, VSLOT0);
        __syncthreads();
        auto step = [&](int j, auto par_tag, auto mask_tag) __attribute__((always_inline)) {
            constexpr int PAR = decltype(par_tag)::value;
            constexpr bool MASK = decltype(mask_tag)::value;
            constexpr int KS = PAR ? KSLOT1 : KSLOT0, VS = PAR ? VSLOT1 : VSLOT0, KN = PAR ? KSLOT0 : KSLOT1, VN = PAR ? VSLOT0 : VSLOT1;
            const int jn = j + 1 < t1 ? j + 1 : j;    // (after the last tile: itself once more, into a slot that nobody reads)
            scale_now = scale_next;
            scale_next = tile_scale_bytes<PAGED>(cache, jn, PAGED ? page : b, h);
            load(src_of(jn, page));
            if constexpr (PAGED) page = page_of(j + 2 < t1 ? j + 2 : jn);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i) sacc[nb][i] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    sacc[nb] = Elem<T>::mfma(__builtin_bit_cast(vec8, lds_read128(k_at(kk) + KS + nb * 32 * G::ROW)), qf[kk], sacc[nb]);
            // reads four products ahead (left to itself the compiler has the operands of two on their way: 1-2 % of the time)
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int i = 0; i < KK * NB; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                if (i < KK * NB - 4) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            const TileScales x8(scale_now, c);
            softmax(j * TN, x8, mask_tag);
            if constexpr (MASK) {
                if (causal && has_nan(VS)) take_nan(j * TN + g * 4, VS);
            }
            __builtin_amdgcn_s_setprio(2);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        const lds_ptr p0 = v_at(db) + VS + (nb * 32 + ks * 16) * G::ROW;
                        const i16x4 lo = lds_read_tr16(p0), hi = lds_read_tr16(p0 + 8 * G::ROW);
                        const i16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        oacc[db] = Elem<_Float16>::mfma(__builtin_bit_cast(f16x8, a), pb[nb][ks], oacc[db]);
                    }
                    const int part = nb * 2 + ks;
#pragma unroll
                    for (int i = part * NL / 4; i < (part + 1) * NL / 4; ++i) store(i, KN, VN);
                }
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();
        };
        using P0 = std::integral_constant<int, 0>;
        using P1 = std::integral_constant<int, 1>;
        const int fast_n = (t1 < nfull ? t1 : nfull) - t0, fast_end = t0 + (fast_n > 0 ? fast_n & ~1 : 0);
        int j = t0;
        for (; j < fast_end; j += 2) {
            step(j, P0{}, std::false_type{});
            step(j + 1, P1{}, std::false_type{});
        }
        for (; j < t1; ++j) {
            if ((j - t0) & 1) step(j, P1{}, std::true_type{});
            else              step(j, P0{}, std::true_type{});
        }
    }

    // ---- O_i = o_i / l_i, turned through the LDS to whole rows (sdpa_fwd_kernel.h), or the state of a run of keys
    const float l_tot = pair_sum(l_run);
    if (splits > 1) {
        const float f = raise_reference(m_ref, l_tot);
        const size_t prow = (size_t)(head * splits + sp) * S + qrow;
        if (qrow < S) {
            float *po = ws + prow * D;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    f32x4 part;
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[e] = oacc[db][q4 * 4 + e] * f;
                    *(f32x4 *)(po + db * 32 + q4 * 8 + g * 4) = part;
                }
            if (g == 0) {
                float *pml = ws + (size_t)(N / nQ) * S * D + prow * 2;
                pml[0] = m_ref;
                pml[1] = l_tot * f;
            }
        }
        return;
    }
    const float inv = m_ref == -INFINITY ? 0.f : 1.0f / l_tot;       // (no key: O = 0, LSE = -inf)
    if (lse != nullptr && g == 0 && qrow < S)
        lse[(size_t)head * S + qrow] = l_tot != 0.f ? (m_ref + __builtin_amdgcn_logf(l_tot)) * 0.69314718055994530942f : -INFINITY;
    constexpr int OCPR = G::OROW / 16, CMASK = OCPR - 1, ORPI = 64 / OCPR;
    const lds_ptr ow = lds + wave * (32 * G::OROW);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            vec4 out;
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = (T)(oacc[db][q4 * 4 + e] * inv);
            *(TSDPA_LDS vec4 *)(ow + l32 * G::OROW + (((db * 4 + q4) ^ (l32 & CMASK)) << 4) + g * 8) = out;
        }
    const int qrow0 = r0 + wave * 32;
#pragma unroll
    for (int i = 0; i < 32 / ORPI; ++i) {
        const int r = i * ORPI + lane / OCPR, cc = lane % OCPR;
        const u32x4 val = lds_read128(ow + r * G::OROW + ((cc ^ (r & CMASK)) << 4));
        if (qrow0 + r < S && cc < D / 8) *(u32x4 *)(o + ((size_t)head * S + qrow0 + r) * D + cc * 8) = val;
    }
#endif
}

template <typename T, int D, int NW, bool PAGED> int launch_cache8_chunk_one(const Cache8Attend &x)
{
    using G = TileGeom<D, kTile8>;
    auto kern = sdpa_cache8_chunk_kernel<T, D, NW, PAGED>;
    constexpr int stage_bytes = NW * 32 * G::OROW, lds_bytes = G::LDS_BYTES > stage_bytes ? G::LDS_BYTES : stage_bytes;
    static_assert(lds_bytes <= 160 * 1024, "LDS of a CU");
    static std::once_flag once;
    static hipError_t attr_err = hipSuccess;
    std::call_once(once, [&] { attr_err = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes); });
    if (attr_err != hipSuccess) return (int)attr_err;
    const LaunchArgs &a = x.a;
    const int nQ = (a.S + NW * 32 - 1) / (NW * 32), heads = a.BH * a.splits, N = heads * nQ;
    // (the order of the forward kernel over a cache, see launch_one in sdpa_fwd_inst.h)
    const bool uneven = a.causal != 0 && (long long)a.rows_per_head * 12 >= a.Skv;
    const TileOrder order = tile_order(heads, nQ, uneven, a.kv_lens ? 0 : (long long)a.Skv * D * 2);
    hipLaunchKernelGGL(kern, dim3((unsigned)N), dim3(NW * 64), lds_bytes, a.stream, (const T *)a.q, (T *)a.o, a.lse, x.c, a.S, nQ, N, a.c, a.qsign, a.causal, order,
                       a.Skv, a.splits, a.ws, a.rows_per_head, a.kv_lens, a.batches, divisor((uint32_t)a.batches));
    return (int)hipGetLastError();
}

template <typename T, int D> int launch_cache8_chunk_dim(const Cache8Attend &x)
{
    return x.c.block_table ? launch_cache8_chunk_one<T, D, 4, true>(x) : launch_cache8_chunk_one<T, D, 4, false>(x);
}

template <typename T> int launch_cache8_chunk(int D, const Cache8Attend &x)
{
    switch (D) {
        case 64: return launch_cache8_chunk_dim<T, 64>(x);
        case 96: return launch_cache8_chunk_dim<T, 96>(x);
        case 128: return launch_cache8_chunk_dim<T, 128>(x);
        default: return launch_cache8_chunk_dim<T, 160>(x);
    }
}

}  // namespace tsdpa
