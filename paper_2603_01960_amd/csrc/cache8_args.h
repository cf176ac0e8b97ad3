// The 8-bit cache: what host code and kernels share.  See include/tiled_sdpa.h for the format.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sdpa_fwd_launch.h"

namespace tsdpa {

constexpr int kScaleRows = 32;                    // rows of a head that share a scale
// Exponents of scales.  A key that matters, 2^0 ... 2^-24 of the row's greatest, times 2^E or 2^-E stays far from the ends of FP32; times 2^(difference of two exponents,
// 124 at most) it may lie below its normal numbers, which the attention kernels look out for (kSmall and raise_reference in sdpa_cache8_values.h).
constexpr int kScaleMost = 62, kScaleBias = 127;

inline int scale_blocks(int rows) { return rows / kScaleRows + (rows % kScaleRows != 0); }

struct Cache8Args {
    void *data[2];                                // K, V
    unsigned char *scales[2];
    const int *block_table;                       // NULL: dense
    int pages, heads, block_rows, blocks;         // blocks: scales per head and page
    int max_blocks;
};

struct Cache8Rows { const void *data; long long batch, row, head; };

struct Cache8Write {
    Cache8Args c;
    Cache8Rows x[2];
    const int *kv_lens, *new_lens;
    int B, S, capacity;
    int windows;                                  // blocks of 32 rows that an entry's S tokens can touch
    hipStream_t stream;
};

struct Cache8Read {
    Cache8Args c;
    const int *slots;
    void *out[2];
    int B, n;
    hipStream_t stream;
};

struct Cache8Attend {
    Cache8Args c;
    LaunchArgs a;                                 // q, o, lse, BH, S, rows_per_head, kv_lens, heads_per_batch, batches, c, qsign, causal, Skv, splits, ws, ticket, stream
};

#if defined(__HIPCC__)
// The maximum over a wavefront's lanes, of numbers that are not negative: within rows of 16 lanes, then across them.
__device__ __forceinline__ int lanes_max(int x)
{
#if defined(__HIP_DEVICE_COMPILE__)
#define TSDPA_MAX_STEP(ctrl, rows) { const int y = __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false); x = x > y ? x : y; }
    TSDPA_MAX_STEP(0x111, 0xf) TSDPA_MAX_STEP(0x112, 0xf) TSDPA_MAX_STEP(0x114, 0xf) TSDPA_MAX_STEP(0x118, 0xf)      // row_shr
    TSDPA_MAX_STEP(0x142, 0xa) TSDPA_MAX_STEP(0x143, 0xc)                                                          // row_bcast
#undef TSDPA_MAX_STEP
    return __builtin_amdgcn_readlane(x, 63);
#else
    return x;
#endif
}
#endif

int launch_cache8_decode_f16(int D, const Cache8Attend &x);
int launch_cache8_decode_bf16(int D, const Cache8Attend &x);
int launch_cache8_rows_f16(int D, const Cache8Attend &x);
int launch_cache8_rows_bf16(int D, const Cache8Attend &x);
int launch_cache8_chunk_f16(int D, const Cache8Attend &x);
int launch_cache8_chunk_bf16(int D, const Cache8Attend &x);

// In tiled_sdpa.hip: splits of tiles of 128 query rows; the states of a.splits runs combined; a number that no other call has.
int row_tile_splits(int heads, int rows, int Skv, int D);
void merge_states(const LaunchArgs &a, int D, int dtype, bool wide);
unsigned long long new_ticket();

}  // namespace tsdpa
