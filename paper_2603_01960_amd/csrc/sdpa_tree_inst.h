// Instantiates the forward kernel for trees of drafted tokens over a cache (KV = 5, 6) for one (element type, head dim): the
// forms that pick_tree and, up to 32 rows, pick_streams_kv (tiled_sdpa.hip) choose.
#pragma once
#include "sdpa_fwd_inst.h"

namespace tsdpa {

constexpr int tree_tile_n(int D) { return D == 160 ? 32 : 64; }

template <typename T, int D> int launch_tree_plain(int tile_m, const LaunchArgs &a)
{
    constexpr int TN = tree_tile_n(D);
    if (tile_m != 128) return (int)hipErrorInvalidValue;
    return a.block_table ? launch_one<T, D, 4, TN, 6>(a) : launch_one<T, D, 4, TN, 5>(a);
}

using LaunchTree = int (*)(int tile_m, const LaunchArgs &a);

// 32 rows with weights in halves (pick_halves): in translation units of their own (sdpa_tree_*_halves.hip), up to D = 128
template <typename T, int D> int launch_tree_halved(int tile_m, const LaunchArgs &a)
{
    if (tile_m != 32 || a.streams != 4) return (int)hipErrorInvalidValue;
    return a.block_table ? launch_one<T, D, 1, 32, 8, 4>(a) : launch_one<T, D, 1, 32, 7, 4>(a);
}

template <typename T, int D, int KV> int launch_tree_streams(int tile_m, const LaunchArgs &a)
{
    switch (tile_m * 10 + a.streams) {
        case 324: return launch_one<T, D, 1, 32, KV, 4>(a);
        case 642: return launch_one<T, D, 2, 32, KV, 2>(a);
    }
    return (int)hipErrorInvalidValue;
}

template <typename T, int D> int launch_tree(int tile_m, const LaunchArgs &a, LaunchTree plain, LaunchTree halved)
{
    if (a.streams <= 1) return plain(tile_m, a);
    if (a.halves) return halved ? halved(tile_m, a) : (int)hipErrorInvalidValue;
    return a.block_table ? launch_tree_streams<T, D, 6>(tile_m, a) : launch_tree_streams<T, D, 5>(tile_m, a);
}

}  // namespace tsdpa
