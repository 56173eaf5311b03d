// What the files of the training operators (lsm_train.h) share on the host's side.
#pragma once
#include "../../include/lsm_train.h"
#include "lsm_block_dev.h"

namespace lsm {

constexpr int kMostExperts = 256, kMostTop = 16, kMostPairs = 1 << 24;

// Stable sort of `count` items into `groups` by their id (lsm_route.hip): item i belongs to group id[i], or with one group to it,
// if id[i] is in [0, limit), else it is left out.  hist: plan_space(count, groups) bytes, or none where that is 0.
size_t plan_space(int64_t count, int groups);
bool enqueue_plan(const int32_t* id, int64_t count, int groups, int limit, int32_t* offsets, int32_t* order, int32_t* place,
                  int32_t* hist, hipStream_t stream);

// The tiles of lsm_product_dev.h: rows and columns, waves along the columns, workgroups of a compute unit at a time.
struct TileSize { int rows, cols, waves, at_once; };
constexpr TileSize kTiles[] = {{256, 256, 2, 1}, {128, 256, 4, 1}, {128, 128, 2, 2}, {64, 256, 4, 2}, {32, 256, 4, 2}, {64, 64, 2, 4}, {32, 128, 4, 4}};
constexpr int kTileKinds = int(sizeof(kTiles) / sizeof(kTiles[0]));
// call(K) with the tile's number as a constant.
#define LSM_KIND(call, kind)                                                                                     \
    ((kind) == 0 ? call(0) : (kind) == 1 ? call(1) : (kind) == 2 ? call(2) : (kind) == 3 ? call(3) : (kind) == 4 ? call(4) \
                                                                                     : (kind) == 5 ? call(5) : call(6))
constexpr int kTileStepBytes = 64;  // of k, a row and step
constexpr int64_t kMostTiles = kAxisThreads / 512;  // of a launch, a workgroup of at most 512 threads each
inline int up(int64_t x, int64_t to) { return int((x + to - 1) / to); }

// The tile with which a product takes least, of those in `kinds` (a bit each): tiles(size) of them, length(size) long.  In microseconds, as
// measured with each tile over sizes from a few tokens to 16384: a compute unit's share of the tiles by the time of a step with its matrix
// cores busy, or the rounds of workgroups by a lone step's latency, or what the steps bring to LDS, rows mostly from the caches; and what
// a round costs beside its steps.  (2047 tokens, 64 experts of 1032 x 2048, 8 a token, backward hidden layer: 398 with 256 rows, 469 with
// 128, 475 with 64; 300 tokens, 1024 x 1024: 103, 92, 104 and 112 with 32.)
template <typename Tiles, typename Length>
int pick_tile_of(bool f32, Tiles tiles, Length length, unsigned kinds) {
    static const float step_bf16[kTileKinds] = {0.78f, 0.5f, 0.26f, 0.3f, 0.18f, 0.085f, 0.1f};
    int best = 0;
    double least = 1e30;
    for (int k = 0; k < kTileKinds; ++k) {
        if (!(kinds >> k & 1)) continue;
        const TileSize& t = kTiles[k];
        const double n = double(tiles(t)), steps = double(up(length(t), f32 ? 16 : 32)), rounds = double(up(int64_t(n), 256 * t.at_once));
        const double share = n > 512 ? n / 256 + 0.3 : double(up(int64_t(n), 256));
        const double busy = share * (f32 ? 3.5 * t.rows * t.cols / 65536. : step_bf16[k]);
        const double brought = n * kTileStepBytes * (t.cols + t.rows / 4) / 12e6;
        // a lone step, and what its workgroups' requests take where there are few of them
        double step = rounds * 0.3 + share * kTileStepBytes * (t.cols + t.rows / 4) / 160e3;
        if (step < busy) step = busy;
        if (step < brought) step = brought;
        const double time = steps * step + rounds * 7.;
        if (time < least) { least = time; best = k; }
    }
    return best;
}
template <typename Tiles>
int pick_tile(bool f32, int64_t K, Tiles tiles, unsigned kinds) {
    return pick_tile_of(f32, tiles, [K](const TileSize&) { return K; }, kinds);
}

}  // namespace lsm
