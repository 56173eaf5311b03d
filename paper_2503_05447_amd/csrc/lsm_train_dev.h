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

}  // namespace lsm
