// The attention kernel for many queries, as the entry point sees it.
#pragma once

#include "ans_attend.cuh"

namespace ansb {
namespace blk {

constexpr uint32_t kAtLongest = 1u << 30;              // tokens of a sequence

struct AtPlan {
  uint32_t tiles, splits;
  size_t room;
};
void plan_tiles(const AttendArgs& a, int sms, AtPlan& p);
int launch_tiles(const AttendArgs& a, const AtPlan& p, cudaStream_t st);

}  // namespace blk
}  // namespace ansb
