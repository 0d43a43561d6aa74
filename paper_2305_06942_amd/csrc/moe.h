// The plan of the tokens-by-expert calls (ebag_a2a_moe_*).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "ebag_a2a.h"
#include "in_flight.h"

namespace ebag {
constexpr int kMaxChoices = 64, kMaxExperts = 512;
}

struct ebag_a2a_moe_plan {
  int device = 0;
  int64_t max_tokens = 0;
  int32_t choices = 0, experts = 0;
  uint32_t* d_counts = nullptr;
  ebag::InFlight sort;
};

namespace ebag {

inline int check_moe_plan(const ebag_a2a_moe_plan* h, int64_t tokens) {
  if (!h) return fail(EBAG_EINVAL, "null plan");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev != h->device)
    return fail(EBAG_EINVAL, "the plan belongs to device %d, but device %d is current", h->device, dev);
  if (tokens < 0 || tokens > h->max_tokens)
    return fail(EBAG_EINVAL, "tokens=%lld outside [0, max_tokens=%lld]", (long long)tokens, (long long)h->max_tokens);
  return EBAG_OK;
}

}  // namespace ebag
