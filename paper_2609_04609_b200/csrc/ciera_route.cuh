// What the layer for a few tokens uses of the router.
#pragma once

#include "ciera_internal.cuh"

namespace ciera {

// the argument checks of ciera_route
int check_route(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens, uint64_t logits_stride,
                const float* bias_dev, const int32_t* experts_dev, const float* weights_dev);

}  // namespace ciera
