// What the layer for a few tokens uses of the router.
#pragma once

#include "ciera_internal.cuh"

namespace ciera {

// the argument checks of ciera_route
int check_route(const ciera_route_config* config, int dtype, const void* logits_dev, uint64_t n_tokens, uint64_t logits_stride,
                const float* bias_dev, const int32_t* experts_dev, const float* weights_dev);

// The layer's kernel comes behind the router's and begins before that has ended.  Other than kernels do otherwise (pdl_wait in
// ciera_internal.cuh), it reads x and writes its workspace before its own pdl_wait().  That holds because each of the router's kernels
// calls pdl_wait() first of all: when all of its blocks have, which is when the layer's kernel may begin, whatever came before the router has
// ended and can be seen.  A router that let others begin before that would have the layer read an x that is still being written.

}  // namespace ciera
