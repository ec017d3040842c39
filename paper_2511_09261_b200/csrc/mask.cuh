// Dropout masks on the host side (dropout.cu), for the kernels that draw them too.
#pragma once

#include "internal.cuh"
#include "philox.cuh"

// The mask of a launch; false: p outside [0, 1].
bool make_mask(const gnnco_dropout_params* d, philox::Mask* m);
void run_dropout(gnnco_handle* h, int32_t dtype, int64_t rows, int32_t F, const void* x, int64_t x_ld, const philox::Mask& m,
                 void* out, int64_t out_ld, cudaStream_t st);
// whether the handle's device is the current one (the launches go there)
bool on_own_device(const gnnco_handle* h);
