// Dropout masks on the host side (dropout.cu), for the kernels that draw them too.
#pragma once

#include "internal.cuh"
#include "philox.cuh"

// The mask of a launch; false: p outside [0, 1].  *drops: whether any word can be below the limit.
bool make_mask(const gnnco_dropout_params* d, philox::Mask* m, bool* drops);
// whether the handle's device is the current one (the launches go there)
bool on_own_device(const gnnco_handle* h);
