// What the files of entry points share.
#pragma once

#include "common.h"

namespace gs {

// The structural check of an access pattern, of its pointer too where kernels will follow it (api.hip).
int check_ap(const gs_ap* a, bool need_data);
// The status of a launch.
int launch_status(hipError_t e);
// Do the bytes of two access patterns overlap?  (Empty tensors overlap nothing.)
bool overlaps(const gs_ap* a, const gs_ap* b);

}  // namespace gs
