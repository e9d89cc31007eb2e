// What the files of entry points share.
#pragma once

#include "common.h"

namespace gs {

// The structural check of an access pattern, of its pointer too where kernels will follow it (api.hip).
int check_ap(const gs_ap* a, bool need_data);
// The status of a launch.
int launch_status(hipError_t e);

}  // namespace gs
