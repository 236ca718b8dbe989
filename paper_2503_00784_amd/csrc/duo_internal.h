// What the library's source files share and nobody else sees.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/duo_verify.h"

// DUO_OK, or DUO_ERR_HIP with the text of duo_last_hip_error.
__attribute__((visibility("hidden"))) int duo_internal_hip_ok(hipError_t e, const char* what);
__attribute__((visibility("hidden"))) int duo_internal_check_config(const duo_model_config* c);
// In front of a launch of class `cls` (DUO_PROF_*), and of nothing else: arms the launch with the timer's next event pair, if the timer is on.
__attribute__((visibility("hidden"))) void duo_internal_prof(int cls);
