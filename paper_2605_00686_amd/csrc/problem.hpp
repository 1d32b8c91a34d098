// What the entry points of both source files share.
#pragma once
#include <stddef.h>

#include "../../include/moe.h"

namespace moe {

// MOE_OK, or why the library takes no such problem: the same checks for every entry point.
__attribute__((visibility("hidden"))) int check_problem(const moe_problem_t *p);

// Allow `kernel` so many bytes of dynamic LDS on the current device (remembered: asked of the runtime once).
__attribute__((visibility("hidden"))) int allow_lds(const void *kernel, size_t bytes);

}  // namespace moe
