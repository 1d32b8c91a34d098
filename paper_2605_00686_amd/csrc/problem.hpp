// What the entry points of both source files ask of a problem.
#pragma once
#include "../../include/moe.h"

namespace moe {

// MOE_OK, or why the library takes no such problem: the same checks for every entry point.
__attribute__((visibility("hidden"))) int check_problem(const moe_problem_t *p);

}  // namespace moe
