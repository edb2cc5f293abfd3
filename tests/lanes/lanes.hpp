#pragma once
#include <hip/hip_runtime.h>

#include <random>

namespace lanes {
extern std::mt19937 order;  // of work groups and waves
}
