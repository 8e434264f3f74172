// What a launch can count.
#pragma once
#include <stdint.h>

namespace psw {

constexpr int64_t kGridThreads = UINT32_MAX;  // threads of a launch in one dimension: workgroups times their threads

}  // namespace psw
