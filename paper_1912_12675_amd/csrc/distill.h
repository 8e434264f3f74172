// A teacher's top logits and the loss over them (top.hip, distill.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace psw {

size_t top_logits_ws_bytes(int n, int classes, int k);
bool top_logits_fits(int n, int classes, int k, int bf16);  // its threads can be counted
hipError_t top_logits(int n, int classes, int bf16, const void* z, int64_t ld, int k, float tau, float* val, int32_t* idx,
                      float* lse, void* ws, hipStream_t st);
size_t distill_ws_bytes(int n, int classes);
bool distill_fits(int n, int classes, int bf16);
hipError_t distill(int n, int classes, int bf16, const void* z, int64_t ld, int k, const int32_t* idx, const float* val,
                   const float* lse, const int32_t* labels, const float* weight, float tau, float alpha, float* loss,
                   float* row_loss, void* dz, int64_t ldd, void* ws, hipStream_t st);

}  // namespace psw
