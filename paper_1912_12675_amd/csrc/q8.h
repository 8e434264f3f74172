// 8-bit operands, their layout (psw_q8_quant in include/psw.h) and their
// products (q8.hip, fc8.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "grid.h"

namespace psw {

constexpr int kQ8Block = 128;

// bytes of a row of values
inline int64_t q8_depth(int k) { return ((int64_t)k + kQ8Block - 1) / kQ8Block * kQ8Block; }
// bytes of a row of scales: whole words, which the products load
inline int q8_scales(int k) { return (int)((q8_depth(k) / kQ8Block + 3) / 4 * 4); }
// rows of scales
inline int q8_scale_rows(int rows, bool tiles) { return tiles ? (int)(((int64_t)rows + kQ8Block - 1) / kQ8Block) : rows; }

size_t q8_quant_ws_bytes(int rows, int cols);  // the column sums of the row tiles
bool q8_quant_fits(int rows, int cols, bool rows_alone);  // its threads can be counted; without transposed rows, tiles and sums
hipError_t q8_quant(int rows, int cols, int bf16, const void* x, int64_t ld, bool tiles, uint8_t* q, uint8_t* s,
                    uint8_t* qt, uint8_t* stp, float* colsum, void* ws, hipStream_t st);
// C[m][n] (+)= sum_k A[m][k] B[n][k] of two 8-bit operands (atiles, btiles:
// square blocks); bf16: C is bfloat16, else float.
size_t mm8_ws_bytes(int M, int N, int depth);
bool mm8_fits(int M, int N, int depth, int bf16);
hipError_t mm8(int M, int N, int depth, const uint8_t* A, const uint8_t* sa, bool atiles, const uint8_t* B,
               const uint8_t* sb, bool btiles, const float* bias, int relu, void* C, int bf16, int accumulate, void* ws,
               hipStream_t st);

}  // namespace psw
