// Quantised rows (fp8_rows.hip) as the products of them (fp8_linear.hip) use them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "winattn_common.hpp"

namespace aeris {

inline bool bad16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15) != 0; }

// AERIS_OK if a quantised matrix may have this size, else an AERIS_ERR_ code.
int fp8_check(int64_t n_rows, int64_t cols);
// 0 on success, -1 if the launch failed.
int launch_fp8_quantize_rows(const void* x, bool f32, long long n_rows, int cols, unsigned char* x8,
                             unsigned char* xs, hipStream_t stream);
int launch_fp8_dequantize(const unsigned char* x8, const unsigned char* xs, long long n_rows, int cols, bf16_t* x,
                          hipStream_t stream);
// The first of dy [n_rows, features] and the second of x [n_rows, channels] in one launch.
int launch_fp8_backward_operands(const bf16_t* dy, int features, unsigned char* dy8, unsigned char* dys,
                                 const unsigned char* x8, const unsigned char* xs, int channels, bf16_t* x,
                                 long long n_rows, hipStream_t stream);

}  // namespace aeris
