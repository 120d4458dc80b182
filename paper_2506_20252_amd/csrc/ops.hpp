// Operators of pat_ops.h: what the C entry points hand to the kernels.  Sizes,
// strides and pointers have been checked when a launch function is called.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace pat {

// Keeps `e` for pat_last_hip_error().
void record_hip_error(hipError_t e);

inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

// Types as template tags' values: the kernels handle float32 and bfloat16.
enum class Elem : int { f32, b16 };

// A row-major matrix: address of its first element, distance of rows in elements.
struct Mat {
  const void* p;
  int64_t stride;
};
struct MatOut {
  void* p;
  int64_t stride;
};

// 4-bit blocks in the stored form, `groups` groups of 128 values a row.
struct MxMat {
  const uint8_t* codes;
  const uint8_t* scales;
};

inline int64_t groups_of(int64_t cols) { return (cols + 127) / 128; }

hipError_t launch_mx_quantize(Mat x, Elem dtype, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream);
hipError_t launch_mx_dequantize(MxMat q, int64_t rows, int64_t cols, MatOut out, Elem dtype, hipStream_t stream);

hipError_t launch_mx_matmul(MxMat a, MxMat b, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype, hipStream_t stream);
size_t mx_linear_workspace(int64_t m, int64_t n, int64_t k);
hipError_t launch_mx_linear(Mat x, Elem x_dtype, MxMat w, int64_t m, int64_t n, int64_t k, MatOut out, Elem dtype,
                            void* workspace, hipStream_t stream);
size_t mx_grad_workspace(int64_t rows, int64_t inner, int64_t cols);
hipError_t launch_mx_grad(Mat g, bool transposed, MxMat q, int64_t rows, int64_t inner, int64_t cols, MatOut out,
                          Elem dtype, void* workspace, hipStream_t stream);

hipError_t launch_embedding(const void* tokens, int token_bytes, int64_t ntokens, Mat table, Elem table_dtype,
                            int64_t first, int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype,
                            hipStream_t stream);
size_t embedding_grad_workspace(int64_t ntokens, int64_t rows, int64_t cols);
hipError_t launch_embedding_grad(const void* tokens, int token_bytes, int64_t ntokens, Mat g, Elem g_dtype, int64_t first,
                                 int64_t rows, int64_t cols, float scale, MatOut out, Elem dtype, void* workspace,
                                 hipStream_t stream);

struct DropoutArgs {
  Mat x;
  Mat residual;  // p == nullptr: none
  MatOut out;
  int64_t rows, cols;
  uint32_t drop;  // P: a place's 16 bits below it drop the element; 65536 drops all
  float scale;    // 65536 / (65536 - P)
  uint64_t seed, index, index_stride;
};
hipError_t launch_dropout(const DropoutArgs& a, Elem dtype, hipStream_t stream);

}  // namespace pat
