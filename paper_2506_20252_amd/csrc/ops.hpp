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

// ---- layer.cpp -----------------------------------------------------------------------------------------------------

// 8-bit blocks in the stored form, groups as above; MxbOut with codes == nullptr: not wanted.
struct MxbMat {
  const uint8_t* codes;
  const uint8_t* scales;
};
struct MxbOut {
  uint8_t* codes;
  uint8_t* scales;
};

hipError_t launch_mxb_quantize(Mat x, Elem dtype, int64_t rows, int64_t cols, MxbOut q, hipStream_t stream);
hipError_t launch_mxb_dequantize(MxbMat q, int64_t rows, int64_t cols, MatOut out, Elem dtype, hipStream_t stream);

// What is done with x w^T before it is stored.  Not gated: plus `residual` (p == nullptr: none), to `out`.  Gated: to `out`
// or, where its p is nullptr, to `blocks`; what a checkpoint keeps to saved_a and saved_b.
enum class Act : int { silu, gelu };
struct Epilogue {
  bool gated;
  Act act;
  Mat residual;
  MatOut out;
  Elem dtype;
  MxbOut blocks, saved_a, saved_b;
};
// w has n rows, 2 n where gated; k > 0 or not.
hipError_t launch_mxb_product(MxbMat x, MxMat w, int64_t m, int64_t n, int64_t k, const Epilogue& e, hipStream_t stream);

hipError_t launch_mxb_weight_grad(Mat g, MxbMat x, int64_t rows, int64_t inner, int64_t cols, MatOut out, Elem dtype,
                                  void* workspace, hipStream_t stream);

hipError_t launch_gated_grad(Mat g, Elem dtype, MxbMat a, MxbMat b, int64_t m, int64_t n, Act act, MatOut out,
                             hipStream_t stream);

struct NormArgs {
  Mat x, residual;  // residual.p == nullptr: none
  const void* weight;
  int64_t rows, cols;
  float eps;
  MatOut total, out;  // p == nullptr: not wanted
  MxbOut blocks;
  Elem dtype, weight_dtype, out_dtype;
};
hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream);

struct NormGradArgs {
  Mat g, x, total_grad;  // total_grad.p == nullptr: none
  const void* weight;
  int64_t rows, cols;
  float eps;
  MatOut out;
  float* dweight;
  Elem dtype, x_dtype, weight_dtype;
};
size_t rms_norm_grad_workspace(int64_t rows, int64_t cols);
hipError_t launch_rms_norm_grad(const NormGradArgs& a, void* workspace, hipStream_t stream);

}  // namespace pat
