// Arguments of the layer norm kernels after host validation (strides in elements).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sva {

constexpr int kNormThreads = 256;  // of a workgroup whose rows are held by 16 to 64 lanes
constexpr int kNormMaxChannels = 16384;

struct RowsView {
  void* p;
  int64_t sb, sn;
};

struct NormArgs {
  RowsView x, dy, y;             // y: the result, or the gradient of x
  const void* w;                 // weight, null: ones
  const void* bias;              // null: zeros
  int64_t w_b, bias_b;           // strides of an entry's weights (0: shared)
  bool w_bf16;
  float unit;                    // added to the weight
  float eps;
  float* mean;                   // [B, N]; forward: written where not null
  float* rstd;
  float* partial;                // [B * parts][2][C]: a workgroup's sums for dw and db (null: an entry has one
                                 // workgroup, which writes them where they belong)
  float* dw;                     // null: not wanted
  float* db;
  int B, N, C;
  int parts;                     // workgroups of an entry
  bool f32, aligned;             // aligned: 16-byte accesses of whole pieces everywhere
};
// How a call's rows are held, and its workspace.
struct NormShape {
  int lanes;                     // of a row: 16, 32, 64, or 0: a workgroup's
  int pieces;                    // of a lane, at most
  int threads, parts;
  size_t ws_bytes;
};
NormShape norm_shape(int B, int N, int C, bool grad, bool per_entry);
hipError_t launch_layer_norm(const NormArgs& a, const NormShape& s, hipStream_t stream);
hipError_t launch_layer_norm_grad(const NormArgs& a, const NormShape& s, int entries, hipStream_t stream);

}  // namespace sva
