// Launch interface of the rotation table and of the norm and rotation of queries and keys.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dit {

constexpr int kMaxRopePairs = 64;  // head_dim 128
constexpr int64_t kMaxRowBlocks = 0xFFFFFFFFll / 256;  // a launch takes under 2^32 threads, 256 a workgroup here

struct RopeTableParams {
  const int32_t* positions;  // [n_rows, n_axes]
  float* table;              // [n_rows, n_pairs, 2]
  int64_t n_rows;
  int32_t n_axes, n_pairs;
  float magnitude;
  // Quarter turns per position of every pair, as the sum of two doubles, and the axis of its position.
  double quarters_hi[kMaxRopePairs], quarters_lo[kMaxRopePairs];
  uint8_t axis[kMaxRopePairs];
};
// Loads the code of these kernels on the current device, which the first launch would otherwise do.
hipError_t qk_norm_rope_prepare();
// Workgroups that a call needs (the caller keeps it at kMaxRowBlocks at most); likewise below.
int64_t rope_table_blocks(const RopeTableParams& p);
hipError_t rope_table_launch(const RopeTableParams& p, hipStream_t stream);

enum class HeadNorm : int { kNone = 0, kRms = 1, kLayer = 2 };

struct NormHeadsParams {
  const char* x;          // bf16 rows of n_heads heads, row_stride_b bytes apart
  char* out;              // likewise
  int64_t row_stride_b, out_stride_b;
  const float* weight;    // [D] or nullptr
  const float* bias;      // [D] or nullptr
  int32_t n_heads;
};
struct QkNormRopeParams {
  NormHeadsParams side[2];  // queries, keys (n_heads 0: none)
  const float* table;       // [n_rows, rot_dim / 2, 2] or nullptr
  int64_t n_rows;
  int32_t rot_dim;          // a multiple of 8
  int32_t half;             // pairs (j, j + rot_dim / 2) instead of (2j, 2j + 1)
  float eps;
};
int64_t qk_norm_rope_blocks(const QkNormRopeParams& p, int head_dim);
hipError_t qk_norm_rope_launch(const QkNormRopeParams& p, HeadNorm norm, int head_dim, hipStream_t stream);

}  // namespace dit
