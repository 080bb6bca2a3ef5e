// Launch interface of masked attention.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_fwd.h"

namespace dit {

// The sequences travel with the kernel: at most this many a launch, further ones in further launches.
constexpr int kMaskedSeqs = 64;
constexpr int kMaskedBlockM = 128;   // query rows of an item
constexpr int kMaskedFewRows = 32;   // (row, head of a group) columns of an item of the few-rows kernel
constexpr int kMaskedMaxParts = 64;  // parts that the keys of a sequence are split into

struct MaskedSeq {
  int64_t part_row;  // with several parts: row of the workspace's partial results where they begin, q_len rows a part
  uint32_t first;    // index of the sequence's first item in the launch
  uint32_t tile0;    // its first 64-key tile in doc_tiles
  uint32_t join0;    // its first workgroup of the join kernel
  int32_t q_start, q_len, kv_start, kv_len, prefix;
  int32_t parts;     // that its keys are split into
};

// Ids of a 64-key tile: the smallest and largest that are documents (hi < lo: none), and the smallest of all.
struct DocTile {
  int32_t lo, hi, any_lo, unused;
};

// The fields of AttnParams: c_log2, negate, q, k, v, out, lse, n_items, n_heads; with parts also part_out and part_lse.
struct MaskedParams : AttnParams {
  int64_t q_stride_b, k_stride_b, v_stride_b;  // bytes from row to row
  const int32_t* q_doc;    // [Tq] or nullptr
  const int32_t* k_doc;    // [Tk]
  DocTile* doc_tiles;
  const float* slopes;     // [n_heads] or nullptr
  float tanh_in;           // 2 * log2(e) * |scale| / cap
  float cap_log2;          // cap * log2(e)
  float poly_up_to, poly[3];  // cap: raw scores up to it are s (poly[0] + poly[1] s^2 + poly[2] s^4)
  float small;                // and where it is at most this, the largest absolute value of a row stands in for its maximum
  int32_t causal;
  int32_t group;           // query heads per key head
  int32_t part_tiles;      // 64-key tiles of a part
  int32_t n;               // sequences
  MaskedSeq seq[kMaskedSeqs];
};

struct MaskedKind {
  int head_dim;
  bool few_rows, cap, bias, lse;
};

// Loads the code of these kernels on the current device and sets their LDS limits.
hipError_t masked_attn_prepare();
// Doc tiles of the launch's sequences, then the attention kernel on p.n_items workgroups.
hipError_t masked_attn_launch(const MaskedParams& p, const MaskedKind& kind, uint32_t n_doc_tiles, hipStream_t stream);
// out, lse (or nullptr) of the launch's first n sequences, those with several parts.
hipError_t masked_join_launch(const MaskedParams& p, int32_t n, uint32_t n_blocks, int head_dim, hipStream_t stream);
uint32_t masked_join_blocks(const MaskedSeq& s, int n_heads);

}  // namespace dit
