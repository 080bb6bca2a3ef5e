// The context behind the C ABI and what its entry points share: errors, the current device, the workspace.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <memory>
#include <string>
#include <vector>

#include "../../include/dit_attn.h"
#include "attn_fwd.h"
#include "plan.h"

namespace dit {

struct CachedPlan {
  std::vector<int32_t> cu;  // key: cu_seqlens contents (of the queries)
  std::vector<int32_t> cu_k;  // key: key boundaries, empty when they are the query boundaries
  int32_t n_heads = 0;
  int32_t head_dim = 0;
  AttnKernel kernel = AttnKernel::kIndependent128;
  int32_t n_splits = 1;  // key chunks per sequence (split-KV); part of the key
  std::vector<WorkItem> host_items;
  WorkItem* dev_items = nullptr;
  uint64_t last_use = 0;
  bool pinned = false;  // a launch that reads dev_items was recorded into a HIP graph: never evicted
};

constexpr size_t kMaxCachedPlans = 32;

}  // namespace dit

struct dit_attn_ctx {
  int device = 0;
  int n_cus = 0;
  uint32_t* sync = nullptr;     // device, 8 words: work counters (zero between launches) and the last launch's clock sample
  uint64_t tick = 0;
  int force_kernel = -1;        // -1: chosen per pack; else a dit::AttnKernel value (dit_attn_set_kernel)
  int last_kernel = -1;         // kernel of the last attention launch (dit_attn_last_launch_kernel)
  int max_splits = 1;           // split-KV: at most this many key chunks per sequence (dit_attn_set_split_kv); 1 = off
  float* workspace = nullptr;   // split-KV partial results and their lse; masked attention's, and its documents by tile
  size_t workspace_bytes = 0;
  bool workspace_pinned = false;        // a captured graph refers to `workspace`: kept until destroy when it is outgrown
  std::vector<float*> retired_workspaces;
  std::vector<std::unique_ptr<dit::CachedPlan>> plans;
  std::string error;
};

namespace dit {

inline int fail(dit_attn_ctx* ctx, int code, const std::string& msg) {
  if (ctx) ctx->error = msg;
  return code;
}

inline int fail_hip(dit_attn_ctx* ctx, hipError_t e, const char* what) {
  // Clear the sticky error so that it is not reported by an unrelated later call.
  (void)hipGetLastError();
  return fail(ctx, DIT_ATTN_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

inline int check_shape_args(const int32_t* cu_seqlens, int32_t n_seqs, int32_t n_heads, int32_t head_dim, std::string& msg) {
  if (!cu_seqlens) {
    msg = "cu_seqlens is NULL";
    return DIT_ATTN_ERR_NULL;
  }
  if (head_dim != 64 && head_dim != 128) {
    msg = "head_dim must be 64 or 128, got " + std::to_string(head_dim);
    return DIT_ATTN_ERR_HEAD_DIM;
  }
  if (n_heads < 1 || n_heads > 65535) {
    msg = "n_heads must be in 1..65535, got " + std::to_string(n_heads);
    return DIT_ATTN_ERR_N_HEADS;
  }
  if (plan_validate(cu_seqlens, n_seqs) != 0) {
    msg = "cu_seqlens must start at 0 and be non-decreasing, n_seqs >= 0";
    return DIT_ATTN_ERR_CU_SEQLENS;
  }
  return DIT_ATTN_OK;
}

struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  hipError_t enter(int dev) {
    hipError_t e = hipGetDevice(&prev);
    if (e != hipSuccess) return e;
    if (prev != dev) {
      e = hipSetDevice(dev);
      if (e != hipSuccess) return e;
      switched = true;
    }
    return hipSuccess;
  }
  ~DeviceGuard() {
    if (switched) (void)hipSetDevice(prev);
  }
};

// Whether `s` is being captured into a graph: such a call may neither allocate nor copy synchronously.
inline bool stream_capturing(hipStream_t s) {
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  const bool capturing = hipStreamIsCapturing(s, &cap) == hipSuccess && cap == hipStreamCaptureStatusActive;
  (void)hipGetLastError();
  return capturing;
}

// Makes the context's workspace at least `need` bytes, on the current device; DIT_ATTN_OK or the error of the call.  What a
// captured call uses stays where it is until the context is destroyed.  `what` names its user in messages.
inline int ensure_workspace(dit_attn_ctx* ctx, size_t need, bool capturing, const char* what) {
  if (need > ctx->workspace_bytes) {
    if (capturing)
      return fail(ctx, DIT_ATTN_ERR_CAPTURE, std::string("the stream is capturing and the ") + what +
                                                 " workspace would have to grow: call once outside the capture first");
    if (ctx->workspace && ctx->workspace_pinned) {
      ctx->retired_workspaces.push_back(ctx->workspace);  // a captured graph still writes there on replay
      ctx->workspace_pinned = false;
    } else if (ctx->workspace) {
      (void)hipFree(ctx->workspace);  // waits for the device: no kernel still uses it
    }
    ctx->workspace = nullptr;
    ctx->workspace_bytes = 0;
    const hipError_t e = hipMalloc(reinterpret_cast<void**>(&ctx->workspace), need);
    if (e != hipSuccess) {
      ctx->workspace = nullptr;
      return fail_hip(ctx, e, (std::string("hipMalloc(") + what + " workspace)").c_str());
    }
    ctx->workspace_bytes = need;
  }
  if (capturing) ctx->workspace_pinned = true;
  return DIT_ATTN_OK;
}

}  // namespace dit
