// Host-side declarations of what runs between the projections of a layer:
// rotary positions, attention over a paged cache, residual norms, low-rank
// adapters (not part of the ABI).  Arguments are validated.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fasq.h"
#include "fasq_internal.h"

namespace fasq {

// One [tokens x heads x D] fp16 tensor: base, token stride, head stride.
struct HeadsView {
  uint16_t* p;
  int64_t ts, hs;
};

// Threads of a launch in x: a grid holds fewer than 2^32 (beyond, some launches
// fail and others run only part of their workgroups), so longer calls go in pieces.
constexpr int64_t kMaxGridThreads = (int64_t(1) << 32) - 1024;

constexpr int kMaxRopeHalf = 128;

struct RopeProblem {
  HeadsView q, q_out, k, v;  // p == nullptr: absent
  int Hq, Hkv;
  int64_t T;
  int D, rot;
  const float* table;
  int64_t table_positions;
  bool interleaved;
  const int32_t* positions;
  const int32_t* slots;
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  float eps;
  fasq_kv_cache cache;
};
hipError_t launch_rope_table(const double* inv_freq, int half, int64_t positions, double scale, float* table,
                             hipStream_t stream);
hipError_t launch_rope_append(const RopeProblem& p, hipStream_t stream);

// What an attention call may have besides scaled products, causality and windows.
struct AttentionMore {
  float softcap;         // 0: none
  const float* slopes;   // NULL: none
  const int32_t* spans;  // NULL: none
  const int32_t* tree;   // NULL: none
  int64_t tree_stride, tree_words;
};

struct AttentionProblem {
  HeadsView q, out;
  int64_t T;
  int Hq, Hkv, D;
  fasq_kv_cache cache;
  const int32_t* pages;
  int64_t page_row_stride, max_pages;
  const int32_t* q_start;
  const int32_t* kv_len;
  int64_t B;
  float scale;
  bool causal;
  int64_t window;
  float* lse;
  void* workspace;
  int64_t workspace_bytes;
  AttentionMore more;
};
int64_t attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D, const DeviceInfo& dev);
hipError_t launch_attention(const AttentionProblem& p, const DeviceInfo& dev, hipStream_t stream);

constexpr int64_t kNormMaxN = 32768;  // values of a row a workgroup holds in registers
struct NormProblem {
  const uint16_t* x;
  const uint16_t* y;
  int64_t M, N;
  const uint16_t* post_weight;
  const uint16_t* gate;
  int64_t gate_stride;
  float scale;
  const uint16_t* weight;
  float eps;
  uint16_t* x_out;
  uint16_t* h;
};
hipError_t launch_residual_norm(const NormProblem& p, hipStream_t stream);

constexpr int kLoraMaxCount = 8;
constexpr int kLoraMaxRank = 256;
constexpr int64_t kLoraMaxN = (int64_t(1) << 31) - (1 << 17);  // a block's features end below 2^31
struct LoraProblem {
  const uint16_t* x;
  int64_t M, K;
  const int32_t* adapters;
  int64_t L;
  int r;
  const float* scales;
  int count;
  const int64_t* N;
  const void* const* A;
  const void* const* B;
  const void* const* base;
  void* const* y;
  void* workspace;
};
int64_t lora_workspace_bytes(int64_t M, int64_t K, int r, int count, const DeviceInfo& dev);
hipError_t launch_lora(const LoraProblem& p, const DeviceInfo& dev, hipStream_t stream);

constexpr int64_t kMaxVocabulary = (int64_t(1) << 30);
struct LogitsProblem {
  const void* logits;
  bool wide;  // fp32
  int64_t stride, R, V;
  fasq_token_rules rules;
  void* out;  // NULL: not written
  bool out_wide;
  int64_t out_stride;
  int32_t* choice;  // NULL: not asked for
  float* lse;
  void* workspace;
};
int64_t logits_workspace_bytes(int64_t R, int64_t V, const DeviceInfo& dev);
hipError_t launch_logits(const LogitsProblem& p, const DeviceInfo& dev, hipStream_t stream);

// The status of a launch, with fasq_last_error() set.
fasq_status launch_status(hipError_t e);

}  // namespace fasq
