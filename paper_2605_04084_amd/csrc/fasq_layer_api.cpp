// libfasq C ABI: what runs between a layer's projections.  Argument checks
// (no HIP call before they pass) and hand-over to the launchers.
#include "fasq.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "fasq_layer.h"

namespace fasq {

namespace {

// No exception leaves a C entry: a text that cannot be kept is dropped.
fasq_status fail(fasq_status s, const char* what, const char* more = "") {
  char text[256];
  std::snprintf(text, sizeof(text), "%s%s", what, more);
  try {
    set_last_error(text);
  } catch (...) {
  }
  return s;
}

fasq_status bad(const char* msg) { return fail(FASQ_ERR_INVALID_ARG, msg); }

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr int kMaxHeads = 65536;
constexpr int64_t kMaxTokens = int64_t(1) << 24;  // tokens of one call
constexpr int64_t kMaxRequests = int64_t(1) << 16;  // each tile of attention is looked up among them
constexpr int64_t kMaxStride = int64_t(1) << 40;

bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride; }

// A heads view of the caller: sizes, alignment of fp16, strides that do not
// fold (a head's D values lie side by side).
const char* check_view(const void* p, int64_t ts, int64_t hs) {
  if (misaligned(p, 2)) return "fp16 tensors must be 2-byte aligned";
  if (!stride_ok(ts) || !stride_ok(hs)) return "strides must lie in [0, 2^40]";
  return nullptr;
}

// Of what is written: neighbouring rows of D values lie apart (a broadcast
// tensor's do not).
bool rows_overlap(int64_t D, int64_t count, int64_t stride) { return count > 1 && stride < D; }

const char* check_cache(const fasq_kv_cache* c) {
  if (c == nullptr) return "cache is NULL";
  if (c->k == nullptr || c->v == nullptr) return "a cache pointer is NULL";
  if (misaligned(c->k, 2) || misaligned(c->v, 2)) return "the cache must be 2-byte aligned";
  if (c->num_pages < 1 || c->page_size < 1) return "num_pages and page_size must be >= 1";
  if (c->num_pages > INT32_MAX / c->page_size) return "num_pages * page_size must fit in 31 bits";
  if (!stride_ok(c->page_stride) || !stride_ok(c->slot_stride) || !stride_ok(c->head_stride))
    return "strides must lie in [0, 2^40]";
  return nullptr;
}

}  // namespace

fasq_status launch_status(hipError_t e) {
  if (e != hipSuccess) return fail(FASQ_ERR_HIP, "kernel launch: ", hipGetErrorString(e));
  set_last_error("");
  return FASQ_OK;
}

}  // namespace fasq

using fasq::bad;

extern "C" {

fasq_status fasq_rope_table(const double* inv_freq, int half, int64_t positions, double scale, float* table,
                            hipStream_t stream) {
  if (inv_freq == nullptr || table == nullptr) return bad("a buffer pointer is NULL");
  if (half < 1 || half > fasq::kMaxRopeHalf) return bad("half must lie in [1, 128]");
  if (positions < 1 || positions > (int64_t(1) << 31)) return bad("positions must lie in [1, 2^31]");
  if (fasq::misaligned(table, 8)) return bad("table must be 8-byte aligned");
  return fasq::launch_status(fasq::launch_rope_table(inv_freq, half, positions, scale, table, stream));
}

fasq_status fasq_rope_append(const void* q, int64_t q_ts, int64_t q_hs, int Hq, void* q_out, int64_t qo_ts,
                             int64_t qo_hs, const void* k, int64_t k_ts, int64_t k_hs, const void* v, int64_t v_ts,
                             int64_t v_hs, int Hkv, int64_t T, int D, const float* table, int64_t table_positions,
                             int rot, int interleaved, const int32_t* positions, const int32_t* slots,
                             const void* q_norm, const void* k_norm, float eps, const fasq_kv_cache* cache,
                             hipStream_t stream) {
  if (T < 0 || T > fasq::kMaxTokens) return bad("T must lie in [0, 2^24]");
  if (D < 1 || D > 256) return bad("D must lie in [1, 256]");
  if (rot < 0 || rot > D || rot % 2 != 0) return bad("rot must be even and lie in [0, D]");
  if (T == 0) return fasq::launch_status(hipSuccess);  // buffers of no tokens may be NULL
  if ((q == nullptr) != (q_out == nullptr)) return bad("q and q_out are given together or not at all");
  if ((k == nullptr) != (v == nullptr)) return bad("k and v are given together or not at all");
  if (q == nullptr && k == nullptr) return bad("there is nothing to do: q and k are NULL");
  if (q != nullptr && (Hq < 1 || Hq > fasq::kMaxHeads)) return bad("Hq must lie in [1, 65536]");
  if (k != nullptr && (Hkv < 1 || Hkv > fasq::kMaxHeads)) return bad("Hkv must lie in [1, 65536]");
  if (rot > 0) {
    if (table == nullptr || positions == nullptr) return bad("a buffer pointer is NULL");
    if (fasq::misaligned(table, 8)) return bad("table must be 8-byte aligned");
    if (table_positions < 1 || table_positions > (int64_t(1) << 31)) return bad("table_positions must lie in [1, 2^31]");
  }
  if ((q_norm != nullptr || k_norm != nullptr) && !(eps > 0.f && std::isfinite(eps)))
    return bad("eps must be positive and finite");
  if (fasq::misaligned(q_norm, 2) || fasq::misaligned(k_norm, 2)) return bad("fp16 tensors must be 2-byte aligned");
  const char* why = nullptr;
  if (q != nullptr) {
    if ((why = fasq::check_view(q, q_ts, q_hs)) || (why = fasq::check_view(q_out, qo_ts, qo_hs))) return bad(why);
    if (q == q_out && (q_ts != qo_ts || q_hs != qo_hs)) return bad("q_out = q needs the strides of q");
    if (fasq::rows_overlap(D, T, qo_ts) || fasq::rows_overlap(D, Hq, qo_hs)) return bad("rows of q_out overlap");
  }
  if (k != nullptr) {
    if ((why = fasq::check_view(k, k_ts, k_hs)) || (why = fasq::check_view(v, v_ts, v_hs)) ||
        (why = fasq::check_cache(cache)))
      return bad(why);
    if (fasq::rows_overlap(D, cache->num_pages, cache->page_stride) ||
        fasq::rows_overlap(D, cache->page_size, cache->slot_stride) || fasq::rows_overlap(D, Hkv, cache->head_stride))
      return bad("rows of the cache overlap");
    if (slots == nullptr) return bad("a buffer pointer is NULL");
  }
  fasq::RopeProblem p = {};
  p.q = {static_cast<uint16_t*>(const_cast<void*>(q)), q_ts, q_hs};
  p.q_out = {static_cast<uint16_t*>(q_out), qo_ts, qo_hs};
  p.k = {static_cast<uint16_t*>(const_cast<void*>(k)), k_ts, k_hs};
  p.v = {static_cast<uint16_t*>(const_cast<void*>(v)), v_ts, v_hs};
  p.Hq = q ? Hq : 0;
  p.Hkv = k ? Hkv : 0;
  p.T = T;
  p.D = D;
  p.rot = rot;
  p.table = table;
  p.table_positions = rot > 0 ? table_positions : 0;
  p.interleaved = interleaved != 0;
  p.positions = positions;
  p.slots = slots;
  p.q_norm = static_cast<const uint16_t*>(q_norm);
  p.k_norm = static_cast<const uint16_t*>(k_norm);
  p.eps = eps;
  if (k != nullptr) p.cache = *cache;
  return fasq::launch_status(fasq::launch_rope_append(p, stream));
}

fasq_status fasq_paged_attention(const void* q, int64_t q_ts, int64_t q_hs, int64_t T, int Hq,
                                 const fasq_kv_cache* cache, int Hkv, int D, const int32_t* pages,
                                 int64_t page_row_stride, int64_t max_pages, const int32_t* q_start,
                                 const int32_t* kv_len, int64_t B, float scale, int causal, int64_t window, void* out,
                                 int64_t out_ts, int64_t out_hs, float* lse, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream) {
  if (T < 0 || T > fasq::kMaxTokens) return bad("T must lie in [0, 2^24]");
  if (B < (T > 0 ? 1 : 0) || B > fasq::kMaxRequests) return bad("B must lie in [1, 2^16] (0 only with T = 0)");
  if (Hkv < 1 || Hq < 1 || Hq > fasq::kMaxHeads || Hq % Hkv != 0) return bad("Hq must be a multiple of Hkv, both >= 1");
  if (T * (Hq / Hkv) > (int64_t(1) << 30)) return bad("T * Hq / Hkv must be at most 2^30");
  if (D < 1) return bad("D must be >= 1");
  if (D % 8 != 0 || D > 256) return fasq::fail(FASQ_ERR_UNSUPPORTED, "attention needs D a multiple of 8, at most 256");
  if (max_pages < (T > 0 ? 1 : 0) || max_pages > INT32_MAX || page_row_stride < 0 || page_row_stride > fasq::kMaxStride)
    return bad("max_pages must be >= 1 and the page table's stride must not be negative");
  if (window < 0) return bad("window must be >= 0");
  if (std::isnan(scale)) return bad("scale must be a number");
  if (workspace_bytes < 0) return bad("workspace_bytes must be >= 0");
  if (T == 0) return fasq::launch_status(hipSuccess);  // buffers of no tokens may be NULL
  if (q == nullptr || out == nullptr || pages == nullptr || q_start == nullptr || kv_len == nullptr)
    return bad("a buffer pointer is NULL");
  const char* why = nullptr;
  if ((why = fasq::check_view(q, q_ts, q_hs)) || (why = fasq::check_view(out, out_ts, out_hs)) ||
      (why = fasq::check_cache(cache)))
    return bad(why);
  if (fasq::rows_overlap(D, T, out_ts) || fasq::rows_overlap(D, Hq, out_hs)) return bad("rows of out overlap");
  if (cache->page_size > (INT32_MAX - 1023) / max_pages)
    return bad("max_pages * page_size must fit in 31 bits, up to 2^31 - 1024");
  if (fasq::misaligned(cache->k, 16) || fasq::misaligned(cache->v, 16) ||
      (cache->page_stride | cache->slot_stride | cache->head_stride) % 8 != 0)
    return bad("the cache must be 16-byte aligned, its strides multiples of 8");
  if (workspace != nullptr && fasq::misaligned(workspace, 16)) return bad("workspace must be 16-byte aligned");
  if (out == q) return bad("out must not be q");
  fasq::DeviceInfo dev;
  const hipError_t e = fasq::device_info(&dev);
  if (e != hipSuccess)
    return fasq::fail(FASQ_ERR_HIP, "querying the current device: ", hipGetErrorString(e));
  fasq::AttentionProblem p = {};
  p.q = {static_cast<uint16_t*>(const_cast<void*>(q)), q_ts, q_hs};
  p.out = {static_cast<uint16_t*>(out), out_ts, out_hs};
  p.T = T;
  p.Hq = Hq;
  p.Hkv = Hkv;
  p.D = D;
  p.cache = *cache;
  p.pages = pages;
  p.page_row_stride = page_row_stride;
  p.max_pages = max_pages;
  p.q_start = q_start;
  p.kv_len = kv_len;
  p.B = B;
  p.scale = scale;
  p.causal = causal != 0;
  p.window = window;
  p.lse = lse;
  p.workspace = workspace;
  p.workspace_bytes = workspace_bytes;
  return fasq::launch_status(fasq::launch_attention(p, dev, stream));
}

int64_t fasq_paged_attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D) {
  if (T < 0 || T > fasq::kMaxTokens || B < (T > 0 ? 1 : 0) || B > fasq::kMaxRequests) return -1;
  if (Hkv < 1 || Hq < 1 || Hq > fasq::kMaxHeads || Hq % Hkv != 0 || D < 8 || D > 256 || D % 8 != 0) return -1;
  if (T * (Hq / Hkv) > (int64_t(1) << 30)) return -1;
  if (T == 0) return 0;
  fasq::DeviceInfo dev;
  if (fasq::device_info(&dev) != hipSuccess) return -1;
  return fasq::attention_workspace_bytes(T, B, Hq, Hkv, D, dev);
}

fasq_status fasq_residual_norm(const void* x, const void* y, int64_t M, int64_t N, const void* post_weight,
                               const void* gate, int64_t gate_stride, float scale, const void* weight, float eps,
                               void* x_out, void* h, hipStream_t stream) {
  if (M < 0 || M > fasq::kMaxTokens) return bad("M must lie in [0, 2^24]");
  if (N < 1) return bad("N must be >= 1");
  if (N > fasq::kNormMaxN) return fasq::fail(FASQ_ERR_UNSUPPORTED, "rows of more than 32768 values");
  if (!(eps > 0.f && std::isfinite(eps))) return bad("eps must be positive and finite");
  if (M == 0) return fasq::launch_status(hipSuccess);  // buffers of no tokens may be NULL
  if (x == nullptr) return bad("a buffer pointer is NULL");
  if (y == nullptr && (post_weight != nullptr || gate != nullptr)) return bad("post_weight and gate need y");
  if ((weight == nullptr) != (h == nullptr)) return bad("weight and h are given together or not at all");
  if (x_out == nullptr && h == nullptr) return bad("there is nothing to write: x_out and h are NULL");
  if (h != nullptr && h == x_out) return bad("h and x_out must differ");
  if (gate != nullptr && gate_stride != 0 && gate_stride != N) return bad("gate_stride must be 0 or N");
  const void* all[] = {x, y, post_weight, gate, weight, x_out, h};
  for (const void* p : all)
    if (fasq::misaligned(p, 2)) return bad("fp16 tensors must be 2-byte aligned");
  fasq::NormProblem p = {};
  p.x = static_cast<const uint16_t*>(x);
  p.y = static_cast<const uint16_t*>(y);
  p.M = M;
  p.N = N;
  p.post_weight = static_cast<const uint16_t*>(post_weight);
  p.gate = static_cast<const uint16_t*>(gate);
  p.gate_stride = gate_stride;
  p.scale = scale;
  p.weight = static_cast<const uint16_t*>(weight);
  p.eps = eps;
  p.x_out = static_cast<uint16_t*>(x_out);
  p.h = static_cast<uint16_t*>(h);
  return fasq::launch_status(fasq::launch_residual_norm(p, stream));
}

int64_t fasq_lora_workspace_bytes(int64_t M, int64_t K, int r, int count) {
  if (M < 0 || M > fasq::kMaxTokens || K < 1 || K > (int64_t(1) << 40) || r < 1 || r > fasq::kLoraMaxRank || count < 1 ||
      count > fasq::kLoraMaxCount)
    return -1;
  if (M == 0) return 0;
  fasq::DeviceInfo dev;
  if (fasq::device_info(&dev) != hipSuccess) return -1;
  return fasq::lora_workspace_bytes(M, K, r, count, dev);
}

fasq_status fasq_lora_batched(const void* x, int64_t M, int64_t K, const int32_t* adapters, int64_t L, int r,
                              const float* scales, int count, const int64_t* N, const void* const* A,
                              const void* const* B, const void* const* base, void* const* y, void* workspace,
                              int64_t workspace_bytes, hipStream_t stream) {
  if (M < 0 || M > fasq::kMaxTokens) return bad("M must lie in [0, 2^24]");
  if (K < 1 || r < 1 || L < 1 || L > INT32_MAX) return bad("K, r and L must be >= 1");
  if (count < 1 || count > fasq::kLoraMaxCount) return bad("count must lie in [1, 8]");
  if (r > fasq::kLoraMaxRank) return fasq::fail(FASQ_ERR_UNSUPPORTED, "adapters of a rank above 256");
  if (K > (int64_t(1) << 40) / r || (M > 0 && K > (int64_t(1) << 40) / M)) return bad("problem too large");
  if (M == 0) return fasq::launch_status(hipSuccess);  // buffers of no tokens may be NULL
  if (N == nullptr || A == nullptr || B == nullptr || base == nullptr || y == nullptr) return bad("an array is NULL");
  if (x == nullptr || adapters == nullptr || scales == nullptr) return bad("a buffer pointer is NULL");
  if (fasq::misaligned(x, 2)) return bad("fp16 tensors must be 2-byte aligned");
  for (int i = 0; i < count; ++i) {
    const char* why = nullptr;
    if (N[i] < 1 || N[i] > fasq::kLoraMaxN) why = "N must lie in [1, 2^31 - 2^17]";
    else if (A[i] == nullptr || B[i] == nullptr || y[i] == nullptr) why = "a buffer pointer is NULL";
    else if (fasq::misaligned(A[i], 2) || fasq::misaligned(B[i], 2) || fasq::misaligned(base[i], 2) ||
             fasq::misaligned(y[i], 2))
      why = "fp16 tensors must be 2-byte aligned";
    if (why != nullptr) {
      char at[32];
      std::snprintf(at, sizeof(at), "projection %d: ", i);
      return fasq::fail(FASQ_ERR_INVALID_ARG, at, why);
    }
  }
  fasq::DeviceInfo dev;
  const hipError_t e = fasq::device_info(&dev);
  if (e != hipSuccess)
    return fasq::fail(FASQ_ERR_HIP, "querying the current device: ", hipGetErrorString(e));
  const int64_t need = fasq::lora_workspace_bytes(M, K, r, count, dev);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need))
    return bad("workspace smaller than fasq_lora_workspace_bytes()");
  if (fasq::misaligned(workspace, 16)) return bad("workspace must be 16-byte aligned");
  fasq::LoraProblem p = {};
  p.x = static_cast<const uint16_t*>(x);
  p.M = M;
  p.K = K;
  p.adapters = adapters;
  p.L = L;
  p.r = r;
  p.scales = scales;
  p.count = count;
  p.N = N;
  p.A = A;
  p.B = B;
  p.base = base;
  p.y = y;
  p.workspace = workspace;
  return fasq::launch_status(fasq::launch_lora(p, dev, stream));
}

}  // extern "C"
