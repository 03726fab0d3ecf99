// Attention of new tokens over a paged cache.
//
// One wave per token and query head, 64 keys at a time with the running
// maximum and sum of a softmax: lanes hold keys for the scores and dimensions
// for the weighted sum of values.
#include <hip/hip_runtime.h>

#include <cmath>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

struct AttentionArgs {
  HeadsView q, out;
  int64_t T, B;
  int Hq, Hkv, D;
  const uint16_t* ck;
  const uint16_t* cv;
  int64_t num_pages;
  uint32_t page_size;
  int64_t page_stride, slot_stride, head_stride;
  const int32_t* pages;
  int64_t page_row_stride;
  int64_t capacity;  // max_pages * page_size
  const int32_t* q_start;
  const int32_t* kv_len;
  float scale;
  bool causal;
  int64_t window;
  float* lse;
};

__device__ __forceinline__ float h2f(uint16_t b) { return (float)__builtin_bit_cast(half_t, b); }

__global__ __launch_bounds__(256) void k_attention_rows(AttentionArgs a) {
  const int64_t row = blockIdx.x * (int64_t)4 + threadIdx.x / kWave;
  if (row >= a.T * a.Hq) return;
  const int lane = threadIdx.x % kWave;
  const int64_t t = row / a.Hq;
  const int h = (int)(row % a.Hq);
  // the request of token t: the last one that starts at or before it
  int64_t lo = 0, hi = a.B;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (a.q_start[mid + 1] <= t) lo = mid + 1;
    else hi = mid;
  }
  if (lo >= a.B || t < a.q_start[lo]) return;
  const int64_t n = a.q_start[lo + 1] - a.q_start[lo];
  int64_t kv = a.kv_len[lo];
  kv = kv < 0 ? 0 : kv > a.capacity ? a.capacity : kv;
  const int64_t pos = kv - n + (t - a.q_start[lo]);
  const int64_t end = a.causal ? (pos + 1 < kv ? pos + 1 : kv) : kv;
  int64_t begin = a.window > 0 ? pos - a.window + 1 : 0;
  if (begin < 0) begin = 0;
  const int32_t* pages = a.pages + lo * a.page_row_stride;
  const int64_t head = (h / (a.Hq / a.Hkv)) * a.head_stride;
  const uint16_t* q = a.q.p + t * a.q.ts + h * a.q.hs;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = begin; j0 < end; j0 += kWave) {
    const int64_t j = j0 + lane;
    float s = -INFINITY;
    int64_t off = 0;
    if (j < end) {
      int64_t page = pages[j / a.page_size];
      page = page < 0 ? 0 : page >= a.num_pages ? a.num_pages - 1 : page;
      off = page * a.page_stride + (j % a.page_size) * a.slot_stride + head;
      s = 0.f;
      for (int i = 0; i < a.D; ++i) s += h2f(q[i]) * h2f(a.ck[off + i]);
      s *= a.scale;
    }
    float top = s;
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
    const float m_new = fmaxf(m, top);
    const float p = j < end ? expf(s - m_new) : 0.f;
    const float keep = m == -INFINITY ? 0.f : expf(m - m_new);
    l = l * keep + wave_sum(p);
    m = m_new;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= keep;
    const int count = (int)(end - j0 < kWave ? end - j0 : kWave);
    for (int c = 0; c < count; ++c) {
      const float pc = __shfl(p, c, kWave);
      const int64_t vo = __shfl(off, c, kWave);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int d = lane + e * kWave;
        if (d < a.D) o[e] += pc * h2f(a.cv[vo + d]);
      }
    }
  }
  uint16_t* out = a.out.p + t * a.out.ts + h * a.out.hs;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int d = lane + e * kWave;
    if (d < a.D) out[d] = begin < end ? f32_to_f16_bits(o[e] / l) : 0;
  }
  if (a.lse != nullptr && lane == 0) a.lse[t * a.Hq + h] = begin < end ? m + logf(l) : -INFINITY;
}

}  // namespace

int64_t attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D, const DeviceInfo& dev) { return 0; }

hipError_t launch_attention(const AttentionProblem& p, const DeviceInfo& dev, hipStream_t stream) {
  AttentionArgs a = {};
  a.q = p.q;
  a.out = p.out;
  a.T = p.T;
  a.B = p.B;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.D = p.D;
  a.ck = static_cast<const uint16_t*>(p.cache.k);
  a.cv = static_cast<const uint16_t*>(p.cache.v);
  a.num_pages = p.cache.num_pages;
  a.page_size = (uint32_t)p.cache.page_size;
  a.page_stride = p.cache.page_stride;
  a.slot_stride = p.cache.slot_stride;
  a.head_stride = p.cache.head_stride;
  a.pages = p.pages;
  a.page_row_stride = p.page_row_stride;
  a.capacity = p.max_pages * p.cache.page_size;
  a.q_start = p.q_start;
  a.kv_len = p.kv_len;
  a.scale = p.scale;
  a.causal = p.causal;
  a.window = p.window;
  a.lse = p.lse;
  return launch_kernel(k_attention_rows, dim3((unsigned)((p.T * p.Hq + 3) / 4)), dim3(256), 0, stream, a);
}

}  // namespace fasq
