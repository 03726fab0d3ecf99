// From logits to tokens: penalties, biases, a grammar's mask and the
// temperature over rows of a vocabulary, the likeliest token and the logarithm
// of the softmax sum.
//
//   k_logits       a slice of a row a workgroup: the slice's tokens are counted
//                  in LDS, then its logits pass once from memory to memory
//   k_logits_join  joins what a row's slices found
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

typedef half8_t half8_any __attribute__((aligned(2)));
typedef float float8_t __attribute__((ext_vector_type(8)));
typedef float8_t float8_any __attribute__((aligned(4)));
typedef int int4_t __attribute__((ext_vector_type(4)));
typedef int4_t int4_any __attribute__((aligned(4)));

constexpr int kThreads = 256, kEach = 8;  // threads of a workgroup, neighbouring logits of a thread
constexpr uint32_t kInPrompt = 0x80000000u;

// What a slice of a row found.
struct Found {
  uint64_t best;  // order_of() of the largest logit, then its index's complement
  float m, sum;   // the largest logit that is a number, the sum of exp(x - m)
};

struct LogitsArgs {
  const void* logits;
  void* out;
  bool out_wide;               // fp32
  int64_t stride, out_stride;  // elements between rows
  int64_t R, first;            // the launch's first workgroup of all
  int V, slices;
  int S;
  const int32_t* requests;
  const int32_t* tokens;
  int64_t token_stride;
  int max_tokens;
  const int32_t* prompt_len;
  const int32_t* token_count;
  const float *repetition, *presence, *frequency, *temperature;
  const int32_t* bias_ids;
  const float* bias_values;
  int max_bias;
  const uint8_t* allowed;
  int64_t allowed_stride;  // bytes
  const int32_t* draft_tokens;
  const int32_t* q_start;
  const int32_t* tree;
  int64_t tree_stride;
  int tree_words;
  bool counted, finds;  // tokens are counted; choice or lse is asked for
  Found* found;         // [R][slices], with more than one
  int32_t* choice;
  float* lse;
};

// Larger for larger logits; NaN above all, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderOfNone = ~0xFF800000u;  // of -inf

// exp(x - m) for a finite m or x <= m = +inf.
__device__ __forceinline__ float weight_of(float x, float m) {
  return x == m ? 1.f : __builtin_amdgcn_exp2f((x - m) * 1.4426950408889634f);
}

__device__ __forceinline__ void join(Found& a, const Found& b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) {
    a.sum += b.sum;  // 0, or NaN
  } else {
    a.sum = (a.m == -INFINITY ? a.sum : a.sum * weight_of(a.m, m)) + (b.m == -INFINITY ? b.sum : b.sum * weight_of(b.m, m));
  }
  a.m = m;
  a.best = a.best > b.best ? a.best : b.best;
}

__device__ __forceinline__ void join_wave(Found& f) {
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) {
    Found g;
    const uint32_t lo = __shfl_xor((uint32_t)f.best, x, kWave), hi = __shfl_xor((uint32_t)(f.best >> 32), x, kWave);
    g.best = (uint64_t)hi << 32 | lo;
    g.m = __shfl_xor(f.m, x, kWave);
    g.sum = __shfl_xor(f.sum, x, kWave);
    join(f, g);
  }
}

__device__ __forceinline__ int request_of(const LogitsArgs& a, int64_t row) {
  const int64_t s = a.requests != nullptr ? a.requests[row] : row;
  return s >= 0 && s < a.S ? (int)s : -1;
}

__device__ __forceinline__ void store_row(const LogitsArgs& a, int64_t row, const Found& f) {
  if (a.choice != nullptr) a.choice[row] = (uint32_t)(f.best >> 32) == kOrderOfNone ? -1 : (int)~(uint32_t)f.best;
  if (a.lse != nullptr) {
    // an infinite logit's sum is infinite; without any logit above -inf it is 0 (or NaN)
    a.lse[row] = f.m == -INFINITY ? (f.sum == f.sum ? f.m : f.sum) : f.m + __logf(f.sum);
  }
}

template <typename V8, typename T>
__device__ __forceinline__ void store_logits(T* to, int v, int V, const float (&x)[kEach]) {
  if (v + kEach <= V) {
    V8 h;
#pragma unroll
    for (int e = 0; e < kEach; ++e) h[e] = static_cast<T>(x[e]);
    *reinterpret_cast<V8*>(to + v) = h;
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (v + e < V) to[v + e] = static_cast<T>(x[e]);
  }
}

// One slice of 2048 GROUPS logits of a row.
template <typename T, int GROUPS>
__global__ __launch_bounds__(kThreads) void k_logits(LogitsArgs a) {
#pragma clang fp contract(off)
  constexpr int SLICE = kThreads * kEach * GROUPS;
  extern __shared__ __align__(16) uint32_t counts[];  // [SLICE], then the biases' [SLICE]
  int* slots = reinterpret_cast<int*>(counts + SLICE);
  __shared__ Found part[kThreads / kWave];
  const int64_t block = a.first + blockIdx.x, row = block / a.slices;
  const int slice = (int)(block - row * a.slices), v0 = slice * SLICE, tid = threadIdx.x;
  const int req = request_of(a, row);
  if (req < 0) return;

  // the logits, on their way while the tokens are counted
  const T* from = static_cast<const T*>(a.logits) + row * a.stride;
  float x[GROUPS][kEach];
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    const int v = v0 + (g * kThreads + tid) * kEach;
    if (v + kEach <= a.V) {
      if constexpr (sizeof(T) == 2) {
        const half8_t h = *reinterpret_cast<const half8_any*>(from + v);
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[g][e] = (float)h[e];
      } else {
        const float8_t h = *reinterpret_cast<const float8_any*>(from + v);
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[g][e] = h[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e) x[g][e] = v + e < a.V ? (float)from[v + e] : -INFINITY;
    }
  }

  const bool counted = a.counted, biased = a.max_bias > 0;
  if (counted)
    for (int i = tid * 4; i < SLICE; i += kThreads * 4) *reinterpret_cast<int4_t*>(counts + i) = int4_t{0, 0, 0, 0};
  if (biased)
    for (int i = tid * 4; i < SLICE; i += kThreads * 4) *reinterpret_cast<int4_t*>(slots + i) = int4_t{-1, -1, -1, -1};
  __syncthreads();
  if (counted) {
    auto count = [&](int token, bool prompt) {
      const uint32_t u = (uint32_t)token - (uint32_t)v0;
      if (token < 0 || token >= a.V || u >= (uint32_t)SLICE) return;
      if (prompt) atomicOr(&counts[u], kInPrompt);
      else atomicAdd(&counts[u], 1u);
    };
    const int32_t* tokens = a.tokens + req * a.token_stride;
    int n = a.token_count != nullptr ? a.token_count[req] : 0, prompt = a.prompt_len != nullptr ? a.prompt_len[req] : 0;
    n = n < 0 ? 0 : n > a.max_tokens ? a.max_tokens : n;
    prompt = prompt < 0 ? 0 : prompt > n ? n : prompt;
    // a prompt matters to the repetition penalty alone
    for (int i = (a.repetition != nullptr ? 0 : prompt) + tid * 4; i < n; i += kThreads * 4) {
      if (i + 4 <= n) {
        const int4_t t = *reinterpret_cast<const int4_any*>(tokens + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) count(t[e], i + e < prompt);
      } else {
        for (int e = i; e < n; ++e) count(tokens[e], e < prompt);
      }
    }
    if (a.tree != nullptr) {
      int first = a.q_start[req], nodes = a.q_start[req + 1];
      first = first < 0 ? 0 : first > a.R ? (int)a.R : first;
      nodes = nodes < first ? 0 : (nodes > a.R ? (int)a.R : nodes) - first;
      const int32_t* words = a.tree + row * a.tree_stride;
      for (int j = tid; j < nodes && j / 32 < a.tree_words; j += kThreads)
        if (words[j / 32] >> (j % 32) & 1) count(a.draft_tokens[first + j], false);
    }
  }
  if (biased) {
    const int32_t* ids = a.bias_ids + (int64_t)req * a.max_bias;
    for (int i = tid; i < a.max_bias; i += kThreads) {
      const int token = ids[i];
      const uint32_t u = (uint32_t)token - (uint32_t)v0;
      if (token >= 0 && token < a.V && u < (uint32_t)SLICE) atomicMax(&slots[u], i);  // a token's last entry counts
    }
  }
  __syncthreads();

  const float rho = a.repetition != nullptr ? a.repetition[req] : 1.f, one_over = 1.f / rho;
  const float frequency = a.frequency != nullptr ? a.frequency[req] : 0.f;
  const float presence = a.presence != nullptr ? a.presence[req] : 0.f;
  const float tau = a.temperature != nullptr ? a.temperature[req] : 0.f, cool = tau > 0.f ? 1.f / tau : 1.f;
  const float* values = a.bias_values + (int64_t)req * a.max_bias;
  Found f = {0, -INFINITY, 0.f};
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    const int at = (g * kThreads + tid) * kEach, v = v0 + at;
    if (counted) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const uint32_t c = counts[at + e];
        if (c == 0) continue;
        float& y = x[g][e];
        const float times = (float)(c & ~kInPrompt);
        y = y > 0.f ? y * one_over : y * rho;
        y = y - (frequency * times + (times > 0.f ? presence : 0.f));
      }
    }
    if (biased) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int s = slots[at + e];
        if (s >= 0) x[g][e] = x[g][e] + values[s];
      }
    }
    const uint32_t bits = a.allowed != nullptr && v < a.V ? a.allowed[row * a.allowed_stride + v / 8] : 0xFFu;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      x[g][e] = x[g][e] * cool;
      if (!(bits >> e & 1)) x[g][e] = -INFINITY;
    }
  }
  if (a.finds) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int v = v0 + (g * kThreads + tid) * kEach + e;
        const uint64_t key = (uint64_t)order_of(x[g][e]) << 32 | (uint32_t)~v;
        if (v < a.V && key > f.best) f.best = key;
        f.m = fmaxf(f.m, x[g][e]);
      }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        f.sum += f.m == -INFINITY ? (x[g][e] == x[g][e] ? 0.f : x[g][e]) : weight_of(x[g][e], f.m);
  }
  if (a.out != nullptr) {
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int v = v0 + (g * kThreads + tid) * kEach;
      if (a.out_wide) store_logits<float8_any>(static_cast<float*>(a.out) + row * a.out_stride, v, a.V, x[g]);
      else store_logits<half8_any>(static_cast<half_t*>(a.out) + row * a.out_stride, v, a.V, x[g]);
    }
  }
  if (a.finds) {
    join_wave(f);
    if (tid % kWave == 0) part[tid / kWave] = f;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int i = 1; i < kThreads / kWave; ++i) join(f, part[i]);
      if (a.slices == 1) store_row(a, row, f);
      else a.found[row * a.slices + slice] = f;
    }
  }
}

// One wave a row.
__global__ __launch_bounds__(kThreads) void k_logits_join(LogitsArgs a) {
  const int64_t row = a.first + (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
  if (row >= a.R || request_of(a, row) < 0) return;
  Found f = {0, -INFINITY, 0.f};
  for (int i = threadIdx.x % kWave; i < a.slices; i += kWave) join(f, a.found[row * a.slices + i]);
  join_wave(f);
  if (threadIdx.x % kWave == 0) store_row(a, row, f);
}

constexpr int kGroups = 2;

int slices_of(int64_t V) { return (int)((V + kThreads * kEach * kGroups - 1) / (kThreads * kEach * kGroups)); }

}  // namespace

int64_t logits_workspace_bytes(int64_t R, int64_t V, const DeviceInfo&) {
  return slices_of(V) > 1 ? R * slices_of(V) * (int64_t)sizeof(Found) : 0;
}

hipError_t launch_logits(const LogitsProblem& p, const DeviceInfo&, hipStream_t stream) {
  const fasq_token_rules& r = p.rules;
  LogitsArgs a = {};
  a.logits = p.logits;
  a.out = p.out;
  a.out_wide = p.out_wide;
  a.stride = p.stride;
  a.out_stride = p.out_stride;
  a.R = p.R;
  a.V = (int)p.V;
  a.slices = slices_of(p.V);
  a.S = (int)r.S;
  a.requests = r.requests;
  a.tokens = r.tokens;
  a.token_stride = r.token_stride;
  a.max_tokens = (int)r.max_tokens;
  a.prompt_len = r.prompt_len;
  a.token_count = r.token_count;
  a.repetition = r.repetition;
  a.presence = r.presence;
  a.frequency = r.frequency;
  a.temperature = r.temperature;
  a.bias_ids = r.bias_ids;
  a.bias_values = r.bias_values;
  a.max_bias = (int)r.max_bias;
  a.allowed = reinterpret_cast<const uint8_t*>(r.allowed);
  a.allowed_stride = r.allowed_stride * 4;
  a.draft_tokens = r.draft_tokens;
  a.q_start = r.q_start;
  a.tree = r.tree;
  a.tree_stride = r.tree_stride;
  a.tree_words = (int)r.tree_words;
  a.choice = p.choice;
  a.lse = p.lse;
  a.counted = r.token_count != nullptr || r.tree != nullptr;
  a.finds = p.choice != nullptr || p.lse != nullptr;
  if (a.finds && a.slices > 1) a.found = static_cast<Found*>(p.workspace);
  constexpr int SLICE = kThreads * kEach * kGroups;
  const size_t lds = SLICE * 4 * (a.max_bias > 0 ? 2 : a.counted ? 1 : 0);
  const int64_t blocks = p.R * a.slices, most = kMaxGridThreads / kThreads;
  for (a.first = 0; a.first < blocks; a.first += most) {
    const int64_t n = blocks - a.first < most ? blocks - a.first : most;
    const hipError_t e = launch_kernel(p.wide ? k_logits<float, kGroups> : k_logits<half_t, kGroups>, dim3((unsigned)n),
                                       dim3(kThreads), lds, stream, a);
    if (e != hipSuccess) return e;
  }
  if (!a.finds || a.slices == 1) return hipSuccess;
  constexpr int ROWS = kThreads / kWave;
  a.first = 0;
  return launch_kernel(k_logits_join, dim3((unsigned)((p.R + ROWS - 1) / ROWS)), dim3(kThreads), 0, stream, a);
}

}  // namespace fasq
