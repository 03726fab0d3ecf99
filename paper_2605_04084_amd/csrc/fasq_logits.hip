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

constexpr int kEach = 8;  // neighbouring logits of a thread
constexpr uint32_t kInPrompt = 0x80000000u;

constexpr float kLog2e = 1.44269504088896341f;

// What some of a row's logits come to.
struct Found {
  uint64_t best;  // order_of() of the largest, then its index's complement
  float m, sum;   // the largest that is a number, the sum of exp(x - m)
};

struct LogitsArgs {
  const void* logits;
  void* out;
  bool out_wide;               // fp32
  int64_t stride, out_stride;  // elements between rows
  int64_t R, first;            // the launch's first workgroup of all
  int V, slices;
  int rows;  // of a workgroup
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
  bool counted;  // tokens are
  Found* found;  // [R][parts]: of each wave that holds some of a row; nullptr: not asked for
  int parts;
  int32_t* choice;
  float* lse;
};

// The kernel's arguments, as if read for the first time: held from the start on they
// would fill the scalar registers, and what does not fit goes through the vector ones.
__device__ __forceinline__ const LogitsArgs& fresh_args() {
  auto p = (__attribute__((address_space(4))) const LogitsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const LogitsArgs*)p;
}

// Larger for larger logits; NaN above all, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderOfNone = ~0xFF800000u;  // of -inf

// A value that no kernel writes while this one runs, at an address that a whole wave shares: a scalar load.
template <typename T>
__device__ __forceinline__ T fixed(const T* p) {
  return *(__attribute__((address_space(4))) const T*)(uintptr_t)p;
}

__device__ __forceinline__ int request_of(const LogitsArgs& a, int64_t row) {
  const int64_t s = a.requests != nullptr ? a.requests[row] : row;
  return s >= 0 && s < a.S ? (int)s : -1;
}

// Eight of them, or the `count` that there are.
template <typename V8, typename T>
__device__ __forceinline__ void store_logits(T* to, uint32_t at, int count, const float (&x)[kEach]) {
  if (count >= kEach) {
    V8 h;
#pragma unroll
    for (int e = 0; e < kEach; ++e) h[e] = static_cast<T>(x[e]);
    *reinterpret_cast<V8*>(to + at) = h;
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (e < count) to[at + e] = static_cast<T>(x[e]);
  }
}

// The larger one that is a number.  As an instruction, because the compiler would
// first make each operand a value that no signalling NaN is.
__device__ __forceinline__ float larger(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ float larger(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Up to here top * kLog2e is off by at most 2^-4 (half an ulp of 2^20.6), so that weights relative to the
// rounded product lie within 2^(2^-4) of those relative to `top`.  From 2^31 on it may be off by 2^7
// and more, which fp32 does not hold as a power of two.
constexpr float kCloseTop = 1048576.f;

// What a wave's logits come to, in its first lane.  first: the index of x[0][0] in lane
// 0; lanes lie side by side, groups `apart`.
template <int GROUPS>
__device__ __forceinline__ Found find(const float (&x)[GROUPS][kEach], int first, int apart) {
  float own[GROUPS], top = -INFINITY;
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    own[g] = larger(x[g][0], x[g][1]);
#pragma unroll
    for (int e = 2; e < kEach; e += 2) own[g] = larger(own[g], x[g][e], x[g][e + 1]);
    top = larger(top, own[g]);
  }
  top = wave_join(top, [](float a, float b) { return larger(a, b); });
  Found f = {0, top, 0.f};
  const float c = top * kLog2e;
  const bool close = fabsf(top) < kCloseTop;
  if (close) {
    // one operation fewer than (x - top) * kLog2e; what the product rounds is made good below
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      float w[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(x[g][e], kLog2e, -c));
#pragma unroll
      for (int e = 0; e < kEach; e += 2) w[e] += w[e + 1];
      f.sum += (w[0] + w[2]) + (w[4] + w[6]);
    }
  } else {  // infinite ones, and masks of large values
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        f.sum += x[g][e] == top ? (top == -INFINITY ? 0.f : 1.f)
                                : __builtin_amdgcn_exp2f((x[g][e] - top) * kLog2e);
  }
  f.sum = wave_join(f.sum, sum_of);
  if (close) f.sum *= __builtin_amdgcn_exp2f(-fmaf(top, kLog2e, -c));
  bool nan = false;  // some logit is: a sum of others is a number
  if (f.sum != f.sum) {
    bool own_nan = false;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
#pragma unroll
      for (int e = 0; e < kEach; ++e) own_nan |= x[g][e] != x[g][e];
    nan = __any(own_nan);
  }
  uint32_t at = 0;
#pragma unroll
  for (int g = GROUPS - 1; g >= 0; --g) {
    // the first lane with one, and the first of its eight
    int e0 = kEach;
    if (nan) {
#pragma unroll
      for (int e = kEach - 1; e >= 0; --e) e0 = x[g][e] != x[g][e] ? e : e0;
    } else if (__ballot(own[g] == top) != 0) {
#pragma unroll
      for (int e = kEach - 1; e >= 0; --e) e0 = x[g][e] == top ? e : e0;
    }
    const uint64_t with = __ballot(e0 < kEach);
    if (with != 0) {
      const int l = __ffsll((unsigned long long)with) - 1;
      at = first + g * apart + l * kEach + __builtin_amdgcn_readlane(e0, l);
    }
  }
  f.best = (uint64_t)order_of(nan ? f.sum : top) << 32 | (uint32_t)~at;
  return f;
}

// A value as if it was new: what follows from it is not kept over a loop (a row's
// end is compared with every index, which filled the scalar registers).
__device__ __forceinline__ int again(int v) {
  v = __builtin_amdgcn_readfirstlane(v);
  asm volatile("" : "+s"(v));
  return v;
}

// Eight logits as they are loaded.
template <typename T>
struct Eight;
template <>
struct Eight<half_t> {
  typedef half8_t Held;
  typedef half8_any InMemory;
};
template <>
struct Eight<float> {
  typedef float8_t Held;
  typedef float8_any InMemory;
};

// One slice of 8 TH GROUPS logits of a.rows rows, one after the other.  Rows of
// one request that follow each other share its counts.
//
// Every workgroup looks at all of its request's tokens, and counts those of its slice
// with LDS atomics (a counter a logit, so that each thread finds its logits' own without
// a search); the logits are on their way meanwhile, pass through registers once, and a
// wave's largest and sum leave for the join.  Eight neighbouring logits a thread are
// one 16-byte load and one byte of a grammar.
//
// 64 rows of 128256 fp16 logits to fp32 with all rules (51 MB): 24.5 us, 2.1 TB/s, bound
// by the counting before the pass and by vector instructions; 256 rows in 16 trees,
// nothing written: 39 us, 22 to 25 of it the pass alone; 5 histories of 20000 to 100000 tokens:
// 19 us, of which LDS atomics of the slice with most of them are the most.
template <typename T, int TH, int GROUPS>
__global__ __launch_bounds__(TH, GROUPS == 2 ? 5 : 7) void k_logits(LogitsArgs) {
#pragma clang fp contract(off)
  const LogitsArgs& a = fresh_args();
  constexpr int SLICE = TH * kEach * GROUPS, WAVES = TH / kWave;
  // counts [SLICE]: occurrences in the answer, kInPrompt.  The biases' entries (-1: none) take
  // their place for a single row, else the place behind them.
  extern __shared__ __align__(16) uint32_t counts[];
  __shared__ int hits;                    // 1: biases fall into the slice, 2: drafted tokens do
  __shared__ int drafts[WAVES * GROUPS];  // the columns in which they do
  const int tid = threadIdx.x, lane = tid % kWave, wave = uniform(tid / kWave);
  int64_t chunk;
  int slice;
  {
    const uint64_t block = a.first + blockIdx.x;
    if (block >> 32 == 0) {
      chunk = (uint32_t)block / (uint32_t)a.slices;
      slice = (int)((uint32_t)block - (uint32_t)chunk * (uint32_t)a.slices);
    } else {
      chunk = block / a.slices;
      slice = (int)(block - chunk * a.slices);
    }
  }
  const int v0 = slice * SLICE, left = a.V - v0;  // of the row, from the slice on
  const int64_t row0 = chunk * a.rows, row1 = row0 + a.rows < a.R ? row0 + a.rows : a.R;
  const bool counted = a.counted, biased = a.max_bias > 0, apart = a.rows > 1 && counted;
  int* const slots = reinterpret_cast<int*>(counts) + (apart ? SLICE : 0);
  // A token's place in the slice, if it is below `limit`.
  const uint32_t limit = left < SLICE ? left : SLICE;
  auto place = [&](int token) { return (uint32_t)token - (uint32_t)v0; };
  // Where it is counted: the k-th logits of a wave's lanes lie side by side.
  auto column = [](uint32_t u) { return (u & ~511u) | (u & 7) << 6 | (u >> 3 & 63); };
  auto fill = [&](int* to, int value) {
#pragma unroll
    for (int i = 0; i < 2 * GROUPS; ++i) *reinterpret_cast<int4_t*>(to + (i * TH + tid) * 4) = int4_t{value, value, value, value};
  };
  // the logits, on their way while the tokens are counted
  typename Eight<T>::Held next[GROUPS];
  int next_bits[GROUPS], next_req;
  auto load = [&](int64_t row) {
    next_req = a.requests != nullptr ? fixed(a.requests + row) : (int)row;
    const T* from = static_cast<const T*>(a.logits) + row * a.stride + v0;
    const uint8_t* allowed = a.allowed + row * a.allowed_stride + v0 / 8;
    if (left >= SLICE) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const uint32_t at = (g * TH + tid) * kEach;
        next[g] = *reinterpret_cast<const typename Eight<T>::InMemory*>(from + at);
        if (a.allowed != nullptr) next_bits[g] = allowed[at / 8];
      }
    } else {
      const int there = again(left);
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int at = (g * TH + tid) * kEach;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const T x = from[at + e < there ? at + e : there - 1];
          next[g][e] = at + e < there ? x : static_cast<T>(-INFINITY);
        }
        if (a.allowed != nullptr) next_bits[g] = allowed[(at < there ? at : 0) / 8];
      }
    }
  };
  load(row0);

  int held = -1;           // the request whose tokens are counted
  int nodes = 0, node0 = 0;  // its drafted tokens
  uint32_t own = ~0u;    // this thread's of them
  bool some_bias = false, some_draft = false;
  int met[GROUPS] = {};  // the columns of this wave in which some token has occurred
  float rho = 1.f, one_over = 1.f, frequency = 0.f, presence = 0.f, cool = 1.f;
  for (int64_t row = row0; row < row1; ++row) {
    const int req = next_req;
    if ((uint32_t)req >= (uint32_t)a.S) {
      if (row + 1 < row1) load(row + 1);
      continue;
    }

    const int32_t* ids = a.bias_ids + (int64_t)req * a.max_bias;
    const int32_t* words = a.tree + row * a.tree_stride;
    // the tokens of this row's nodes, once more or once less
    auto drafted = [&](uint32_t change) {
      for (int j = tid; j < nodes && j / 32 < a.tree_words; j += TH)
        if (words[j / 32] >> (j % 32) & 1) {
          const uint32_t u = j == tid ? own : place(a.draft_tokens[node0 + j]);
          if (u < limit) atomicAdd(&counts[column(u)], change);
        }
    };
    if (req != held) {
      held = req;
      if (counted) {
        if (a.repetition != nullptr) rho = fixed(a.repetition + req);
        if (a.frequency != nullptr) frequency = fixed(a.frequency + req);
        if (a.presence != nullptr) presence = fixed(a.presence + req);
      }
      float tau = 0.f;
      if (a.temperature != nullptr) tau = fixed(a.temperature + req);
      if (counted || biased) {
        if (row > row0) __syncthreads();  // nobody reads the last request's
        int n = 0, prompt = 0;
        if (counted && a.token_count != nullptr) {
          n = fixed(a.token_count + req);
          prompt = a.prompt_len != nullptr ? fixed(a.prompt_len + req) : 0;
          n = n < 0 ? 0 : n > a.max_tokens ? a.max_tokens : n;
          prompt = prompt < 0 ? 0 : prompt > n ? n : prompt;
        }
        const int32_t* tokens = a.tokens + req * a.token_stride;
        int drafted_one = -1, bias_one = -1;  // of this thread
        if (a.tree != nullptr) {
          node0 = fixed(a.q_start + req);
          nodes = fixed(a.q_start + req + 1);
          node0 = node0 < 0 ? 0 : node0 > a.R ? (int)a.R : node0;
          nodes = nodes < node0 ? 0 : (nodes > a.R ? (int)a.R : nodes) - node0;
          if (tid < nodes) drafted_one = a.draft_tokens[node0 + tid];
        }
        if (tid < a.max_bias) bias_one = ids[tid];
        if (counted) fill(reinterpret_cast<int*>(counts), 0);
        if (biased && (apart || !counted)) fill(slots, -1);
        if (tid == 0) hits = 0;
        if (tid < WAVES * GROUPS) drafts[tid] = 0;
        __syncthreads();
        auto scan = [&](int i, int end, auto count) __attribute__((always_inline)) {
          constexpr int AHEAD = 4;
          // most slices hold few of a text's tokens: four are looked at together
          auto four = [&](int4_t t) __attribute__((always_inline)) {
            uint32_t u[4];
            bool any = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              u[e] = place(t[e]);
              any |= u[e] < limit;
            }
            if (!__any(any)) return;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (u[e] < limit) count(&counts[column(u[e])]);
          };
#pragma unroll 1
          for (; i + AHEAD * TH * 4 <= end; i += AHEAD * TH * 4) {
            int4_t t[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) t[k] = *reinterpret_cast<const int4_any*>(tokens + i + (k * TH + tid) * 4);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) four(t[k]);
          }
#pragma unroll 1
          for (i += wave * kWave * 4; i < end; i += TH * 4) {
            const int at = i + lane * 4;
            int4_t t = {-1, -1, -1, -1};
            if (at + 4 <= end) {
              t = *reinterpret_cast<const int4_any*>(tokens + at);
            } else {
#pragma unroll
              for (int e = 0; e < 3; ++e)
                if (at + e < end) t[e] = tokens[at + e];
            }
            four(t);
          }
        };
        // a prompt matters to the repetition penalty alone
        if (a.repetition != nullptr) scan(0, prompt, [](uint32_t* c) { atomicOr(c, kInPrompt); });
        scan(prompt, n, [](uint32_t* c) { atomicAdd(c, 1u); });
        own = place(drafted_one);
        int hit = 0;
        for (int i = tid; i < a.max_bias; i += TH) {
          const uint32_t u = place(i == tid ? bias_one : ids[i]);
          if (u >= limit) continue;
          hit = 1;
          if (apart || !counted) atomicMax(&slots[u], i);  // a token's last entry counts
        }
        for (int j = tid; j < nodes; j += TH) {
          const uint32_t u = j == tid ? own : place(a.draft_tokens[node0 + j]);
          if (u >= limit) continue;
          hit |= 2;
          atomicOr(&drafts[u >> 9], 1 << (u & 7));
        }
        if (hit != 0) atomicOr(&hits, hit);
        __syncthreads();
        some_bias = (uniform(hits) & 1) != 0;
        some_draft = (uniform(hits) & 2) != 0;
        if (counted) {
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) {
            met[g] = uniform(drafts[g * WAVES + wave]);
#pragma unroll
            for (int e = 0; e < kEach; ++e) met[g] |= __any(counts[(g * WAVES + wave) * 512 + e * kWave + lane] != 0) ? 1 << e : 0;
          }
        }
      }
      one_over = 1.f / rho;
      // fp32 holds no reciprocal of less than 2^-128; an infinite one would make NaN of zeros
      cool = tau > 0.f ? fminf(1.f / tau, 3.402823466e38f) : 1.f;
    }

    int bits[GROUPS];
    float x[GROUPS][kEach];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) x[g][e] = (float)next[g][e];
      bits[g] = next_bits[g];
    }
    if (row + 1 < row1) load(row + 1);
    if (counted) {
      if (some_draft) {
        drafted(1u);
        __syncthreads();
      }
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        if (met[g] == 0) continue;  // few columns have any
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          if (!(met[g] >> e & 1)) continue;
          const uint32_t k = counts[(g * WAVES + wave) * 512 + e * kWave + lane];
          const float y = x[g][e], times = (float)(k & ~kInPrompt);
          const float z = y * (y > 0.f ? one_over : rho) - (times > 0.f ? frequency * times + presence : 0.f);
          x[g][e] = k != 0 ? z : y;
        }
      }
      if (some_draft) {
        __syncthreads();
        drafted(0xFFFFFFFFu);
      }
    }
    if (some_bias) {
      if (counted && !apart) {
        __syncthreads();
        fill(slots, -1);
        __syncthreads();
        for (int i = tid; i < a.max_bias; i += TH) {
          const uint32_t u = place(ids[i]);
          if (u < limit) atomicMax(&slots[u], i);
        }
        __syncthreads();
      }
      const float* values = a.bias_values + (int64_t)req * a.max_bias;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int4_t* at = reinterpret_cast<const int4_t*>(slots + (g * TH + tid) * kEach);
        const int4_t c[2] = {at[0], at[1]};
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (c[e / 4][e % 4] >= 0) x[g][e] = x[g][e] + values[c[e / 4][e % 4]];
      }
    }
    if (a.temperature != nullptr) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g)
#pragma unroll
        for (int e = 0; e < kEach; ++e) x[g][e] = x[g][e] * cool;
      if (left < SLICE) {  // what lies past the vocabulary stays -inf: an infinite temperature makes NaN of it
        const int there = again(left);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
          for (int e = 0; e < kEach; ++e) x[g][e] = (g * TH + tid) * kEach + e < there ? x[g][e] : -INFINITY;
      }
    }
    if (a.allowed != nullptr) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          // all ones or none, then x or -inf bit by bit (which the compiler makes four operations of)
          const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe(bits[g], e, 1);
          asm("v_bfi_b32 %0, %1, %0, %2" : "+v"(x[g][e]) : "v"(keep), "s"(0xFF800000u));
        }
      }
    }
    if (a.out != nullptr) {
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        const int at = (g * TH + tid) * kEach, count = left >= SLICE ? kEach : again(left) - at;
        if (a.out_wide) store_logits<float8_any>(static_cast<float*>(a.out) + row * a.out_stride + v0, at, count, x[g]);
        else store_logits<half8_any>(static_cast<half_t*>(a.out) + row * a.out_stride + v0, at, count, x[g]);
      }
    }
    if (a.found != nullptr) {
      // what lies past the vocabulary is -inf, and no choice where all is
      const Found f = find<GROUPS>(x, v0 + wave * kWave * kEach, TH * kEach);
      if (lane == 0) a.found[(row * a.slices + slice) * WAVES + wave] = f;
    }
  }
}

// One wave a row.
constexpr int kJoinThreads = 256;
__global__ __launch_bounds__(kJoinThreads) void k_logits_join(LogitsArgs a) {
  const int64_t row = a.first + (int64_t)blockIdx.x * (kJoinThreads / kWave) + threadIdx.x / kWave;
  if (row >= a.R || request_of(a, row) < 0) return;
  const int lane = threadIdx.x % kWave;
  const Found* parts = a.found + row * a.parts;
  constexpr int HELD = 4;
  Found f[HELD];
  uint32_t order = 0, index = 0xFFFFFFFFu;
  float m = -INFINITY, sum = 0.f;
  for (int i0 = 0; i0 < a.parts; i0 += HELD * kWave) {
#pragma unroll
    for (int k = 0; k < HELD; ++k) f[k] = i0 + k * kWave + lane < a.parts ? parts[i0 + k * kWave + lane] : Found{0, -INFINITY, 0.f};
    float top = m;
#pragma unroll
    for (int k = 0; k < HELD; ++k) top = fmaxf(top, f[k].m);
    top = wave_join(top, [](float a, float b) { return larger(a, b); });
    sum *= m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * kLog2e);
    m = top;
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
      sum += f[k].sum * (f[k].m == m ? 1.f : __builtin_amdgcn_exp2f((f[k].m - m) * kLog2e));
      const uint32_t o = (uint32_t)(f[k].best >> 32), at = ~(uint32_t)f[k].best;
      index = o > order ? at : o == order && at < index ? at : index;
      order = o > order ? o : order;
    }
  }
  sum = wave_join(sum, sum_of);
  const uint32_t best = wave_join(order, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  index = wave_join(order == best ? index : 0xFFFFFFFFu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
  if (lane != 0) return;
  if (a.choice != nullptr) a.choice[row] = best == kOrderOfNone ? -1 : (int)index;
  if (a.lse != nullptr) a.lse[row] = sum == 0.f ? -INFINITY : m + __log2f(sum) * 0.693147180559945309f;
}

// How a call's rows are cut.
struct LogitsPlan {
  int threads, groups;
  int slices, rows;
};

// 512 threads with one group of eight logits a thread up to 16 logits a lane of the chip,
// else two.  One row of 128256, 64 rows, 16 trees of 16 rows, 5 rows with histories of
// 20000 to 100000: 7.0 / 25 / 47 / 19 us with one group, 8.7 / 23.9 / 39 / 22 with two; 9 / 23 /
// 41 / 31 with 256 threads, 11.6 / 26.6 / 49 / 24 with 1024 and two groups (kernel
// times).  Up to eight rows of a request share the counts of a slice: with one row a
// workgroup 16 trees take 60 us in all, with eight 42.
LogitsPlan plan_logits(int64_t R, int64_t V, int64_t rows_of_request, const DeviceInfo& dev) {
  LogitsPlan p;
  p.threads = 512;
  p.groups = R * V > (int64_t)dev.num_cus * 4096 ? 2 : 1;
  p.slices = (int)((V + p.threads * p.groups * kEach - 1) / (p.threads * p.groups * kEach));
  // Rows one after the other share what is counted, but only what the chip does not hold
  // at once (two workgroups a compute unit).  3 requests of 53 rows of 8550: 20 us, 47
  // eight by eight; 3 of 36 rows of 146672 25.6 and 31.8; 4 of 16 rows of 128256 19 and
  // 33; 16 of 16 rows take 50 with three workgroups a unit in place of 40.
  const int64_t rows = R * p.slices / (2 * dev.num_cus);
  p.rows = (int)(rows < rows_of_request ? rows : rows_of_request);
  p.rows = p.rows < 1 ? 1 : p.rows > 8 ? 8 : p.rows;
  return p;
}

template <typename T, int TH, int GROUPS>
hipError_t launch_slices(LogitsArgs a, hipStream_t stream) {
  const int64_t blocks = (a.R + a.rows - 1) / a.rows * a.slices, most = kMaxGridThreads / TH;
  const int arrays = a.counted && a.max_bias > 0 && a.rows > 1 ? 2 : a.counted || a.max_bias > 0 ? 1 : 0;
  const size_t lds = arrays * TH * GROUPS * kEach * sizeof(uint32_t);
  for (a.first = 0; a.first < blocks; a.first += most) {
    const int64_t n = blocks - a.first < most ? blocks - a.first : most;
    const hipError_t e = launch_kernel(k_logits<T, TH, GROUPS>, dim3((unsigned)n), dim3(TH), lds, stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T>
hipError_t launch_planned(const LogitsPlan& pl, const LogitsArgs& a, hipStream_t stream) {
  return pl.groups == 1 ? launch_slices<T, 512, 1>(a, stream) : launch_slices<T, 512, 2>(a, stream);
}

}  // namespace

int64_t logits_workspace_bytes(int64_t R, int64_t V, const DeviceInfo& dev) {
  const LogitsPlan p = plan_logits(R, V, 1, dev);
  return R * p.slices * (p.threads / kWave) * (int64_t)sizeof(Found);
}

hipError_t launch_logits(const LogitsProblem& p, const DeviceInfo& dev, hipStream_t stream) {
  const fasq_token_rules& r = p.rules;
  const LogitsPlan pl = plan_logits(p.R, p.V, r.S > 0 ? (p.R + r.S - 1) / r.S : 1, dev);
  LogitsArgs a = {};
  a.logits = p.logits;
  a.out = p.out;
  a.out_wide = p.out_wide;
  a.stride = p.stride;
  a.out_stride = p.out_stride;
  a.R = p.R;
  a.V = (int)p.V;
  a.slices = pl.slices;
  a.rows = pl.rows;
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
  a.parts = pl.slices * (pl.threads / kWave);
  if (p.choice != nullptr || p.lse != nullptr) a.found = static_cast<Found*>(p.workspace);
  const hipError_t e = p.wide ? launch_planned<float>(pl, a, stream) : launch_planned<half_t>(pl, a, stream);
  if (e != hipSuccess) return e;
  if (a.found == nullptr) return hipSuccess;
  constexpr int ROWS = kJoinThreads / kWave;
  a.first = 0;
  return launch_kernel(k_logits_join, dim3((unsigned)((p.R + ROWS - 1) / ROWS)), dim3(kJoinThreads), 0, stream, a);
}

}  // namespace fasq
