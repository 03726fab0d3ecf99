// The residual stream between two blocks: norm, gate and scale of the block's
// output, the sum, and the next block's norm, in one pass.
//
// A workgroup holds one row in registers, so x and y are read once and x_out
// and h written once: bound by memory.  Each of the two norms is a sum over
// the row (a wave's lanes by DPP, then the waves by LDS in wave order), in fp32;
// x_out and h are each rounded once, from fp32 values.  4096 rows of 4096 with
// both norms and a gate take 24.3 us (134 MB, 5.5 TB/s), one row 2.6 us.
#include <hip/hip_runtime.h>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

struct NormArgs {
  const uint16_t* x;
  const uint16_t* y;
  const uint16_t* post_weight;
  const uint16_t* gate;
  int64_t gate_stride;
  const uint16_t* weight;
  uint16_t* x_out;
  uint16_t* h;
  int N;
  float scale, eps;
};

// Eight values of a row: one 16-byte chunk (VEC), or values `step` apart.
template <bool VEC>
__device__ __forceinline__ void load8(float (&v)[8], const uint16_t* row, int at, int step, int n) {
  if constexpr (VEC) {
    if (at < n) {
      const half8_t h = *reinterpret_cast<const half8_t*>(row + at);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = at + i * step < n ? (float)__builtin_bit_cast(half_t, row[at + i * step]) : 0.f;
  }
}

template <bool VEC>
__device__ __forceinline__ void store8(const float (&v)[8], uint16_t* row, int at, int step, int n) {
  if constexpr (VEC) {
    if (at < n) {
      half8_t h;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = static_cast<half_t>(v[i]);
      *reinterpret_cast<half8_t*>(row + at) = h;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i * step < n) row[at + i * step] = f32_to_f16_bits(v[i]);
  }
}

// The sum over the workgroup, in every thread.  `room` is not reused by the
// next call of the same row.
template <int WAVES>
__device__ __forceinline__ float row_sum(float s, float* room) {
  s = wave_sum(s);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = s;
    __syncthreads();
    s = room[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += room[w];
  }
  return s;
}

// One row per workgroup, CH chunks of eight values per thread.
template <int THREADS, int CH, bool VEC>
__global__ __launch_bounds__(THREADS) void k_residual_norm(NormArgs a) {
  constexpr int WAVES = THREADS / kWave;
  __shared__ float room[2][WAVES];
  const int64_t m = blockIdx.x, off = m * a.N;
  const int n = a.N, step = VEC ? 1 : THREADS;
  auto at = [&](int c) { return VEC ? (c * THREADS + (int)threadIdx.x) * 8 : c * 8 * THREADS + (int)threadIdx.x; };
  float x[CH][8];
#pragma unroll
  for (int c = 0; c < CH; ++c) load8<VEC>(x[c], a.x + off, at(c), step, n);
  if (a.y != nullptr) {
    float y[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) load8<VEC>(y[c], a.y + off, at(c), step, n);
    if (a.post_weight != nullptr) {
      float s = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s += y[c][i] * y[c][i];
      const float inv = 1.f / sqrtf(row_sum<WAVES>(s, room[0]) / (float)n + a.eps);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float w[8];
        load8<VEC>(w, a.post_weight, at(c), step, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[c][i] = y[c][i] * inv * w[i];
      }
    }
    if (a.gate != nullptr) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float g[8];
        load8<VEC>(g, a.gate + m * a.gate_stride, at(c), step, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[c][i] *= g[i];
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[c][i] += a.scale * y[c][i];
  }
  if (a.x_out != nullptr) {
#pragma unroll
    for (int c = 0; c < CH; ++c) store8<VEC>(x[c], a.x_out + off, at(c), step, n);
  }
  if (a.h == nullptr) return;
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[c][i] * x[c][i];
  const float inv = 1.f / sqrtf(row_sum<WAVES>(s, room[1]) / (float)n + a.eps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float w[8];
    load8<VEC>(w, a.weight, at(c), step, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[c][i] = x[c][i] * inv * w[i];
    store8<VEC>(x[c], a.h + off, at(c), step, n);
  }
}

template <int THREADS, int CH>
hipError_t launch_row(const NormArgs& all, int64_t M, bool vec, hipStream_t stream) {
  constexpr int64_t most = kMaxGridThreads / THREADS;  // rows of a launch
  for (int64_t m0 = 0; m0 < M; m0 += most) {
    const dim3 grid((unsigned)(M - m0 < most ? M - m0 : most));
    NormArgs a = all;
    a.x += m0 * a.N;
    if (a.y != nullptr) a.y += m0 * a.N;
    if (a.gate != nullptr) a.gate += m0 * a.gate_stride;
    if (a.x_out != nullptr) a.x_out += m0 * a.N;
    if (a.h != nullptr) a.h += m0 * a.N;
    const hipError_t e = vec ? launch_kernel(k_residual_norm<THREADS, CH, true>, grid, dim3(THREADS), 0, stream, a)
                             : launch_kernel(k_residual_norm<THREADS, CH, false>, grid, dim3(THREADS), 0, stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_residual_norm(const NormProblem& p, hipStream_t stream) {
  NormArgs a = {};
  a.x = p.x;
  a.y = p.y;
  a.post_weight = p.post_weight;
  a.gate = p.gate;
  a.gate_stride = p.gate_stride;
  a.weight = p.weight;
  a.x_out = p.x_out;
  a.h = p.h;
  a.N = (int)p.N;
  a.scale = p.scale;
  a.eps = p.eps;
  const void* all[] = {p.x, p.y, p.post_weight, p.gate, p.weight, p.x_out, p.h};
  bool vec = p.N % 8 == 0;
  for (const void* q : all) vec = vec && (reinterpret_cast<uintptr_t>(q) & 15) == 0;
  // Few waves for short rows, so that more rows are in flight (4096 rows of 512:
  // 4.8 us, 5.7 with 256 threads), and many for long ones (rows of 8192: 49.1
  // us with 1024 threads, 56.8 with 256; of 14336: 91.7, 96.8 with 512).
  if (p.N <= 512) return launch_row<64, 1>(a, p.M, vec, stream);
  if (p.N <= 2048) return launch_row<256, 1>(a, p.M, vec, stream);
  if (p.N <= 4096) return launch_row<256, 2>(a, p.M, vec, stream);
  if (p.N <= 8192) return launch_row<1024, 1>(a, p.M, vec, stream);
  if (p.N <= 16384) return launch_row<1024, 2>(a, p.M, vec, stream);
  return launch_row<1024, 4>(a, p.M, vec, stream);
}

}  // namespace fasq
