// Low-rank adapters of many requests beside shared projections.
//
// y = base + s_a B_a (A_a x): first the low-rank values t = A_a x (fp32, in
// the workspace), then the second product on the projection's output.
#include <hip/hip_runtime.h>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

struct LoraProjection {
  const uint16_t* A;
  const uint16_t* B;
  const uint16_t* base;
  uint16_t* y;
  int64_t N;
};

struct LoraArgs {
  const uint16_t* x;
  const int32_t* adapters;
  const float* scales;
  float* t;  // [count x M x r]
  int64_t M, K, L;
  int r;
  LoraProjection p[kLoraMaxCount];
};

__device__ __forceinline__ float h2f(uint16_t b) { return (float)__builtin_bit_cast(half_t, b); }

// t[i][m][j]: one wave each.
__global__ __launch_bounds__(256) void k_lora_down(LoraArgs a) {
  const int64_t row = blockIdx.x * (int64_t)4 + threadIdx.x / kWave;
  if (row >= a.M * a.r) return;
  const int lane = threadIdx.x % kWave;
  const int64_t m = row / a.r;
  const int ad = a.adapters[m];
  if (ad < 0 || ad >= a.L) return;
  const uint16_t* A = a.p[blockIdx.y].A + ((int64_t)ad * a.r + row % a.r) * a.K;
  const uint16_t* x = a.x + m * a.K;
  float s = 0.f;
  for (int64_t k = lane; k < a.K; k += kWave) s += h2f(A[k]) * h2f(x[k]);
  s = wave_sum(s);
  if (lane == 0) a.t[blockIdx.y * a.M * a.r + row] = s;
}

// y[i][m][n]: one thread each.
__global__ __launch_bounds__(256) void k_lora_up(LoraArgs a) {
  const LoraProjection& p = a.p[blockIdx.y];
  const int64_t total = a.M * p.N;
  for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / p.N, n = i % p.N;
    const int ad = a.adapters[m];
    const float b = p.base ? h2f(p.base[i]) : 0.f;
    float s = 0.f;
    const bool has = ad >= 0 && ad < a.L;
    if (has) {
      const float* t = a.t + (blockIdx.y * a.M + m) * a.r;
      const uint16_t* B = p.B + ((int64_t)ad * p.N + n) * a.r;
      for (int j = 0; j < a.r; ++j) s += t[j] * h2f(B[j]);
    }
    p.y[i] = f32_to_f16_bits(has ? b + a.scales[ad] * s : b);
  }
}

}  // namespace

int64_t lora_workspace_bytes(int64_t M, int64_t K, int r, int count, const DeviceInfo& dev) {
  return M * r * count * (int64_t)sizeof(float);
}

hipError_t launch_lora(const LoraProblem& p, const DeviceInfo& dev, hipStream_t stream) {
  LoraArgs a = {};
  a.x = p.x;
  a.adapters = p.adapters;
  a.scales = p.scales;
  a.t = static_cast<float*>(p.workspace);
  a.M = p.M;
  a.K = p.K;
  a.L = p.L;
  a.r = p.r;
  int64_t most = 0;
  for (int i = 0; i < p.count; ++i) {
    a.p[i].A = static_cast<const uint16_t*>(p.A[i]);
    a.p[i].B = static_cast<const uint16_t*>(p.B[i]);
    a.p[i].base = static_cast<const uint16_t*>(p.base[i]);
    a.p[i].y = static_cast<uint16_t*>(p.y[i]);
    a.p[i].N = p.N[i];
    if (p.N[i] > most) most = p.N[i];
  }
  const int64_t rows = (p.M * p.r + 3) / 4;
  hipError_t e = launch_kernel(k_lora_down, dim3((unsigned)rows, p.count), dim3(256), 0, stream, a);
  if (e != hipSuccess) return e;
  const int64_t blocks = (p.M * most + 255) / 256;
  return launch_kernel(k_lora_up, dim3((unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), p.count), dim3(256), 0,
                       stream, a);
}

}  // namespace fasq
