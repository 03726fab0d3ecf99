// Rotary positions, the per-head norm before them and the write of new keys
// and values to a paged cache, in one pass over q, k and v.
//
// A head is held by L lanes, 16 values each: a lane owns both values of every
// pair it turns, so a head needs no exchange for the rotation and one sum over
// its L lanes for the norm.  The pass is bound by memory: it reads and writes
// each value once and the table's row once per token.  4096 tokens of 32 + 8 + 8
// heads of 128 with head norms take 21 us (101 MB, 4.8 TB/s), 16 tokens 3.4 us.
#include <hip/hip_runtime.h>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

struct RopeFreqs {
  double w[kMaxRopeHalf];
};

// table[p][i] = (cos, sin)(p * w[i]) * scale; one thread per pair.
__global__ void k_rope_table(RopeFreqs f, int half, int64_t positions, double scale, float* __restrict__ table) {
  const int64_t n = positions * half;
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    double s, c;
    sincos((double)(i / half) * f.w[i % half], &s, &c);
    table[2 * i] = (float)(c * scale);
    table[2 * i + 1] = (float)(s * scale);
  }
}

struct RopeArgs {
  HeadsView q, q_out, k, v;
  int Hq, Hkv;
  uint32_t rows;  // T * (Hq + 2 Hkv) heads
  int D, half;
  const float* table;
  int64_t table_positions;
  const int32_t* positions;
  const int32_t* slots;
  const uint16_t* q_norm;
  const uint16_t* k_norm;
  float eps;
  uint16_t* ck;
  uint16_t* cv;
  int64_t num_slots;
  uint32_t page_size;
  int64_t page_stride, slot_stride, head_stride;
};

// One head of one token: its kind, source, destination and norm weights.
struct RopeRow {
  const uint16_t* src;
  uint16_t* dst;  // nullptr: not written
  const uint16_t* norm;
  uint32_t token;
  bool turned;
};

__device__ __forceinline__ RopeRow rope_row(const RopeArgs& a, uint32_t row) {
  const uint32_t heads = a.Hq + 2 * a.Hkv;
  RopeRow r;
  r.token = row / heads;
  uint32_t h = row - r.token * heads;
  if (h < (uint32_t)a.Hq) {
    r.src = a.q.p + r.token * a.q.ts + h * a.q.hs;
    r.dst = a.q_out.p + r.token * a.q_out.ts + h * a.q_out.hs;
    r.norm = a.q_norm;
    r.turned = true;
    return r;
  }
  h -= a.Hq;
  r.turned = h < (uint32_t)a.Hkv;
  if (!r.turned) h -= a.Hkv;
  const HeadsView& s = r.turned ? a.k : a.v;
  r.src = s.p + r.token * s.ts + h * s.hs;
  r.norm = r.turned ? a.k_norm : nullptr;
  const int64_t slot = a.slots[r.token];
  r.dst = nullptr;
  if (slot >= 0 && slot < a.num_slots) {
    const uint32_t page = (uint32_t)slot / a.page_size;
    r.dst = (r.turned ? a.ck : a.cv) + page * a.page_stride + ((uint32_t)slot - page * a.page_size) * a.slot_stride +
            h * a.head_stride;
  }
  return r;
}

// The table's row of a token, or nullptr where its position lies outside.
__device__ __forceinline__ const float* rope_cs(const RopeArgs& a, uint32_t token) {
  const int64_t p = a.positions[token];
  return p >= 0 && p < a.table_positions ? a.table + p * (2 * a.half) : nullptr;
}

__device__ __forceinline__ float h2f(uint16_t b) { return (float)__builtin_bit_cast(half_t, b); }

struct Chunk {
  float v[8];
  __device__ __forceinline__ void load(const uint16_t* p) {
    const half8_t h = *reinterpret_cast<const half8_t*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
  }
  __device__ __forceinline__ void store(uint16_t* p) const {
    half8_t h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = static_cast<half_t>(v[i]);
    *reinterpret_cast<half8_t*>(p) = h;
  }
  __device__ __forceinline__ float squares() const {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i] * v[i];
    return s;
  }
  __device__ __forceinline__ void scale(float r, const uint16_t* w) {
    Chunk c;
    c.load(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] * r * c.v[i];
  }
};

// L lanes per head, two 16-byte chunks per lane: chunks c and half / 8 + c
// (the two values of 8 pairs) in the half layout, 2 c and 2 c + 1 in the
// interleaved one and behind the turned part.  Needs D and the layout's
// chunks whole and aligned (the launcher checks).
template <int L, bool INTERLEAVED>
__global__ __launch_bounds__(256) void k_rope_vec(RopeArgs a) {
  const uint32_t row = blockIdx.x * (256 / L) + threadIdx.x / L;
  if (row >= a.rows) return;  // whole groups of L lanes leave together
  const int lane = threadIdx.x % L;
  const RopeRow r = rope_row(a, row);
  const int chunks = a.D / 8, turned = a.half / 4;  // chunks of the head, of its turned part
  int c0 = 2 * lane, c1 = 2 * lane + 1;
  if (!INTERLEAVED && c1 < turned) {
    c0 = lane;
    c1 = turned / 2 + lane;
  }
  const bool has0 = c0 < chunks, has1 = c1 < chunks;
  Chunk x0 = {}, x1 = {};
  if (has0) x0.load(r.src + c0 * 8);
  if (has1) x1.load(r.src + c1 * 8);
  if (r.norm != nullptr) {
    const float s = group_sum<L>(x0.squares() + x1.squares());
    const float inv = 1.f / sqrtf(s / (float)a.D + a.eps);
    if (has0) x0.scale(inv, r.norm + c0 * 8);
    if (has1) x1.scale(inv, r.norm + c1 * 8);
  }
  if (r.dst == nullptr) return;
  if (r.turned && a.half > 0) {
    const float* cs = rope_cs(a, r.token);
    if (cs == nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x0.v[i] = x1.v[i] = __builtin_nanf("");
    } else if (INTERLEAVED) {
      // pair 4 c + i of chunk c
      auto turn = [&](Chunk& x, int c) {
        const float4_t* t = reinterpret_cast<const float4_t*>(cs + c * 8);
        const float4_t t0 = t[0], t1 = t[1];
        const float co[4] = {t0[0], t0[2], t1[0], t1[2]}, si[4] = {t0[1], t0[3], t1[1], t1[3]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = x.v[2 * i], q = x.v[2 * i + 1];
          x.v[2 * i] = p * co[i] - q * si[i];
          x.v[2 * i + 1] = q * co[i] + p * si[i];
        }
      };
      if (c0 < turned) turn(x0, c0);
      if (c1 < turned) turn(x1, c1);
    } else if (c1 < turned) {
      const float4_t* t = reinterpret_cast<const float4_t*>(cs + c0 * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4_t v = t[i];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float p = x0.v[2 * i + e], q = x1.v[2 * i + e];
          x0.v[2 * i + e] = p * v[2 * e] - q * v[2 * e + 1];
          x1.v[2 * i + e] = q * v[2 * e] + p * v[2 * e + 1];
        }
      }
    }
  }
  if (has0) x0.store(r.dst + c0 * 8);
  if (has1) x1.store(r.dst + c1 * 8);
}

// Any D, strides and alignment: one wave per head, single values.  Every lane
// holds its values before the first store (q_out may be q).
__global__ __launch_bounds__(256) void k_rope_any(RopeArgs a, bool interleaved) {
  const uint32_t row = blockIdx.x * 4 + threadIdx.x / kWave;
  if (row >= a.rows) return;
  const int lane = threadIdx.x % kWave;
  const RopeRow r = rope_row(a, row);
  // lane's values: pairs lane and lane + 64 (two values each), then the tail
  constexpr int kE = 4;
  float x[kE + 4];
  int at[kE + 4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + j * kWave;
    at[2 * j] = i < a.half ? (interleaved ? 2 * i : i) : -1;
    at[2 * j + 1] = i < a.half ? (interleaved ? 2 * i + 1 : i + a.half) : -1;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 2 * a.half + lane + j * kWave;
    at[kE + j] = i < a.D ? i : -1;
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < kE + 4; ++j) {
    x[j] = at[j] >= 0 ? h2f(r.src[at[j]]) : 0.f;
    s += x[j] * x[j];
  }
  if (r.norm != nullptr) {
    const float inv = 1.f / sqrtf(wave_sum(s) / (float)a.D + a.eps);
#pragma unroll
    for (int j = 0; j < kE + 4; ++j)
      if (at[j] >= 0) x[j] = x[j] * inv * h2f(r.norm[at[j]]);
  }
  if (r.dst == nullptr) return;
  if (r.turned && a.half > 0) {
    const float* cs = rope_cs(a, r.token);
    if (cs == nullptr) {
#pragma unroll
      for (int j = 0; j < kE + 4; ++j) x[j] = __builtin_nanf("");
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = lane + j * kWave;
        if (i < a.half) {
          const float c = cs[2 * i], sn = cs[2 * i + 1], p = x[2 * j], q = x[2 * j + 1];
          x[2 * j] = p * c - q * sn;
          x[2 * j + 1] = q * c + p * sn;
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kE + 4; ++j)
    if (at[j] >= 0) r.dst[at[j]] = f32_to_f16_bits(x[j]);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool view16(const HeadsView& v) { return v.p == nullptr || (aligned16(v.p) && (v.ts | v.hs) % 8 == 0); }

template <int L>
hipError_t launch_vec(const RopeArgs& a, bool interleaved, hipStream_t stream) {
  const dim3 grid((a.rows + 256 / L - 1) / (256 / L));
  return interleaved ? launch_kernel(k_rope_vec<L, true>, grid, dim3(256), 0, stream, a)
                     : launch_kernel(k_rope_vec<L, false>, grid, dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_rope_table(const double* inv_freq, int half, int64_t positions, double scale, float* table,
                             hipStream_t stream) {
  RopeFreqs f = {};
  for (int i = 0; i < half; ++i) f.w[i] = inv_freq[i];
  const int64_t blocks = (positions * half + 255) / 256;
  return launch_kernel(k_rope_table, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream, f, half,
                       positions, scale, table);
}

hipError_t launch_rope_append(const RopeProblem& p, hipStream_t stream) {
  RopeArgs a = {};
  a.q = p.q;
  a.q_out = p.q_out;
  a.k = p.k;
  a.v = p.v;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.D = p.D;
  a.half = p.rot / 2;
  a.table = p.table;
  a.table_positions = p.table_positions;
  a.positions = p.positions;
  a.slots = p.slots;
  a.q_norm = p.q_norm;
  a.k_norm = p.k_norm;
  a.eps = p.eps;
  if (p.k.p != nullptr) {
    a.ck = static_cast<uint16_t*>(p.cache.k);
    a.cv = static_cast<uint16_t*>(p.cache.v);
    a.num_slots = p.cache.num_pages * p.cache.page_size;
    a.page_size = (uint32_t)p.cache.page_size;
    a.page_stride = p.cache.page_stride;
    a.slot_stride = p.cache.slot_stride;
    a.head_stride = p.cache.head_stride;
  }
  const int64_t heads = p.Hq + 2 * (int64_t)p.Hkv;
  const bool vec = p.D % 8 == 0 && p.rot % (p.interleaved ? 8 : 16) == 0 && view16(p.q) && view16(p.q_out) &&
                   view16(p.k) && view16(p.v) && aligned16(p.q_norm) && aligned16(p.k_norm) && aligned16(p.table) &&
                   (p.k.p == nullptr || (aligned16(a.ck) && aligned16(a.cv) &&
                                         (a.page_stride | a.slot_stride | a.head_stride) % 8 == 0));
  const int lanes = !vec ? kWave : p.D <= 64 ? 4 : p.D <= 128 ? 8 : 16;  // of a head
  const int64_t most = kMaxGridThreads / lanes / heads;  // tokens of a launch
  for (int64_t t0 = 0; t0 < p.T; t0 += most) {
    const int64_t n = p.T - t0 < most ? p.T - t0 : most;
    RopeArgs b = a;
    b.rows = (uint32_t)(n * heads);
    if (b.q.p != nullptr) {
      b.q.p += t0 * b.q.ts;
      b.q_out.p += t0 * b.q_out.ts;
    }
    if (b.k.p != nullptr) {
      b.k.p += t0 * b.k.ts;
      b.v.p += t0 * b.v.ts;
      b.slots += t0;
    }
    if (b.positions != nullptr) b.positions += t0;
    hipError_t e;
    if (!vec) e = launch_kernel(k_rope_any, dim3((b.rows + 3) / 4), dim3(256), 0, stream, b, p.interleaved);
    else if (p.D <= 64) e = launch_vec<4>(b, p.interleaved, stream);
    else if (p.D <= 128) e = launch_vec<8>(b, p.interleaved, stream);
    else e = launch_vec<16>(b, p.interleaved, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fasq
