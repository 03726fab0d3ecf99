// Low-rank adapters of many requests beside shared projections:
// y = base + s_a B_a (A_a x), two or three launches.
//
//   k_lora_down  t = A_a x, fp32 in the workspace, K split over workgroups
//   k_lora_fold  beyond 128 tokens and 16 ranks: t summed over the splits and in
//                the form the matrix cores take, which k_lora_up makes itself
//                otherwise
//   k_lora_up    y = base + s_a B_a t, one pass over the projection's output
//
// They work on blocks of 16 to 128 tokens in the order given.  A block's
// adapters are found by comparing the tokens' ids (a lane holds a token), so
// requests may come in any order and nothing is planned beforehand: the
// adapters of a block are dealt to J workgroups, each of which computes the
// tokens of its own ones and writes those only.  Both products run on the
// matrix cores (v_mfma_f32_16x16x32_f16, tokens across); a token is a column
// and never meets another one's values.
#include <hip/hip_runtime.h>

#include <cmath>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

namespace {

constexpr int kLoraMaxSplits = 8;  // of K
constexpr int kU = 8;              // neighbouring features of a lane
constexpr int kSlice = 64 * kU;    // output features of a workgroup at a time

struct LoraProjection {
  const uint16_t* A;
  const uint16_t* B;
  const uint16_t* base;
  uint16_t* y;
  int N;
};

struct LoraArgs {
  const uint16_t* x;
  const int32_t* adapters;
  const float* scales;
  float* t;  // [splits][count][M][r]
  half_t* low;     // folded: [count][M][2][rp], rp = r up to a multiple of 32
  float* factors;  // folded: [count][M]
  int M;
  int64_t K, L;
  int r, J, splits, count, slices;
  int64_t k_share;  // K values of a split, a multiple of 32
  LoraProjection p[kLoraMaxCount];
};

// A quotient that is the same in every lane: the division leaves it in a vector
// register.
__device__ __forceinline__ int scalar(uint32_t v) { return __builtin_amdgcn_readfirstlane((int)v); }

typedef half8_t half8_any __attribute__((aligned(2)));

// Eight values at p[at ...] of a row of n (zeros behind its end).  Without
// VEC the row may start anywhere and end inside the eight: they are read at
// once all the same, past the row's end too, but not past `last`, the end of
// the tensor.  There is one load in any case (of the tensor's last values where
// there is nothing to read), so that the loads of different rows follow each
// other without a branch between them.  RAW: what lies behind the row's end,
// or of a row that is not live, is anything, and nothing has to wait for the
// loaded values yet.
template <bool VEC, bool RAW = false>
__device__ __forceinline__ half8_t row8(const uint16_t* p, int64_t at, int64_t n, const uint16_t* last, int64_t total,
                                        bool live) {
  const bool has = live && at < n;
  const uint16_t* q = p + at;
  if constexpr (VEC) {
    const half8_t v = *reinterpret_cast<const half8_t*>(has ? q : last - 8);
    return RAW || has ? v : half8_t{};
  }
  const bool end = has && last - q < 8;
  half8_t v = {};
  if (total >= 8) v = *reinterpret_cast<const half8_any*>(has && !end ? q : last - 8);
  u32x4 w = __builtin_bit_cast(u32x4, v);
  if (end) {
    w = u32x4{};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 2] |= (uint32_t)(q + i < last ? q[i] : 0) << (i % 2 * 16);
  }
  if constexpr (RAW) return __builtin_bit_cast(half8_t, w);
  const int keep = !has ? 0 : n - at < 8 ? (int)(n - at) : 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= keep >= 2 * i + 2 ? ~0u : keep == 2 * i + 1 ? 0xFFFFu : 0u;
  return __builtin_bit_cast(half8_t, w);
}

// The adapters of a block of TM tokens: lane l holds the ids of tokens l, l +
// 64, ... (-1: none).
template <int TM>
struct BlockIds {
  static constexpr int W = (TM + kWave - 1) / kWave;
  int id[W];

  __device__ __forceinline__ BlockIds(const LoraArgs& a, int m0) {
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int at = w * kWave + threadIdx.x % kWave, m = m0 + at;
      const int v = at < TM && m < a.M ? a.adapters[m] : -1;
      id[w] = v >= 0 && v < a.L ? v : -1;
    }
  }

  // Calls f(adapter, masks of its tokens) for every J-th adapter, from the
  // j-th on, in the order of their first tokens.
  template <typename F>
  __device__ __forceinline__ void each(int j, int J, F f) const {
    uint64_t left[W];
#pragma unroll
    for (int w = 0; w < W; ++w) left[w] = __ballot(id[w] >= 0);
    int i = 0;
#pragma unroll
    for (int w = 0; w < W; ++w)
      for (; left[w] != 0; ++i) {
        const int a = __builtin_amdgcn_readlane(id[w], __ffsll((unsigned long long)left[w]) - 1);
        uint64_t mask[W];
#pragma unroll
        for (int v = 0; v < W; ++v) {
          mask[v] = __ballot(id[v] == a);
          left[v] &= ~mask[v];
        }
        if (i % J == j) f(a, mask);
      }
  }
};

// ---------------------------------------------------------------------------
// t[split][i][m][rank] over ranks [16 RT z, 16 RT (z + 1)), 16 TT tokens and a
// share of K, which the four waves split once more and add in wave order.
// Adapters and activations go from memory to the operands: a wave reads 16
// rows of 64 bytes at a time.  2048 tokens of 4096 values, two projections of 64
// ranks take 17.5 us (more splits, or shares of K begun at different places,
// were no faster: not the order of memory's channels), 16 tokens with an
// adapter each on three projections of 16 ranks 4.8 us.
// ---------------------------------------------------------------------------
template <int TT, int RT, bool VEC>
__global__ __launch_bounds__(256) void k_lora_down(LoraArgs a) {
  constexpr int TM = 16 * TT;
  __shared__ float4_t sums[3][RT * TT][kWave];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane % 16, g = lane / 16;
  const int m0 = blockIdx.x * TM, j = scalar(blockIdx.z / a.splits), z = blockIdx.z - j * a.splits;
  const int rank_part = scalar(blockIdx.y / a.count), i = blockIdx.y - rank_part * a.count, r0 = rank_part * (16 * RT);
  const int64_t begin = z * a.k_share, end = begin + a.k_share < a.K ? begin + a.k_share : a.K;
  const BlockIds<TM> ids(a, m0);
  ids.each(j, a.J, [&](int ad, const uint64_t (&masks)[1]) {
    const uint64_t mask = masks[0];
    const uint16_t* x = a.x + (int64_t)(m0 + l16) * a.K;
    const uint16_t* A = a.p[i].A + ((int64_t)ad * a.r + r0 + l16) * a.K;
    float4_t acc[RT][TT] = {};
    // UN steps' loads before their products; steps past the end are zeros
    constexpr int UN = RT * TT >= 8 ? 2 : 4;
    const int64_t x_all = (int64_t)a.M * a.K, A_all = a.L * a.r * a.K;
    for (int64_t k = begin + wave * (32 * UN); k < end; k += 4 * 32 * UN) {
      half8_t b[UN][TT], w[UN][RT];
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        const int64_t at = k + u * 32 + g * 8;
#pragma unroll
        for (int q = 0; q < TT; ++q) b[u][q] = row8<VEC>(x + q * 16 * a.K, at, end, a.x + x_all, x_all, mask >> (q * 16 + l16) & 1);
#pragma unroll
        for (int t = 0; t < RT; ++t) w[u][t] = row8<VEC>(A + t * 16 * a.K, at, end, a.p[i].A + A_all, A_all, r0 + t * 16 + l16 < a.r);
      }
#pragma unroll
      for (int u = 0; u < UN; ++u)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int q = 0; q < TT; ++q)
            acc[t][q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[u][t], b[u][q], acc[t][q], 0, 0, 0);
    }
    __syncthreads();  // the last adapter's sums have been read
    if (wave > 0) {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int q = 0; q < TT; ++q) sums[wave - 1][t * TT + q][lane] = acc[t][q];
    }
    __syncthreads();
    if (wave > 0) return;
    // ranks 4 g .. 4 g + 3 of each 16, token l16 of each 16
#pragma unroll
    for (int q = 0; q < TT; ++q) {
      const bool mine = mask >> (q * 16 + l16) & 1;
      float* out = a.t + (((int64_t)z * a.count + i) * a.M + m0 + q * 16 + l16) * a.r;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
#pragma unroll
        for (int s = 0; s < 3; ++s) acc[t][q] += sums[s][t * TT + q][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int rank = r0 + t * 16 + g * 4 + e;
          if (mine && rank < a.r) out[rank] = acc[t][q][e];
        }
      }
    }
  });
}

// A token's low-rank values for the matrix cores: scaled by a power of two so
// that the largest lies in [2^14, 2^15), each is the sum of two fp16 values (the
// value and what its rounding left): 22 bits down to 2^-17 of the largest,
// steps of 2^-38 of it below (with the largest in [1/2, 1) the second value
// would run out of exponent 15 bits earlier).  power: the scale undone.
struct LowScale {
  float down, power;
  __device__ __forceinline__ explicit LowScale(float top) {
    int e = 0;
    if (top > 0.f && top < INFINITY) frexpf(top, &e);
    if (top == INFINITY) e = 120;  // nothing finite may become infinite beside it
    e = e < -100 ? -100 : e > 120 ? 120 : e;
    down = ldexpf(1.f, 15 - e);
    power = ldexpf(1.f, e - 15);
  }
  __device__ __forceinline__ void split(float v, half_t& hi, half_t& lo) const {
    const float x = v * down;
    hi = static_cast<half_t>(x);
    const float rest = x - (float)hi;
    lo = static_cast<half_t>(rest - rest == 0.f ? rest : 0.f);  // not finite: hi says it
  }
};

// One wave per token and projection (4.9 us for 2048 tokens of 2 x 64 ranks).
__global__ __launch_bounds__(256) void k_lora_fold(LoraArgs a) {
  const int m = blockIdx.x * 4 + threadIdx.x / kWave;
  if (m >= a.M) return;
  const int64_t row = (int64_t)blockIdx.y * a.M + m;  // of [count][M]
  const int lane = threadIdx.x % kWave, ad = a.adapters[m];
  if (ad < 0 || ad >= a.L) return;
  const int rp = (a.r + 31) / 32 * 32;
  const int64_t split = (int64_t)a.count * a.M * a.r;
  float v[4] = {}, top = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int rank = q * kWave + lane;
    if (rank < a.r)
      for (int z = 0; z < a.splits; ++z) v[q] += a.t[z * split + row * a.r + rank];
    top = fmaxf(top, fabsf(v[q]));
  }
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
  const LowScale scale(top);
  half_t* out = a.low + row * (2 * rp);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int rank = q * kWave + lane;
    if (rank < rp) scale.split(v[q], out[rank], out[rp + rank]);
  }
  if (lane == 0) a.factors[row] = a.scales[ad] * scale.power;
}

// ---------------------------------------------------------------------------
// y over `slices` times 512 output features and TM tokens.  The low-rank values
// come as LowScale has them, so that the matrix cores take them without
// losing the fp32 sums; both products add up in fp32.  Tokens go down the
// MFMA tile and features across: column q of tile u of a wave's eight is
// feature 8 q + u of its 128, so that a lane ends with 8 neighbouring features
// of 4 tokens, and base and y move in runs of 256 bytes, base a tile ahead.
// Bound by that pass over base and y: 2048 tokens, 2 x 14336 features, 64
// ranks take 67 us (3.5 TB/s).  Measured slower there: runs of 128 bytes (80
// us), blocks of 64 tokens (71 us), base two tiles ahead (70 us, registers
// spill), low-rank values folded by every workgroup instead of once (97 us).
// 16 tokens with an adapter each on 4096 + 1024 + 1024 features: 7.4 us.
// ---------------------------------------------------------------------------
template <int TM, int NQ, bool VEC>
__global__ __launch_bounds__(256, 2) void k_lora_up(LoraArgs a) {
  constexpr int TT = TM / 16;
  constexpr bool FOLDED = TM > 16;
  extern __shared__ uint8_t smem[];
  const int j = scalar(blockIdx.z / a.count), i = blockIdx.z - j * a.count;
  const LoraProjection& p = a.p[i];
  const int n_block = blockIdx.y * (kSlice * a.slices);
  if (n_block >= p.N) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane % 16, g = lane / 16;
  const int m0 = blockIdx.x * TM;
  const int rp = (a.r + 31) / 32 * 32;
  // not folded: the block's low-rank values in LDS
  const int pitch = rp + 8;
  half_t* hi = reinterpret_cast<half_t*>(smem);  // [TM][pitch]
  half_t* lo = hi + TM * pitch;                  // [TM][pitch]
  float* factor = reinterpret_cast<float*>(lo + TM * pitch);  // [TM]
  const int n_end = n_block + kSlice * a.slices < p.N ? n_block + kSlice * a.slices : p.N;
  const BlockIds<TM> ids(a, m0);
  constexpr int W = BlockIds<TM>::W;

  const int64_t B_all = a.L * p.N * a.r, y_all = (int64_t)a.M * p.N;
  // the kU features n ... of token m
  auto load = [&](int m, int n, bool live) {
    if (p.base == nullptr) return half8_t{};
    return row8<VEC, true>(p.base + (int64_t)m * p.N, n, p.N, p.base + y_all, y_all, live);
  };
  auto store = [&](int m, int n, half8_t v) {
    uint16_t* at = p.y + (int64_t)m * p.N + n;
    if (VEC || n + 8 <= p.N) {
      if (VEC && n < p.N) *reinterpret_cast<half8_t*>(at) = v;
      if (!VEC) *reinterpret_cast<half8_any*>(at) = v;
      return;
    }
    const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int e = 0; e < kU; ++e)
      if (n + e < p.N) at[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
  };

  ids.each(j, a.J, [&](int ad, const uint64_t (&mask)[W]) {
    if constexpr (!FOLDED) {  // 16 lanes a token
      __syncthreads();  // the last adapter's values have been read
      const int64_t split = (int64_t)a.count * a.M * a.r;
      const int tok = threadIdx.x / 16;
      const float* src = a.t + ((int64_t)i * a.M + m0 + tok) * a.r;
      float v[NQ] = {}, top = 0.f;
      auto add = [&](int z) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const int rank = q * 16 + threadIdx.x % 16;
          const bool has = (mask[0] >> tok & 1) && rank < a.r;
          const float x = *(has ? src + z * split + rank : a.t);
          v[q] += has ? x : 0.f;
        }
      };
      if constexpr (NQ <= 4) {  // all loads at once
#pragma unroll
        for (int z = 0; z < kLoraMaxSplits; ++z)
          if (z < a.splits) add(z);
      } else {
        for (int z = 0; z < a.splits; ++z) add(z);
      }
#pragma unroll
      for (int q = 0; q < NQ; ++q) top = fmaxf(top, fabsf(v[q]));
#pragma unroll
      for (int x = 1; x < 16; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
      const LowScale scale(top);
#pragma unroll
      for (int q = 0; q < (NQ + 1) / 2 * 2; ++q) {
        const int at = tok * pitch + q * 16 + threadIdx.x % 16;
        if (q * 16 < rp) scale.split(q < NQ ? v[q < NQ ? q : 0] : 0.f, hi[at], lo[at]);
      }
      if (threadIdx.x % 16 == 0) factor[tok] = a.scales[ad] * scale.power;
      __syncthreads();
    }
    // ---- the product
    for (int n0 = n_block + wave * (16 * kU); n0 < n_end; n0 += kSlice) {
      const int n = n0 + l16 * kU;
      const uint16_t* B = p.B + ((int64_t)ad * p.N + n) * a.r;
      auto rank8 = [&](int k, int u) { return row8<VEC>(B + u * a.r, k + g * 8, a.r, p.B + B_all, B_all, n + u < p.N); };
      auto low = [&](int t, int k, half8_t& th, half8_t& tl) {
        if constexpr (FOLDED) {
          const int m = m0 + t * 16 + l16;
          const half_t* h = a.low + ((int64_t)i * a.M + (m < a.M ? m : a.M - 1)) * (2 * rp) + k + g * 8;
          th = *reinterpret_cast<const half8_t*>(h);
          tl = *reinterpret_cast<const half8_t*>(h + rp);
        } else {
          th = *reinterpret_cast<const half8_t*>(hi + (t * 16 + l16) * pitch + k + g * 8);
          tl = *reinterpret_cast<const half8_t*>(lo + (t * 16 + l16) * pitch + k + g * 8);
        }
      };
      auto tile_of = [&](int t) {  // the tile's 16 tokens that are this adapter's
        return t < TT ? (uint32_t)((t < 4 ? mask[0] : mask[W - 1]) >> (t % 4 * 16)) & 0xFFFF : 0u;
      };
      auto bases = [&](int t, half8_t (&b)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          b[e] = load(m0 + t * 16 + g * 4 + e, n, (tile_of(t) >> (g * 4 + e) & 1) != 0);
      };
      // up to 64 ranks: this adapter's rows stay in registers for all tokens
      constexpr int KR = NQ <= 4 ? (NQ + 1) / 2 : 1;
      half8_t w[KR][kU];
      if constexpr (NQ <= 4) {
#pragma unroll
        for (int k = 0; k < KR; ++k)
#pragma unroll
          for (int u = 0; u < kU; ++u) w[k][u] = rank8(k * 32, u);
      }
      struct Ahead {  // what a tile of 16 tokens reads
        half8_t b[4];
        half8_t th[KR], tl[KR];
        float f[4];
      };
      auto read = [&](int t, Ahead& r) {
        bases(t, r.b);
        if constexpr (FOLDED) {
          t = t < TT ? t : TT - 1;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int m = m0 + t * 16 + g * 4 + e;
            r.f[e] = a.factors[(int64_t)i * a.M + (m < a.M ? m : a.M - 1)];
          }
          if constexpr (NQ <= 4) {
#pragma unroll
            for (int k = 0; k < KR; ++k) low(t, k * 32 < rp ? k * 32 : 0, r.th[k], r.tl[k]);
          }
        }
      };
      Ahead now, next;
      read(0, now);
#pragma unroll 1
      for (int t = 0; t < TT; ++t) {
        if (TT > 1) read(t + 1, next);
        const uint32_t tile = tile_of(t);
        if (tile != 0) {
          float4_t acc[kU] = {};
          auto product = [&](half8_t th, half8_t tl, const half8_t (&v)[kU]) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
              acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(tl, v[u], acc[u], 0, 0, 0);
              acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(th, v[u], acc[u], 0, 0, 0);
            }
          };
          if constexpr (NQ <= 4) {
#pragma unroll
            for (int k = 0; k < KR; ++k) {
              if (k * 32 < rp) {
                if constexpr (!FOLDED) low(t, k * 32, now.th[k], now.tl[k]);
                product(now.th[k], now.tl[k], w[k]);
              }
            }
          } else {
            for (int k = 0; k < rp; k += 32) {
#pragma unroll
              for (int u = 0; u < kU; ++u) w[0][u] = rank8(k, u);
              low(t, k, now.th[0], now.tl[0]);
              product(now.th[0], now.tl[0], w[0]);
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (tile >> (g * 4 + e) & 1) {
              const float f = FOLDED ? now.f[e] : factor[g * 4 + e];
              half8_t v;
#pragma unroll
              for (int u = 0; u < kU; ++u) v[u] = static_cast<half_t>((float)now.b[e][u] + f * acc[u][e]);
              store(m0 + t * 16 + g * 4 + e, n, v);
            }
        }
        now = next;
      }
    }
  });

  // tokens without an adapter
  if (j == 0 && p.base != p.y) {
    uint64_t has[W];
#pragma unroll
    for (int w = 0; w < W; ++w) has[w] = __ballot(ids.id[w] >= 0);
    for (int n0 = n_block + wave * (16 * kU); n0 < n_end; n0 += kSlice) {
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int tok = t * 16 + g * 4 + e;
          if (m0 + tok < a.M && !((t < 4 ? has[0] : has[W - 1]) >> (tok % 64) & 1))
            store(m0 + tok, n0 + l16 * kU, load(m0 + tok, n0 + l16 * kU, true));
        }
    }
  }
}

// Blocks of tokens, splits of K.
struct LoraPlan {
  int TD, TU;  // tokens of a block of k_lora_down, k_lora_up
  int RT, splits;
  int64_t k_share;
};

int64_t up_to(int64_t n, int64_t of) { return (n + of - 1) / of; }

LoraPlan plan_lora(int64_t M, int64_t K, int r, int count, const DeviceInfo& dev) {
  LoraPlan p;
  // More tokens share what a block reads of an adapter (700 tokens 30.5 us,
  // 31.8 with blocks of 16; 37 tokens 12.4, 12.7 with blocks of 32).
  p.TD = M > 64 ? 32 : 16;
  // Up to 16 ranks a workgroup sums its few low-rank values itself (1000 tokens
  // of 16 ranks 24.8 us, 32.8 folded in blocks of 128; 400 tokens of 64 ranks
  // 50 and 40).
  p.TU = M > 128 && r > 16 ? 128 : 16;
  p.RT = r <= 16 ? 1 : r <= 32 ? 2 : 4;
  // splits of at least 512 values, up to a workgroup a compute unit
  const int64_t wide = up_to(M, p.TD) * count * up_to(r, 16 * p.RT);
  int64_t s = up_to(dev.num_cus, wide);
  s = s > up_to(K, 512) ? up_to(K, 512) : s;
  s = s > kLoraMaxSplits ? kLoraMaxSplits : s;
  p.k_share = up_to(up_to(K, s), 32) * 32;
  p.splits = (int)up_to(K, p.k_share);
  return p;
}

// Workgroups that share the adapters of a block of TM tokens, which may hold
// one per token: as many as there is room for on the chip.  (They are the
// grid's slowest dimension: those that find nothing to do end together, and do
// not leave every other XCD idle.)
int sharers(int64_t M, int64_t L, int TM, int64_t wide, const DeviceInfo& dev) {
  int64_t j = up_to(2 * dev.num_cus, wide);
  j = j < L ? j : L;
  j = j < TM ? j : TM;
  return (int)(j < M ? j : M);
}

template <int TT, int RT>
hipError_t launch_down(const LoraArgs& a, dim3 grid, bool vec, hipStream_t stream) {
  return vec ? launch_kernel(k_lora_down<TT, RT, true>, grid, dim3(256), 0, stream, a)
             : launch_kernel(k_lora_down<TT, RT, false>, grid, dim3(256), 0, stream, a);
}

template <int TM, int NQ>
hipError_t launch_up(const LoraArgs& a, dim3 grid, bool vec, hipStream_t stream) {
  const size_t lds = TM > 16 ? 0 : TM * (up_to(a.r, 32) * 32 + 8) * 4 + TM * 4;  // at most 17 KB
  return launch_kernel(vec ? k_lora_up<TM, NQ, true> : k_lora_up<TM, NQ, false>, grid, dim3(256), lds, stream, a);
}

}  // namespace

int64_t lora_workspace_bytes(int64_t M, int64_t K, int r, int count, const DeviceInfo& dev) {
  const LoraPlan pl = plan_lora(M, K, r, count, dev);
  const int64_t t = up_to(pl.splits * M * r * count, 4) * 4;
  return (t + (pl.TU > 16 ? M * count * (up_to(r, 32) * 32 + 1) : 0)) * (int64_t)sizeof(float);
}

hipError_t launch_lora(const LoraProblem& p, const DeviceInfo& dev, hipStream_t stream) {
  const LoraPlan pl = plan_lora(p.M, p.K, p.r, p.count, dev);
  LoraArgs a = {};
  a.x = p.x;
  a.adapters = p.adapters;
  a.scales = p.scales;
  a.t = static_cast<float*>(p.workspace);
  a.M = (int)p.M;
  a.K = p.K;
  a.L = p.L;
  a.r = p.r;
  a.count = p.count;
  a.splits = pl.splits;
  a.k_share = pl.k_share;
  auto aligned = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  bool vec_k = p.K % 8 == 0 && aligned(p.x), vec_r = p.r % 8 == 0;
  int most_n = 0;
  for (int i = 0; i < p.count; ++i) {
    a.p[i].A = static_cast<const uint16_t*>(p.A[i]);
    a.p[i].B = static_cast<const uint16_t*>(p.B[i]);
    a.p[i].base = static_cast<const uint16_t*>(p.base[i]);
    a.p[i].y = static_cast<uint16_t*>(p.y[i]);
    a.p[i].N = (int)p.N[i];
    vec_k = vec_k && aligned(p.A[i]);
    vec_r = vec_r && aligned(p.B[i]) && p.N[i] % 8 == 0 && aligned(p.base[i]) && aligned(p.y[i]);
    if (a.p[i].N > most_n) most_n = a.p[i].N;
  }
  hipError_t e;
  const int64_t ranks = up_to(a.r, 16 * pl.RT);
  const int64_t td = up_to(p.M, pl.TD);
  a.J = sharers(p.M, p.L, pl.TD, td * a.count * ranks * pl.splits, dev);
  const dim3 down((unsigned)td, (unsigned)(a.count * ranks), (unsigned)(pl.splits * a.J));
  switch (pl.RT * 100 + pl.TD) {
    case 116: e = launch_down<1, 1>(a, down, vec_k, stream); break;
    case 216: e = launch_down<1, 2>(a, down, vec_k, stream); break;
    case 416: e = launch_down<1, 4>(a, down, vec_k, stream); break;
    case 132: e = launch_down<2, 1>(a, down, vec_k, stream); break;
    case 232: e = launch_down<2, 2>(a, down, vec_k, stream); break;
    default: e = launch_down<2, 4>(a, down, vec_k, stream); break;
  }
  if (e != hipSuccess) return e;
  if (pl.TU > 16) {
    a.low = reinterpret_cast<half_t*>(a.t + up_to(pl.splits * p.M * p.r * p.count, 4) * 4);
    a.factors = reinterpret_cast<float*>(a.low + p.M * p.count * 2 * (up_to(p.r, 32) * 32));
    e = launch_kernel(k_lora_fold, dim3((unsigned)up_to(p.M, 4), (unsigned)p.count), dim3(256), 0, stream, a);
    if (e != hipSuccess) return e;
  }
  // several slices share what a workgroup makes of the low-rank values, where
  // enough workgroups are left
  const int64_t slices = up_to(most_n, kSlice);
  // blocks of 64 where those of 128 leave compute units without work (200 tokens
  // of 64 ranks 29.6 us, 34 with 128; 1000 tokens 79 and 71)
  int64_t all_slices = 0;
  for (int i = 0; i < p.count; ++i) all_slices += up_to(p.N[i], kSlice);
  const int TU = pl.TU > 16 && 2 * up_to(p.M, 128) * all_slices < 3 * dev.num_cus ? 64 : pl.TU;
  const int64_t blocks = up_to(p.M, TU) * p.count;
  a.slices = 1;
  while (a.slices < 8 && blocks * up_to(slices, 2 * a.slices) >= 4 * dev.num_cus) a.slices *= 2;
  const int64_t tu = up_to(p.M, TU), ny = up_to(slices, a.slices);
  a.J = sharers(p.M, p.L, TU, tu * ny * a.count, dev);
  const dim3 up((unsigned)tu, (unsigned)ny, (unsigned)(a.count * a.J));
  if (TU == 16)
    return a.r <= 16   ? launch_up<16, 1>(a, up, vec_r, stream)
           : a.r <= 64 ? launch_up<16, 4>(a, up, vec_r, stream)
                       : launch_up<16, 16>(a, up, vec_r, stream);
  if (TU == 64)
    return a.r <= 64 ? launch_up<64, 4>(a, up, vec_r, stream) : launch_up<64, 16>(a, up, vec_r, stream);
  return a.r <= 64 ? launch_up<128, 4>(a, up, vec_r, stream) : launch_up<128, 16>(a, up, vec_r, stream);
}

}  // namespace fasq
