// Attention over a paged cache: the work of one wave, and where a workgroup's
// work lies in the batch.
//
// A wave holds 32 query rows.  A row is a (token, query head) pair of one
// cache head: with G = Hq / Hkv query heads per cache head, row r of a request
// is its token r / G and head r % G, so the heads of a group share the keys
// and values that a tile brings on chip, from one token (G rows) to a chunk.
//
// Scores are computed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_f16, keys
// down, queries across): lane l then holds 16 of every 32 keys of query l % 32,
// and its softmax statistics are its own but for one exchange with lane l ^ 32.
// The weights leave the score registers already in the layout of the second
// product's operand, O^T = V^T P^T, if V's rows are taken in the order the
// score registers have them, which is free: V^T comes from LDS through the
// transposing read (ds_read_b64_tr_b16), four rows at a time from anywhere.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fasq_device.h"
#include "fasq_layer.h"

namespace fasq {

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef half8_t half8_any __attribute__((aligned(2)));

// A request as the kernels read it: lengths cut to what exists.
struct Request {
  int q0, n, kv;
};

// A tile whose keys several shares of the batch hold (see Place), as its first
// share's workgroup leaves it for k_attention_join.
struct CutTile {
  int64_t start, end, share;
  Request r;
  int tile, head, cut;  // cut = 0: none starts in that share
};

struct AttentionArgs {
  HeadsView q, out;
  int64_t T, B;
  int Hq, Hkv, G, D;
  const uint16_t* ck;
  const uint16_t* cv;
  int num_pages;
  uint32_t page_size;
  int page_shift;  // log2(page_size), -1 where it is no power of two
  int g_shift;     // the same of G
  int64_t page_stride, slot_stride, head_stride;
  const int32_t* pages;
  int64_t page_row_stride;
  int capacity;  // max_pages * page_size: at most 2^31 - 1024, so that no key's number overflows, steps past the end too
  const int32_t* q_start;
  const int32_t* kv_len;
  float c;  // |scale| * log2(e), at least 1e-30 so that -inf stays -inf
  bool negate;  // scale < 0: the queries change sign instead
  bool causal;
  bool out_vec;  // 8-byte stores of out
  bool whole_units;     // pages hold whole units of 16 keys, within 2^31 bytes
  int window;  // 0: none, or all that there can be
  float* lse;
  // Split over workgroups (part_o != nullptr): workgroup w of `parts` takes
  // the w-th equal share of the batch's keys; see Place.
  int parts;
  int64_t first;  // without a split: the launch's first workgroup of all
  float* part_o;  // [2 * parts][rows][DP], not divided by the sum
  float* part_ml;  // [2 * parts][rows][2]: maximum (in powers of two), sum
  CutTile* cuts;   // [parts]
};

// The kernel's arguments (its only parameter), as if read for the first time:
// where a kernel starts a new phase it reads what it needs again, a scalar load
// or two, instead of holding all of it and what follows from it in registers
// from the start on (which cost hundreds of instructions before the first key).
__device__ __forceinline__ const AttentionArgs& fresh_args() {
  auto p = (__attribute__((address_space(4))) const AttentionArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttentionArgs*)p;
}

// ---------------------------------------------------------------------------
// Where work lies
// ---------------------------------------------------------------------------

// Quotients without the long way round that a 64-bit division, or one by a
// value that is no constant, takes (about a microsecond of a short call).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}
__device__ __forceinline__ int token_of(const AttentionArgs& a, int row) {
  return a.g_shift >= 0 ? row >> a.g_shift : (int)((uint32_t)row / (uint32_t)a.G);
}

__device__ __forceinline__ Request read_request(const AttentionArgs& a, int64_t b) {
  const int T = (int)a.T;
  int q0 = a.q_start[b], q1 = a.q_start[b + 1], kv = a.kv_len[b];
  q0 = q0 < 0 ? 0 : q0 > T ? T : q0;
  q1 = q1 < q0 ? q0 : q1 > T ? T : q1;
  kv = kv < 0 ? 0 : kv > a.capacity ? a.capacity : kv;
  return {q0, q1 - q0, kv};
}

// The batch as a wave sees it: lane l keeps requests l, l + 64, ..., the first
// of them in registers (all there are in most batches).
struct Batch {
  Request first;
  __device__ __forceinline__ explicit Batch(const AttentionArgs& a) {
    const int lane = threadIdx.x % kWave;
    first = lane < a.B ? read_request(a, lane) : Request{0, 0, 0};
  }
  __device__ __forceinline__ Request of(const AttentionArgs& a, int64_t b) const {
    return b < kWave ? first : read_request(a, b);
  }
};

// Keys [begin, end) that token i of a request sees.
struct Span {
  int begin, end;
};

__device__ __forceinline__ Span token_span(const AttentionArgs& a, const Request& r, int i) {
  const int pos = r.kv - r.n + i;  // may be negative: more new tokens than keys
  int end = a.causal && pos + 1 < r.kv ? pos + 1 : r.kv;
  int begin = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  end = end < 0 ? 0 : end;
  return {begin < end ? begin : end, end};
}

// Keys that some token of tile t (ROWS rows) sees.
template <int ROWS>
__device__ __forceinline__ Span tile_span(const AttentionArgs& a, const Request& r, int t) {
  const int rows = r.n * a.G;
  const int last = (t + 1) * ROWS < rows ? (t + 1) * ROWS : rows;
  const Span s0 = token_span(a, r, token_of(a, t * ROWS)), s1 = token_span(a, r, token_of(a, last - 1));
  return {s0.begin < s1.begin ? s0.begin : s1.begin, s1.end > s0.end ? s1.end : s0.end};
}

// The batch as a line of positions.  With `parts` shares, every cache head
// has the same stretch, in it the requests in order, in them their tiles, and
// a tile is as long as the keys its request can need (a multiple of STEP, at
// least one).  Share w holds the positions [w * share, (w + 1) * share): each
// workgroup has the same number of keys to read, whatever the lengths, and a
// tile is cut only where two shares meet.  Without shares a tile is one
// position long.
struct Place {
  int b, tile, head;
  Request r;
  int64_t start, end;  // the tile's positions
};

template <int ROWS, int STEP>
__device__ __forceinline__ int64_t tile_length(const AttentionArgs& a, const Request& r, bool shared) {
  if (!shared) return 1;
  int keys = r.kv;
  if (a.window > 0) {
    // of the tile's tokens, from a multiple of 32 on; without causality the
    // request's first token sees the window before it and all that follows
    const int besides = (a.causal ? token_of(a, ROWS) : r.n) + 32;
    keys = keys - besides > a.window ? a.window + besides : keys;
  }
  return keys <= STEP ? STEP : ((int64_t)keys + STEP - 1) / STEP * STEP;
}

// A value that every lane of the wave holds, as a scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)v), hi = (uint32_t)uniform((int)(uint32_t)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// Lane l's value (l uniform), as a scalar.
__device__ __forceinline__ int lane_value(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ int64_t lane_value(int64_t v, int l) {
  const uint32_t lo = (uint32_t)lane_value((int)(uint32_t)v, l), hi = (uint32_t)lane_value((int)(uint32_t)(v >> 32), l);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ int64_t wave_total(int64_t v) {
#pragma unroll
  for (int x = 1; x < kWave; x *= 2) v += __shfl_xor(v, x, kWave);
  return v;
}

template <int ROWS>
__device__ __forceinline__ int tiles_of(const AttentionArgs& a, const Request& r) {
  return (r.n * a.G + ROWS - 1) / ROWS;
}

// Positions of one cache head.
template <int ROWS, int STEP>
__device__ __forceinline__ int64_t head_length(const AttentionArgs& a, const Batch& batch, bool shared) {
  int64_t sum = 0;
  for (int64_t b = threadIdx.x % kWave; b < a.B; b += kWave) {
    const Request r = batch.of(a, b);
    sum += tiles_of<ROWS>(a, r) * tile_length<ROWS, STEP>(a, r, shared);
  }
  return a.B == 1 ? lane_value(sum, 0) : uniform(wave_total(sum));
}

// The tile at a position within a head's stretch, in every lane of the wave.
// pos < head_length.
template <int ROWS, int STEP>
__device__ __forceinline__ Place locate(const AttentionArgs& a, const Batch& batch, int64_t pos, bool shared) {
  Place p = {};
  int64_t base = 0;
  for (int64_t b0 = 0; b0 < a.B; b0 += kWave) {
    const int64_t b = b0 + threadIdx.x % kWave;
    Request r = {};
    int64_t one = 0, own = 0;
    if (b < a.B) {
      r = batch.of(a, b);
      one = tile_length<ROWS, STEP>(a, r, shared);
      own = tiles_of<ROWS>(a, r) * one;
    }
    int64_t upto = own;  // positions up to and with this lane's request
    if (a.B > 1) {
#pragma unroll
      for (int x = 1; x < kWave; x *= 2) {
        const int64_t below = __shfl_up(upto, x, kWave);
        if ((int)(threadIdx.x % kWave) >= x) upto += below;
      }
    }
    const uint64_t hit = __ballot(base + upto > pos && b < a.B);
    if (hit != 0) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      p.b = (int)(b0 + l);
      p.r.q0 = lane_value(r.q0, l);
      p.r.n = lane_value(r.n, l);
      p.r.kv = lane_value(r.kv, l);
      one = lane_value(one, l);
      const int64_t first = base + lane_value(upto - own, l);
      p.tile = (int)quotient(pos - first, one);
      p.start = first + p.tile * one;
      p.end = p.start + one;
      return p;
    }
    base += lane_value(upto, kWave - 1);
  }
  p.b = -1;
  return p;
}

// Element offset of key j's row in a cache head (page table row `pages`).
__device__ __forceinline__ int64_t key_offset(const AttentionArgs& a, int page, int j) {
  const uint32_t in_page = a.page_shift >= 0 ? (uint32_t)j & (a.page_size - 1) : (uint32_t)j % a.page_size;
  page = page < 0 ? 0 : page >= a.num_pages ? a.num_pages - 1 : page;
  return page * a.page_stride + in_page * a.slot_stride;
}

__device__ __forceinline__ int page_of(const AttentionArgs& a, const int32_t* pages, int j) {
  return pages[a.page_shift >= 0 ? (uint32_t)j >> a.page_shift : (uint32_t)j / a.page_size];
}

// ---------------------------------------------------------------------------
// Keys and values in LDS: rows of DP values, 16-byte chunks permuted within a
// row so that both readers meet all banks: 16 lanes reading one chunk column
// of 16 rows (scores), and 32 lanes reading four chunks of four neighbouring
// rows (the transposing read).
// ---------------------------------------------------------------------------
template <int DP>
__device__ __forceinline__ int chunk_swap(int row) {
  if constexpr (DP == 64) return ((row & 2) << 1) | ((row >> 2) & 3);
  else return ((row & 3) << 2) | ((row >> 2) & 3);
}

// Wait until at most N of this wave's vector-memory operations are in flight
// (gfx9 encoding), and a barrier that neither waits for them nor lets the
// compiler move memory accesses across.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
  asm volatile("" ::: "memory");
}
// Wait for this wave's reads of LDS: before copies that overwrite what they read.
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (0x7 << 4) | (0 << 8));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// LDS by its address: rows are powers of two long, so the permuted chunk of a
// column is one exclusive or away from the lane's first address, and rows
// and blocks are immediate offsets.
typedef __attribute__((address_space(3))) const half8_t* lds_half8;
typedef __attribute__((address_space(3))) short4_t* lds_short4;
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// Copies of 16 bytes a lane from memory to LDS (address `to`, uniform, plus 16
// bytes a lane).  Written out because the compiler holds every transposing
// read of LDS back until all copies it knows of have landed, also those of
// other stages; the kernels wait for their copies themselves (wait_loads).
__device__ __forceinline__ void copy16_to_lds(const uint16_t* src, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory");
}
// The same from a uniform base and a byte offset per lane.
__device__ __forceinline__ void copy16_to_lds(const uint16_t* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base)
               : "memory");
}

// Copies of 16 rows of a cache head to LDS by one wave, INSTR copies of RPI
// rows.  FULL: D is DP.
template <int DP, bool FULL>
struct RowCopy {
  static constexpr int CH = DP / 8, RPI = kWave / CH, INSTR = 16 / RPI;
  uint32_t offset[INSTR];  // of this lane, where the 16 rows lie in one page
  uint32_t on;             // bit i: copy i brings a chunk below D

  __device__ __forceinline__ explicit RowCopy(const AttentionArgs& a) {
    const int lane = threadIdx.x % kWave;
    on = 0;
#pragma unroll
    for (int i = 0; i < INSTR; ++i) {
      const int row = i * RPI + lane / CH, chunk = (lane % CH) ^ chunk_swap<DP>(row);
      offset[i] = (uint32_t)(row * a.slot_stride + chunk * 8) * 2;
      on |= (chunk * 8 < a.D ? 1u : 0u) << i;
    }
  }

  // Whether keys k .. k + 15 (k a multiple of 16) lie in one page and in
  // [first, last], so that they can be copied from one base.
  __device__ __forceinline__ static bool whole(const AttentionArgs& a, int k, int first, int last) {
    return a.whole_units && k >= first && k + 15 <= last;
  }
  // Their offset in the cache: `page` is their page, in any lane.
  __device__ __forceinline__ static int64_t whole_offset(const AttentionArgs& a, int64_t head_off, int page, int k) {
    return uniform(key_offset(a, uniform(page), k) + head_off);
  }
  // Copy i of them.  to: the LDS address of the first row.
  __device__ __forceinline__ void one(const uint16_t* base, int i, uint32_t to) const {
    if (FULL || (on >> i & 1)) copy16_to_lds(base, offset[i], to + i * 1024);
  }
  // Any keys k .. k + 15, those outside [first, last] in the place of the
  // nearest inside.  `page`: lane l's page of key k + l % 16 as cut (page_of).
  __device__ __forceinline__ void each(const AttentionArgs& a, const uint16_t* cache, int64_t head_off, int page, int k,
                                       int first, int last, uint32_t to) const {
    const int lane = threadIdx.x % kWave, j = k + lane % 16;
    const int64_t own = key_offset(a, page, j < first ? first : j < last ? j : last) + head_off;
    int64_t off[INSTR];
#pragma unroll
    for (int i = 0; i < INSTR; ++i) off[i] = __shfl(own, i * RPI + lane / CH, kWave);
#pragma unroll
    for (int i = 0; i < INSTR; ++i) {
      const int chunk = (lane % CH) ^ chunk_swap<DP>(i * RPI + lane / CH);
      if (FULL || (on >> i & 1)) copy16_to_lds(cache + off[i] + chunk * 8, to + i * 1024);
    }
  }
  __device__ __forceinline__ void run(const AttentionArgs& a, const uint16_t* cache, int64_t head_off, int page, int k,
                                      int first, int last, uint32_t to) const {
    if (whole(a, k, first, last)) {
      const uint16_t* from = cache + whole_offset(a, head_off, page, k);
#pragma unroll
      for (int i = 0; i < INSTR; ++i) one(from, i, to);
    } else {
      each(a, cache, head_off, page, k, first, last, to);
    }
  }
};

// Values of a tile that some of its rows do not see: a weight of zero leaves a
// finite value out of a sum, but not NaN or an infinity.  Where rows of a tile
// see different keys (only there), the tile's values are cut to finite ones in
// LDS before they are used.  Returns whether any was not (in any lane): then
// rows are checked key by key at the end (SlowRow).  One wave, rows [0, ROWS)
// of DP values that it has copied itself.
template <int DP, int ROWS>
__device__ __forceinline__ bool cut_to_finite(uint16_t* values) {
  constexpr int N = ROWS * DP / 8 / kWave;
  const half_t most = static_cast<half_t>(65504.f);
  half8_t bad = {};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    half8_t* at = reinterpret_cast<half8_t*>(values) + i * kWave + threadIdx.x % kWave;
    const half8_t v = *at;
    bad += v * half8_t{};  // NaN where v is not finite
    *at = __builtin_elementwise_min(__builtin_elementwise_max(v, half8_t(-most)), half8_t(most));
  }
  bool nan = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) nan = nan || !(bad[e] == static_cast<half_t>(0.f));
  return __any(nan);
}

// ---------------------------------------------------------------------------
// One wave: 32 rows against KB blocks of 32 keys at a time
// ---------------------------------------------------------------------------

// Weights enter the second product in fp16, 2^kLift times larger than relative
// to the running maximum: then they have 11 bits down to 2^-21 of the row's
// largest, and vanish (while the fp32 sum still counts them) only below 2^-32 of it
// rather than 2^-25, which a sum over 131072 keys beside one far larger shows.
// With kLift 7 and a maximum up to 2^8 behind they stay below fp16's largest
// value, but for scores of 2^24 powers of two and more, whose rounding may pass
// it: such rows end not finite and are computed again (SlowRow).
constexpr float kLift = 7.f;

template <int DP, int KB>
struct WaveTile {
  half8_t q[DP / 16];
  float16_t o[DP / 32];
  // running maximum of the scores (this row), and m * c - kLift (0 without one)
  float m, mc;
  float l, rest;  // sum of this lane's weights, and what its last addition rounded up

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    m = -INFINITY;
    mc = 0.f;
    l = rest = 0.f;
  }

  // A block's weights to the sum.  In fp32 alone, 65536 weights of 2^-24.6 beside one
  // of 1 leave it at 1: it is held with what each addition rounds (compensated
  // summation), so that it is off by a few roundings whatever the length.
  __device__ __forceinline__ void add_block(float sum) {
    const float more = sum - rest, next = l + more;
    rest = (next - l) - more;
    l = next;
  }
  __device__ __forceinline__ void scale_sum(float keep) {
    l *= keep;
    rest *= keep;
  }

  // Row `row` of the request, which exists (lane l and l ^ 32 hold one row;
  // zeros unless `live`, and past D).
  __device__ __forceinline__ void load_q(const AttentionArgs& a, const Request& r, int head, int row, bool live) {
    const int h = (threadIdx.x % kWave) / 32;
    const int t = token_of(a, row);
    const uint16_t* src = a.q.p + (r.q0 + t) * a.q.ts + (head * a.G + row - t * a.G) * a.q.hs;
    // all loads first (wherever rows start), then what they have to wait for
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      const int d = s * 16 + h * 8;
      q[s] = *reinterpret_cast<const half8_any*>(src + (d < a.D ? d : 0));
    }
    const uint32_t flip = a.negate ? 0x80008000u : 0u;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      u32x4 w = __builtin_bit_cast(u32x4, q[s]);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = live && s * 16 + h * 8 < a.D ? w[e] ^ flip : 0u;
      q[s] = __builtin_bit_cast(half8_t, w);
    }
  }

  // keys, values: the tile's rows in LDS (KB * 32 of them); key0: its first
  // key.  A row sees keys [begin, end); `masked` (uniform): not every live row
  // sees all of the tile.  Operands are read from LDS a step or two ahead of
  // the products that take them; the scheduling barriers keep them there.
  __device__ __forceinline__ void step(const uint16_t* keys, const uint16_t* values, int key0, int begin, int end,
                                       bool masked, float c) {
    const int lane = threadIdx.x % kWave, l32 = lane % 32, h = lane / 32;
    constexpr int KT = DP / 16, AHEAD = 2;
    const uint32_t k_at = lds_address(keys) + l32 * (DP * 2) + (h ^ chunk_swap<DP>(l32)) * 16;
    half8_t k[AHEAD + 1][KB];
    auto read_k = [&](int t) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        k[t % (AHEAD + 1)][kb] = *(lds_half8)(uintptr_t)((k_at ^ (t % 8 * 32)) + t / 8 * 256 + kb * 32 * DP * 2);
    };
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) read_k(t);
    float16_t s[KB];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      if (t + AHEAD < KT) read_k(t + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[t % (AHEAD + 1)][kb], q[t], t == 0 ? float16_t{} : s[kb], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    // rows of V in the order of the score registers: weight j of slab u is
    // key 16 u + (j / 4) * 8 + h * 4 + j % 4; operands in groups of four
    // blocks of 32 dimensions
    constexpr int GI = DP / 32 < 4 ? DP / 32 : 4, GROUPS = 2 * KB * (DP / 32) / GI;
    const int r = (lane % 16) / 4, x = (lane / 16 & 1) * 2 + (lane & 3) / 2;
    uint32_t v_at[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = j * 8 + h * 4 + r;
      v_at[j] = lds_address(values) + row * (DP * 2) + (x ^ chunk_swap<DP>(row)) * 16 + (lane & 1) * 8;
    }
    short4_t v[2][GI][2];
    auto read_v = [&](int g) {
      const int u = g * GI / (DP / 32), i0 = g * GI % (DP / 32);
#pragma unroll
      for (int i = 0; i < GI; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          v[g % 2][i][j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_short4)(uintptr_t)((v_at[j] ^ ((i0 + i) % 4 * 64)) + (i0 + i) / 4 * 256 + u * 16 * DP * 2));
    };
    read_v(0);
    __builtin_amdgcn_sched_barrier(0);
    if (masked) {
      const int first = begin - key0 - h * 4, last = end - key0 - h * 4;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = kb * 32 + (e / 4) * 8 + e % 4;
          s[kb][e] = key < first || key >= last ? -INFINITY : s[kb][e];
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
    {
      const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      top = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
    }
    // The maximum need not be the newest one: weights up to 2^15 are as exact
    // in fp16 as weights up to 2^7, so a row is rescaled only where its maximum
    // has grown by more than 2^8 (each row by its own scores alone).
    const bool grown = (top - m) * c > 8.f;  // from -inf too; not from -inf to -inf
    if (__any(grown)) {
      // the weights are 2^(s c - mc) with the rounded mc, here too
      const float next_c = top * c - kLift;
      const float keep = !grown ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - next_c);
      scale_sum(keep);
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= keep;
      m = grown ? top : m;
      mc = grown ? next_c : mc;
    }
    half8_t p[2 * KB];
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = __builtin_amdgcn_exp2f(s[kb][e] * c - mc);
        sum += w;
        p[2 * kb + e / 8][e % 8] = static_cast<half_t>(w);
      }
    add_block(sum);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      if (g + 1 < GROUPS) read_v(g + 1);
      __builtin_amdgcn_sched_barrier(0);
      const int u = g * GI / (DP / 32), i0 = g * GI % (DP / 32);
#pragma unroll
      for (int i = 0; i < GI; ++i) {
        const half8_t vv = __builtin_bit_cast(
            half8_t, __builtin_shufflevector(v[g % 2][i][0], v[g % 2][i][1], 0, 1, 2, 3, 4, 5, 6, 7));
        o[i0 + i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv, p[u], o[i0 + i], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // -------------------------------------------------------------------------
  // The same as a pipeline of blocks of 32 keys, for rows whose work the
  // matrix cores bound: while the vector ALUs turn block b's scores into
  // weights, the matrix cores compute the scores of block b + 1 and add the
  // weighted values of block b - 1.  The two do not depend on each other, and
  // one step is one MFMA (32 cycles), its share of the block's 16 scores per
  // lane, and the LDS reads of an operand three steps ahead.  With two waves a
  // SIMD, which is what the registers allow, a step takes a wave 114 cycles, what
  // lies between blocks included (2048 tokens after 6144: 411000 cycles for
  // 3616 steps on average, with 7.4 vector instructions each): the
  // exponential, the LDS read, the copies and the wait for the last sum add up in it.
  // -------------------------------------------------------------------------
  static constexpr int N = DP / 16;  // products of a block with the keys, and with the values
  static constexpr int OPS = 4;      // operands held: the current one and three ahead
  u32x4 ops[OPS];

  // The steps: a product with the keys adds to the one before it, and the matrix
  // cores take one that has to wait for its sum at half their rate, so two
  // of them are followed by one with the values (which add to DP / 32 sums in
  // turn); at DP = 64, where the scores would come too late for their maximum,
  // the keys come first.
  static constexpr bool MIXED = N > 4;
  static constexpr bool is_key(int i) { return MIXED ? i < N / 2 * 3 && i % 3 < 2 : i < N; }
  static constexpr int nth(int i) {  // of its kind
    return !MIXED ? i % N : i >= N / 2 * 3 ? i - N : i % 3 < 2 ? i / 3 * 2 + i % 3 : i / 3;
  }
  static constexpr int SCORED = MIXED ? N / 2 * 3 - 2 : N - 1;  // the last step with the keys

  // This lane's addresses of the operands in the first rows of LDS; stages and
  // blocks of rows are constant offsets from there.
  struct Lanes {
    uint32_t k[N < 8 ? N : 8], v[2][DP / 32 < 4 ? DP / 32 : 4];
    __device__ __forceinline__ explicit Lanes(const uint16_t* first) {
#pragma unroll
      for (int t = 0; t < N && t < 8; ++t) k[t] = key_lane(first) ^ (t * 32);
#pragma unroll
      for (int d = 0; d < DP / 32 && d < 4; ++d)
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j][d] = value_lane(first, j) ^ (d * 64);
    }
  };

  // The operand of step i: keys and values at these byte offsets.
  __device__ __forceinline__ void read_op(const Lanes& at, uint32_t k_off, uint32_t v_off, int i) {
    if (is_key(i)) {
      const int t = nth(i);
      ops[i % OPS] = __builtin_bit_cast(u32x4, *(lds_half8)(uintptr_t)(at.k[t % 8] + (k_off + t / 8 * 256)));
      return;
    }
    const int u = nth(i) / (DP / 32), d = nth(i) % (DP / 32);
    short4_t part[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_short4)(uintptr_t)(at.v[j][d % 4] + (v_off + d / 4 * 256 + u * 16 * DP * 2)));
    ops[i % OPS] = __builtin_bit_cast(u32x4, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }

  // This lane's first addresses in a block of 32 rows of keys and of values.
  static __device__ __forceinline__ uint32_t key_lane(const uint16_t* keys) {
    const int lane = threadIdx.x % kWave, l32 = lane % 32;
    return lds_address(keys) + l32 * (DP * 2) + (lane / 32 ^ chunk_swap<DP>(l32)) * 16;
  }
  static __device__ __forceinline__ uint32_t value_lane(const uint16_t* values, int j) {
    const int lane = threadIdx.x % kWave, x = (lane / 16 & 1) * 2 + (lane & 3) / 2;
    const int row = j * 8 + lane / 32 * 4 + lane % 16 / 4;
    return lds_address(values) + row * (DP * 2) + (x ^ chunk_swap<DP>(row)) * 16 + (lane & 1) * 8;
  }

  // Scores of a block alone.
  __device__ __forceinline__ void scores(uint32_t k_at, float16_t& s) {
    auto read = [&](int t) {
      ops[t % OPS] = __builtin_bit_cast(u32x4, *(lds_half8)(uintptr_t)((k_at ^ (t % 8 * 32)) + t / 8 * 256));
    };
#pragma unroll
    for (int t = 0; t < OPS - 1; ++t) read(t);
#pragma unroll
    for (int t = 0; t < N; ++t) {
      if (t + OPS - 1 < N) read(t + OPS - 1);
      __builtin_amdgcn_sched_barrier(0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, ops[t % OPS]), q[t],
                                                 t == 0 ? float16_t{} : s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Weights of scores alone.
  __device__ __forceinline__ void weights(const float16_t& s, half8_t (&p)[2], float c) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = __builtin_amdgcn_exp2f(s[e] * c - mc);
      sum += w;
      p[e / 8][e % 8] = static_cast<half_t>(w);
    }
    add_block(sum);
  }

  // The larger of this lane's value and the other's of its row.
  static __device__ __forceinline__ float row_max(float top) {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
  }

  // Before a block's weights: its mask and the running maximum.  top, over:
  // the row's largest score, and by how much it passes the maximum, in powers
  // of two (where nothing is masked).  p: weights that have not met their
  // values yet.
  __device__ __forceinline__ void settle(float16_t& s, float top, float over, half8_t (&p)[2], int key0, int begin,
                                         int end, bool masked, float c) {
    if (masked) {
      const int h4 = threadIdx.x % kWave / 32 * 4, first = begin - key0 - h4, last = end - key0 - h4;
      top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = (e / 4) * 8 + e % 4;
        s[e] = key < first || key >= last ? -INFINITY : s[e];
        top = fmaxf(top, s[e]);
      }
      top = row_max(top);
      over = (top - m) * c;
    }
    const bool grown = over > 8.f;  // as in step()
    if (__any(grown)) {
      const float next_c = top * c - kLift;
      const float keep = !grown ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - next_c);
      scale_sum(keep);
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= keep;
      // these weights are now below 2^-8 of the largest: one more rounding of theirs is nothing
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e / 8][e % 8] = static_cast<half_t>((float)p[e / 8][e % 8] * keep);
      m = grown ? top : m;
      mc = grown ? next_c : mc;
    }
  }

  // One block: the weights `made` of its scores s, the scores `next` of the
  // block at k_off, the values at v_off weighted with `p`, and next's largest score
  // of the row (top) and by how much it passes the maximum (over).  The operands
  // of the first three steps are there; those of the block after this one are
  // read if `more` (32 rows further).  at_step(i): what else step i issues.
  template <typename F>
  __device__ __forceinline__ void block(const float16_t& s, float16_t& next, const half8_t (&p)[2], half8_t (&made)[2],
                                        const Lanes& at, uint32_t k_off, uint32_t v_off, bool more, float c,
                                        float& top, float& over, F at_step) {
    constexpr int STEPS = 2 * N;
    float w[16], sum;
    u32x4 packed[2];
    auto add = [&](int e) {
      sum = e == 0 ? w[0] : sum + w[e];
      asm volatile("" : "+v"(sum));
      if (e % 2 == 1) {
        typedef _Float16 pair_t __attribute__((ext_vector_type(2)));
        uint32_t pair = __builtin_bit_cast(uint32_t, pair_t{static_cast<half_t>(w[e - 1]), static_cast<half_t>(w[e])});
        asm volatile("" : "+v"(pair));
        packed[e / 8][e % 8 / 2] = pair;
      }
    };
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int j = i + OPS - 1;
      if (j < STEPS) read_op(at, k_off, v_off, j);
      else if (more) read_op(at, k_off + 32 * DP * 2, v_off + 32 * DP * 2, j - STEPS);
      __builtin_amdgcn_sched_barrier(0);
      const half8_t op = __builtin_bit_cast(half8_t, ops[i % OPS]);
      if (is_key(i)) next = __builtin_amdgcn_mfma_f32_32x32x16_f16(op, q[nth(i)], i == 0 ? float16_t{} : next, 0, 0, 0);
      else {
        const int u = nth(i) / (DP / 32), d = nth(i) % (DP / 32);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(op, p[u], o[d], 0, 0, 0);
      }
#pragma unroll
      for (int e = 16 * i / STEPS; e < 16 * (i + 1) / STEPS; ++e) {
        // computed here, not where it is used: the compiler would move it
        // there (the empty asm statements); a weight is added up a step later,
        // when the exponential is there
        w[e] = __builtin_amdgcn_exp2f(s[e] * c - mc);
        asm volatile("" : "+v"(w[e]));
        if (e >= 1) add(e - 1);
      }
      // the maximum, from the second step after the scores are complete on
      if (i == SCORED + 2 || i == SCORED + 3) {
#pragma unroll
        for (int e = i == SCORED + 2 ? 0 : 8; e < (i == SCORED + 2 ? 8 : 16); ++e) top = e == 0 ? next[0] : fmaxf(top, next[e]);
        asm volatile("" : "+v"(top));
      }
      if (i == SCORED + 4) {
        top = row_max(top);
        over = (top - m) * c;
        asm volatile("" : "+v"(top), "+v"(over));
      }
      at_step(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    add(15);
    add_block(sum);
    made[0] = __builtin_bit_cast(half8_t, packed[0]);
    made[1] = __builtin_bit_cast(half8_t, packed[1]);
  }

  // What partial results' weights are relative to, in powers of two.
  __device__ __forceinline__ float top() const { return m == -INFINITY ? m : mc; }

  // Sum of the row's weights, in both its lanes.
  __device__ __forceinline__ float total() const {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }

  // Whether this lane's part of the row holds a value that is not finite.
  __device__ __forceinline__ bool broken() const {
    float z = (l - l) + (mc - mc);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) z += o[i][e] - o[i][e];
    return !(z == 0.f);
  }
};

// fp16 bits to fp32.
__device__ __forceinline__ float half_value(uint16_t b) { return (float)__builtin_bit_cast(half_t, b); }

// What a finished row holds: its sum of weighted values still has to be
// divided by l.  A row that sees keys but whose scores are all -inf is 0 / 0.
__device__ __forceinline__ float row_factor(float l, bool sees) {
  return l == 0.f ? (sees ? __builtin_nanf("") : 0.f) : 1.f / l;
}
__device__ __forceinline__ float row_lse(float mc, float l, bool sees) {
  if (l == 0.f) return sees ? __builtin_nanf("") : -INFINITY;
  return (mc + __log2f(l)) * 0.69314718055994530942f;
}

// One row over the keys [begin, end), key by key, by a whole wave: for rows
// whose result is not finite, or whose masked tiles held values that are not.
// Only keys that the row sees are touched.  Lane l holds dimensions l, l + 64, ...
template <int DP>
struct SlowRow {
  float m = -INFINITY, l = 0.f, o[(DP + kWave - 1) / kWave] = {};

  __device__ __forceinline__ void run(const AttentionArgs& a, const uint16_t* q, int64_t head_off,
                                      const int32_t* pages, int begin, int end) {
    const int lane = threadIdx.x % kWave;
    for (int j0 = begin; j0 < end; j0 += kWave) {
      const int j = j0 + lane;
      float s = -INFINITY;
      int64_t off = 0;
      if (j < end) {
        off = key_offset(a, page_of(a, pages, j), j) + head_off;
        s = 0.f;
        for (int i = 0; i < a.D; ++i) s += half_value(q[i]) * half_value(a.ck[off + i]);
        s *= a.negate ? -a.c : a.c;
      }
      float top = s;
#pragma unroll
      for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
      const float next = fmaxf(m, top);
      const float p = j < end ? exp2f(s - (next == -INFINITY ? 0.f : next)) : 0.f;
      const float keep = l == 0.f ? 0.f : exp2f(m - next);
      l = l * keep + wave_sum(p);
      m = next;
#pragma unroll
      for (float& v : o) v = keep == 0.f ? 0.f : v * keep;
      const int count = end - j0 < kWave ? end - j0 : kWave;
      for (int e = 0; e < count; ++e) {
        const float w = __shfl(p, e, kWave);
        const int64_t vo = __shfl(off, e, kWave);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(o) / sizeof(float)); ++i)
          if (lane + i * kWave < a.D) o[i] += w * half_value(a.cv[vo + lane + i * kWave]);
      }
    }
  }

  // Writes the row, to the output (slot < 0) or as row `at` of a slot, if it
  // holds a value that is not finite or the one there does (`broken`): the
  // tiles' result stands for rows that see finite values alone.
  template <int ROWS>
  __device__ __forceinline__ void store(const AttentionArgs& a, const Request& r, int head, int row, int at,
                                        int64_t slot, bool sees, bool broken) const {
    const int lane = threadIdx.x % kWave;
    constexpr int N = (DP + kWave - 1) / kWave;
    float z = l - l;
#pragma unroll
    for (int i = 0; i < N; ++i) z += o[i] - o[i];
    if (!broken && !__any(!(z == 0.f))) return;
    if (slot >= 0) {
      const int64_t to = slot * ROWS + at;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (lane + i * kWave < DP) a.part_o[to * DP + lane + i * kWave] = o[i];
      if (lane == 0) {
        a.part_ml[to * 2] = m;
        a.part_ml[to * 2 + 1] = l;
      }
      return;
    }
    const float f = row_factor(l, sees);
    const int t = token_of(a, row);
    uint16_t* dst = a.out.p + (r.q0 + t) * a.out.ts + (head * a.G + row - t * a.G) * a.out.hs;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + i * kWave < a.D) dst[lane + i * kWave] = f32_to_f16_bits(o[i] * f);
    if (lane == 0 && a.lse != nullptr)
      a.lse[(int64_t)(r.q0 + t) * a.Hq + head * a.G + row - t * a.G] = row_lse(m, l, sees);
  }
};

}  // namespace fasq
