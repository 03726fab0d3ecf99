// Attention of new tokens over a paged cache: kernels, and the launch of one variant.
//
//   k_attention_few   up to 32 rows of a cache head (decode, a few tokens): the
//                     waves of a workgroup share the rows and split the keys
//   k_attention_tile  128 rows: the waves share the keys and split the rows
//   k_attention_join  joins what shares of a tile's keys gave
#pragma once

#include <hip/hip_runtime.h>

#include "fasq_attention.h"

namespace fasq {

// Which kernel a call takes, and its grid.
struct AttentionPlan {
  bool few;       // k_attention_few
  int DP;
  int rows;       // of a tile
  int64_t tiles;  // at most, of one cache head
  int parts;      // shares of a split call
  bool split;     // worth splitting
  int classes;    // of tiles in a split call with masks or scores of its own
  int64_t bytes;  // of the workspace
};

namespace {

// Stores four consecutive values of an output row.
__device__ __forceinline__ void store4(const AttentionArgs& a, uint16_t* dst, int d, const float (&v)[4]) {
  if (d >= a.D) return;  // D is a multiple of 8
  if (a.out_vec) {
    half4_t h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = static_cast<half_t>(v[i]);
    *reinterpret_cast<half4_t*>(dst + d) = h;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[d + i] = f32_to_f16_bits(v[i]);
  }
}

__device__ __forceinline__ uint16_t* out_row(const AttentionArgs& a, const Request& r, int head, int row) {
  const int t = token_of(a, row);
  return a.out.p + (r.q0 + t) * a.out.ts + (head * a.G + row - t * a.G) * a.out.hs;
}

__device__ __forceinline__ const uint16_t* query_row(const AttentionArgs& a, const Request& r, int head, int row) {
  const int t = token_of(a, row);
  return a.q.p + (r.q0 + t) * a.q.ts + (head * a.G + row - t * a.G) * a.q.hs;
}

__device__ __forceinline__ int64_t lse_at(const AttentionArgs& a, const Request& r, int head, int row) {
  const int t = token_of(a, row);
  return (int64_t)(r.q0 + t) * a.Hq + head * a.G + row - t * a.G;
}

// Chunks past D are zero and stay so.
template <int DP>
__device__ __forceinline__ void clear_lds(uint16_t* at, int rows) {
  const u32x4 zero = {0, 0, 0, 0};
  for (int i = threadIdx.x % kWave; i < rows * DP / 8; i += kWave) reinterpret_cast<u32x4*>(at)[i] = zero;
  wait_lds();  // before copies that land beside them
}

// The rows a share of a tile's keys gives: a slot of the partial results.
// Share w has at most two cut tiles: one that it starts with (slot 2 w) and
// one that starts within it (slot 2 w + 1).
__device__ __forceinline__ int64_t slot_of(int64_t w, int64_t share, int64_t tile_start) {
  return 2 * w + (tile_start > w * share ? 1 : 0);
}

// Leaves the tile that starts in share w and goes on past it for the join (or
// that there is none).  One thread.
__device__ __forceinline__ void leave_cut(const AttentionArgs& a, int64_t w, int64_t share, const Place& p, int tile,
                                          int head, int64_t t0, int64_t t1, bool cut) {
  a.cuts[w] = CutTile{t0, t1, share, p.r, tile, head, cut ? 1 : 0};
}

template <int STEP>
__device__ __forceinline__ int64_t share_of(int64_t total, int parts, int least) {
  const int64_t s = quotient(total + parts - 1, parts);
  return s <= least ? least : (s + STEP - 1) / STEP * STEP;
}

constexpr int kXcds = 8;
// Keys a share has at least.  One token on 1531 keys: 12.1 us with 128, 13.4 with
// 256.  512 tokens: 33 us with 256, 44 with 384; a ragged batch 49 and 62, and 49
// with 128.
constexpr int kFewShare = 128;
constexpr int kTileShare = 256;

// ---------------------------------------------------------------------------
// Up to 32 rows: NW waves, each 32 keys at a time with its own two stages of
// LDS, so that no wave waits for another until the end, where their results
// are joined in wave order.  Bound by the keys and values read: 64 requests of
// 300 to 8192 keys (8 heads of 128 for 32) take 126 us (633 MB, 5.0 TB/s), two
// of 65536 to 131072 149 us (5.4 TB/s).  One token on 1531 keys takes 9.1 us, of
// which reading lengths, finding its keys and the first copies are the most.
// ---------------------------------------------------------------------------
template <class V, int DP, int NW, bool FULL>
__global__ __launch_bounds__(NW * kWave, 1) void k_attention_few(AttentionArgs) {
  const AttentionArgs given = fresh_args();
  constexpr int ROWS = 32, STEP = NW * 32, OS = DP + 4, COPIES = 4 * RowCopy<DP, FULL>::INSTR;  // of a stage
  extern __shared__ uint8_t smem[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane % 32, h = lane / 32;
  uint16_t* ring = reinterpret_cast<uint16_t*>(smem) + wave * (2 * 2 * 32 * DP);
  float* jo = reinterpret_cast<float*>(smem);           // [NW][32][OS]
  float* jm = jo + NW * 32 * OS;                        // [NW][32]
  float* jl = jm + NW * 32;                             // [NW][32]
  int* flag = reinterpret_cast<int*>(jl + NW * 32);     // [32], then [NW] of the waves

  const RowCopy<DP, FULL> copy(given);
  const bool shared = given.part_o != nullptr;
  const Batch<V> batch(given, ROWS, nullptr);
  const int64_t head_len = head_length<V, ROWS, STEP>(given, batch, shared);
  int64_t pos, pos_end, share = 0, w = blockIdx.x;
  int head;
  if (shared) {
    share = share_of<STEP>(head_len * given.Hkv, given.parts, kFewShare);
    pos = w * share;
    pos_end = pos + share < head_len * given.Hkv ? pos + share : head_len * given.Hkv;
    head = pos < pos_end ? (int)quotient(pos, head_len) : 0;
  } else {
    w += given.first;
    const int64_t tile = quotient(w, given.Hkv);
    head = (int)(w - tile * given.Hkv);
    pos = head * head_len + tile;
    pos_end = tile < head_len ? pos + 1 : pos;
  }
  if (shared && pos >= pos_end && threadIdx.x == 0) leave_cut(given, w, share, Place{}, 0, 0, 0, 0, false);
  Place p = {};
  bool placed = false;
  while (pos < pos_end) {
    const AttentionArgs a = fresh_args();
    if (!placed) {
      p = locate<V, ROWS, STEP>(a, batch, pos - head * head_len, shared);
      if (p.b < 0) {
        if (shared && threadIdx.x == 0) leave_cut(a, w, share, p, 0, 0, 0, 0, false);
        return;
      }
    }
    const int64_t t0 = head * head_len + p.start, t1 = head * head_len + p.end;
    const int64_t seg_end = t1 < pos_end ? t1 : pos_end;
    const int rows = p.r.n * a.G, row0 = p.tile * ROWS, live = rows - row0 < ROWS ? rows - row0 : ROWS;
    const bool alive = l32 < live;
    Span mine = token_span<V>(a, p.r, token_of(a, row0 + (alive ? l32 : live - 1)));
    // keys that some live row sees, and every one
    const Spans spans = row_spans<V>(a, p.r, row0, live, mine, alive);
    const Span span = spans.any.begin < spans.any.end ? spans.any : Span{0, 0};
    const int base = span.begin / 32 * 32;
    int lo = base, hi = span.end;
    if (shared) {
      const int64_t from = base + (pos - t0), most = base + (seg_end - t0);  // may lie behind the last key
      lo = from < hi ? (int)from : hi;
      hi = most < hi ? (int)most : hi;
    }
    const int all_begin = spans.all.begin;
    int all_end = spans.all.end;
    const bool mixed = spans.all.begin != span.begin || spans.all.end != span.end;  // rows see different keys
    bool suspect = false;
    if (mine.end > hi) mine.end = hi;
    if (all_end > hi) all_end = hi;
    const int32_t* pages = a.pages + p.b * a.page_row_stride;
    const int64_t head_off = head * a.head_stride;

    if constexpr (!FULL) clear_lds<DP>(ring, 2 * 2 * 32);
    WaveTile<V, DP, 1> t;
    int k0 = lo + wave * 32;
    auto page_at = [&](int k) {
      const int j = k + l32;
      return k < hi ? page_of(a, pages, j < span.begin ? span.begin : j < hi ? j : hi - 1) : 0;
    };
    auto issue = [&](int k, int page, int stage) {  // page: lane l's of key k + l % 32
      const uint32_t to = lds_address(ring) + stage * (2 * 32 * DP * 2);
      const int page1 = __shfl_down(page, 16, kWave);
      copy.run(a, a.ck, head_off, page, k, span.begin, hi - 1, to);
      copy.run(a, a.ck, head_off, page1, k + 16, span.begin, hi - 1, to + 16 * DP * 2);
      copy.run(a, a.cv, head_off, page, k, span.begin, hi - 1, to + 32 * DP * 2);
      copy.run(a, a.cv, head_off, page1, k + 16, span.begin, hi - 1, to + 48 * DP * 2);
    };
    int page = page_at(k0), stage = 0;
    t.fetch_q(a, p.r, head, row0 + (alive ? l32 : live - 1));
    if (k0 < hi) issue(k0, page, 0);
    page = page_at(k0 + STEP);
    t.finish_q(a, alive);
    t.load_row(a, p.r, head, row0 + (alive ? l32 : live - 1));
    t.clear();
    for (; k0 < hi; k0 += STEP, stage ^= 1) {
      const int next = k0 + STEP;
      if (next < hi) {
        const int now = page;
        page = page_at(next + STEP);
        wait_lds();  // the other stage's readers are done
        issue(next, now, stage ^ 1);
        wait_loads<COPIES>();  // the copies of this stage
      } else {
        wait_loads<0>();
      }
      uint16_t* keys = ring + stage * (2 * 32 * DP);
      const bool masked = k0 < all_begin || k0 + 32 > all_end;
      if (masked && mixed) suspect |= cut_to_finite<DP, 32>(keys + 32 * DP);
      t.step(keys, keys + 32 * DP, k0, alive ? mine.begin : 0, alive ? mine.end : 0, masked, a);
    }
    // ---- join the waves
    __syncthreads();
    const float l = t.total(a);
    if (alive) {
      float* o = jo + (wave * 32 + l32) * OS;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<float4_t*>(o + i * 32 + e * 8 + h * 4) =
              float4_t{t.o[i][4 * e], t.o[i][4 * e + 1], t.o[i][4 * e + 2], t.o[i][4 * e + 3]};
      if (h == 0) {
        jm[wave * 32 + l32] = t.top();
        jl[wave * 32 + l32] = l;
      }
    }
    if (lane == 0) flag[32 + wave] = suspect;
    if (threadIdx.x < 32) flag[threadIdx.x] = 0;
    __syncthreads();
    const bool cut = shared && (t0 < pos || seg_end < t1);
    const int64_t slot = cut ? slot_of(w, share, t0) : 0;
    if (shared && seg_end == pos_end && threadIdx.x == 0)
      leave_cut(a, w, share, p, p.tile, head, t0, t1, t0 >= w * share && t1 > seg_end);
#pragma unroll 2
    for (int u = threadIdx.x; u < live * (DP / 4); u += NW * kWave) {
      const int row = u / (DP / 4), d = u % (DP / 4) * 4;
      float top = jm[row];
#pragma unroll
      for (int i = 1; i < NW; ++i) top = fmaxf(top, jm[i * 32 + row]);
      float v[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const float m = jm[i * 32 + row], f = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
        const float4_t o = *reinterpret_cast<const float4_t*>(jo + (i * 32 + row) * OS + d);
        sum += f * jl[i * 32 + row];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += f * o[e];
      }
      const float z = (v[0] - v[0]) + (v[1] - v[1]) + (v[2] - v[2]) + (v[3] - v[3]) + (sum - sum);
      if (!(z == 0.f)) flag[row] = 1;
      if (cut) {
        *reinterpret_cast<float4_t*>(a.part_o + (slot * ROWS + row) * DP + d) = float4_t{v[0], v[1], v[2], v[3]};
        if (d == 0) {
          a.part_ml[(slot * ROWS + row) * 2] = top;
          a.part_ml[(slot * ROWS + row) * 2 + 1] = sum;
        }
      } else {
        const bool sees = sum != 0.f || token_sees<V>(a, p.r, token_of(a, row0 + row));
        const float f = row_factor(sum, sees);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= f;
        store4(a, out_row(a, p.r, head, row0 + row), d, v);
        if (d == 0 && a.lse != nullptr)
          a.lse[lse_at(a, p.r, head, row0 + row)] = final_lse<V>(top, sum, sees, a, p.r, head, row0 + row);
      }
    }
    // nobody waits for the stores above, but for rows that are stored again
    wait_lds();
    barrier_only();
    const bool again = __any(lane < 32 + NW && flag[lane < 32 + NW ? lane : 0] != 0);
    if (again) __syncthreads();
    int any_suspect = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) any_suspect |= flag[32 + i];
    for (int row = wave; row < live && again; row += NW) {
      if ((flag[row] | any_suspect) == 0) continue;
      const Span s = token_span<V>(a, p.r, token_of(a, row0 + row));
      SlowRow<V, DP> slow;
      slow.run(a, query_row(a, p.r, head, row0 + row), head_off, pages, p.r, head, row0 + row,
               s.begin > lo ? s.begin : lo, s.end < hi ? s.end : hi);
      slow.template store<ROWS>(a, p.r, head, row0 + row, row, cut ? slot : -1, flag[row] != 0);
    }
    pos = seg_end;
    if (pos < pos_end) {
      __syncthreads();  // the stages are free
      placed = advance<V, ROWS, STEP>(a, batch, p, head);
      if (!placed) head = (int)quotient(pos, head_len);
    }
  }
}

// ---------------------------------------------------------------------------
// 128 rows: four waves of 32 rows over shared tiles of 64 keys, two stages.
// Bound by what one wave does in turn (see WaveTile::block): 2048 tokens after
// 6144, 32 heads of 128 on 8, take 261 to 275 us from card to card (241 GFLOP,
// 925 to 878 TFLOP/s; the matrix cores are busy half of the time, at 1.78 GHz).
// Of 285 us at the time the copies were 30, the LDS reads 30, the maximum 12, the
// sum of the weights 10 (each left out, for timing).  64 rows a wave would halve
// the LDS reads, but leave one wave a SIMD.  A tile costs 10 us besides its keys.
// ---------------------------------------------------------------------------
template <class V, int DP, bool FULL>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void k_attention_tile(AttentionArgs) {
  const AttentionArgs given = fresh_args();
  constexpr int ROWS = 128, STEP = 64;
  extern __shared__ uint8_t smem[];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l32 = lane % 32, h = lane / 32;
  uint16_t* ring = reinterpret_cast<uint16_t*>(smem);
  int* flag = reinterpret_cast<int*>(smem + 512 * DP);  // a value of a mixed tile was not finite

  const RowCopy<DP, FULL> copy(given);
  const bool shared = given.part_o != nullptr;
  const Batch<V> batch(given, ROWS, flag + 4);
  // With two classes every request's even tiles lie in the first half of the line,
  // its odd ones at the same places of the second: workgroups of one compute unit
  // then read the same keys at the same time, once from memory (see plan_attention).
  const int classes = V::kMore && shared ? given.classes : 1;
  const int64_t head_len = head_length<V, ROWS, STEP>(given, batch, shared, classes);
  int64_t pos, pos_end, share = 0, base = 0, w = blockIdx.x;
  int head, cls = 0;
  if (shared) {
    // Workgroups go to the XCDs in turn, and each XCD has its own L2: its
    // shares lie side by side, so that they read the keys of few heads (2048
    // tokens after 6144 in shares: 285 us, 296 without).  A compute unit gets
    // two of them, half of the XCD's shares apart: the second half runs
    // backwards, so that a share with a prompt's last tiles, which see the most
    // keys, meets one with its first (2048 tokens in shares: 69 us, 75 without).
    if (given.parts % kXcds == 0) {
      const int per = given.parts / kXcds;
      int v = (int)w / kXcds;
      if (classes == 2) {
        w = v < per / 2 ? w % kXcds * (per / 2) + v : given.parts / 2 + w % kXcds * (per / 2) + v - per / 2;
      } else {
        if (DP <= 128 && v >= per / 2) v = per / 2 + (per - 1 - v);
        w = w % kXcds * per + v;
      }
    }
    // Short tiles are left whole where all have one length (300 tokens: 28 us, 38
    // with each cut; 1207 tokens in a window of 107 27.5 and 42.6; but 224 rows
    // of 256 dimensions in a window of 432 50 and 42).
    int64_t length = 0;
    if (given.B == 1) {
      const Request one = {uniform(batch.first.q0), uniform(batch.first.n), uniform(batch.first.kv)};
      length = tile_length<V, ROWS, STEP>(given, one, uniform(batch.keys), true);
    } else if (given.window > 0 && given.causal) {  // the longest there can be
      length = tile_length<V, ROWS, STEP>(given, Request{0, 0, INT32_MAX}, INT32_MAX, true);
    }
    const bool whole = length > 0 && (length - tile_extra<V, ROWS>(given)) * DP <= 384 * 128;
    const int parts = classes == 2 ? given.parts / 2 : given.parts;  // of a class
    share = share_of<STEP>(head_len * given.Hkv, parts, whole ? (int)length : kTileShare);
    if (whole) share = quotient(share - 1, length) * length + length;
    if (classes == 2 && w >= parts) cls = 1;
    base = cls * parts * share;
    pos = w * share;
    pos_end = base + head_len * given.Hkv;
    if (pos + share < pos_end) pos_end = pos + share;
    head = pos < pos_end ? (int)quotient(pos - base, head_len) : 0;
  } else {
    w += given.first;
    const int64_t tile = quotient(w, given.Hkv);
    head = (int)(w - tile * given.Hkv);
    pos = head * head_len + tile;
    pos_end = tile < head_len ? pos + 1 : pos;
  }
  if (shared && pos >= pos_end && threadIdx.x == 0) leave_cut(given, w, share, Place{}, 0, 0, 0, 0, false);
  if constexpr (!FULL) {
    clear_lds<DP>(ring + wave * (64 * DP), 64);
    __syncthreads();
  }
  Place p = {};
  bool placed = false;
  while (pos < pos_end) {
    const AttentionArgs a = fresh_args();
    if (!placed) {
      p = locate<V, ROWS, STEP>(a, batch, pos - base - head * head_len, shared, classes);
      if (p.b < 0) {
        if (shared && threadIdx.x == 0) leave_cut(a, w, share, p, 0, 0, 0, 0, false);
        return;
      }
    }
    // the tiles with the most keys first
    const int tile = !shared ? tiles_of<ROWS>(a, p.r) - 1 - p.tile : p.tile * classes + cls;
    const int64_t t0 = base + head * head_len + p.start, t1 = base + head * head_len + p.end;
    const int64_t seg_end = t1 < pos_end ? t1 : pos_end;
    if (V::kMore && classes == 2 && tile >= tiles_of<ROWS>(a, p.r)) {  // a request of an odd number
      if (seg_end == pos_end && threadIdx.x == 0) leave_cut(a, w, share, p, tile, head, t0, t1, false);
      pos = seg_end;
      if (pos < pos_end) {
        placed = advance<V, ROWS, STEP>(a, batch, p, head, classes);
        if (!placed) head = (int)quotient(pos - base, head_len);
      }
      continue;
    }
    const int rows = p.r.n * a.G, tile_rows = rows - tile * ROWS < ROWS ? rows - tile * ROWS : ROWS;
    const int row0 = tile * ROWS + wave * 32;
    const int live = rows - row0 < 32 ? rows - row0 : 32;  // may be <= 0
    const bool alive = l32 < live;
    Span mine = {0, 0}, all = {0, 0};
    if (alive) mine = token_span<V>(a, p.r, token_of(a, row0 + l32));
    // over the four waves: the keys that some row sees, and that all see
    Spans of_tile;
    if (V::kMore && a.spans != nullptr) {
      Spans* const of_waves = reinterpret_cast<Spans*>(flag + 4);
      of_tile = row_spans<V>(a, p.r, row0, live, mine, alive);
      all = of_tile.all;
      if (lane == 0) of_waves[wave] = of_tile;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Spans s = of_waves[i];
        of_tile.all = {max(of_tile.all.begin, s.all.begin), min(of_tile.all.end, s.all.end)};
        of_tile.any = {min(of_tile.any.begin, s.any.begin), max(of_tile.any.end, s.any.end)};
      }
      of_tile = {{uniform(of_tile.all.begin), uniform(of_tile.all.end)}, {uniform(of_tile.any.begin), uniform(of_tile.any.end)}};
      if (of_tile.any.begin >= of_tile.any.end) of_tile.any = {0, 0};
    } else {
      of_tile = row_spans<V>(a, p.r, tile * ROWS, tile_rows, mine, alive);
      if (live > 0) all = row_spans<V>(a, p.r, row0, live, mine, alive).all;
    }
    const Span span = of_tile.any;
    const int key0 = span.begin / 32 * 32;
    int lo = key0, hi = span.end;
    if (shared) {
      const int64_t from = key0 + (pos - t0), most = key0 + (seg_end - t0);  // may lie behind the last key
      lo = from < hi ? (int)from : hi;
      hi = most < hi ? (int)most : hi;
    }
    const bool mixed = of_tile.all.begin != span.begin || of_tile.all.end != span.end;  // rows see different keys
    const int most_begin = of_tile.all.begin, least_end = of_tile.all.end;
    if (mine.end > hi) mine.end = hi;
    if (all.end > hi) all.end = hi;
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    const int32_t* pages = a.pages + p.b * a.page_row_stride;
    const int64_t head_off = head * a.head_stride;

    WaveTile<V, DP, 1> t;
    auto page_at = [&](int k) {
      const int j = k + wave * 16 + lane % 16;
      return k < hi ? page_of(a, pages, j < span.begin ? span.begin : j < hi ? j : hi - 1) : 0;
    };
    // Keys and values have two stages each.  Keys run a tile ahead: while the
    // pipeline takes the scores of tile i + 1 it weights the values of tile i.
    const uint32_t rows_at = lds_address(ring) + wave * (16 * DP * 2);
    uint16_t* vring = ring + 2 * 64 * DP;
    auto copy_keys = [&](int k, int page, int stage) {
      copy.run(a, a.ck, head_off, page, k + wave * 16, span.begin, hi - 1, rows_at + stage * (64 * DP * 2));
    };
    auto copy_values = [&](int k, int page, int stage) {
      copy.run(a, a.cv, head_off, page, k + wave * 16, span.begin, hi - 1, rows_at + (2 + stage) * (64 * DP * 2));
    };
    // values that some rows do not see are cut to finite ones by the wave that copied them
    auto cut_values = [&](int k, int stage) {
      if (mixed && (k < most_begin || k + STEP > least_end)) {
        if (cut_to_finite<DP, 16>(vring + stage * (64 * DP) + wave * 16 * DP)) *flag = 1;
      }
    };
    auto masked = [&](int k) { return k < all.begin || k + 32 > all.end; };
    int page[3] = {page_at(lo), page_at(lo + STEP), 0};
    int ahead[2] = {page_at(lo + 2 * STEP), page_at(lo + 3 * STEP)};  // with them: one wait less
    t.fetch_q(a, p.r, head, alive ? row0 + l32 : tile * ROWS);
    t.load_row(a, p.r, head, alive ? row0 + l32 : tile * ROWS);
    t.clear();
    if (lo < hi) {
      asm volatile("" : "+v"(page[0]), "+v"(page[1]), "+v"(ahead[0]), "+v"(ahead[1]));  // one wait, and not for copies
      copy_keys(lo, page[0], 0);
      copy_keys(lo + STEP, page[1], 1);  // behind the end: any key, masked
      copy_values(lo, page[0], 0);
      // offsets of the units that the next tile's copies bring: values of tile
      // 1, keys of tile 2; pages of this one and the next two
      int page_v = page[1];
      int64_t off_v = copy.whole_offset(a, head_off, page_v, lo + STEP + wave * 16);
      page[0] = ahead[0];
      page[1] = ahead[1];
      int64_t off_k = copy.whole_offset(a, head_off, page[0], lo + 2 * STEP + wave * 16);
      t.finish_q(a, alive);
      wait_loads<0>();
      barrier_only();
      float16_t s0, s1;
      half8_t p0[2], p1[2] = {};
      t.scores(WaveTile<V, DP, 1>::key_lane(ring), lo, s0);
      t.scores(WaveTile<V, DP, 1>::key_lane(ring + 32 * DP), lo + 32, s1);
      float top = s0[0], top1 = s1[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) {
        top = fmaxf(top, s0[e]);
        top1 = fmaxf(top1, s1[e]);
      }
      top = t.row_max(top);
      top1 = t.row_max(top1);
      t.settle(s0, top, (top - t.m) * a.c, p1, lo, mine.begin, mine.end, masked(lo), a);
      t.weights(s0, p0, a);
      t.settle(s1, top1, (top1 - t.m) * a.c, p0, lo + 32, mine.begin, mine.end, masked(lo + 32), a);
      const typename WaveTile<V, DP, 1>::Lanes lanes(ring);
      auto turn = [&](int k0, int stage) __attribute__((always_inline)) {
        // here: values of tile k0 in `stage`, keys of the next in the other
        // one; p0, s1: weights and scores of the tile's two blocks
        wait_lds();
        wait_loads<0>();  // this wave's copies
        cut_values(k0, stage);
        wait_lds();
        barrier_only();   // everyone's; nobody reads what is overwritten now
        // The next copies: one every third step below, since memory takes a
        // copy in 16 cycles and the eight waves of a compute unit would stand
        // in line for it here (2048 tokens after 6144: 324 us, spread 291 at
        // the time); all at once where keys lie in several pages or past the end.
        const int kk = k0 + 2 * STEP + wave * 16;
        const bool spread = copy.whole(a, kk, span.begin, hi - 1);  // then the values' unit is whole too
        const uint16_t *from_k = a.ck + off_k, *from_v = a.cv + off_v;
        if (!spread) {
          copy_keys(k0 + 2 * STEP, page[0], stage);
          copy_values(k0 + STEP, page_v, stage ^ 1);
        }
        const uint32_t to_k = rows_at + stage * (64 * DP * 2), to_v = rows_at + (2 + (stage ^ 1)) * (64 * DP * 2);
        page[2] = page_at(k0 + 4 * STEP);
        auto at_step = [&](int i) {
          constexpr int C = RowCopy<DP, FULL>::INSTR;
          const int n = i / 3;
          if (i == 6 * C + 1) {  // the next tile's offsets; its page came a tile ago
            off_v = off_k;
            off_k = copy.whole_offset(a, head_off, page[1], kk + STEP);
            asm volatile("" : "+s"(off_k));
          }
          if (i % 3 != 0 || n >= 2 * C || !spread) return;
          if (n < C) copy.one(from_k, n, to_k);
          else copy.one(from_v, n - C, to_v);
        };
        const uint32_t k_off = (stage ^ 1) * (64 * DP * 2), v_off = (2 + stage) * (64 * DP * 2), next = 32 * DP * 2;
#pragma unroll
        for (int i = 0; i < WaveTile<V, DP, 1>::OPS - 1; ++i) t.read_op(lanes, k_off, v_off, i);
        float over = 0.f;
        t.block(s1, s0, p0, p1, lanes, k_off, v_off, true, a, k0 + STEP, top, over, at_step);
        t.settle(s0, top, over, p1, k0 + STEP, mine.begin, mine.end, masked(k0 + STEP), a);
        t.block(s0, s1, p1, p0, lanes, k_off + next, v_off + next, false, a, k0 + STEP + 32, top, over,
                [&](int i) { at_step(i + DP / 8); });
        t.settle(s1, top, over, p0, k0 + STEP + 32, mine.begin, mine.end, masked(k0 + STEP + 32), a);
        page_v = page[0];
        page[0] = page[1];
        page[1] = page[2];
      };
      // the stages are constants in each half of the loop
      for (int k0 = lo; k0 < hi; k0 += 2 * STEP) {
        turn(k0, 0);
        if (k0 + STEP >= hi) break;
        turn(k0 + STEP, 1);
      }
      wait_loads<0>();  // copies behind the end
    }
    const AttentionArgs end = fresh_args();
    const float l = t.total(end);
    const bool cut = shared && (t0 < pos || seg_end < t1);
    const int64_t slot = cut ? slot_of(w, share, t0) : 0;
    if (shared && seg_end == pos_end && threadIdx.x == 0)
      leave_cut(end, w, share, p, tile, head, t0, t1, t0 >= w * share && t1 > seg_end);
    if (alive) {
      if (cut) {
        const int64_t at = slot * ROWS + wave * 32 + l32;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float4_t*>(end.part_o + at * DP + i * 32 + e * 8 + h * 4) =
                float4_t{t.o[i][4 * e], t.o[i][4 * e + 1], t.o[i][4 * e + 2], t.o[i][4 * e + 3]};
        if (h == 0) {
          end.part_ml[at * 2] = t.top();
          end.part_ml[at * 2 + 1] = l;
        }
      } else {
        const bool sees = l != 0.f || token_sees<V>(end, p.r, token_of(end, row0 + l32));
        const float f = row_factor(l, sees);
        uint16_t* dst = out_row(end, p.r, head, row0 + l32);
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v[4] = {t.o[i][4 * e] * f, t.o[i][4 * e + 1] * f, t.o[i][4 * e + 2] * f, t.o[i][4 * e + 3] * f};
            store4(end, dst, i * 32 + e * 8 + h * 4, v);
          }
        if (h == 0 && end.lse != nullptr)
          end.lse[lse_at(end, p.r, head, row0 + l32)] =
              final_lse<V>(t.top(), l, sees, end, p.r, head, row0 + l32);
      }
    }
    uint64_t broken = __ballot(alive && t.broken(l));
    broken = (broken | broken >> 32) & 0xFFFFFFFFu;
    __syncthreads();
    uint64_t again = *flag != 0 && live > 0 ? (uint64_t(1) << live) - 1 : broken;
    if (again != 0) {
      wait_loads<0>();  // the stores above come first
      while (again != 0) {
        const int i = __ffsll((unsigned long long)again) - 1, row = row0 + i;
        again &= again - 1;
        const Span s = token_span<V>(end, p.r, token_of(end, row));
        SlowRow<V, DP> slow;
        slow.run(end, query_row(end, p.r, head, row), head_off, pages, p.r, head, row,
                 s.begin > lo ? s.begin : lo, s.end < hi ? s.end : hi);
        slow.template store<ROWS>(end, p.r, head, row, wave * 32 + i, cut ? slot : -1, (broken >> i & 1) != 0);
      }
    }
    pos = seg_end;
    if (pos < pos_end) {
      __syncthreads();  // the stages are free
      placed = advance<V, ROWS, STEP>(end, batch, p, head, classes);
      if (!placed) head = (int)quotient(pos - base, head_len);
    }
  }
}

// ---------------------------------------------------------------------------
// Joins the shares of one cut tile: workgroup x takes the one that starts in
// share x, y cuts the tile's values.  Shares are added in their order, by groups
// of threads that take every so-manieth share where there are few rows.  4.6 us
// for one token on 1531 keys, 5.4 for two on 131072, 7.5 for a ragged batch of
// 24 requests, mostly the launch.
// ---------------------------------------------------------------------------
template <class V, int DP, int ROWS, int YS>
__global__ __launch_bounds__(256) void k_attention_join(AttentionArgs a) {
  constexpr int TH = 256, CH = DP / 4, MOST = 8;
  __shared__ float so[TH * 4], sm[TH], sl[TH];
  const CutTile p = a.cuts[blockIdx.x];
  if (!p.cut) return;
  const int head = p.head;
  const int64_t t0 = p.start, t1 = p.end, share = p.share, w0 = blockIdx.x;
  const int nparts = (int)(quotient(t1 - 1, share) - w0 + 1);
  const int rows = p.r.n * a.G, row0 = p.tile * ROWS, live = rows - row0 < ROWS ? rows - row0 : ROWS;
  // units (row, four values) of this workgroup; a few workgroups do where there
  // are few shares (5 requests of one token, up to 28701 keys in 90 shares, on one
  // cache head: 22 us, 25 without the rest; a ragged batch 1 us less with few)
  int per = (live * CH + YS - 1) / YS;
  if (nparts <= 16 && per < TH / 2) per = TH / 2;
  const int first = blockIdx.y * per;
  const int units = live * CH - first < per ? live * CH - first : per;
  if (units <= 0) return;
  int groups = TH / units;
  groups = groups < 1 ? 1 : groups > MOST ? MOST : groups;
  groups = groups < nparts ? groups : nparts;
  for (int u0 = 0; u0 < units; u0 += TH) {
    // thread: its unit and its group of shares
    const int u = groups > 1 ? (int)threadIdx.x % units : u0 + (int)threadIdx.x;
    const int g = groups > 1 ? (int)threadIdx.x / units : 0;
    const bool active = u < units && g < groups;
    const int row = (first + u) / CH, d = (first + u) % CH * 4;
    float m = -INFINITY, l = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
    if (active) {
#pragma unroll 4
      for (int i = g; i < nparts; i += groups) {
        const int64_t at = slot_of(w0 + i, share, t0) * ROWS + row;
        const float pm = a.part_ml[at * 2], pl = a.part_ml[at * 2 + 1];
        const float4_t o = *reinterpret_cast<const float4_t*>(a.part_o + at * DP + d);
        const float top = fmaxf(m, pm);
        const float fm = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
        const float fp = pm == top ? 1.f : __builtin_amdgcn_exp2f(pm - top);
        l = l * fm + pl * fp;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = v[e] * fm + o[e] * fp;
        m = top;
      }
    }
    if (groups > 1) {
      sm[threadIdx.x] = m;
      sl[threadIdx.x] = l;
      *reinterpret_cast<float4_t*>(so + threadIdx.x * 4) = float4_t{v[0], v[1], v[2], v[3]};
      __syncthreads();
      if (g > 0 || !active) return;
      for (int i = 1; i < groups; ++i) {
        const int t = i * units + u;
        const float pm = sm[t], top = fmaxf(m, pm);
        const float fm = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
        const float fp = pm == top ? 1.f : __builtin_amdgcn_exp2f(pm - top);
        const float4_t o = *reinterpret_cast<const float4_t*>(so + t * 4);
        l = l * fm + sl[t] * fp;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = v[e] * fm + o[e] * fp;
        m = top;
      }
    }
    if (!active) continue;
    const bool sees = l != 0.f || token_sees<V>(a, p.r, token_of(a, row0 + row));
    const float f = row_factor(l, sees);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= f;
    store4(a, out_row(a, p.r, head, row0 + row), d, v);
    if (d == 0 && a.lse != nullptr)
      a.lse[lse_at(a, p.r, head, row0 + row)] = final_lse<V>(m, l, sees, a, p.r, head, row0 + row);
  }
}

// All workgroups of a call, in as many launches as they need.
hipError_t launch_blocks(void (*kernel)(AttentionArgs), int64_t blocks, int threads, size_t lds, hipStream_t stream,
                         AttentionArgs a) {
  const int64_t most = kMaxGridThreads / threads;
  for (; a.first < blocks; a.first += most) {
    const int64_t n = blocks - a.first < most ? blocks - a.first : most;
    const hipError_t e = launch_kernel(kernel, dim3((unsigned)n), dim3(threads), lds, stream, a);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class V, int DP, bool FULL>
hipError_t launch_planned(const AttentionPlan& pl, const AttentionArgs& a, hipStream_t stream) {
  constexpr int NW = DP == 256 ? 2 : 4, JY = 8;
  const bool shared = a.part_o != nullptr;
  const int64_t blocks = shared ? pl.parts : pl.tiles * a.Hkv;
  hipError_t e;
  if (pl.few) {
    if ((e = prepare_kernel(k_attention_few<V, DP, NW, FULL>)) != hipSuccess) return e;
    e = launch_blocks(k_attention_few<V, DP, NW, FULL>, blocks, NW * kWave, NW * 256 * DP, stream, a);
    if (e != hipSuccess || !shared) return e;
    return launch_kernel(k_attention_join<V, DP, 32, JY>, dim3((unsigned)blocks - 1, JY), dim3(256), 0, stream, a);
  }
  if ((e = prepare_kernel(k_attention_tile<V, DP, FULL>)) != hipSuccess) return e;
  e = launch_blocks(k_attention_tile<V, DP, FULL>, blocks, 256, 512 * DP + (V::kMore ? 16 + 4 * (int)sizeof(Spans) : 16), stream, a);
  if (e != hipSuccess || !shared) return e;
  return launch_kernel(k_attention_join<V, DP, 128, 16>, dim3((unsigned)blocks - 1, 16), dim3(256), 0, stream, a);
}

}  // namespace

template <class V>
hipError_t launch_variant(const AttentionPlan& pl, const AttentionArgs& a, hipStream_t stream) {
  const bool full = a.D == pl.DP;
  switch (pl.DP) {
    case 64: return full ? launch_planned<V, 64, true>(pl, a, stream) : launch_planned<V, 64, false>(pl, a, stream);
    case 128: return full ? launch_planned<V, 128, true>(pl, a, stream) : launch_planned<V, 128, false>(pl, a, stream);
    default: return full ? launch_planned<V, 256, true>(pl, a, stream) : launch_planned<V, 256, false>(pl, a, stream);
  }
}

}  // namespace fasq
