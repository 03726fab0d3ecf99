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
typedef int int2_any __attribute__((ext_vector_type(2), aligned(4)));

// What a kernel's variant has besides scaled products, causality and windows.
// MORE: masks of a call's own (runs of keys, trees of drafted tokens); CAP:
// scores capped by a tanh; SLOPES: scores with a bias that grows with the distance.
template <bool MORE, bool CAP, bool SLOPES>
struct Variant {
  static constexpr bool kMore = MORE, kCap = CAP, kSlopes = SLOPES;
};
using Plain = Variant<false, false, false>;

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
  // Of variants besides Plain:
  const int32_t* spans;  // [T][2]: the keys that each token sees, or NULL (causal, window)
  const int32_t* tree;   // [T][tree_words]: which new tokens each one sees, or NULL
  int64_t tree_stride;
  int tree_words;
  const float* slopes;  // [Hq]
  float slope_unit;     // a slope times this is one in units of the raw products
  float cap, cap_unit;  // softcap in powers of two; a raw product (with its bias) times this is the tanh's argument
  int classes;  // 1, or 2: see k_attention_tile
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

// Quotients without the long way round that a 64-bit division takes (about a
// microsecond of a short call): in 32 bits, or through fp64, for 0 <= a < 2^53,
// b > 0.  Positions are at most the keys that all tiles of all heads can need, which
// no call could read if they were more.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  const int64_t q = (int64_t)((double)a / (double)b);  // or its neighbour
  const int64_t rest = a - q * b;
  return rest < 0 ? q - 1 : rest >= b ? q + 1 : q;
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

// Keys [begin, end) that token i of a request sees.
struct Span {
  int begin, end;
};

template <class V>
__device__ __forceinline__ Span token_span(const AttentionArgs& a, const Request& r, int i) {
  if constexpr (V::kMore) {
    if (a.spans != nullptr) {
      const int2_any both = *reinterpret_cast<const int2_any*>(a.spans + 2 * ((int64_t)r.q0 + i));
      int begin = both[0], end = both[1];
      end = end < 0 ? 0 : end < r.kv ? end : r.kv;
      begin = begin < 0 ? 0 : begin < end ? begin : end;
      return {begin, end};
    }
    if (a.tree != nullptr) return {0, r.kv};
  }
  const int pos = r.kv - r.n + i;  // may be negative: more new tokens than keys
  int end = a.causal && pos + 1 < r.kv ? pos + 1 : r.kv;
  int begin = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  end = end < 0 ? 0 : end;
  return {begin < end ? begin : end, end};
}

// Keys of a wave's rows, lane by lane: what all of them see, and some.
struct Spans {
  Span all, any;
};
// `live`: the lane has a row.  Without any key, `any` ends before it begins.
__device__ __forceinline__ Spans join_spans(Span s, bool live) {
  auto most = [](int a, int b) { return a > b ? a : b; };
  auto least = [](int a, int b) { return a < b ? a : b; };
  const Span some = live && s.begin < s.end ? s : Span{INT32_MAX, 0};
  if (!live) s = {0, INT32_MAX};
  return {{wave_join(s.begin, most), wave_join(s.end, least)}, {wave_join(some.begin, least), wave_join(some.end, most)}};
}

// The same of the rows [row, row + count) of a request, of which lane l holds the
// one that sees `mine`, if `live` (which counts where a call has spans).
template <class V>
__device__ __forceinline__ Spans row_spans(const AttentionArgs& a, const Request& r, int row, int count, Span mine,
                                           bool live) {
  Spans s;
  if (V::kMore && a.spans != nullptr) {
    s = join_spans(mine, live);
  } else {
    const Span s0 = token_span<V>(a, r, token_of(a, row)), s1 = token_span<V>(a, r, token_of(a, row + count - 1));
    s.all = {s0.begin > s1.begin ? s0.begin : s1.begin, s0.end < s1.end ? s0.end : s1.end};
    s.any = {s0.begin < s1.begin ? s0.begin : s1.begin, s1.end > s0.end ? s1.end : s0.end};
  }
  if constexpr (V::kMore) {
    // of the new tokens, which a tree's words tell about, none is seen by all
    if (a.tree != nullptr && s.all.end > r.kv - r.n) s.all.end = r.kv - r.n;
  }
  return s;
}

// Which new tokens a row of a tree sees: bit j % 32 of word j / 32 tells about
// the request's j-th new token, which is key `first` + j.
struct TreeRow {
  const int32_t* words;
  int count, first;
  // The bits of keys key0 .. key0 + 31; those before `first` are set.
  __device__ __forceinline__ uint32_t block(int key0) const {
    const int64_t at = (int64_t)key0 - first;
    const int w = (int)(at >> 5), shift = (int)(at & 31);
    const uint32_t lo = word(w), hi = word(w + 1);
    return shift == 0 ? lo : lo >> shift | hi << (32 - shift);
  }
  __device__ __forceinline__ uint32_t word(int w) const {
    return w < 0 ? 0xFFFFFFFFu : w < count ? (uint32_t)words[w] : 0u;
  }
};
__device__ __forceinline__ TreeRow tree_row(const AttentionArgs& a, const Request& r, int i) {
  return {a.tree + ((int64_t)r.q0 + i) * a.tree_stride, a.tree_words, r.kv - r.n};
}

// Whether token i sees any key.  Only rows without a weight need to know.
template <class V>
__device__ __forceinline__ bool token_sees(const AttentionArgs& a, const Request& r, int i) {
  const Span s = token_span<V>(a, r, i);
  if constexpr (V::kMore) {
    if (a.tree != nullptr && s.begin < s.end) {
      const TreeRow row = tree_row(a, r, i);
      if (s.begin < row.first) return true;
      for (int k = s.begin; k < s.end; k += 32) {
        const uint32_t bits = row.block(k);
        if ((s.end - k < 32 ? bits & ((1u << (s.end - k)) - 1) : bits) != 0) return true;
      }
      return false;
    }
  }
  return s.begin < s.end;
}

// The bias of a row's scores: slope * -|position - key|, in units of the raw
// products, less that of the nearest key it may see (so that a row far from all
// its keys loses nothing to it; not where scores are capped).
struct RowBias {
  float slope;      // negative for positive slopes
  int pos, nearest; // the distance of the nearest key
};
template <class V>
__device__ __forceinline__ RowBias row_bias(const AttentionArgs& a, const Request& r, int head, int row) {
  const int t = token_of(a, row), pos = r.kv - r.n + t;
  const float slope = -a.slopes[head * a.G + row - t * a.G] * a.slope_unit;
  int nearest = 0;
  if constexpr (!V::kCap) {
    const Span s = token_span<V>(a, r, t);
    if (s.begin < s.end) nearest = pos >= s.end ? pos - s.end + 1 : pos < s.begin ? s.begin - pos : 0;
  }
  return {slope, pos, nearest};
}
// What the nearest key's bias adds to a logarithm of a sum.
template <class V>
__device__ __forceinline__ float lse_bias(const AttentionArgs& a, const Request& r, int head, int row) {
  const RowBias b = row_bias<V>(a, r, head, row);
  return b.nearest == 0 ? 0.f : b.slope * a.c * (float)b.nearest * 0.69314718055994530942f;
}

// The batch as a wave sees it: lane l keeps requests l, l + 64, ..., the first
// of them in registers (all there are in most batches).
template <class V>
struct Batch {
  Request first;
  int keys;  // that one of its tiles can need
  // rows: of a tile; of_waves: LDS for a value of each of four waves, or nullptr.
  __device__ __forceinline__ Batch(const AttentionArgs& a, int rows, int* of_waves) {
    const int lane = threadIdx.x % kWave;
    first = lane < a.B ? read_request(a, lane) : Request{0, 0, 0};
    keys = first.kv;
    if constexpr (V::kMore) {
      // Where tokens see runs of keys of their own: the keys that some of a few tokens
      // sees; for a single request the most that a tile's tokens see together.  2030
      // tokens of 7 heads on 1 (96 dimensions): 40 us in 5 documents, 51 with shares as
      // if each saw all keys; 29 and 46 in 40 documents, 58 and 57 in one; 1024 tokens of
      // 32 heads on 8 31.6 and 37 in 11, 42.3 and 40.9 in one.
      if (a.spans != nullptr && a.part_o != nullptr) {
        Request r = first;
        const bool one = a.B == 1;
        if (one) r = {__builtin_amdgcn_readfirstlane(first.q0), __builtin_amdgcn_readfirstlane(first.n), __builtin_amdgcn_readfirstlane(first.kv)};
        // a single request's tokens by four waves, if that many are there; all those of the
        // tiles that start among a wave's
        const int besides = (rows - 1) / a.G + 1, waves = one && r.n > 256 && of_waves != nullptr ? 4 : 1;
        const int wave = waves == 4 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) : 0;
        const int part = (r.n + waves - 1) / waves, from = wave * part;
        const int upto = waves == 4 ? min(from + part + besides, r.n) : r.n;
        const int per = one ? max((upto - from + kWave - 1) / kWave, 1) : r.n;  // of a lane, side by side
        const int begin = one ? from + lane * per : 0, end = min(begin + per, upto);
        const bool few = r.n <= (one ? (waves == 4 ? 4096 : 256) : 32);
        Span s = {INT32_MAX, 0};
#pragma unroll 8
        for (int i = begin; i < end && few; ++i) {
          const Span t = token_span<V>(a, r, i);
          if (t.begin < t.end) s = {min(s.begin, t.begin), max(s.end, t.end)};
        }
        if (one && few) {
          // lanes that the tokens of a tile lie in, at most; as many or more are joined
          const int lanes = besides / per + 2;
          for (int x = 1; x < lanes && x < kWave; x *= 2) {
            s.begin = min(s.begin, __shfl_down(s.begin, x, kWave));
            s.end = max(s.end, __shfl_down(s.end, x, kWave));
          }
        }
        if (few) keys = s.begin < s.end ? s.end - s.begin / 32 * 32 : 0;
        if (one && few) {
          keys = wave_join(keys, [](int x, int y) { return x > y ? x : y; });
          if (waves == 4) {
            if (lane == 0) of_waves[wave] = keys;
            __syncthreads();
            keys = max(max(of_waves[0], of_waves[1]), max(of_waves[2], of_waves[3]));
            __syncthreads();
          }
        }
      }
    }
  }
  __device__ __forceinline__ Request of(const AttentionArgs& a, int64_t b) const {
    return b < kWave ? first : read_request(a, b);
  }
  __device__ __forceinline__ int keys_of(const Request& r, int64_t b) const { return V::kMore && b < kWave ? keys : r.kv; }
};

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

// Positions behind a tile's last key, for what a tile of 128 rows costs besides its
// keys (queries to fetch, rows to leave): without them the share that gets several
// tiles of few keys is the last to end.  A prompt's 509 tokens, a short prompt and 22
// single tokens on 77 to 3001 keys (12/4 heads of 80, pages of 20, slopes): 71.3 us without, 56.8 /
// 56.1 / 60.6 with 192 / 256 / 384; 16 trees of 32 nodes on 300 to 8192 keys (32/8
// heads of 128): 72.5, and 68.9 / 71.3 / 66.1.  One request's tiles are all of a kind,
// and the plain variant's shares stay as they were.
constexpr int kTileExtra = 256;
template <class V, int ROWS>
__device__ __forceinline__ int tile_extra(const AttentionArgs& a) {
  return V::kMore && ROWS == 128 && a.B > 1 ? kTileExtra : 0;
}

template <class V, int ROWS, int STEP>
__device__ __forceinline__ int64_t tile_length(const AttentionArgs& a, const Request& r, int keys, bool shared) {
  if (!shared) return 1;
  if (a.window > 0) {
    // of the tile's tokens, from a multiple of 32 on; without causality the
    // request's first token sees the window before it and all that follows
    const int besides = (a.causal ? token_of(a, ROWS) : r.n) + 32;
    keys = keys - besides > a.window ? a.window + besides : keys;
  }
  return (keys <= STEP ? STEP : ((int64_t)keys + STEP - 1) / STEP * STEP) + tile_extra<V, ROWS>(a);
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
__device__ __forceinline__ int tiles_of(const AttentionArgs& a, const Request& r, int classes = 1) {
  const int tiles = (r.n * a.G + ROWS - 1) / ROWS;
  return classes == 2 ? (tiles + 1) / 2 : tiles;
}

// Positions of one cache head; of every classes-th tile.
template <class V, int ROWS, int STEP>
__device__ __forceinline__ int64_t head_length(const AttentionArgs& a, const Batch<V>& batch, bool shared, int classes = 1) {
  int64_t sum = 0;
  if (a.B == 1) {
    const Request r = {uniform(batch.first.q0), uniform(batch.first.n), uniform(batch.first.kv)};  // of lane 0
    return tiles_of<ROWS>(a, r, classes) * tile_length<V, ROWS, STEP>(a, r, uniform(batch.keys), shared);
  }
  for (int64_t b = threadIdx.x % kWave; b < a.B; b += kWave) {
    const Request r = batch.of(a, b);
    sum += tiles_of<ROWS>(a, r, classes) * tile_length<V, ROWS, STEP>(a, r, batch.keys_of(r, b), shared);
  }
  return uniform(wave_total(sum));
}

// The tile at a position within a head's stretch, in every lane of the wave.
// pos < head_length.
template <class V, int ROWS, int STEP>
__device__ __forceinline__ Place locate(const AttentionArgs& a, const Batch<V>& batch, int64_t pos, bool shared,
                                         int classes = 1) {
  Place p = {};
  int64_t base = 0;
  if (a.B == 1) {
    p.b = 0;
    p.r = {uniform(batch.first.q0), uniform(batch.first.n), uniform(batch.first.kv)};  // of lane 0
    const int64_t one = tile_length<V, ROWS, STEP>(a, p.r, uniform(batch.keys), shared);
    p.tile = (int)(shared ? quotient(pos, one) : pos);
    p.start = p.tile * one;
    p.end = p.start + one;
    return p;
  }
  for (int64_t b0 = 0; b0 < a.B; b0 += kWave) {
    const int64_t b = b0 + threadIdx.x % kWave;
    Request r = {};
    int64_t one = 0, own = 0;
    if (b < a.B) {
      r = batch.of(a, b);
      one = tile_length<V, ROWS, STEP>(a, r, batch.keys_of(r, b), shared);
      own = tiles_of<ROWS>(a, r, classes) * one;
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

// The tile behind `p`, of the next request or the next head where that was the
// last; there is one.  false: not among the next few requests, use locate().
template <class V, int ROWS, int STEP>
__device__ __forceinline__ bool advance(const AttentionArgs& a, const Batch<V>& batch, Place& p, int& head,
                                        int classes = 1) {
  const int64_t one = p.end - p.start;
  if (++p.tile < tiles_of<ROWS>(a, p.r, classes)) {
    p.start = p.end;
    p.end += one;
    return true;
  }
  p.tile = 0;
  p.start = p.end;
  for (int tries = 0; tries < 4; ++tries) {
    if (++p.b == a.B) {
      p.b = 0;
      p.start = 0;
      ++head;
    }
    if (p.b < kWave) p.r = {lane_value(batch.first.q0, p.b), lane_value(batch.first.n, p.b), lane_value(batch.first.kv, p.b)};
    else p.r = read_request(a, p.b);
    if (p.r.n > 0) {
      const int keys = V::kMore && p.b < kWave ? lane_value(batch.keys, p.b) : p.r.kv;
      p.end = p.start + tile_length<V, ROWS, STEP>(a, p.r, keys, true);
      return true;
    }
  }
  return false;
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
// it, or take the weights below what they need: such rows end not finite (total)
// and are computed again (SlowRow).
constexpr float kLift = 7.f;

// Capped scores cap * tanh(x), in powers of two.  Arguments up to kSmall by a
// polynomial in x^2 that is as near to tanh(x) / x as fp32 is (weighted least squares
// of the relative error over [0, kSmall]: 7.3e-8); it takes half as long as the others',
// cap - 2 cap / (1 + 2^(2 x log2(e))), whose exponential and reciprocal are off by an
// ulp each, which makes 2^-22 of the cap.
constexpr float kSmall = 0.6f;
__device__ __forceinline__ float capped_small(const AttentionArgs& a, float s) {
  const float x = s * a.cap_unit, t = x * x;
  float p = fmaf(t, 0.0154754265905575f, -0.05210147946762546f);
  p = fmaf(t, p, 0.1331017364332229f);
  p = fmaf(t, p, -0.33332309973340374f);
  p = fmaf(t, p, 0.9999999268688409f);
  return (a.cap * x) * p;
}
__device__ __forceinline__ float capped_large(const AttentionArgs& a, float s) {
  const float e = __builtin_amdgcn_exp2f(s * a.cap_unit * 2.88539008177792681f);
  return fmaf(-2.f * a.cap, __builtin_amdgcn_rcpf(1.f + e), a.cap);
}
// Which formula a score takes is its own matter alone: it must not depend on the others of a block,
// which its row may not see.
__device__ __forceinline__ bool is_small(const AttentionArgs& a, float s) { return fabsf(s * a.cap_unit) < kSmall; }
__device__ __forceinline__ float capped(const AttentionArgs& a, float s) {
  const float small = capped_small(a, s), large = capped_large(a, s);
  return is_small(a, s) ? small : large;
}

template <class V, int DP, int KB>
struct WaveTile {
  half8_t q[DP / 16];
  float16_t o[DP / 32];
  // running maximum of the scores (this row), and m * c - kLift (0 without one)
  float m, mc;
  float l, rest;  // sum of this lane's weights, and what its last addition rounded up
  RowBias bias;   // with SLOPES
  TreeRow tree;   // with MORE, in calls with a tree
  bool has_tree;

  // Caps a block's scores, of which `top` is the row's largest, and that too.  2048 tokens after their
  // like take 168 us where all are small, 178 / 190 / 204 / 217 where 0.03 / 0.3 / 1.6 / 13 % are not
  // (194 / 215 / 216 / 217 with both formulas for every score of a block that has a large one;
  // 217 / 255 / 265 / 272 with a third way for scores that are large in all lanes).
  __device__ __forceinline__ void cap_scores(const AttentionArgs& a, float16_t& s, float& top) const {
    float low = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) low = fminf(low, s[e]);
    if (__all(fmaxf(top, -low) * a.cap_unit < kSmall)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = capped_small(a, s[e]);
      top = capped_small(a, top);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        // the second formula only where some lane needs it
        const float v = s[e];
        const bool large = !is_small(a, v);
        s[e] = capped_small(a, v);
        if (__any(large)) s[e] = large ? capped_large(a, v) : s[e];
      }
      top = capped(a, top);
    }
  }

  // What variants need of row `row`, which exists.
  __device__ __forceinline__ void load_row(const AttentionArgs& a, const Request& r, int head, int row) {
    if constexpr (V::kSlopes) bias = row_bias<V>(a, r, head, row);
    if constexpr (V::kMore) {
      has_tree = a.tree != nullptr;
      if (has_tree) tree = tree_row(a, r, token_of(a, row));
    }
  }

  // The scores that the products with a block's keys are added to.
  __device__ __forceinline__ float16_t before(int key0) const {
    float16_t s = {};
    if constexpr (V::kSlopes) {
      const int h4 = threadIdx.x % kWave / 32 * 4;
      // at most 2^31 - 1024 + 64: keys behind the last one may be named
      const int back = bias.pos - key0 - h4 - bias.nearest;
      if (__all(bias.pos - key0 - 31 >= 0)) {
        // each key's distance as a number first, exact below 2^24: from one key to the next by
        // sums of slopes, the last of a block would keep what rounded the first one's bias
        const float far = (float)back;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = bias.slope * (far - (float)((e / 4) * 8 + e % 4));
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = back + bias.nearest - ((e / 4) * 8 + e % 4);
          s[e] = bias.slope * (float)((d < 0 ? -d : d) - bias.nearest);
        }
      }
    }
    return s;
  }

  // Scores times this are powers of two; capped ones are already.
  __device__ __forceinline__ static float unit(const AttentionArgs& a) { return V::kCap ? 1.f : a.c; }

  // A block's scores with those that the row does not see taken out; returns the largest of this lane's.
  __device__ __forceinline__ float mask(float16_t& s, int key0, int begin, int end) const {
    const int h4 = threadIdx.x % kWave / 32 * 4, first = begin - key0 - h4, last = end - key0 - h4;
    uint32_t bits = 0xFFFFFFFFu;
    if constexpr (V::kMore) {
      if (has_tree && key0 + 32 > tree.first) bits = tree.block(key0) >> h4;
    }
    bits &= last >= 32 ? ~0u : last <= 0 ? 0u : ~(~0u << last);
    bits &= first <= 0 ? ~0u : first >= 32 ? 0u : ~0u << first;
    const float unseen = -INFINITY;
    float top = unseen;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      // all ones or none, then the score or `unseen` bit by bit: half the operations of comparisons
      const uint32_t seen = (uint32_t)__builtin_amdgcn_sbfe((int)bits, (e / 4) * 8 + e % 4, 1);
      float v = s[e];
      asm("v_bfi_b32 %0, %1, %0, %2" : "+v"(v) : "v"(seen), "s"(unseen));
      s[e] = v;
      top = fmaxf(top, v);
    }
    return top;
  }

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

  // Row `row` of the request, which exists (lane l and l ^ 32 hold one row): the loads
  // (wherever rows start), and later what waits for them.
  __device__ __forceinline__ void fetch_q(const AttentionArgs& a, const Request& r, int head, int row) {
    const int h = (threadIdx.x % kWave) / 32;
    const int t = token_of(a, row);
    const uint16_t* src = a.q.p + (r.q0 + t) * a.q.ts + (head * a.G + row - t * a.G) * a.q.hs;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      const int d = s * 16 + h * 8;
      q[s] = *reinterpret_cast<const half8_any*>(src + (d < a.D ? d : 0));
    }
  }
  // Zeros unless `live`, and past D.
  __device__ __forceinline__ void finish_q(const AttentionArgs& a, bool live) {
    const int h = (threadIdx.x % kWave) / 32;
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
                                       bool masked, const AttentionArgs& a) {
    const float c = unit(a);
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
    if constexpr (V::kSlopes)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = before(key0 + kb * 32);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      if (t + AHEAD < KT) read_k(t + AHEAD);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[t % (AHEAD + 1)][kb], q[t],
                                                       t == 0 && !V::kSlopes ? float16_t{} : s[kb], 0, 0, 0);
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
    float top;
    if constexpr (V::kCap || V::kMore) {
      top = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        float most = s[kb][0];
        if (V::kCap || !masked) {
#pragma unroll
          for (int e = 1; e < 16; ++e) most = fmaxf(most, s[kb][e]);
        }
        if constexpr (V::kCap) cap_scores(a, s[kb], most);
        if (masked) most = mask(s[kb], key0 + kb * 32, begin, end);
        top = fmaxf(top, most);
      }
    } else {
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
      top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[kb][e]);
    }
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
  __device__ __forceinline__ void scores(uint32_t k_at, int key0, float16_t& s) {
    if constexpr (V::kSlopes) s = before(key0);
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
                                                 t == 0 && !V::kSlopes ? float16_t{} : s, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // Weights of scores alone.
  __device__ __forceinline__ void weights(const float16_t& s, half8_t (&p)[2], const AttentionArgs& a) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float w = __builtin_amdgcn_exp2f(s[e] * unit(a) - mc);
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
                                         int end, bool masked, const AttentionArgs& a) {
    const float c = unit(a);
    if constexpr (V::kCap || V::kMore) {
      if constexpr (V::kCap) {
        cap_scores(a, s, top);
        over = top - m;
      }
      if (masked) {
        top = row_max(mask(s, key0, begin, end));
        over = (top - m) * c;
      }
    } else if (masked) {
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
  // next_key: the first key of the scores `next`.
  template <typename F>
  __device__ __forceinline__ void block(const float16_t& s, float16_t& next, const half8_t (&p)[2], half8_t (&made)[2],
                                        const Lanes& at, uint32_t k_off, uint32_t v_off, bool more,
                                        const AttentionArgs& a, int next_key, float& top, float& over, F at_step) {
    const float c = unit(a);
    constexpr int STEPS = 2 * N;
    float w[16], sum;
    u32x4 packed[2];
    if constexpr (V::kSlopes) next = before(next_key);
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
      if (is_key(i)) next = __builtin_amdgcn_mfma_f32_32x32x16_f16(op, q[nth(i)], i == 0 && !V::kSlopes ? float16_t{} : next, 0, 0, 0);
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

  // Sum of the row's weights, in both its lanes; NaN where even the largest has lost 2^2
  // of its 2^kLift to the rounding of mc, which takes fp16's bits from all of them, or all of them
  // to zero (scores of 2^26 powers of two and more).
  __device__ __forceinline__ float total(const AttentionArgs& a) const {
    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const bool lost = m > -INFINITY && fmaf(m, unit(a), -mc) < kLift - 2.f;
    return lost ? __builtin_nanf("") : __uint_as_float(w[0]) + __uint_as_float(w[1]);
  }

  // Whether this lane's part of the row, whose sum is `sum`, holds a value that is not finite.
  __device__ __forceinline__ bool broken(float sum) const {
    float z = (sum - sum) + (mc - mc);
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

// The logarithm of a row's sum as it is returned.
template <class V>
__device__ __forceinline__ float final_lse(float mc, float l, bool sees, const AttentionArgs& a, const Request& r,
                                           int head, int row) {
  const float lse = row_lse(mc, l, sees);
  if constexpr (V::kSlopes && !V::kCap) return lse + lse_bias<V>(a, r, head, row);
  return lse;
}

// One row over the keys [begin, end), key by key, by a whole wave: for rows
// whose result is not finite, or whose masked tiles held values that are not.
// Only keys that the row sees are touched.  Lane l holds dimensions l, l + 64, ...
template <class V, int DP>
struct SlowRow {
  float m = -INFINITY, l = 0.f, o[(DP + kWave - 1) / kWave] = {};

  // r, head, row: as in query_row
  __device__ __forceinline__ void run(const AttentionArgs& a, const uint16_t* q, int64_t head_off,
                                      const int32_t* pages, const Request& r, int head, int row, int begin, int end) {
    RowBias bias = {};
    if constexpr (V::kSlopes) bias = row_bias<V>(a, r, head, row);
    const bool has_tree = V::kMore && a.tree != nullptr;
    TreeRow tree = {};
    if (has_tree) tree = tree_row(a, r, token_of(a, row));
    const int lane = threadIdx.x % kWave;
    for (int j0 = begin; j0 < end; j0 += kWave) {
      const int j = j0 + lane;
      float s = -INFINITY;
      int64_t off = 0;
      const bool seen = j < end && (!has_tree || (tree.block(j) & 1) != 0);
      if (seen) {
        off = key_offset(a, page_of(a, pages, j), j) + head_off;
        s = 0.f;
        for (int i = 0; i < a.D; ++i) s += half_value(q[i]) * half_value(a.ck[off + i]);
        if constexpr (V::kSlopes || V::kCap) {
          s = a.negate ? -s : s;
          if constexpr (V::kSlopes) {
            const int d = bias.pos - j;
            s += bias.slope * (float)((d < 0 ? -d : d) - bias.nearest);
          }
          s = V::kCap ? capped(a, s) : s * a.c;
        } else {
          s *= a.negate ? -a.c : a.c;
        }
      }
      float top = s;
#pragma unroll
      for (int x = 1; x < kWave; x *= 2) top = fmaxf(top, __shfl_xor(top, x, kWave));
      const float next = fmaxf(m, top);
      const float p = seen ? exp2f(s - (next == -INFINITY ? 0.f : next)) : 0.f;
      const float keep = l == 0.f ? 0.f : exp2f(m - next);
      l = l * keep + wave_sum(p);
      m = next;
#pragma unroll
      for (float& v : o) v = keep == 0.f ? 0.f : v * keep;
      const int count = end - j0 < kWave ? end - j0 : kWave;
      for (int e = 0; e < count; ++e) {
        const float w = __shfl(p, e, kWave);
        if (V::kMore && !__shfl((int)seen, e, kWave)) continue;
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
                                        int64_t slot, bool broken) const {
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
    const int t = token_of(a, row);
    const bool sees = l != 0.f || token_sees<V>(a, r, t);
    const float f = row_factor(l, sees);
    uint16_t* dst = a.out.p + (r.q0 + t) * a.out.ts + (head * a.G + row - t * a.G) * a.out.hs;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + i * kWave < a.D) dst[lane + i * kWave] = f32_to_f16_bits(o[i] * f);
    if (lane == 0 && a.lse != nullptr)
      a.lse[(int64_t)(r.q0 + t) * a.Hq + head * a.G + row - t * a.G] = final_lse<V>(m, l, sees, a, r, head, row);
  }
};

}  // namespace fasq
