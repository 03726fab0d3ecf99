// Attention of new tokens over a paged cache: which kernel a call takes, and its plain variant.
#include <hip/hip_runtime.h>

#include <cmath>

#include "fasq_attention_kernels.h"

namespace fasq {

// The other variants, a source file each.
extern template hipError_t launch_variant<Variant<true, false, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
extern template hipError_t launch_variant<Variant<true, true, false>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
extern template hipError_t launch_variant<Variant<true, false, true>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);
extern template hipError_t launch_variant<Variant<true, true, true>>(const AttentionPlan&, const AttentionArgs&, hipStream_t);

namespace {

AttentionPlan plan_attention(int64_t T, int64_t B, int Hq, int Hkv, int D, const DeviceInfo& dev) {
  AttentionPlan p;
  const int64_t G = Hq / Hkv, rows = T * G;
  p.DP = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  // Tiles of 32 rows for up to 32 of a request on average (16 requests of one
  // token 37 us, 42 in tiles of 128), or 64 in all: keys split further make up
  // for keys read twice (16 tokens of one request on 4000 keys 20 us, 35; on
  // 40000 keys 71, 65; 32 tokens there 117, 71).
  p.few = rows <= 32 * B || rows <= 64;
  p.rows = p.few ? 32 : 128;
  p.tiles = (rows + (p.rows - 1) * (B < T ? B : T)) / p.rows;
  // Workgroups that the chip holds at once (by LDS).  16 requests of one token,
  // 64 dimensions: 23.2 us with two a compute unit, 26.6 with one.
  p.parts = dev.num_cus * (p.few ? (p.DP == 64 ? 2 : 1) : (p.DP == 256 ? 1 : 2));
  // Whole tiles are left whole where they fill the chip: at least twice (4096
  // tokens of 32 heads on 8 take 182 us, split 215), or one request's, once
  // (2048 tokens 67 us, split 71).
  const int64_t whole = rows / p.rows * Hkv;
  const bool once = B == 1 && p.tiles * Hkv <= p.parts && 16 * whole >= 15 * p.parts;
  p.split = p.few || !(once || whole >= 2 * p.parts);
  // Two to four tiles of a request's rows at most (trees): its even and odd ones go to
  // a half of the workgroups each, and both come by the same keys at the same time, so
  // one reads them from memory and the other from the last-level cache.  2 trees of 64
  // nodes on 65536 to 131072 keys (32 heads on 8): 333 us in one line of tiles, 292 in
  // two; only in the variants with masks, caps or slopes, whose shares are their own.  It
  // goes by the average request: 4 capped requests of 90 tokens (three tiles) on 8192 keys take 113 us
  // and 111 in one line, one of 500 tokens beside three single ones on 8192 keys, which have no odd
  // tiles, 67 and 54.
  p.classes = !p.few && p.split && p.parts % 16 == 0 && rows > p.rows * B && rows <= 4 * p.rows * B ? 2 : 1;
  const int64_t of_share = int64_t(2) * p.rows * (p.DP + 2) * (int64_t)sizeof(float) + (int64_t)sizeof(CutTile);
  p.bytes = p.split ? p.parts * of_share : 0;
  return p;
}

}  // namespace

int64_t attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D, const DeviceInfo& dev) {
  return plan_attention(T, B, Hq, Hkv, D, dev).bytes;
}

hipError_t launch_attention(const AttentionProblem& p, const DeviceInfo& dev, hipStream_t stream) {
  const AttentionPlan pl = plan_attention(p.T, p.B, p.Hq, p.Hkv, p.D, dev);
  AttentionArgs a = {};
  a.q = p.q;
  a.out = p.out;
  a.T = p.T;
  a.B = p.B;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.Hq / p.Hkv;
  a.D = p.D;
  a.ck = static_cast<const uint16_t*>(p.cache.k);
  a.cv = static_cast<const uint16_t*>(p.cache.v);
  a.num_pages = (int)p.cache.num_pages;
  a.page_size = (uint32_t)p.cache.page_size;
  a.page_shift = -1;
  for (int s = 0; s < 31; ++s)
    if (p.cache.page_size == int64_t(1) << s) a.page_shift = s;
  a.g_shift = -1;
  for (int s = 0; s < 31; ++s)
    if (a.G == 1 << s) a.g_shift = s;
  a.page_stride = p.cache.page_stride;
  a.slot_stride = p.cache.slot_stride;
  a.head_stride = p.cache.head_stride;
  a.pages = p.pages;
  a.page_row_stride = p.page_row_stride;
  a.capacity = (int)(p.max_pages * p.cache.page_size);
  a.q_start = p.q_start;
  a.kv_len = p.kv_len;
  a.c = (float)(std::fabs((double)p.scale) * 1.4426950408889634074);
  if (a.c < 1e-30f) a.c = 1e-30f;
  a.negate = p.scale < 0.f;
  a.causal = p.causal;
  a.window = p.window < a.capacity ? (int)p.window : 0;
  auto aligned = [](const HeadsView& v, int bytes) {
    return reinterpret_cast<uintptr_t>(v.p) % bytes == 0 && v.ts % (bytes / 2) == 0 && v.hs % (bytes / 2) == 0;
  };
  a.out_vec = aligned(p.out, 8);
  a.whole_units = p.cache.page_size % 16 == 0 && p.cache.slot_stride < int64_t(1) << 25;
  a.lse = p.lse;
  if (pl.split && p.workspace != nullptr && p.workspace_bytes >= pl.bytes) {
    a.parts = pl.parts;
    a.part_o = static_cast<float*>(p.workspace);
    a.part_ml = a.part_o + int64_t(2) * pl.parts * pl.rows * pl.DP;
    a.cuts = reinterpret_cast<CutTile*>(a.part_ml + int64_t(2) * pl.parts * pl.rows * 2);
  }
  const AttentionMore& more = p.more;
  const bool cap = more.softcap > 0.f, slopes = more.slopes != nullptr;
  if (!cap && !slopes && more.spans == nullptr && more.tree == nullptr) return launch_variant<Plain>(pl, a, stream);
  a.spans = more.spans;
  a.tree = more.tree;
  a.tree_stride = more.tree_stride;
  a.tree_words = (int)more.tree_words;
  a.slopes = more.slopes;
  a.slope_unit = (float)(1.4426950408889634074 / a.c);
  a.cap = (float)(more.softcap * 1.4426950408889634074);
  a.classes = pl.classes;
  a.cap_unit = cap ? (float)(a.c / (more.softcap * 1.4426950408889634074)) : 0.f;
  if (cap) return slopes ? launch_variant<Variant<true, true, true>>(pl, a, stream) : launch_variant<Variant<true, true, false>>(pl, a, stream);
  return slopes ? launch_variant<Variant<true, false, true>>(pl, a, stream) : launch_variant<Variant<true, false, false>>(pl, a, stream);
}

}  // namespace fasq
