// Host planner of the AdamW operators: blocks and state layout of every tensor, tiles of a slot's
// gradients.  HIP-free.
#include "adamw_internal.hpp"

#include <algorithm>

#include "plan.hpp"

namespace acp {
namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t align_up(int64_t x, int64_t a) { return cdiv(x, a) * a; }
bool words(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace

std::string adamw_plan(AwPlan& plan, int32_t num_tensors, const int32_t* ndims, const int64_t* dims,
                       int32_t bits, const uint8_t* no_decay, uint64_t seed) {
  if (num_tensors < 1) return "no tensors";
  if (!ndims || !dims) return "null shape arrays";
  if (bits != 32 && bits != 8) return "moments have 32 or 8 bits";
  plan.bits = bits;
  plan.seed = seed;
  int64_t off = 0, blk = 0, at = 0;
  for (int32_t t = 0; t < num_tensors; ++t) {
    if (ndims[t] < 1 || ndims[t] > 8) return "a tensor has 1 to 8 dimensions";
    int64_t rest = 1;
    for (int32_t i = 0; i < ndims[t]; ++i) {
      const int64_t d = dims[at + i];
      if (d < 1 || d > (int64_t(1) << 38)) return "dimension out of range";
      if (i > 0 || ndims[t] == 1) {
        if (rest > kAwMaxCols / d) return "a row is too long";
        rest *= d;
      }
    }
    AwTensor x{};
    x.n = ndims[t] == 1 ? 1 : dims[at];
    x.m = rest;
    at += ndims[t];
    if (x.n > kAwMaxElems / x.m) return "a tensor is too large";
    if (x.m < kAwScaleBlock) {
      x.k = static_cast<int32_t>(kAwScaleBlock / x.m);
      x.nb = 1;
      x.w = static_cast<int32_t>(x.k * x.m);
      x.blocks = cdiv(x.n, x.k);
    } else {
      const int64_t nb = cdiv(x.m, kAwScaleBlock);
      x.k = 1;
      x.nb = static_cast<int32_t>(nb);
      x.w = static_cast<int32_t>(align_up(cdiv(x.m, nb), 4));
      x.blocks = x.n * nb;
      x.slack = nb * x.w - x.m;
    }
    x.off = off;
    x.blk = blk;
    x.decay = no_decay && no_decay[t] ? 0 : 1;
    off += align_up(x.n * x.m, kAwAlign);
    blk += x.blocks;
    if (off > kAwMaxElems || blk > kAwMaxElems) return "too many elements";
    plan.tensors.push_back(x);
  }
  plan.elems = off;
  plan.blocks = blk;
  const int64_t each = bits / 8;
  int64_t b = 0;
  plan.off_m = b;       b = align_up(b + off * each, 256);
  plan.off_v = b;       b = align_up(b + off * each, 256);
  plan.off_ms = b;      b = align_up(b + (bits == 8 ? blk * 4 : 0), 256);
  plan.off_vs = b;      b = align_up(b + (bits == 8 ? blk * 4 : 0), 256);
  plan.off_tensors = b; b = align_up(b + num_tensors * static_cast<int64_t>(sizeof(AwTensor)), 256);
  plan.total_bytes = b;
  return "";
}

namespace {

// the lists of a slot's tiles, in their order
enum { kDenseWide, kDense, kProductWide, kProduct, kNarrow, kJoined, kNorm, kGram, kTrace, kLists };

// rows of a narrow tile: as many whole blocks as kAwRows rows hold, at least one
int64_t narrow_rows(const AwTensor& x) { return x.k * std::max<int64_t>(1, kAwRows / x.k); }

// Whether every row of the tensor, of its copy and of its gradient is whole words, of the values of two bytes and
// one byte too (32 bits, values: but for the end of the last).
bool whole_words(const AwPlan& plan, const AwTensor& x, const AwGrad& g) {
  return words(x.copy) && words(g.g) &&
         ((plan.bits == 32 && g.rank == 0) || ((x.w & 3) == 0 && ((x.slack ? x.m : x.n * x.m) & 3) == 0));
}

}  // namespace

std::string adamw_slot(AwSlotPlan& s, const AwPlan& plan) {
  const int32_t count = static_cast<int32_t>(plan.tensors.size());
  int64_t doubles = 0, all_groups = 0, dense_elems = 0;
  for (int32_t t = 0; t < count; ++t) {
    const AwTensor& x = plan.tensors[t];
    if (s.grads[t].rank && x.m >= kAwScaleBlock) all_groups += cdiv(x.n, kAwRows) * x.nb;
    if (!s.grads[t].rank) dense_elems += x.n * x.m;
    s.rank = std::max(s.rank, s.grads[t].rank);
  }
  const bool join = all_groups > 0 && dense_elems <= kAwJoined;
  const int64_t row_groups = std::max<int64_t>(1, std::min<int64_t>(aw_row_groups(plan.bits, s.rank), all_groups / kAwProductTiles));
  const int64_t per = plan.bits == 8 ? kAwTileBlocks : kAwTile, span = aw_norm_tile(plan.elems);
  const int gt = aw_gram_t(s.rank);
  // how many tiles there will be, before any list of them is made: init takes more than fits any host's memory
  int64_t counts[kLists] = {};
  for (int32_t t = 0; t < count; ++t) {
    const AwTensor& x = plan.tensors[t];
    const AwGrad& g = s.grads[t];
    const int64_t numel = x.n * x.m;
    const bool wide = whole_words(plan, x, g);
    if (g.rank == 0) {
      const int64_t all = plan.bits == 8 ? x.blocks : numel, tiles = cdiv(all, per);
      // (32 bits: a tensor's last tile can end inside a word)
      const int64_t last = wide && plan.bits == 32 && (all & 3) != 0;
      counts[join ? kJoined : wide ? kDenseWide : kDense] += join ? tiles : tiles - last;
      if (!join) counts[kDense] += last;
      counts[kNorm] += cdiv(numel, span);
      continue;
    }
    if (x.m < kAwScaleBlock)
      counts[kNarrow] += cdiv(x.n, narrow_rows(x));
    else
      counts[wide ? kProductWide : kProduct] += cdiv(cdiv(x.n, kAwRows), row_groups) * x.nb;
    const int64_t q = aw_gram_side(g.rank, gt), rows = aw_gram_rows(g.rank);
    counts[kGram] += (cdiv(x.n, rows) + cdiv(x.m, rows)) * (q * (q + 1) / 2);
    counts[kTrace] += aw_gram_entries(g.rank, gt) / 256;
  }
  // a launch has fewer than 2^32 threads, a tile at most 1024 of them; the last launch of products takes the
  // narrow and joined tiles along
  const int64_t waves = aw_product_waves(s.rank);
  const int64_t along = counts[kNarrow] + counts[kJoined] * aw_joined_groups(plan.bits, waves);
  const int64_t last_products = counts[kProduct] ? counts[kProduct] : counts[kProductWide];
  bool fits = (align_up(along, 64) + align_up(last_products, 64)) * 64 * waves < int64_t(1) << 32;
  for (int64_t k : counts) fits = fits && k < int64_t(1) << 22;
  if (!fits) return "too many elements for one slot";

  std::vector<AwTile> lists[kLists];
  for (int32_t i = 0; i < kLists; ++i) lists[i].reserve(counts[i]);
  for (int32_t t = 0; t < count; ++t) {
    const AwTensor& x = plan.tensors[t];
    AwGrad& g = s.grads[t];
    const int64_t numel = x.n * x.m;
    const bool wide = whole_words(plan, x, g);
    if (g.rank == 0) {
      const int64_t all = plan.bits == 8 ? x.blocks : numel;
      for (int64_t f = 0; f < all; f += per) {
        const bool words_only = wide && (plan.bits == 8 || ((all - f) & 3) == 0 || all - f >= per);
        lists[join ? kJoined : words_only ? kDenseWide : kDense].push_back(
            AwTile{t, static_cast<int32_t>(std::min(per, all - f)),
                   plan.bits == 8 && x.slack ? f / x.nb | f % x.nb << kAwSegShift : f});
      }
      for (int64_t f = 0; f < numel; f += span)
        lists[kNorm].push_back(AwTile{t, static_cast<int32_t>(std::min(span, numel - f)), f});
      continue;
    }
    if (x.m < kAwScaleBlock) {
      const int64_t rows = narrow_rows(x);
      for (int64_t r0 = 0; r0 < x.n; r0 += rows)
        lists[kNarrow].push_back(AwTile{t, static_cast<int32_t>(std::min(rows, x.n - r0)), r0});
    } else {  // rows of one block column
      const int64_t groups = cdiv(x.n, kAwRows), step = cdiv(groups, row_groups);
      for (int64_t g0 = 0; g0 < step; ++g0)
        for (int64_t seg = 0; seg < x.nb; ++seg)
          lists[wide ? kProductWide : kProduct].push_back(
              AwTile{t, static_cast<int32_t>(step * kAwRows), g0 * kAwRows | seg << kAwSegShift});
    }
    const int q = aw_gram_side(g.rank, gt);
    for (int32_t side = 0; side < 2; ++side) {
      g.slices[side] = static_cast<int32_t>(cdiv(side ? x.m : x.n, aw_gram_rows(g.rank)));
      g.gram[side] = doubles;
      doubles += g.slices[side] * aw_gram_entries(g.rank, gt);
      for (int32_t sl = 0; sl < g.slices[side]; ++sl)
        for (int32_t bi = 0; bi < q; ++bi)
          for (int32_t bj = bi; bj < q; ++bj) lists[kGram].push_back(AwTile{t, side + 2 * bi + 256 * bj, sl});
    }
    for (int32_t bi = 0; bi < q; ++bi)
      for (int32_t bj = bi; bj < q; ++bj) {
        int64_t at = aw_gram_at(g.rank, gt, bi, bj);
        for (int32_t i = 0; i < gt; ++i)
          for (int32_t j = bi == bj ? i : 0; j < gt; ++j, at += 256)
            lists[kTrace].push_back(AwTile{t, bi == bj && i == j ? 1 : 2, at});
      }
  }
  int64_t* to[kLists] = {&s.dense[1], &s.dense[0], &s.product[1], &s.product[0], &s.narrow, &s.joined, &s.norm, &s.gram, &s.trace};
  for (int32_t i = 0; i < kLists; ++i) {
    *to[i] = static_cast<int64_t>(lists[i].size());
    s.tiles.insert(s.tiles.end(), lists[i].begin(), lists[i].end());
  }
  int64_t b = 0;
  s.off_grads = b; b = align_up(b + count * static_cast<int64_t>(sizeof(AwGrad)), 256);
  s.off_tiles = b; b = align_up(b + static_cast<int64_t>(s.tiles.size() * sizeof(AwTile)), 256);
  s.off_sums = b;  b = align_up(b + (s.norm + s.trace) * 8, 256);
  s.off_gram = b;  b = align_up(b + doubles * 8, 256);
  s.total_bytes = b;
  return "";
}

// The key of a step's rounding; each tensor's follows from it on the device.
uint32_t adamw_step_key(uint64_t seed, int64_t step) {
  return static_cast<uint32_t>(splitmix64_mix(seed ^ splitmix64_mix(static_cast<uint64_t>(step))) >> 32);
}

}  // namespace acp
