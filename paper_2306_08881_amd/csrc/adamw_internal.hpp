// Descriptors of the AdamW operators, shared by their host planner (HIP-free) and the gfx950 kernels.
//
// State block (one per optimiser, allocated by the caller), regions in order, each 256-byte aligned:
//   m, v      the moments.  32 bits: fp32 values, tensor k's element i at AwTensor::off + i.  8 bits:
//             m and sqrt(v) as e4m3 codes at the same places, a byte each.
//   scales    8 bits: one fp32 scale per block, of m and then of sqrt(v), tensor k's block j at
//             AwTensor::blk + j.
//   tensors   AwTensor[].
// Gradient block (one per gradient slot): AwGrad[], the launches' tiles, partial sums of the norm.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

namespace acp {

constexpr int kAwBlock = 256;           // threads per workgroup (4 waves of 64)
constexpr int kAwScaleBlock = 256;      // values per block of 8-bit moments, at most: one wave, four a lane
constexpr int64_t kAwAlign = 256;       // elements: where tensors start in the m and v regions
constexpr int64_t kAwMaxCols = int64_t(1) << 38;
constexpr int64_t kAwMaxElems = int64_t(1) << 40;
constexpr int kAwMaxRank = 256;
constexpr int64_t kAwMaxFactorRows = int64_t(1) << 30;
constexpr int64_t kAwMaxFactorCols = int64_t(1) << 24;  // 16 rows' byte offsets then stay below 2^31
constexpr int kAwSlots = 4;             // gradient slots of an optimiser

constexpr int kAwPart = 256;            // elements a wave takes of a dense tile (32-bit moments)
constexpr int kAwPartBlocks = 2;        // blocks it takes (8-bit moments, rows of whole words)
constexpr int64_t kAwTile = 2048;       // elements of a dense tile
constexpr int64_t kAwTileBlocks = 16;   // blocks of one
// Elements of a tile of the norm: longer ones where the optimiser has enough elements.  us with 16384 and 32768,
// one tensor of values: fp32 8 M elements 9.3 and 10.5, 32 M 23.0 and 24.1, 64 M 43.1 and 43.7, 128 M 82.4 and
// 82.3, 512 M 319 and 312; bfloat16 8 M 8.2 and 9.0, 32 M 14.5 and 14.5, 64 M 24.5 and 24.0, 512 M 168 and 162.
constexpr int64_t aw_norm_tile(int64_t elems) { return elems >= int64_t(1) << 26 ? 32768 : 16384; }
constexpr int kAwRows = 16;             // rows of A B^T that go through LDS at a time
// Groups of kAwRows rows that a tile of A B^T has, at most: its wave loads B's part once for them.  They
// lie as many groups apart as there are tiles in the column, so that all workgroups together sweep
// through the tensor in step (8 bits, BERT-large rank 32: neighbouring groups 1116 us, these 1055).
// BERT-large, us with 1, 2, 4 and 16 groups:
//   8 bits   rank 4   794  735  718  779     rank 32   974  856  814  811     rank 64 1452 1243 1117 1012
//            rank 128 2284 1782 1581 1362    rank 256 5305 3886 3086 2528
//   32 bits  rank 4  1277 1327 1427 1511     rank 16  1327 1324 1416 1511     rank 32 1308 1357 1410 1513
//            rank 64 1555 1428 1428 1492     rank 128 2228 1848 1670 1573     rank 256 4895 3652 3161 2824
// With 32 bits HBM is what counts up to rank 32, and one group is best.  Above, B's part, loaded for 16 rows only,
// costs more than that gains: there the rule for 32 bits is not the best one.
// A slot with few groups has fewer a tile, so that there are kAwProductTiles tiles: 8 bits, us with 1024, 2048,
// 4096 and 8192, BERT-base rank 32 272 272 272 277, rank 64 366 354 363 381, rank 128 484 473 497 531,
// ResNet-50 rank 4 67.5 66.3 66.7 66.8, rank 64 104 107 121 121.
constexpr int aw_row_groups(int bits, int rank) { return bits == 32 ? 1 : rank <= 32 ? 4 : 16; }
constexpr int64_t kAwProductTiles = 4096;
// Dense tensors beside factored ones go with the products' launch up to this many elements (the vectors of a
// model, or what else a launch of its own would cost more than their lower occupancy there).  us in their launch and
// in one of their own, beside factors of 4096 x 4096: 8 bits 64 K elements 45.3 and 49.1, 1 M 48.4 and 50.9, 2 M
// 52.1 and 52.9, 8 M 69.5 and 70.1; 32 bits 64 K 67.1 and 69.6, 2 M 76.6 and 78.7, 8 M 102.6 and 105.0.
constexpr int64_t kAwJoined = int64_t(1) << 21;

// Waves of a workgroup of A B^T that share a tile's columns: four, which meet at fewer barriers (8 bits, BERT-large
// rank 32 959 us, with eight 1036), but eight above rank 128, where B's part would leave a SIMD one wave (rank
// 256 2701 us, with eight 2495).
constexpr int aw_product_waves(int rank) { return rank <= 128 ? 4 : 8; }
// Workgroups of `waves` waves that share a joined dense tile, a wave taking kAwPart elements or one block.
constexpr int64_t aw_joined_groups(int bits, int64_t waves) { return (bits == 32 ? kAwTile / kAwPart : kAwTileBlocks) / waves; }

struct AwTensor {
  float* p;       // parameters
  uint16_t* copy; // bfloat16 copy, or null
  int64_t n, m;   // rows, columns
  int64_t off;    // first element in the m and v regions
  int64_t blk;    // first block
  int64_t blocks; // number of blocks
  int64_t slack;  // nb * w - m (rows that blocks do not fill; 0 where blocks follow each other)
  int32_t w;      // elements of a block (the last of a row, or of the tensor, may be shorter)
  int32_t nb;     // blocks of a row (1 where a block holds whole rows)
  int32_t k;      // rows of a block
  int32_t decay;  // weight decay applies
};

struct AwGrad {
  const void* g;   // the gradient's values, or null
  const float *a, *b;  // its factors, n x rank and m x rank
  int64_t gram[2]; // first partial Gram matrix of a and b (doubles, in the gradient block's partials)
  int32_t slices[2];  // row slices of a and b
  int32_t bf16;    // g holds bfloat16 values
  int32_t rank;    // 0: g
};

// Dense tiles: elements [first, first + count) (32 bits, and the norm) or blocks (8 bits; where rows end
// inside a block, slack > 0, the first is row | block of the row << kAwSegShift) of a tensor.
// Tiles of A B^T: rows [row, row + count) and block column seg, first = row | seg << kAwSegShift; where
// blocks hold whole rows (narrow), first = row.
// Gram tiles: count = side + 2 bi + 256 bj, first = slice.  Trace tiles: count = how often the tile of 256
// entries counts, first = its first entry.
struct AwTile {
  int32_t tensor, count;
  int64_t first;
};
constexpr int kAwSegShift = 32;
constexpr int64_t kAwRowMask = (int64_t(1) << kAwSegShift) - 1;

// Gram matrices are formed in square blocks of 16 t columns, a wave each, over slices of aw_gram_rows(r)
// factor rows.  t, in 16-column tiles, is the slot's: that of its largest rank.  A block has t^2 tiles
// of 256 entries, one on the diagonal of the matrix those on and above its own diagonal.
constexpr int aw_gram_t(int r) { return r <= 16 ? 1 : r <= 32 ? 2 : 4; }
constexpr int aw_gram_rows(int r) { return r <= 64 ? 256 : 1024; }
constexpr int aw_gram_side(int r, int t) { return (r + 16 * t - 1) / (16 * t); }  // blocks of a side
constexpr int64_t aw_gram_entries(int r, int t) {  // of a whole matrix
  const int64_t q = aw_gram_side(r, t);
  return (q * (t * (t + 1) / 2) + q * (q - 1) / 2 * (t * t)) * 256;
}
constexpr int64_t aw_gram_at(int r, int t, int bi, int bj) {  // first entry of block (bi, bj), bi <= bj
  const int64_t q = aw_gram_side(r, t), d = t * (t + 1) / 2, f = t * t, i = bi;
  return (i * d + (i * q - i * (i + 1) / 2) * f + (bj > bi ? d + (bj - bi - 1) * f : 0)) * 256;
}

struct AwPlan {
  int32_t bits = 32;
  uint64_t seed = 0;
  std::vector<AwTensor> tensors;
  int64_t elems = 0, blocks = 0;  // of the m and v regions, and of the scales
  int64_t off_m = 0, off_v = 0, off_ms = 0, off_vs = 0, off_tensors = 0, total_bytes = 0;
};

// Launches on one slot's gradients
struct AwSlotPlan {
  std::vector<AwGrad> grads;
  std::vector<AwTile> tiles;  // dense, product, narrow product, joined dense, norm, gram and trace tiles, in that order
  // [1]: every row of the tensor, of its copy and of its gradient is whole words; these come first
  int64_t dense[2] = {0, 0}, product[2] = {0, 0};
  int64_t narrow = 0, joined = 0;  // joined: dense tiles that go with the last launch of products
  int64_t norm = 0, gram = 0, trace = 0;  // their numbers
  int32_t rank = 0;           // the largest of the slot
  int64_t off_grads = 0, off_tiles = 0, off_sums = 0, off_gram = 0, total_bytes = 0;
};

struct AwArgs {
  const AwTensor* tensors;
  const AwGrad* grads;
  const AwTile* tiles;
  uint8_t *m, *v;     // regions of the moments
  float *ms, *vs;     // and of their scales
  const float* clip;  // norm and clip coefficient, or null
  float b1, c1, b2, c2;  // betas and 1 - betas
  float lr;           // lr / (1 - beta1^t)
  float rs;           // 1 / sqrt(1 - beta2^t)
  float eps, decay;   // 1 - lr * weight decay
  float scale;        // of the gradients
  uint32_t key;       // of the rounding
  // tiles of products of a launch, narrow and joined dense ones that go with it, and workgroups of those
  uint32_t count, narrow, joined, others;
};

struct AwNormArgs {
  const AwTensor* tensors;
  const AwGrad* grads;
  const AwTile* tiles;
  double* sums;   // one per norm tile, then one per trace tile
  double* gram;   // partial Gram matrices
  float* clip;
  int64_t count;  // of sums
  int64_t norm, gram_tiles;  // tiles of the norm of values, and of Gram matrices
  int32_t t;      // aw_gram_t of the slot
  float scale, max_norm;
};

std::string adamw_plan(AwPlan& plan, int32_t num_tensors, const int32_t* ndims, const int64_t* dims,
                       int32_t bits, const uint8_t* no_decay, uint64_t seed);
std::string adamw_slot(AwSlotPlan& slot, const AwPlan& plan);  // slot.grads' pointers and ranks are set
uint32_t adamw_step_key(uint64_t seed, int64_t step);

}  // namespace acp
