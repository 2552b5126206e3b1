// AdamW over many tensors at once, with moments of 32 or 8 bits, on gradients as values or as the two
// factors that the compressor holds, and the norm of all gradients together.
//
// Arithmetic of a step, all in fp32, the same in every kernel, c = scale * clip coefficient:
//   g' = c g;  m' = b1 m + (1 - b1) g';  v' = b2 v + (1 - b2) g'^2
//   p' = d p - s m' / (sqrt(v') rs + eps),  d = 1 - lr wd (1 without decay), s = lr / (1 - b1^t),
//   rs = 1 / sqrt(1 - b2^t)
#include <hip/hip_runtime.h>

#include "adamw_internal.hpp"
#include "device.hpp"

#pragma clang fp contract(off)

namespace acp {
namespace {

constexpr int kNormLoads = 4;   // loads of a lane in flight in the norm
constexpr int kLdsPitch = 260;  // floats from a row of a product tile to the next: 16 lanes' 16-byte
                                // writes of 16 rows then cover all banks

typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef double d4 __attribute__((ext_vector_type(4)));

__device__ inline float bf16_value(unsigned short h) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(h) << 16);
}
__device__ inline unsigned short to_bf16(float x) {
  return __builtin_bit_cast(unsigned short, static_cast<__bf16>(x));
}

// Arrays are read and written through buffer resources, whose base is the same in every lane: values past
// the end read as zero and are not written (each 32-bit word of an access by itself), and no branch keeps
// the compiler from having many loads in flight.  Offsets `at` count elements; kNowhere is past every end.
// WIDE: the values of 2 bytes and 1 byte lie in whole words.  WIDE accesses are streamed; others share memory
// lines with their neighbours' and are cached on the way in (odd-sized layers, 8 bits, 119 us with every load
// streamed, 115 so).
constexpr uint32_t kNowhere = 0x20000000u;
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

__device__ inline Rsrc span(const void* base, uint32_t bytes) { return tile_rsrc(static_cast<const float*>(base), bytes); }

template <bool WIDE>
__device__ inline void ld4(Rsrc r, uint32_t at, float (&x)[4]) {
  const float4 v = WIDE ? bld4_nt(r, 4 * at) : bld4(r, 4 * at);
  x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
}
__device__ inline void st4(Rsrc r, uint32_t at, const float (&x)[4]) {
  bst4_nt(r, 4 * at, make_float4(x[0], x[1], x[2], x[3]));
}
// Ragged rows (not WIDE): a lane that has all four takes them at once, at whatever address; where the length
// is no multiple of four one lane has fewer, and takes them one by one (odd-sized layers, 8 bits, 109 us;
// every value by itself 129).
__device__ inline bool whole(uint32_t at, int len) { return static_cast<int>(at) + 4 <= len; }

template <bool WIDE>
__device__ inline void ld4_bf16(Rsrc r, uint32_t at, int len, float (&x)[4]) {
  const u2 v = __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(
      r, WIDE ? 2 * at : whole(at, len) ? 2 * at : kOut, 0, WIDE ? kAuxNT : 0));
  x[0] = __builtin_bit_cast(float, v[0] << 16);
  x[1] = __builtin_bit_cast(float, v[0] & 0xFFFF0000u);
  x[2] = __builtin_bit_cast(float, v[1] << 16);
  x[3] = __builtin_bit_cast(float, v[1] & 0xFFFF0000u);
  if (!WIDE && (len & 3) != 0) {
#pragma unroll
    for (uint32_t i = 0; i < 3; ++i) {
      const float y = bf16_value(static_cast<unsigned short>(
          __builtin_amdgcn_raw_buffer_load_b16(r, whole(at, len) ? kOut : 2 * (at + i), 0, 0)));
      x[i] = whole(at, len) ? x[i] : y;
    }
  }
}
template <bool WIDE>
__device__ inline void st4_bf16(Rsrc r, uint32_t at, int len, const float (&x)[4]) {
  const u2 v = {to_bf16(x[0]) | static_cast<uint32_t>(to_bf16(x[1])) << 16,
                to_bf16(x[2]) | static_cast<uint32_t>(to_bf16(x[3])) << 16};
  __builtin_amdgcn_raw_buffer_store_b64(v, r, WIDE ? 2 * at : whole(at, len) ? 2 * at : kOut, 0, kAuxNT);
  if (!WIDE && (len & 3) != 0) {
#pragma unroll
    for (uint32_t i = 0; i < 3; ++i)
      __builtin_amdgcn_raw_buffer_store_b16(to_bf16(x[i]), r, whole(at, len) ? kOut : 2 * (at + i), 0, 0);
  }
}
// four bytes
template <bool WIDE>
__device__ inline uint32_t ld4_bytes(Rsrc r, uint32_t at, int len) {
  uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(r, WIDE ? at : whole(at, len) ? at : kOut, 0, WIDE ? kAuxNT : 0);
  if (!WIDE && (len & 3) != 0) {
#pragma unroll
    for (uint32_t i = 0; i < 3; ++i)
      v |= static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b8(r, whole(at, len) ? kOut : at + i, 0, 0)) << (8 * i);
  }
  return v;
}
template <bool WIDE>
__device__ inline void st4_bytes(Rsrc r, uint32_t at, int len, uint32_t v) {
  __builtin_amdgcn_raw_buffer_store_b32(v, r, WIDE ? at : whole(at, len) ? at : kOut, 0, kAuxNT);
  if (!WIDE && (len & 3) != 0) {
#pragma unroll
    for (uint32_t i = 0; i < 3; ++i)
      __builtin_amdgcn_raw_buffer_store_b8(static_cast<unsigned char>(v >> (8 * i)), r, whole(at, len) ? kOut : at + i, 0, 0);
  }
}
// elements at .. of the `len` of a gradient from e on
template <bool WIDE>
__device__ inline void ld4_grad(const AwGrad& g, int64_t e, int len, uint32_t at, float (&x)[4]) {
  if (g.bf16)
    ld4_bf16<WIDE>(span(static_cast<const unsigned short*>(g.g) + e, 2u * len), at, len, x);
  else
    ld4<WIDE>(span(static_cast<const float*>(g.g) + e, 4u * len), at, x);
}

// A table entry that the whole wave reads, in scalar registers: where a kernel's branches read different
// entries the compiler no longer sees by itself that it is the same in every lane, and would loop over the
// lanes at every access through a resource made from it.
template <class E>
__device__ inline E same(const E& x) {
  static_assert(sizeof(E) % 4 == 0, "whole words");
  struct Words {
    int w[sizeof(E) / 4];
  };
  Words w = __builtin_bit_cast(Words, x);
#pragma unroll
  for (size_t i = 0; i < sizeof(E) / 4; ++i) w.w[i] = __builtin_amdgcn_readfirstlane(w.w[i]);
  return __builtin_bit_cast(E, w);
}

// ---- one lane's four elements ------------------------------------------------------------------

struct Coef {
  float c, decay;
};
// the gradients' factor; false if the norm was not finite, when nothing is to be updated
__device__ inline bool grad_factor(const AwArgs& a, float& c) {
  c = a.scale;
  if (!a.clip) return true;
  const float k = a.clip[1];
  c = k * a.scale;
  return k == k;
}

// sqrt(x) correctly rounded for x >= 2^-100: the instruction's result (1 ulp), or the neighbour beside
// which the residual x - s s' says the root lies.  Below, where fp32 does not hold all residuals, within 2 ulp;
// subnormal x the instruction takes for 0.  0, infinity and NaN fail both tests and stay.
__device__ inline float root(float x) {
  const float s = __builtin_amdgcn_sqrtf(x);
  const float lo = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) - 1u);
  const float hi = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, s) + 1u);
  const float below = __builtin_fmaf(-lo, s, x), above = __builtin_fmaf(-hi, s, x);
  return above > 0.f ? hi : below <= 0.f ? lo : s;
}

// m, v and p of a lane's four elements updated in place; r: sqrt(v').  What goes into the moments is rounded
// operation by operation, as anyone would write it: 8-bit moments turn a difference in the last bit into one of a
// whole code now and then, which another program's replay of the step would see (fused and with the bare
// instruction for the root: BERT-large rank 32 937 us, so 944).  p's quotient is m' times the hardware's
// reciprocal (1 ulp; eps > 0 keeps the denominator a normal number, and an infinite one gives 0).
// Subnormal v' are scaled for their roots, in waves that have any (8 bits, BERT-base 341 us without, 347 so;
// BERT-large rank 64 1016 and 1035, 256 2548 and 2536, others within 1 %; with every element scaled or not by a
// select rank 4 744 and 760, rank 256 3093).  They are found by the least of the bits less one, where 0 counts as
// large: a class test of each value took more scalar registers (rank 256 2805 us).
__device__ inline void update4(const AwArgs& a, const Coef& k, const float (&g)[4], float (&p)[4], float (&m)[4],
                               float (&v)[4], float (&r)[4]) {
  uint32_t least = ~0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float c = g[i] * k.c;
    m[i] = m[i] * a.b1 + c * a.c1;
    v[i] = v[i] * a.b2 + (c * c) * a.c2;
    r[i] = root(v[i]);
    const uint32_t b = __builtin_bit_cast(uint32_t, v[i]) - 1u;
    least = b < least ? b : least;
  }
  if (__builtin_expect(__any(least < 0x007FFFFFu), 0)) {  // (2^-126)
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = v[i] < 0x1p-126f ? __builtin_amdgcn_sqrtf(v[i] * 0x1p64f) * 0x1p-32f : r[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float den = __builtin_fmaf(r[i], a.rs, a.eps);
    p[i] = __builtin_fmaf(-(m[i] * __builtin_amdgcn_rcpf(den)), a.lr, p[i] * k.decay);
  }
}

// ---- 8-bit moments -----------------------------------------------------------------------------

// The 32-bit finaliser of MurmurHash3 (A. Appleby, public domain).
__device__ inline uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x85EBCA6Bu;
  x ^= x >> 13;
  x *= 0xC2B2AE35u;
  return x ^ (x >> 16);
}
__device__ inline uint32_t tensor_key(uint32_t key, int tensor) {
  return mix32(key + static_cast<uint32_t>(tensor) * 0x9E3779B1u);
}
// 32 random bits of element e, x = key + e * kElementStep (elements 2^32 apart share theirs).  Shifts and
// multiplier are those of the first of two rounds of a published integer hash; one round, for its price (of 56
// vector instructions an element 11 are the rounding's).  What it has to do is to leave the mean of the rounding's
// errors at zero, over elements and over steps.
constexpr uint32_t kElementStep = 0x9E3779B1u;
__device__ inline uint32_t random_bits(uint32_t x) {
  x ^= x >> 15;
  x *= 0x2C1B3C6Du;
  return x ^ (x >> 12);
}

// The largest of the wave's values, in every lane: rows of 16 lanes by butterflies, then from row to row.
template <int CTRL, int ROWS>
__device__ inline uint32_t max_step(uint32_t v) {
  const uint32_t x = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false));
  return x > v ? x : v;
}
__device__ inline uint32_t wave_max(uint32_t v) {
  v = max_step<0xB1, 0xF>(v);   // quad_perm [1,0,3,2]
  v = max_step<0x4E, 0xF>(v);   // quad_perm [2,3,0,1]
  v = max_step<0x141, 0xF>(v);  // row_half_mirror
  v = max_step<0x140, 0xF>(v);  // row_mirror
  v = max_step<0x142, 0xA>(v);  // rows 1 and 3 take lane 15 of the row before
  v = max_step<0x143, 0xC>(v);  // rows 2 and 3 take lane 31
  return __builtin_amdgcn_readlane(v, 63);
}

// The scales of a block's m and sqrt(v) and their inverses, from the bits of the block's largest magnitudes
// (which order like the values, NaN above infinity): formed once, in even lanes for m and in odd ones for
// sqrt(v).  A block that holds a value that is not finite, or above 2^126 where the reciprocal leaves the
// normal numbers, becomes NaN as a whole: a scale from its other values would hide it.  One below 2^-100
// becomes zero: its inverse would overflow, and such moments are nothing beside any eps.  The quotient
// is the reciprocal's, corrected by its residual.
struct Scales {
  float scale;          // of the lane's kind
  float inv_m, inv_r;
  uint32_t live_m, live_r;  // masks of the codes: none of a NaN block
};
constexpr uint32_t kDead = 0x7E800000u;  // bits of 2^126
__device__ inline Scales block_scales(uint32_t top_m, uint32_t top_r) {
  const uint32_t bits = (tid() & 1) ? top_r : top_m;
  const float top = __builtin_bit_cast(float, bits);
  const bool dead = bits > kDead, none = dead || bits < 0x0D800000u;  // 2^-100
  const float rcp = __builtin_amdgcn_rcpf(top), q = 448.f * rcp;
  const float inv = none ? 0.f : __builtin_fmaf(__builtin_fmaf(-top, q, 448.f), rcp, q);
  Scales s;
  s.scale = dead ? __builtin_bit_cast(float, 0x7FC00000u) : none ? 0.f : top * (1.f / 448.f);
  const int bi = __builtin_bit_cast(int, inv);
  s.inv_m = __builtin_bit_cast(float, __builtin_amdgcn_readlane(bi, 0));
  s.inv_r = __builtin_bit_cast(float, __builtin_amdgcn_readlane(bi, 1));
  s.live_m = top_m > kDead ? 0u : ~0u;
  s.live_r = top_r > kDead ? 0u : ~0u;
  return s;
}

// A magnitude's largest over a lane's four values, NaN if one is.
__device__ inline uint32_t top4(const float (&x)[4]) {
  const float t = __builtin_elementwise_maximum(
      __builtin_elementwise_maximum(fabsf(x[0]), fabsf(x[1])), __builtin_elementwise_maximum(fabsf(x[2]), fabsf(x[3])));
  return __builtin_bit_cast(uint32_t, t) & 0x7FFFFFFFu;
}

// y, at most 448 in magnitude, as an e4m3 code in byte I of `codes`, rounded up in magnitude with the
// probability of the fraction dropped: the instruction adds its random operand, of which 16 bits are
// given, below the last bit kept.  Rounding to nearest would lose every change of less than half a
// step, 3 % and more, of a moment that moves by 0.1 % a step.
template <int I>
__device__ inline uint32_t put_code(uint32_t codes, float y, uint32_t random) {
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_sr_fp8_f32(y, static_cast<int>(random), static_cast<int>(codes), I));
}

// The codes of a lane's element I, m and sqrt(v) over their scales; e0: the hash's input for element 0.
// sqrt(v) > 0 stays so (the smallest code is 2^-9): a zero beside a moment m that is none would make a
// step of m / eps.
template <int I>
__device__ inline void put_pair(uint32_t& cm, uint32_t& cr, float m, float r, uint32_t e0) {
  const uint32_t random = random_bits(e0 + I * kElementStep);
  cm = put_code<I>(cm, __builtin_amdgcn_fmed3f(m, -448.f, 448.f), random & 0xFFFF0000u);
  cr = put_code<I>(cr, __builtin_amdgcn_fmed3f(r, fminf(r * 0x1p100f, 0x1p-9f), 448.f), random << 16);
}

// the values of four codes
__device__ inline void values_of(uint32_t codes, float (&x)[4]) {
  const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), false);
  const f2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

// What a lane reads of its four elements besides the gradient.
template <int BITS>
struct Lane;
template <>
struct Lane<32> {
  float p[4], m[4], v[4];
};
template <>
struct Lane<8> {
  float p[4], ms, vs;
  uint32_t m, v;
};

// The arrays of a step from element e of a tensor on, `len` elements of them, and the scales of `blocks`
// blocks from blk on.
struct Streams {
  Rsrc p, copy, m, v, ms, vs;
};
template <int BITS>
__device__ inline Streams streams(const AwArgs& a, const AwTensor& t, int64_t e, uint32_t len, int64_t blk, uint32_t blocks) {
  Streams s;
  s.p = span(t.p + e, 4 * len);
  s.copy = span(t.copy + e, t.copy ? 2 * len : 0);
  s.m = span(a.m + (t.off + e) * (BITS / 8), BITS / 8 * len);
  s.v = span(a.v + (t.off + e) * (BITS / 8), BITS / 8 * len);
  if constexpr (BITS == 8) {
    s.ms = span(a.ms + t.blk + blk, 4 * blocks);
    s.vs = span(a.vs + t.blk + blk, 4 * blocks);
  }
  return s;
}

template <int BITS, bool WIDE>
__device__ inline void load_lane(const Streams& s, uint32_t at, int len, uint32_t blk, Lane<BITS>& x) {
  ld4<WIDE>(s.p, at, x.p);
  if constexpr (BITS == 32) {
    ld4<WIDE>(s.m, at, x.m);
    ld4<WIDE>(s.v, at, x.v);
  } else {
    x.m = ld4_bytes<WIDE>(s.m, at, len);
    x.v = ld4_bytes<WIDE>(s.v, at, len);
    x.ms = bld1(s.ms, 4 * blk);
    x.vs = bld1(s.vs, 4 * blk);
  }
}

// The step of a wave's elements (`len` of them, not WIDE); with 8 bits they are block blk of the streams.  e0:
// the hash's input for the lane's first element.
template <int BITS, bool WIDE>
__device__ inline void step_lane(const AwArgs& a, const AwTensor& t, const Coef& k, uint32_t e0, const Streams& s,
                                 uint32_t at, int len, uint32_t blk, Lane<BITS>& x, const float (&g)[4]) {
  if constexpr (BITS == 32) {
    float r[4];
    update4(a, k, g, x.p, x.m, x.v, r);
    st4(s.p, at, x.p);
    st4(s.m, at, x.m);
    st4(s.v, at, x.v);
  } else {
    float m[4], v[4], r[4];
    values_of(x.m, m);
    values_of(x.v, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = m[i] * x.ms;
      r[i] = r[i] * x.vs;
      v[i] = r[i] * r[i];
    }
    update4(a, k, g, x.p, m, v, r);
    // elements past the end have zeros, or NaN beside a dead block's others
    const Scales sc = block_scales(wave_max(top4(m)), wave_max(top4(r)));
    uint32_t cm = 0, cr = 0;
    put_pair<0>(cm, cr, m[0] * sc.inv_m, r[0] * sc.inv_r, e0);
    put_pair<1>(cm, cr, m[1] * sc.inv_m, r[1] * sc.inv_r, e0);
    put_pair<2>(cm, cr, m[2] * sc.inv_m, r[2] * sc.inv_r, e0);
    put_pair<3>(cm, cr, m[3] * sc.inv_m, r[3] * sc.inv_r, e0);
    st4(s.p, at, x.p);
    st4_bytes<WIDE>(s.m, at, len, cm & sc.live_m);
    st4_bytes<WIDE>(s.v, at, len, cr & sc.live_r);
    const uint32_t lane = tid() & 63;
    bst1(s.ms, lane == 0 ? 4 * blk : kOut, sc.scale);
    bst1(s.vs, lane == 1 ? 4 * blk : kOut, sc.scale);
  }
  if (t.copy) st4_bf16<WIDE>(s.copy, at, len, x.p);
}

// First element, length and index of block j of a dense tile.
__device__ inline void block_at(const AwTensor& t, const AwTile& tile, int j, int64_t& first, int& len, int64_t& blk) {
  int64_t left;
  if (t.slack == 0) {  // blocks follow each other
    blk = tile.first + j;
    first = blk * t.w;
    left = t.n * t.m - first;
  } else {
    int64_t row = tile.first & kAwRowMask, seg = (tile.first >> kAwSegShift) + j;
    while (seg >= t.nb) seg -= t.nb, ++row;
    blk = row * t.nb + seg;
    first = row * t.m + seg * t.w;
    left = t.m - seg * t.w;
  }
  len = left < t.w ? static_cast<int>(left) : t.w;
}

// ---- step on gradients given as values ---------------------------------------------------------

// Dense tiles are shared by waves: kAwPart elements or kAwPartBlocks blocks each, whose loads are all made
// before the first is updated (8 bits, BERT-large: two blocks 863 us, one 904).
//
// Where all rows are whole words (WIDE) a workgroup is one wave, and LDS that is asked for and not used
// keeps the CU to 16 waves: with more in flight per workgroup and CU the reads and writes of seven streams
// get in each other's way in HBM.  BERT-large, 32 bits: workgroups of 256 threads and 1024 elements
// 1627 us, with 16 waves a CU 1539; of one wave and 256 elements 1506 and 1435.
// Else neighbouring blocks share memory lines, which are best written from one CU: workgroups of four
// waves, at full occupancy (odd-sized layers, 8 bits: one wave a workgroup 142 us, four 118).
//
// Bound by HBM: BERT-large (334 M elements), 32 bits, 28 bytes an element, 1440 us, 6.5 TB/s; 8 bits, 16.1
// bytes, 853 us, 6.3 TB/s with the vector units 60 % busy; odd-sized layers, 8 bits, 110 us, 5.2 TB/s.
constexpr int kDenseLds = 10240;
template <bool WIDE>
constexpr int dense_threads() { return WIDE ? 64 : kAwBlock; }
template <int BITS, bool WIDE>
constexpr int dense_part() { return BITS == 32 ? kAwPart : WIDE ? kAwPartBlocks : 1; }

// Workgroups of `waves` waves that share a tile.
template <int BITS, bool WIDE>
constexpr int dense_groups(int waves) { return (BITS == 32 ? kAwTile : kAwTileBlocks) / dense_part<BITS, WIDE>() / waves; }

// Part `part` of a dense tile, by one wave.
template <int BITS, bool WIDE>
__device__ inline void dense_wave(const AwArgs& a, const AwTile& tile, int part, float c) {
  constexpr int per = dense_part<BITS, WIDE>();
  const int o = 4 * (tid() & 63), first = part * per;
  if (first >= tile.count) return;
  const AwTensor t = same(a.tensors[tile.tensor]);
  const AwGrad gr = same(a.grads[tile.tensor]);
  const Coef k{c, t.decay ? a.decay : 1.f};
  if constexpr (BITS == 32) {
    const int64_t e = tile.first + first;
    const int len = tile.count - first < per ? tile.count - first : per;
    const Streams str = streams<32>(a, t, e, len, 0, 0);
    Lane<32> x;
    float g[4];
    load_lane<32, WIDE>(str, o, len, 0, x);
    ld4_grad<WIDE>(gr, e, len, o, g);
    step_lane<32, WIDE>(a, t, k, 0, str, o, len, 0, x, g);
  } else {
    const uint32_t key = tensor_key(a.key, tile.tensor) + o * kElementStep;
    Lane<8> x[per];
    float g[per][4];
    int64_t e[per], blk[per];
    int len[per];
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const bool in = first + i < tile.count;
      block_at(t, tile, in ? first + i : first, e[i], len[i], blk[i]);
      if (!in) len[i] = 0;
      load_lane<8, WIDE>(streams<8>(a, t, e[i], len[i], blk[i], in), o, len[i], 0, x[i]);
      ld4_grad<WIDE>(gr, e[i], len[i], o, g[i]);
    }
#pragma unroll
    for (int i = 0; i < per; ++i)
      step_lane<8, WIDE>(a, t, k, key + static_cast<uint32_t>(e[i]) * kElementStep,
                         streams<8>(a, t, e[i], len[i], blk[i], len[i] > 0), o, len[i], 0, x[i], g[i]);
  }
}

template <int BITS, bool WIDE>
__global__ __launch_bounds__(dense_threads<WIDE>()) void k_adamw(AwArgs a) {
  float c;
  if (!grad_factor(a, c)) return;
  constexpr int waves = dense_threads<WIDE>() / 64, groups = dense_groups<BITS, WIDE>(waves);
  const int wave = waves > 1 ? __builtin_amdgcn_readfirstlane(tid() >> 6) : 0;
  dense_wave<BITS, WIDE>(a, a.tiles[blockIdx.x / groups], blockIdx.x % groups * waves + wave, c);
}

// ---- step on gradients given as factors --------------------------------------------------------

constexpr int product_group(int kc) { return aw_product_waves(16 * kc); }

// The operands of a product for 16 rows of A or B, 16 KC values of the inner dimension, row l of a factor's
// rows in `r` from value `row` on: lane 16 q + l has the values 4 q .. 4 q + 3 of each 16, or below rank 16 the
// values 4 s + q, so that whole steps of four can be left out; at rank 16 the values 2 q, 2 q + 1 of each 8.
// Values from `rank` on, and of rows past the end, are zero.  Any order of the sum would do for its error bound; with
// these, sums over ranks up to 16 and of 32 came out bit for bit as those of the BLAS library that this was
// measured beside, which says nothing of another version of it.
template <int KC>
__device__ inline void load_operand(f4 (&x)[KC], Rsrc r, uint32_t row, int q, int rank) {
  if (KC == 1 && rank == 16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f2 v = __builtin_bit_cast(f2, __builtin_amdgcn_raw_buffer_load_b64(r, 4 * (row + 2 * q) + 32 * h, 0, 0));
      x[0][2 * h] = v[0];
      x[0][2 * h + 1] = v[1];
    }
    return;
  }
  if (rank == 16 * KC) {
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const float4 v = bld4(r, 4 * (row + 4 * q) + 64 * k);
      x[k] = f4{v.x, v.y, v.z, v.w};
    }
    return;
  }
  // made anew at every call: the compiler would keep the lanes' conditions of all k beside the loop
  int in = KC == 1 && rank < 16 ? rank - q : rank - 4 * q;
  asm volatile("" : "+v"(in));
  if (KC == 1 && rank < 16) {
#pragma unroll
    for (int s = 0; s < 4; ++s) x[0][s] = bld1(r, 4 * s < in ? 4 * (row + 4 * s + q) : kOut);
  } else if ((rank & 3) == 0) {
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const float4 v = bld4(r, 16 * k < in ? 4 * (row + 16 * k + 4 * q) : kOut);
      x[k] = f4{v.x, v.y, v.z, v.w};
    }
  } else {
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[k][i] = bld1(r, 16 * k + i < in ? 4 * (row + 16 * k + 4 * q + i) : kOut);
  }
}
// D of a lane: columns 4 q .. 4 q + 3 of row l (B's rows are the first operand)
template <int KC, int J>
__device__ inline void multiply(f4 (&acc)[J], const f4 (&a)[KC], const f4 (&b)[J][KC], int steps) {
#pragma unroll
  for (int k = 0; k < KC; ++k)
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (KC > 1 || s < steps)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j][k][s], a[k][s], acc[j], 0, 0, 0);
}

// A tile of rows of one block column of G = A B^T.  A wave keeps B's part for its 64 columns in registers
// and forms 16 rows at a time, which go through LDS from the matrix cores' order (four neighbouring
// columns of row `lane % 16` in a lane) to whole rows, four columns a lane, as the step reads and writes.
// The product of the next 16 rows runs beside the step of these, and the next row's state is requested as
// soon as a row is done.
//
// BERT-large: 32 bits, rank 4, 24 bytes an element, 1277 us, 6.3 TB/s: HBM.  8 bits, 12.1 bytes: rank 4 718 us
// (5.6 TB/s), rank 32 814 and with a bfloat16 copy 870 us (5.4 TB/s): the vector units (74 % busy), which share
// their SIMD with the matrix cores' turns and the barriers.  Rank 64 1012 us, 128 1362 us, 256 2530 us: the
// fp32 matrix cores (for which alone 272, 544 and 1088 us are needed) and the few waves that B's registers
// leave.  With 32 bits a tile has one group of 16 rows, whose product nothing runs beside: rank 64 1555 us, 128
// 2228, 256 4895.  A whole step from the compress call on, 8 bits, with M_hat written and without: rank 4 1739 and
// 1397 us, rank 32 1909 and 1610, rank 64 2171 and 2083, rank 128 3085 and 3250, rank 256 5834 and 7034.
template <int BITS, int KC, bool WIDE>
__device__ inline void product_rows(const AwArgs& a, const AwTensor& t, const AwTile& tile, const Coef& k,
                                    const AwGrad& gr, float (*lds)[kAwRows * kLdsPitch]) {
  constexpr int W = product_group(KC), N = kAwRows / W, J = 16 / W;  // rows and 16-column blocks of a wave
  const int wave = __builtin_amdgcn_readfirstlane(tid() >> 6), lane = tid() & 63;
  const int l16 = lane & 15, q = lane >> 4, o = 4 * lane;
  const int64_t row0 = tile.first & kAwRowMask, col0 = (tile.first >> kAwSegShift) * t.w;
  const int m = static_cast<int>(t.m), nb = t.nb;
  const int cols = m - col0 < t.w ? static_cast<int>(m - col0) : t.w;
  const int left = static_cast<int>(t.n - row0), stride = tile.count;  // rows from row0 on; from 16 to the next
  const int rank = gr.rank, steps = (rank + 3) / 4;
  f4 bf[J][KC], af[KC], acc[J];
  const Rsrc brows = span(gr.b + col0 * rank, 4u * cols * rank);
#pragma unroll
  for (int j = 0; j < J; ++j) load_operand<KC>(bf[j], brows, (16 * (J * wave + j) + l16) * rank, q, rank);
  auto load_a = [&](int r0) {
    const int rows = left - r0 < 16 ? (left - r0 > 0 ? left - r0 : 0) : 16;
    load_operand<KC>(af, span(gr.a + (row0 + r0) * rank, 4u * rows * rank), l16 * rank, q, rank);
  };
  auto to_lds = [&](float* to) {
#pragma unroll
    for (int j = 0; j < J; ++j) *reinterpret_cast<f4*>(&to[l16 * kLdsPitch + 16 * (J * wave + j) + 4 * q]) = acc[j];
  };
  auto zero = [&] {
#pragma unroll
    for (int j = 0; j < J; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};
  };
  // The arrays of 16 rows from r0 on (WIDE), or of one row, whose end may lie inside a lane's four.
  auto rows_from = [&](int r0, int most) {
    const int rows = left - r0 < most ? left - r0 : most;
    const int64_t r = row0 + r0;
    return streams<BITS>(a, t, r * m + col0, rows > 0 ? (rows - 1) * m + cols : 0, r * nb + (tile.first >> kAwSegShift),
                         rows > 0 ? (rows - 1) * nb + 1 : 0);
  };
  const uint32_t lane_at = !WIDE || o < cols ? o : kNowhere;
  Lane<BITS> x[N];
  auto request = [&](int i, const Streams& s, int r0) {
    const int r = N * wave + i;
    if constexpr (WIDE)
      load_lane<BITS, true>(s, lane_at + r * m, 0, r * nb, x[i]);
    else
      load_lane<BITS, false>(rows_from(r0 + r, 1), o, r0 + r < left ? cols : 0, 0, x[i]);
  };
  Streams cur = rows_from(0, 16);
  load_a(0);
#pragma unroll
  for (int i = 0; i < N; ++i) request(i, cur, 0);
  zero();
  multiply<KC, J>(acc, af, bf, steps);
  to_lds(lds[0]);
  load_a(stride);
  __syncthreads();
  const uint32_t key = BITS == 8 ? tensor_key(a.key, tile.tensor) + o * kElementStep : 0;
  for (int r0 = 0, at = 0; r0 < left; r0 += stride, at ^= 1) {
    if (r0 + stride < left) {
      zero();
      multiply<KC, J>(acc, af, bf, steps);
      load_a(r0 + 2 * stride);
    }
    const Streams next = rows_from(r0 + stride, 16);
    const uint32_t e0 = key + static_cast<uint32_t>((row0 + r0) * m + col0) * kElementStep;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = N * wave + i;
      const f4 v = *reinterpret_cast<const f4*>(&lds[at][r * kLdsPitch + o]);
      float g[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) g[h] = o + h < cols ? v[h] : 0.f;
      const uint32_t e = e0 + static_cast<uint32_t>(r) * static_cast<uint32_t>(m) * kElementStep;
      if constexpr (WIDE)
        step_lane<BITS, true>(a, t, k, e, cur, lane_at + r * m, 0, r * nb, x[i], g);
      else
        step_lane<BITS, false>(a, t, k, e, rows_from(r0 + r, 1), o, r0 + r < left ? cols : 0, 0, x[i], g);
      request(i, next, r0 + stride);
    }
    cur = next;
    if (r0 + stride < left) to_lds(lds[at ^ 1]);
    __syncthreads();
  }
}

// Logical workgroup: eight neighbours go to one XCD (workgroups go round the eight in turn), since
// neighbouring tiles read the same rows of A and share memory lines.
__device__ inline uint32_t near_block(uint32_t b) {
  return (b & ~63u) | (b & 7u) << 3 | (b >> 3 & 7u);
}

// Waves per SIMD: what the registers allow that hold B's part, 16 KC of them (rank 32, 8 bits: four waves,
// with spills, 962 us, three 925).
constexpr int product_waves(int kc) { return kc == 1 ? 4 : kc == 2 ? 3 : 2; }
// 32-bit moments: LDS asked for and not used keeps a CU to three workgroups, for HBM's sake as in the
// dense step (BERT-large rank 4 1392 us with four, 1387 with three, 1424 with two).
constexpr int kProductLds = 20000;

// A tile of narrower rows: whole blocks, of several rows each.
template <int BITS, int W>
__device__ inline void narrow_tile(const AwArgs& a, const AwTile& tile, float c, float* lds) {
  const AwTensor t = same(a.tensors[tile.tensor]);
  const AwGrad gr = same(a.grads[tile.tensor]);
  const Coef k{c, t.decay ? a.decay : 1.f};
  const int wave = __builtin_amdgcn_readfirstlane(tid() >> 6), lane = tid() & 63;
  const int l16 = lane & 15, q = lane >> 4;
  const int64_t row0 = tile.first;
  const int cols = static_cast<int>(t.m), rank = gr.rank;
  const Rsrc arows = span(gr.a + row0 * rank, 4u * tile.count * rank), brows = span(gr.b, 4u * cols * rank);
  for (int rb = 0; rb < tile.count; rb += 16) {
    for (int cb = 16 * wave; cb < cols; cb += 16 * W) {
      f4 acc = {0.f, 0.f, 0.f, 0.f};
      for (int k0 = 0; k0 < rank; k0 += 16) {
        f4 x, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (load_operand's orders)
          const int kk = k0 + (rank < 16 ? 4 * i + q : rank == 16 ? 8 * (i >> 1) + 2 * q + (i & 1) : 4 * q + i);
          x[i] = bld1(brows, kk < rank ? 4u * ((cb + l16) * rank + kk) : kOut);
          y[i] = bld1(arows, kk < rank ? 4u * ((rb + l16) * rank + kk) : kOut);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], acc, 0, 0, 0);
      }
      if (rb + l16 < tile.count) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (cb + 4 * q + i < cols) lds[(rb + l16) * cols + cb + 4 * q + i] = acc[i];
      }
    }
  }
  __syncthreads();
  const uint32_t o = 4 * lane;
  const uint32_t key = BITS == 8 ? tensor_key(a.key, tile.tensor) + o * kElementStep : 0;
  for (int j = wave; j * t.k < tile.count; j += W) {
    const int rows = tile.count - j * t.k < t.k ? tile.count - j * t.k : t.k;
    const int len = rows * cols;
    const int64_t e = (row0 + int64_t(j) * t.k) * t.m;
    const Streams s = streams<BITS>(a, t, e, len, row0 / t.k + j, 1);
    Lane<BITS> x;
    float g[4];
    load_lane<BITS, false>(s, o, len, 0, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = static_cast<int>(o) + i < len ? lds[j * t.k * cols + o + i] : 0.f;
    step_lane<BITS, false>(a, t, k, key + static_cast<uint32_t>(e) * kElementStep, s, o, len, 0, x, g);
  }
}

// Rows of 256 columns or more, ranks up to 16 KC; before them the slot's narrow and joined dense tiles.
template <int BITS, int KC, bool WIDE>
__global__ __launch_bounds__(64 * product_group(KC), product_waves(KC)) void k_adamw_product(AwArgs a) {
  __shared__ __align__(16) float lds[2][kAwRows * kLdsPitch];
  constexpr int W = product_group(KC);
  float c;
  if (!grad_factor(a, c)) return;
  if (blockIdx.x < a.others) {
    const uint32_t b = blockIdx.x;
    if (b < a.narrow) {
      narrow_tile<BITS, W>(a, same(a.tiles[a.count + b]), c, lds[0]);
    } else {
      constexpr int groups = dense_groups<BITS, false>(W);
      const uint32_t d = b - a.narrow;
      if (d >= a.joined * groups) return;
      dense_wave<BITS, false>(a, same(a.tiles[a.count + a.narrow + d / groups]),
                              d % groups * W + __builtin_amdgcn_readfirstlane(tid() >> 6), c);
    }
    return;
  }
  const uint32_t b = near_block(blockIdx.x - a.others);
  if (b >= a.count) return;
  const AwTile tile = same(a.tiles[b]);
  const AwTensor t = same(a.tensors[tile.tensor]);
  const AwGrad gr = same(a.grads[tile.tensor]);
  const Coef k{c, t.decay ? a.decay : 1.f};
  product_rows<BITS, KC, WIDE>(a, t, tile, k, gr, lds);
}

// Narrow tiles of a slot that has no others.
template <int BITS>
__global__ __launch_bounds__(kAwBlock) void k_adamw_narrow(AwArgs a) {
  __shared__ __align__(16) float lds[kAwRows * kAwScaleBlock];
  float c;
  if (!grad_factor(a, c)) return;
  narrow_tile<BITS, kAwBlock / 64>(a, a.tiles[blockIdx.x], c, lds);
}

// ---- norm --------------------------------------------------------------------------------------

// Sums over the workgroup in a fixed order; thread 0 has the result.
__device__ inline double block_sum(double v) {
  __shared__ double part[16];
  v = wave_sum(v);
  const int wave = tid() >> 6;
  if ((tid() & 63) == 0) part[wave] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < static_cast<int>(blockDim.x >> 6); ++i) s += part[i];
  return s;
}

// Squares and their sums are in 64 bits: no finite gradient overflows, and the result does not
// depend on how the tiles are cut beyond its last bits.  bfloat16 values' squares are exact in fp32
// where they are normal numbers there; two of them are added in fp32 (2^-24 of their sum at most, 2^-25 of the norm)
// before they go on in 64 bits, unless the wave has values too large or small for that (BERT-large, eight bytes
// a load: 133 us with every square in 64 bits, 121 so). A lane loads 16 bytes of either type: bfloat16 103 us
// (6.5 TB/s), 121 with eight; fp32 197 us (6.8 TB/s). HBM bounds both.
__device__ inline void norm_tile(const AwNormArgs& a, const AwTile& tile, double* out) {
  const AwGrad gr = a.grads[tile.tensor];
  double s = 0.0;
  if (gr.bf16) {
    const unsigned short* src = static_cast<const unsigned short*>(gr.g) + tile.first;
    const bool pairs = (reinterpret_cast<uintptr_t>(src) & 3) == 0 && (tile.count & 1) == 0;  // whole words
    const Rsrc r = span(src, 2u * tile.count);
    for (int o = 8 * tid(); o < tile.count; o += 8 * kAwBlock * kNormLoads) {
      v4u g[kNormLoads];
#pragma unroll
      for (int u = 0; u < kNormLoads; ++u) {
        const uint32_t at = o + 8 * kAwBlock * u;
        if (pairs) {
          g[u] = __builtin_amdgcn_raw_buffer_load_b128(r, 2 * at, 0, kAuxNT);
        } else {
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i)
            g[u][i] = static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(r, 2 * (at + 2 * i), 0, 0)) |
                      static_cast<uint32_t>(__builtin_amdgcn_raw_buffer_load_b16(r, 2 * (at + 2 * i + 1), 0, 0)) << 16;
        }
      }
      float top = 0.f;
      auto low = [](uint32_t w) { return __builtin_bit_cast(float, w << 16); };
      auto high = [](uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); };
#pragma unroll
      for (int u = 0; u < kNormLoads; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(low(g[u][i])), fabsf(high(g[u][i]))));
      // (a smaller value's square is lost beside one of 2^-40 and more)
      if (__any(top >= 0x1p60f || (top < 0x1p-40f && top > 0.f))) {
#pragma unroll
        for (int u = 0; u < kNormLoads; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const double x = low(g[u][i]), y = high(g[u][i]);
            s = __builtin_fma(x, x, s);
            s = __builtin_fma(y, y, s);
          }
      } else {
#pragma unroll
        for (int u = 0; u < kNormLoads; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = low(g[u][i]), y = high(g[u][i]);
            s += __builtin_fmaf(x, x, y * y);
          }
      }
    }
  } else {
    const Rsrc r = span(static_cast<const float*>(gr.g) + tile.first, 4u * tile.count);
    for (int o = 4 * tid(); o < tile.count; o += 4 * kAwBlock * kNormLoads) {
      float g[kNormLoads][4];
#pragma unroll
      for (int u = 0; u < kNormLoads; ++u) ld4<true>(r, o + 4 * kAwBlock * u, g[u]);
#pragma unroll
      for (int u = 0; u < kNormLoads; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_fma(static_cast<double>(g[u][i]), static_cast<double>(g[u][i]), s);
    }
  }
  s = block_sum(s);
  if (tid() == 0) *out = s;
}

// |A B^T|^2 = sum of (A^T A) o (B^T B), so the norm of a factored gradient needs its factors' Gram
// matrices alone.  In 64 bits: where the factors' columns nearly cancel, so do the products.
// One wave forms a block of 16 T columns squared over one slice of rows on the fp64 matrix cores, 16 x 16
// tiles at a time, on the diagonal of the matrix those on and above the diagonal only.  A lane loads T
// neighbouring columns at once and gives one to each tile: the order of columns and rows does not matter, as
// long as A and B have the same.  Slices of 256 rows: longer ones leave CUs idle, shorter ones
// write more partial sums (rank 4: 36 us with 256 rows, 39 with 512, 41 with 128).
// BERT-large rank 64: 76 us of the norm's 92, a third of the fp64 matrix cores' peak: one wave per SIMD, for
// the registers of the blocks off the diagonal (368), which ranks above 64 have, in the same kernel.  Rank 256: 964 us
// in all.
template <int T>
__device__ inline void load_columns(float (&x)[T], Rsrc r, uint32_t at, int left) {
  if (left >= T) {
    if constexpr (T == 4) {
      const float4 v = bld4(r, at);
      x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else {
#pragma unroll
      for (int c = 0; c < T; ++c) x[c] = bld1(r, at + 4 * c);
    }
  } else {  // the last columns of a rank that 16 T does not divide
#pragma unroll
    for (int c = 0; c < T; ++c) x[c] = bld1(r, c < left ? at + 4 * c : kOut);
  }
}

template <int T, bool DIAG>
__device__ inline void gram_tile(const AwGrad& gr, const float* x, int rows, int bi, int bj, double* out) {
  constexpr int U = T == 4 ? 8 : 16 / T;  // steps of four rows loaded at a time
  const int r = gr.rank, l16 = tid() & 15, q = (tid() >> 4) & 3;
  // rows past the slice read as zero
  const Rsrc rs = tile_rsrc(x, 4u * rows * r);
  const int ci = 16 * T * bi + T * l16, cj = 16 * T * bj + T * l16;
  d4 acc[DIAG ? T * (T + 1) / 2 : T * T] = {};
  float fi[U][T], fj[U][T];
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t row = 4u * r * (k0 + 4 * u + q);
      load_columns<T>(fi[u], rs, row + 4 * ci, r - ci);
      if (!DIAG) load_columns<T>(fj[u], rs, row + 4 * cj, r - cj);
    }
  };
  load(0);
  for (int k0 = 0; k0 < rows; k0 += 4 * U) {
    double di[U][T], dj[U][T];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < T; ++c) {
        di[u][c] = fi[u][c];
        dj[u][c] = DIAG ? di[u][c] : fj[u][c];
      }
    load(k0 + 4 * U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = DIAG ? i : 0; j < T; ++j, ++n)
          acc[n] = __builtin_amdgcn_mfma_f64_16x16x4f64(di[u][i], dj[u][j], acc[n], 0, 0, 0);
    }
  }
  constexpr int N = DIAG ? T * (T + 1) / 2 : T * T;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) out[n * 256 + 64 * e + (tid() & 63)] = acc[n][e];
}

// The first workgroups each have a tile of the norm of values, the others four of Gram matrices.
template <int T>
__global__ __launch_bounds__(kAwBlock) void k_norm(AwNormArgs a) {
  if (static_cast<int64_t>(blockIdx.x) < a.norm) {
    norm_tile(a, a.tiles[blockIdx.x], a.sums + blockIdx.x);
    return;
  }
  if constexpr (T > 0) {
    const int wave = __builtin_amdgcn_readfirstlane(tid() >> 6);
    const int64_t i = 4 * (static_cast<int64_t>(blockIdx.x) - a.norm) + wave;
    if (i >= a.gram_tiles) return;
    const AwTile tile = a.tiles[a.norm + i];
    const AwGrad gr = a.grads[tile.tensor];
    const AwTensor t = a.tensors[tile.tensor];
    const int side = tile.count & 1, bi = (tile.count >> 1) & 127, bj = tile.count >> 8;
    const int per = aw_gram_rows(gr.rank);
    const int64_t row0 = tile.first * per, left = (side ? t.m : t.n) - row0;
    const int rows = static_cast<int>(left < per ? left : per);
    const float* x = (side ? gr.b : gr.a) + row0 * gr.rank;
    double* out = a.gram + gr.gram[side] + tile.first * aw_gram_entries(gr.rank, T) + aw_gram_at(gr.rank, T, bi, bj);
    // (a block of fewer columns holds the slot's whole matrices)
    if constexpr (T == 4) {
      if (bi != bj) {
        gram_tile<T, false>(gr, x, rows, bi, bj, out);
        return;
      }
    }
    gram_tile<T, true>(gr, x, rows, bi, bj, out);
  }
}

// One tile of both Gram matrices, summed over their slices (a quarter of them by each 256 threads) and
// multiplied; tiles off the diagonal count twice.
__global__ __launch_bounds__(1024) void k_trace(AwNormArgs a) {
  __shared__ double part[2][4][256];
  const AwTile tile = a.tiles[blockIdx.x];
  const AwGrad gr = a.grads[tile.tensor];
  const int64_t entries = aw_gram_entries(gr.rank, a.t);
  const int entry = tid() & 255, quarter = tid() >> 8;
  for (int side = 0; side < 2; ++side) {
    const double* x = a.gram + gr.gram[side] + tile.first + entry;
    double s = 0.0;
#pragma unroll 4
    for (int k = quarter; k < gr.slices[side]; k += 4) s += x[k * entries];
    part[side][quarter][entry] = s;
  }
  __syncthreads();
  double s = 0.0;
  if (quarter == 0) {
    double g[2];
    for (int side = 0; side < 2; ++side)
      g[side] = (part[side][0][entry] + part[side][1][entry]) + (part[side][2][entry] + part[side][3][entry]);
    s = g[0] * g[1] * tile.count;
  }
  s = block_sum(s);
  if (tid() == 0) a.sums[a.norm + blockIdx.x] = s;
}

// The norm and the clip coefficient, NaN where the norm is not finite.
__global__ __launch_bounds__(1024) void k_clip(AwNormArgs a) {
  double s = 0.0;
  for (int64_t i = tid(); i < a.count; i += 1024) s += a.sums[i];
  s = block_sum(s);
  if (tid() == 0) {
    // a trace of products that cancel to nothing may come out below zero by rounding
    const float norm = static_cast<float>(sqrt(s < 0.0 ? 0.0 : s) * fabs(static_cast<double>(a.scale)));
    a.clip[0] = norm;
    const bool finite = fabsf(norm) < __builtin_inff();
    a.clip[1] = !finite ? __builtin_nanf("") : norm > a.max_norm ? a.max_norm / norm : 1.f;
  }
}

template <int BITS, bool WIDE>
void launch_dense(int64_t tiles, const AwArgs& a, hipStream_t st) {
  constexpr int threads = dense_threads<WIDE>(), groups = dense_groups<BITS, WIDE>(threads / 64);
  hipLaunchKernelGGL((k_adamw<BITS, WIDE>), dim3(static_cast<uint32_t>(tiles * groups)), dim3(threads), WIDE ? kDenseLds : 0,
                     st, a);
}

// `narrow` and `joined` tiles lie behind the products' in the table, and their workgroups come first: they are
// short, and would leave the last ones alone on the GPU.
template <int BITS, int KC, bool WIDE>
void launch_products(int64_t tiles, int64_t narrow, int64_t joined, AwArgs a, hipStream_t st) {
  constexpr int W = product_group(KC);
  static_assert(dense_groups<BITS, false>(W) == aw_joined_groups(BITS, W), "the planner counts a launch's threads");
  a.count = static_cast<uint32_t>(tiles);
  a.narrow = static_cast<uint32_t>(narrow);
  a.joined = static_cast<uint32_t>(joined);
  const int64_t others = (narrow + joined * dense_groups<BITS, false>(W) + 63) / 64 * 64;
  a.others = static_cast<uint32_t>(others);
  const int64_t grid = others + (tiles + 63) / 64 * 64;
  hipLaunchKernelGGL((k_adamw_product<BITS, KC, WIDE>), dim3(static_cast<uint32_t>(grid)), dim3(64 * W),
                     BITS == 32 ? kProductLds : 0, st, a);
}

template <int BITS, bool WIDE>
void launch_product(int rank, int64_t tiles, int64_t narrow, int64_t joined, const AwArgs& a, hipStream_t st) {
  if (rank <= 16)
    launch_products<BITS, 1, WIDE>(tiles, narrow, joined, a, st);
  else if (rank <= 32)
    launch_products<BITS, 2, WIDE>(tiles, narrow, joined, a, st);
  else if (rank <= 64)
    launch_products<BITS, 4, WIDE>(tiles, narrow, joined, a, st);
  else if (rank <= 128)
    launch_products<BITS, 8, WIDE>(tiles, narrow, joined, a, st);
  else
    launch_products<BITS, 16, WIDE>(tiles, narrow, joined, a, st);
}

template <int BITS>
void launch_step(const AwSlotPlan& s, AwArgs a, hipStream_t st) {
  if (s.dense[1]) launch_dense<BITS, true>(s.dense[1], a, st);
  a.tiles += s.dense[1];
  if (s.dense[0]) launch_dense<BITS, false>(s.dense[0], a, st);
  a.tiles += s.dense[0];
  const bool last = s.product[0] == 0;  // the launch that the narrow and joined tiles go with
  if (s.product[1]) launch_product<BITS, true>(s.rank, s.product[1], last ? s.narrow : 0, last ? s.joined : 0, a, st);
  a.tiles += s.product[1];
  if (s.product[0])
    launch_product<BITS, false>(s.rank, s.product[0], s.narrow, s.joined, a, st);
  else if (s.narrow && !s.product[1])
    hipLaunchKernelGGL(k_adamw_narrow<BITS>, dim3(static_cast<uint32_t>(s.narrow)), dim3(kAwBlock), 0, st, a);
}

}  // namespace

hipError_t adamw_launch_step(const AwSlotPlan& s, int bits, const AwArgs& a, hipStream_t st) {
  if (bits == 32)
    launch_step<32>(s, a, st);
  else
    launch_step<8>(s, a, st);
  return hipGetLastError();
}

hipError_t adamw_launch_norm(const AwSlotPlan& s, AwNormArgs a, hipStream_t st) {
  a.count = s.norm + s.trace;
  a.norm = s.norm;
  a.gram_tiles = s.gram;
  a.t = aw_gram_t(s.rank);
  a.tiles += s.dense[0] + s.dense[1] + s.product[0] + s.product[1] + s.narrow + s.joined;
  const dim3 grid(static_cast<uint32_t>(s.norm + (s.gram + 3) / 4)), block(kAwBlock);
  if (!s.gram)
    hipLaunchKernelGGL(k_norm<0>, grid, block, 0, st, a);
  else if (a.t == 1)
    hipLaunchKernelGGL(k_norm<1>, grid, block, 0, st, a);
  else if (a.t == 2)
    hipLaunchKernelGGL(k_norm<2>, grid, block, 0, st, a);
  else
    hipLaunchKernelGGL(k_norm<4>, grid, block, 0, st, a);
  if (s.trace) {
    AwNormArgs b = a;
    b.tiles += s.norm + s.gram;
    hipLaunchKernelGGL(k_trace, dim3(static_cast<uint32_t>(s.trace)), dim3(1024), 0, st, b);
  }
  hipLaunchKernelGGL(k_clip, dim3(1), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace acp
