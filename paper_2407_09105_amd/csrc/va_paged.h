// Attention of one new token of every sequence over the paged key-value cache: the kernel (instantiated in va_paged_*.hip, one
// file per type of the queries) and what it shares with the joining of parts (va_paged.hip).
//
// A wave takes 32 keys at a time for the (up to 16) query heads of a KV head, straight from memory into registers: no barrier, and no
// LDS but for the queries where registers do not hold them, until the waves' results are joined at the end.  With
// v_mfma_f32_16x16x32 (lane l: i = l % 16, h = l / 16; operand A row i, B column i, both at k = 8 h + 0..7; result: column i, rows
// 4 h + 0..3):
//   - S^T = K Q^T, two products of 16 keys: lane (i, h) holds 16-byte chunks h, h + 4, ... of key i's row (loaded as whole 128-byte
//     lines, then swapped between lanes 8 apart) - which columns share a k-step does not matter as long as q's fragments hold the
//     same ones - and ends up with scores of head i, keys 4 h + 0..3.
//   - O^T += V^T P^T: those 2 x 4 keys are k = 8 h + 0..7, so P^T needs no exchange between lanes.  Lane (i, h) loads columns
//     8 i + 0..7 of its 8 keys (16 lanes together a whole row of 128 columns); the fragment of the m-th product, whose rows are the
//     columns 8 i + m, is the m-th element of each of them: four byte permutations, half an instruction per element.
// fp32 queries over a cache of fp32 do both products with v_mfma_f32_16x16x4_f32, an element of a lane's chunk per step; over 8 bits,
// which are exact in bf16, queries and P are three bf16 parts each, 24 bits (30 sequences of 4000, 8 heads of 64, int8: 51 us with the
// former, 29 so; of 256 261, 125).
// Softmax: fp32, running maximum and sum per head, the maximum moved only when it grows by more than 2^kLazyLog2.  O is as exact as fp32
// products make it, whatever the elements.  Against bf16 and 8-bit values P enters the matrix unit in three bf16 parts, which hold all its
// 24 bits: with two, 16 bits, one of some hundred 16-bit results was rounded the other way.  The matrix unit is idle most of the time; the
// third part costs nothing that can be measured (16 sequences of up to 4000, 16 heads of 256: 109.5 us with two, 110 with three).
// fp16 has no room for P: two fp16 parts keep 22 bits of the largest and none of what lies 2^-31 below, of which a long context may be made.
// fp16 values are widened instead, and O^T += V^T P^T runs in v_mfma_f32_16x16x4_f32, an element of a column per step: 131072 keys of 8
// heads of 128 105 -> 109 us, 48 sequences of about 700 41.7 -> 44.3, 16 of up to 4000 with 16 heads of 256 110 -> 126.  Values in two bf16
// parts against P in three would cost as much (108, 42.7, 127) and its registers spill.
//
// Bound by memory: keys and values are read once, 2 d elements each key against 4 d flops per query head.  Measured, with the
// joining: 131072 keys of 8 heads of 128 in bf16 87 us (6.1 TB/s; the kernel alone 6.6, the card reads 7.0), 128 sequences of
// 1024 to 8192 in e4m3 221 us (5.9), 16 of up to 4096 with 16 heads of 256 113 us (5.7).
#pragma once
#include "va_kv_cache.h"

namespace va {
namespace paged {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 32;               // keys of a wave's step
constexpr int kUnit = kTile * kWaves;   // sequences are cut at multiples of this
constexpr int kHeads = 16;              // query heads of a workgroup
constexpr int kMostUnits = 1 << 24;     // of the longest sequence, 2^31 tokens
constexpr float kLazyLog2 = 8.f;
constexpr float kMostFloat = 3.402823466e38f;

// How the sequences are cut into parts, one workgroup's work per KV head: see find_part.
struct Split {
  int slots;        // room for parts; n_seqs where no sequence is cut
  int least_units;  // least length of a part
  FastDiv extra;    // slots - n_seqs
};
Split split_of(int n_seqs, long long capacity, int hq, int hkv);

// Of every sequence where its parts begin and how many it has; then of all parts in order [slots, hq] pairs (reference score before it
// is scaled, sum of P) and [slots, hq, d] sums of P V.
struct Workspace {
  int2 *parts;
  float2 *ml;
  float *o;
};
static inline size_t workspace_bytes(const Split &s, int n_seqs, int hq, int d) {
  return s.slots == n_seqs ? 0 : (size_t)n_seqs * sizeof(int2) + (size_t)s.slots * hq * (sizeof(float2) + d * sizeof(float));
}
static inline Workspace workspace(void *p, const Split &s, int n_seqs, int hq) {
  int2 *const parts = (int2 *)p;
  float2 *const ml = (float2 *)(parts + n_seqs);
  return {parts, ml, (float *)(ml + (size_t)s.slots * hq)};
}

struct Part {
  int b, first, parts;  // sequence, its first part's slot, how many it has
  int units;            // of kUnit keys in a part
  int n;                // tokens of the sequence
};

// Sum of a wave's values up to each lane: shifts within rows of 16, then the rows' totals (data-parallel primitives, no LDS).
__device__ __forceinline__ int sum_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes before
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // last lane of row 0 / 2 to row 1 / 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
  return x;
}

// The part that a slot holds; false where it holds none.  A sequence of u units has max(1, ceil(u / c)) parts of c units, where
// c = max(least_units, ceil(all units / (slots - n_seqs))): no more than slots in all, whatever the lengths are, and of equal
// size but for the last of each sequence.  A wave reads 64 lengths at a time and adds them up across its lanes.
__device__ __forceinline__ bool find_part(const int32_t *__restrict__ lens, const PageMap &map, const Split &split, int slot, Part &part) {
  const int lane = threadIdx.x & 63, B = map.n_seqs;
  auto length = [&](int b) { return min(max(lens[min(b, B - 1)], 0), map.capacity); };
  if (split.slots == B) {
    if (slot >= B) return false;
    part = {slot, slot, 1, kMostUnits, uniform(length(slot))};
    return true;
  }
  const int mine0 = length(lane);
  auto units_of = [](int n) { return (int)((uint32_t)(n + kUnit - 1) / kUnit); };
  auto units_at = [&](int b0, int n) { return b0 + lane < B ? units_of(n) : 0; };
  long long total = __builtin_amdgcn_readlane(sum_upto(units_at(0, mine0)), 63);  // 64 x 2^24 at most
  for (int b0 = 64; b0 < B; b0 += 64) total += __builtin_amdgcn_readlane(sum_upto(units_at(b0, length(b0 + lane))), 63);
  const int drop = total >= 1 << 30 ? 10 : 0;  // to what a 32-bit division takes, rounded up
  const int share = ((int)((total + (1 << drop) - 1) >> drop) + (int)split.extra.d - 1) / split.extra;
  const int c = max(split.least_units, min(share, kMostUnits >> drop) << drop);
  const float inv = 1.f / (float)c;
  int before = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int mine = b0 == 0 ? mine0 : length(b0 + lane), units = units_of(mine);
    int parts = (int)((float)units * inv);  // units <= 2^24 are exact, the quotient is off by one at most
    const int rest = units - parts * c;
    parts += rest > c ? 2 : rest > 0 ? 1 : 0;
    parts = b0 + lane < B ? max(1, parts) : 0;
    const int upto = before + sum_upto(parts);
    const uint64_t past = __ballot(upto > slot);
    if (past) {
      const int at = __builtin_ctzll(past), has = __builtin_amdgcn_readlane(parts, at);
      part = {b0 + at, __builtin_amdgcn_readlane(upto, at) - has, has, c, __builtin_amdgcn_readlane(mine, at)};
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// max / sum over the four lanes that hold a head
__device__ __forceinline__ float head_max(float x) {
  x = pair_max(x);
  return fmaxf(x, __shfl_xor(x, 16));
}
__device__ __forceinline__ float head_sum(float x) {
  x = pair_sum(x);
  return x + __shfl_xor(x, 16);
}

// ---- element types ----------------------------------------------------------------------------------

template <class E> struct is_f32 { static constexpr bool value = false; };
template <> struct is_f32<F32> { static constexpr bool value = true; };

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Four cached 8-bit elements (one dword) as 16-bit elements of E, two dwords; exact.
__device__ __forceinline__ void widen(E4m3, Bf16, uint32_t x, uint32_t (&y)[2]) {
  y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
  y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true));
}
__device__ __forceinline__ void widen(E4m3, F16, uint32_t x, uint32_t (&y)[2]) {
  y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false));
  y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true));
}
__device__ __forceinline__ void floats(I8, uint32_t x, float (&y)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (float)(int8_t)(x >> (8 * e));
}
__device__ __forceinline__ void widen(I8, Bf16, uint32_t x, uint32_t (&y)[2]) {
  float f[4];
  floats(I8(), x, f);  // eight significant bits at most: the upper halves hold them
  y[0] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
  y[1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
}
__device__ __forceinline__ void widen(I8, F16, uint32_t x, uint32_t (&y)[2]) {
  // the bytes 128 higher, behind the exponent of 1024: 1024 + 128 + x, exactly
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
  x ^= 0x80808080u;
  y[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - off);
  y[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - off);
}

// Numbers in three parts of bf16, all 24 bits: fp32 queries (+-) against 8-bit keys, and P (times the scale of V over 8 bits).  Each part is
// cut off, not rounded; of an infinity or a NaN the first is that and the others are 0.
// kPositive: P against values of bf16, which may be infinite: the later parts also hold 2^-30 of P, so that they are positive like P and an
// infinity in V comes out as one (zero times it would be NaN).
template <bool kPositive> __device__ __forceinline__ void three_parts(const float (&p)[8], bf16x8 (&y)[3]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = p[e];
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    u32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * e + 1]), __float_as_uint(rest[2 * e]), 0x07060302u);
    y[part] = as_x8<Bf16>(h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float cut = rest[e] - __uint_as_float(__float_as_uint(rest[e]) & 0xffff0000u);
      if constexpr (kPositive) rest[e] = fmaf(p[e], 0x1p-30f, cut);
      else rest[e] = fabsf(p[e]) < INFINITY ? cut : 0.f;
    }
  }
}

// ---- the kernel ---------------------------------------------------------------------------------------

// How a tile's rows are found and read.
//   kWholeRows: page_size is a multiple of 16, so that the 16 keys of a product lie next to each other, and head_dim is kDh itself
//   kInPage:    the pages likewise, any head_dim that 16-byte chunks fit
//   kPerKey:    each key is found on its own
//   kDwords:    likewise, and rows are at least four whole dwords, which 16-byte chunks do not fit: the chunk that a row ends in is
//               loaded from its end and moved (82 sequences of 4259, 4 heads of 33 fp32 elements: 223 us in single dwords, 95 so;
//               30 of 4000, 8 heads of 100 bf16 elements 132, 81)
//   kElements:  likewise, and rows are read element by element
enum Look { kWholeRows, kInPage, kPerKey, kDwords, kElements };

struct Args {
  const void *Q;
  void *O;
  float *LSE;
  const void *k, *v;
  const float *ks, *vs;
  PageMap map;
  const int32_t *lens;
  Split split;
  Workspace ws;
  FastDiv hkv, groups;  // KV heads; groups of kHeads query heads of one KV head
  int hq, G, d;         // G = hq / hkv
  float scale, scale_log2;
};

// log sum exp(S) of a row from its reference score and the sum of P.  (Scores are scaled on their own: as exponents of two the
// largest would pass fp32's range, by 1.44.)
__device__ __forceinline__ float lse_of(float m, float sum, float scale) {
  return sum != 0.f ? fmaf(m, scale, log2f(sum) * 0.6931471805599453f) : -INFINITY;
}

// Between lanes 8 apart in a row of 16 (i and i + 8): before, lane l holds a of row l % 8 and b of row 8 + l % 8; after, the lower
// lane both a's of its row, its own and the upper one's, and the upper lane both b's, the lower one's first.
__device__ __forceinline__ void own_row(uint32_t &a, uint32_t &b) {
  constexpr int kRotateBy8 = 0x128;
  const int x = __builtin_amdgcn_update_dpp((int)a, (int)b, kRotateBy8, 0xf, 0xc, false);  // upper lanes: b of the lower
  b = (uint32_t)__builtin_amdgcn_update_dpp((int)b, (int)a, kRotateBy8, 0xf, 0x3, false);  // lower lanes: a of the upper
  a = (uint32_t)x;
}
// a = b = x of this lane's i -> a of i % 8, b of 8 + i % 8
__device__ __forceinline__ void other_half(int &a, int &b) {
  const int x = a;
  a = __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xc, false);
  b = __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0x3, false);
}

// What the lanes know of the 16 keys of a product, lane (i, h) of key i; turned: of key (i + 4 h) % 16; four_of: a turned value of
// key 4 h + kV, which in each row of 16 lanes is lane kV's.
__device__ __forceinline__ int turned(int x) {
  const int lane = threadIdx.x & 63;
  return __shfl(x, (lane + (lane >> 4) * 4) & 15);
}
template <int kV> __device__ __forceinline__ int four_of(int turned_x) {
  return __builtin_amdgcn_update_dpp(turned_x, turned_x, 0x150 + kV, 0xf, 0xf, false);
}
__device__ __forceinline__ void four_of(float turned_x, f32x4 &y) {
  const int x = (int)__float_as_uint(turned_x);
  y = f32x4{__uint_as_float((uint32_t)four_of<0>(x)), __uint_as_float((uint32_t)four_of<1>(x)), __uint_as_float((uint32_t)four_of<2>(x)),
            __uint_as_float((uint32_t)four_of<3>(x))};
}

template <int kBytes> struct Piece {
  uint32_t x[kBytes / 4];
};
template <int kBytes, int kPolicy> __device__ __forceinline__ Piece<kBytes> buffer_piece(buffer_t b, uint32_t off) {
  Piece<kBytes> p;
  if constexpr (kBytes == 16) {
    const u32x4 r = __builtin_amdgcn_raw_buffer_load_b128(b, (int)off, 0, kPolicy);
#pragma unroll
    for (int i = 0; i < 4; ++i) p.x[i] = r[i];
  } else if constexpr (kBytes == 8) {
    const u32x2 r = __builtin_amdgcn_raw_buffer_load_b64(b, (int)off, 0, kPolicy);
    p.x[0] = r[0], p.x[1] = r[1];
  } else {
    p.x[0] = __builtin_amdgcn_raw_buffer_load_b32(b, (int)off, 0, kPolicy);
  }
  return p;
}
template <int kBytes> __device__ __forceinline__ Piece<kBytes> memory_piece(const char *p) {
  struct __attribute__((packed, aligned(4))) Raw { uint32_t x[kBytes / 4]; };
  const Raw r = *(const Raw *)p;
  Piece<kBytes> q;
#pragma unroll
  for (int i = 0; i < kBytes / 4; ++i) q.x[i] = r.x[i];
  return q;
}
// A row's bytes from `at` on, which may end inside the piece: the row's last kBytes, its words moved down once they are here.
template <int kBytes> __device__ __forceinline__ Piece<kBytes> last_piece(const char *row, int at, int row_bytes) {
  return memory_piece<kBytes>(row + min(at, row_bytes - kBytes));
}
template <int kBytes> __device__ __forceinline__ void move_down(Piece<kBytes> &p, int at, int row_bytes) {
  const int by = max(at - (row_bytes - kBytes), 0) / 4;  // what moves in at the end is not there: any value
  constexpr int kWords = kBytes / 4;
#pragma unroll
  for (int step = 1; step < kWords; step *= 2)
#pragma unroll
    for (int w = 0; w + step < kWords; ++w) {
      const uint32_t here = p.x[w], next = p.x[w + step];
      p.x[w] = (by & step) != 0 ? next : here;
    }
}
// elements `column` .. of a row of d elements, zeros behind it
template <class T, int kBytes> __device__ __forceinline__ Piece<kBytes> element_piece(const T *row, int column, int d) {
  constexpr int kEach = 4 / sizeof(T);
  Piece<kBytes> p;
#pragma unroll
  for (int i = 0; i < kBytes / 4; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int c = column + i * kEach + e;
      uint32_t bits = 0;
      if (c < d) {
        if constexpr (sizeof(T) == 1) bits = *(const uint8_t *)(row + c);
        else if constexpr (sizeof(T) == 2) bits = *(const uint16_t *)(row + c);
        else bits = *(const uint32_t *)(row + c);
      }
      w |= bits << (8 * sizeof(T) * e % 32);
    }
    p.x[i] = w;
  }
  return p;
}

// Waves that share a SIMD.  Scattered keys of 8 bits gain from a fourth (33 sequences of 4096, pages of 24, 8 heads of 128: 92 us with
// three, 78 so); keys that lie together do not (56, 57; 16 bits 95, 110 with four, which spill).
template <class E, class C> constexpr int waves_per_simd(int dh, Look look) {
  if (is_f32<E>::value) return dh == 256 ? 1 : 2;
  return dh == 256 ? 2 : is_8bit<C>::value && look == kPerKey ? 4 : 3;
}

// E: type of the queries; C: of the cache (E itself or 8 bits); kDh: head_dim rounded up to 64, 128 or 256.
template <class E, class C, int kDh, Look kLook>
__global__ void __launch_bounds__(kThreads, (waves_per_simd<E, C>(kDh, kLook)))
kernel(Args a) {
  constexpr bool kF32 = is_f32<E>::value, k8 = is_8bit<C>::value, kTogether = kLook <= kInPage;  // a product's keys
  typedef typename E::elem elem;
  typedef typename C::elem cached;
  constexpr int kSize = sizeof(cached);
  // K: chunks of 16 bytes, chunk n of lane (i, h) = columns (4 n + h) kCpc ..
  constexpr int kCpc = 16 / kSize, kKn = kDh / (4 * kCpc);
  // V: kVC columns of a row for a lane at a time, kHf times
  constexpr int kVC = kF32 || kDh == 64 ? 4 : 8, kHf = kDh / (16 * kVC), kVBytes = kVC * kSize;
  typedef typename std::conditional<kF32, Bf16, E>::type E16;  // matrix operands of S over 16 and 8 bits
  // fp32 matrix instructions: S of fp32 alone, O also of fp16, whose range small probabilities leave
  constexpr bool kMat32 = kF32 && !k8, kMat32V = !k8 && !std::is_same<C, Bf16>::value;
  constexpr int kParts = kF32 ? 3 : 1;       // of a query's element over 8 bits

  constexpr int kStride = 16 * kVC + 4;
  __shared__ __attribute__((aligned(16))) float part_o[kWaves][kHeads][kStride];
  __shared__ float part_m[kWaves][kHeads], part_l[kWaves][kHeads];

  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), i = lane & 15, h = lane >> 4;
  const PageMap &map = a.map;
  const int hkv = map.hkv, d = kLook == kWholeRows ? kDh : a.d, G = a.G, page = map.page.d;

  // Workgroup ids go to the 8 XCDs in turn: the groups of 16 query heads of one KV head, which read the same keys, 8 ids apart.
  const int turn = blockIdx.x >> 3, pair = turn / a.groups * 8 + (blockIdx.x & 7), head0 = turn % a.groups * kHeads;
  if (pair >= a.split.slots * hkv) return;
  const int slot = pair / a.hkv, g = pair - slot * hkv;
  Part part;
  if (!find_part(a.lens, map, a.split, slot, part)) return;
  const int b = part.b, n = part.n;
  const int heads = min(G - head0, kHeads);  // rows of this workgroup
  const size_t first_head = (size_t)b * a.hq + g * G + head0;

  // q as operand B, head i, the columns of the K chunks: kQn times 16 bytes a lane.  They stay in registers but where
  // those do not suffice, head_dim 256 of 16 or 32 bits and the four waves above: there every tile reads them from LDS anew (16
  // sequences of 500 to 4000 tokens, 16 heads of 256: 114 us with spills, 107 with one wave per SIMD, 107 so; scattered keys 120,
  // 112, 107).
  constexpr int kEach = 16 / (int)sizeof(elem), kQn = kKn * kCpc / kEach;
  constexpr bool kQInLds = kDh == 256 ? !k8 : kDh == 128 && waves_per_simd<E, C>(kDh, kLook) == 4;
  __shared__ u32x4 q_lds[kQInLds ? kQn : 1][64];
  u32x4 q_reg[kQn];
  bf16x8 q_parts[kF32 && k8 ? kQn / 2 : 1][kParts];  // of 8 columns, where they are three
  {
    const buffer_t q = make_buffer((const elem *)a.Q + first_head * d, (size_t)heads * d * sizeof(elem));  // no rows behind `heads`
#pragma unroll
    for (int x = 0; x < kQn; ++x) {
      const int column = (4 * (x * kEach / kCpc) + h) * kCpc + x * kEach % kCpc;
      u32x4 y;
      if constexpr (kLook >= kDwords) {
        const Piece<16> piece = element_piece<elem, 16>((const elem *)a.Q + (first_head + min(i, heads - 1)) * d, column, i < heads ? d : 0);
        y = u32x4{piece.x[0], piece.x[1], piece.x[2], piece.x[3]};
      } else {
        y = buffer_load16(q, column < d ? (uint32_t)((i * d + column) * sizeof(elem)) : kPastEnd);
      }
      q_reg[x] = y;
    }
  }
  if constexpr (kF32 && k8) {
#pragma unroll
    for (int x = 0; x < kQn; x += 2) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = __builtin_canonicalizef(__uint_as_float(q_reg[x + e / 4][e % 4]));  // a NaN's first part shall be one
      three_parts<false>(f, q_parts[x / 2]);
    }
  }
  auto q_at = [&](int x) {
    if constexpr (kQInLds) return q_lds[x][lane];
    else return q_reg[x];
  };

  // keys j0 .. j1 - 1, tiles wave, wave + kWaves, ...
  const long long j0l = (long long)(slot - part.first) * part.units * kUnit;
  const int j0 = (int)min(j0l, (long long)n), j1 = (int)min(j0l + (long long)part.units * kUnit, (long long)n);
  const int tile_end = (j1 + kTile - 1) / kTile;
  const int32_t *const table = map.table + (int64_t)b * map.stride;

  // ---- rows of a tile: the entries are requested two tiles ahead, the rows one ----
  struct Entries {
    int j[2], at[2], id[2];  // key (kTogether: the product's first, else this lane's own), the page's place in the table, the page
  };
  struct Rows {
    int row[2];    // of that key; row 0 where it does not exist (kTogether: not read then)
    int count[2];  // kTogether: how many of the product's 16 keys exist; else which, a bit each
  };
  auto entries = [&](int tile) {
    Entries t;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      t.j[s] = tile * kTile + 16 * s + (kTogether ? 0 : i);
      t.at[s] = min(t.j[s], j1 - 1) / map.page;
      t.id[s] = table[t.at[s]];
    }
    return t;
  };
  auto rows_of = [&](const Entries &t) {
    Rows r;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const bool ok = t.j[s] < j1 && (uint32_t)t.id[s] < (uint32_t)map.n_pages;
      r.row[s] = ok ? (t.id[s] * hkv + g) * page + (t.j[s] - t.at[s] * page) : 0;
      if constexpr (kTogether) r.count[s] = ok ? min(j1 - t.j[s], 16) : 0;
      else r.count[s] = (int)((uint32_t)__ballot(ok) & 0xffffu);  // the four groups of 16 lanes have the same keys
    }
    return r;
  };

  const uint32_t row_bytes = (uint32_t)d * kSize;
  // A load of K takes whole 128-byte lines: chunks 8 x .. 8 x + 7 of rows 0..7 (a) or 8..15 (b), lane (i, h) chunk 4 (i / 8) + h of
  // row i % 8.  The lanes 8 apart then swap what is the other's row (own_row), and hold chunks 4 n + h, n = 2 x and 2 x + 1, of
  // their own row i.  Rows of 64 bytes have 4 chunks: a load takes the 16 rows as they are.
  constexpr bool kLines = kKn > 1;
  constexpr int kLoads = kLines ? kKn / 2 : 1;  // of one kind
  const int k_row = kLines ? i & 7 : i, k_chunk = kLines ? 4 * (i >> 3) + h : h;
  uint32_t k_off[kLoads], v_off[kHf];  // column offsets in a row, kPastEnd for columns that do not exist
#pragma unroll
  for (int x = 0; x < kLoads; ++x) k_off[x] = (8 * x + k_chunk) * kCpc < d ? (uint32_t)(k_row * row_bytes + (8 * x + k_chunk) * 16) : kPastEnd;
#pragma unroll
  for (int x = 0; x < kHf; ++x) v_off[x] = (16 * x + i) * kVC < d ? (uint32_t)(4 * h * row_bytes + (16 * x + i) * kVBytes) : kPastEnd;
  const bool half_chunk = k8 && (d & 8) != 0;  // rows end in the middle of a 16-byte chunk
  // Rows pass by the caches (non-temporal loads) where a load takes whole 128-byte lines: this card reads 7.0 TB/s so, 6.1 otherwise (64
  // sequences of 4096, 32 / 8 heads of 128, 192 us without and 171 so).  Right where rows are read once, and kept where they are not: if
  // those sequences share half their pages 126 and 120; 15 of 16 pages 90 and 102; and with 64 query heads to each of two KV heads, whose keys
  // four workgroups read, 104 and 132.  A line fetched in pieces would be fetched again: with rows of 160 bytes 250 us became 266.
  constexpr int kPolicyK = kLook == kWholeRows ? kOnce : 0, kPolicyV = kDh * kSize >= 128 ? kOnce : 0;

  typedef Piece<16> KPiece;
  typedef Piece<kVBytes> VPiece;
  KPiece kr[2][kKn];
  VPiece vr[8][kHf];
  // scales: kTogether of keys 4 h + 0..3; else of key (i + 4 h) % 16, handed round (four_of) when they are used
  f32x4 ksr[2], vsr[2];
  float ks_turned[2], vs_turned[2];

  auto load_k = [&](const Rows &r) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (kTogether) {
        const buffer_t buf = make_buffer((const char *)a.k + (size_t)r.row[s] * row_bytes, (size_t)r.count[s] * row_bytes);
#pragma unroll
        for (int x = 0; x < kKn; ++x) {  // a, b, a, b, ...
          const uint32_t base = k_off[x / 2], off = base == kPastEnd ? kPastEnd : base + (x % 2) * 8 * row_bytes;
          if (!half_chunk) {
            kr[s][x] = buffer_piece<16, kPolicyK>(buf, off);
          } else {
            const Piece<8> lo = buffer_piece<8, 0>(buf, off);
            const Piece<8> hi = buffer_piece<8, 0>(buf, (8 * (x / 2) + k_chunk) * kCpc + 8 < d ? off + 8 : kPastEnd);
            kr[s][x] = {{lo.x[0], lo.x[1], hi.x[0], hi.x[1]}};
          }
        }
        if constexpr (k8) {
          const buffer_t sb = make_buffer(a.ks + r.row[s], r.count[s] > 0 ? 64 : 0);
          const Piece<16> y = buffer_piece<16, 0>(sb, 16 * h);
#pragma unroll
          for (int v = 0; v < 4; ++v) ksr[s][v] = __uint_as_float(y.x[v]);
        }
      } else {
        // rows of the two kinds of loads; row 0 for a key that does not exist
        int from[2] = {r.row[s], r.row[s]};
        if constexpr (kLines) other_half(from[0], from[1]);
#pragma unroll
        for (int x = 0; x < kKn; ++x) {
          const char *row = (const char *)a.k + (size_t)from[x % 2] * row_bytes;
          const int column = (8 * (x / 2) + k_chunk) * kCpc;
          // (columns that do not exist are loaded from the row's end; what is not q's to see is cleared before it is used)
          if constexpr (kLook == kElements) {
            kr[s][x] = element_piece<cached, 16>((const cached *)row, column, d);
          } else if constexpr (kLook == kDwords) {
            kr[s][x] = last_piece<16>(row, column * kSize, (int)row_bytes);
          } else if (!half_chunk) {
            kr[s][x] = memory_piece<16>(row + min(column, d - kCpc) * kSize);
          } else {
            const Piece<8> lo = memory_piece<8>(row + min(column, d - 8) * kSize), hi = memory_piece<8>(row + min(column + 8, d - 8) * kSize);
            kr[s][x] = {{lo.x[0], lo.x[1], hi.x[0], hi.x[1]}};
          }
        }
        if constexpr (k8) ks_turned[s] = a.ks[turned(r.row[s])];
      }
    }
  };
  auto load_v = [&](const Rows &r) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (kTogether) {
        const buffer_t buf = make_buffer((const char *)a.v + (size_t)r.row[s] * row_bytes, (size_t)r.count[s] * row_bytes);
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int x = 0; x < kHf; ++x) vr[4 * s + v][x] = buffer_piece<kVBytes, kPolicyV>(buf, v_off[x] == kPastEnd ? kPastEnd : v_off[x] + v * row_bytes);
        if constexpr (k8) {
          const buffer_t sb = make_buffer(a.vs + r.row[s], r.count[s] > 0 ? 64 : 0);
          const Piece<16> y = buffer_piece<16, 0>(sb, 16 * h);
#pragma unroll
          for (int v = 0; v < 4; ++v) vsr[s][v] = __uint_as_float(y.x[v]);
        }
      } else {
        const int turned_row = turned(r.row[s]);
        const int from[4] = {four_of<0>(turned_row), four_of<1>(turned_row), four_of<2>(turned_row), four_of<3>(turned_row)};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const char *row = (const char *)a.v + (size_t)from[v] * row_bytes;
#pragma unroll
          for (int x = 0; x < kHf; ++x) {
            if constexpr (kLook == kElements)
              vr[4 * s + v][x] = element_piece<cached, kVBytes>((const cached *)row, (16 * x + i) * kVC, d);
            else if constexpr (kLook == kDwords)
              vr[4 * s + v][x] = last_piece<kVBytes>(row, (16 * x + i) * kVBytes, (int)row_bytes);
            else
              vr[4 * s + v][x] = memory_piece<kVBytes>(row + min((16 * x + i) * kVC, d - kVC) * kSize);
          }
        }
        if constexpr (k8) vs_turned[s] = a.vs[turned_row];
      }
    }
  };

  f32x4 acc[kHf][kVC];
#pragma unroll
  for (int x = 0; x < kHf; ++x)
#pragma unroll
    for (int m = 0; m < kVC; ++m) acc[x][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m_ref = -INFINITY, m_thr = -INFINITY;  // raw score that exponents are relative to, and the one that moves it
  float l_run = 0.f;                           // this lane's share of the sum of P

  // In flight: the entries of tile + 2 kWaves, the keys of tile + kWaves, the values of tile.  Behind the last tile no key exists;
  // its loads are made all the same (a branch around them would make the compiler wait for all that is in flight).
  int tile = j0 / kTile + wave;
  Rows now = {};
  Entries ahead = {};
  if (tile < tile_end) {
    now = rows_of(entries(tile));
    load_k(now);
    ahead = entries(tile + kWaves);
  }
  if constexpr (kQInLds) {
#pragma unroll
    for (int x = 0; x < kQn; ++x)
      if (x % kWaves == wave) q_lds[x][lane] = q_reg[x];
    __syncthreads();
  }
  for (; tile < tile_end; tile += kWaves) {
    const Rows next = rows_of(ahead);
    ahead = entries(tile + 2 * kWaves);
    load_v(now);
    __builtin_amdgcn_sched_barrier(0);  // they are on their way before the keys are waited for
    if constexpr (kQInLds) asm volatile("" ::: "memory");  // q is read within the loop
    // ---- S^T = K Q^T ----
    f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if constexpr (kLook == kDwords) {
#pragma unroll
      for (int x = 0; x < kKn; ++x)
#pragma unroll
        for (int t = 0; t < 2; ++t) move_down(kr[t][x], (8 * (x / 2) + k_chunk) * 16, (int)row_bytes);
    }
    if constexpr (kLines) {
#pragma unroll
      for (int x = 0; x < kKn; x += 2)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) own_row(kr[t][x].x[w], kr[t][x + 1].x[w]);
    }
    if constexpr (kLook == kPerKey || kLook == kDwords) {
      if (d != kDh) {
#pragma unroll
        for (int x = 0; x < kKn; ++x)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int w = 0; w < 4; ++w) kr[t][x].x[w] = (4 * x + h) * kCpc + w * 4 / kSize < d ? kr[t][x].x[w] : 0u;
      }
    }
#pragma unroll
    for (int x = 0; x < kKn; ++x) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const KPiece &p = kr[t][x];
        if constexpr (kMat32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t] = mfma16(__uint_as_float(p.x[e]), __uint_as_float(q_at(x)[e]), s[t]);
        } else if constexpr (k8) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint32_t w0[2], w1[2];
            widen(C(), E16(), p.x[2 * y], w0);
            widen(C(), E16(), p.x[2 * y + 1], w1);
            const auto key = as_x8<E16>(u32x4{w0[0], w0[1], w1[0], w1[1]});
            if constexpr (kF32) {
#pragma unroll
              for (int part = kParts - 1; part >= 0; --part) s[t] = mfma16(key, q_parts[2 * x + y][part], s[t]);
            } else {
              s[t] = mfma16(key, as_x8<E16>(q_at(2 * x + y)), s[t]);
            }
          }
        } else {
          s[t] = mfma16(as_x8<E16>(u32x4{p.x[0], p.x[1], p.x[2], p.x[3]}), as_x8<E16>(q_at(x)), s[t]);
        }
      }
    }
    if constexpr (k8) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (!kTogether) four_of(ks_turned[t], ksr[t]);
        s[t] *= ksr[t];
      }
    }
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    // ---- keys that do not exist ----
    if constexpr (kTogether) {
      if (now.count[0] + now.count[1] < kTile) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const bool there = 4 * h + v < now.count[t];
            s[t][v] = there ? s[t][v] : -INFINITY;
            if constexpr (k8) vsr[t][v] = there ? vsr[t][v] : 0.f;
          }
      }
    } else {
      if (now.count[0] != 0xffff || now.count[1] != 0xffff) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t mine = (uint32_t)now.count[t] >> (4 * h);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const bool there = mine >> v & 1;
            s[t][v] = there ? s[t][v] : -INFINITY;
#pragma unroll
            for (int x = 0; x < kHf; ++x)  // row 0 was read instead
#pragma unroll
              for (int w = 0; w < kVBytes / 4; ++w) vr[4 * t + v][x].x[w] = there ? vr[4 * t + v][x].x[w] : 0u;
          }
        }
      }
    }
    // ---- softmax ----
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__any(mx > m_thr)) {
      // (finite: an infinite score then has the exponential infinity and not NaN, and so has LSE)
      const float m_new = fminf(fmaxf(m_ref, head_max(mx)), kMostFloat);
      const float alpha = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_ref - m_new) * a.scale_log2);
      l_run *= alpha;  // a NaN of before stays
#pragma unroll
      for (int x = 0; x < kHf; ++x)
#pragma unroll
        for (int m = 0; m < kVC; ++m) acc[x][m] *= alpha;
      m_ref = m_new;
      m_thr = m_new + kLazyLog2 / a.scale_log2;
    }
    const float base = m_ref == -INFINITY ? 0.f : m_ref;
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = __builtin_amdgcn_exp2f((s[e >> 2][e & 3] - base) * a.scale_log2);
      l_run += p[e];
    }
    if constexpr (k8) {
      if constexpr (!kTogether) {
        four_of(vs_turned[0], vsr[0]);
        four_of(vs_turned[1], vsr[1]);
        if (now.count[0] != 0xffff || now.count[1] != 0xffff) {
#pragma unroll
          for (int e = 0; e < 8; ++e) vsr[e >> 2][e & 3] = (uint32_t)now.count[e >> 2] >> (4 * h + (e & 3)) & 1 ? vsr[e >> 2][e & 3] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] *= vsr[e >> 2][e & 3];
    }
    // ---- O^T += V^T P^T ----
    if constexpr (kLook == kDwords) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int x = 0; x < kHf; ++x) move_down(vr[e][x], (16 * x + i) * kVBytes, (int)row_bytes);
    }
    if constexpr (kMat32V) {
      if constexpr (kSize == 2) __builtin_amdgcn_sched_barrier(0);  // values are waited for behind the softmax
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int x = 0; x < kHf; ++x)
#pragma unroll
          for (int w = 0; w < kVBytes / 4; ++w) {
            struct Columns { cached x[4 / kSize]; };
            uint32_t two = vr[e][x].x[w];
            if constexpr (kSize == 2) asm("" : "+v"(two));  // converted here, not where the word comes from, which would take twice its registers
            const Columns c = __builtin_bit_cast(Columns, two);
#pragma unroll
            for (int m = 0; m < 4 / kSize; ++m) acc[x][w * 4 / kSize + m] = mfma16((float)c.x[m], p[e], acc[x][w * 4 / kSize + m]);
          }
    } else {
      bf16x8 parts[3];
      three_parts<!k8>(p, parts);
      __builtin_amdgcn_sched_barrier(0);  // values are waited for behind the softmax
#pragma unroll
      for (int x = 0; x < kHf; ++x) {
        uint32_t w[8][kVC / 2];  // columns in pairs
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (k8) {
#pragma unroll
            for (int y = 0; y < kVC / 4; ++y) {
              uint32_t two[2];
              widen(C(), Bf16(), vr[e][x].x[y], two);
              w[e][2 * y] = two[0], w[e][2 * y + 1] = two[1];
            }
          } else {
#pragma unroll
            for (int y = 0; y < kVC / 2; ++y) w[e][y] = vr[e][x].x[y];
          }
        }
#pragma unroll
        for (int m = 0; m < kVC; ++m) {
          u32x4 f;
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = __builtin_amdgcn_perm(w[2 * e + 1][m / 2], w[2 * e][m / 2], m % 2 ? 0x07060302u : 0x05040100u);
          const bf16x8 vf = as_x8<Bf16>(f);
#pragma unroll
          for (int part = 2; part >= 0; --part) acc[x][m] = mfma16(vf, parts[part], acc[x][m]);
        }
      }
    }
    now = next;
  }

  if (a.split.slots != map.n_seqs && slot == part.first && g == 0 && head0 == 0 && threadIdx.x == 0)
    a.ws.parts[b] = make_int2(part.first, part.parts);

  // ---- the waves' results: relative to the largest reference, added in order ----
  l_run = head_sum(l_run);
  if (h == 0) part_m[wave][i] = m_ref, part_l[wave][i] = l_run;
#pragma unroll
  for (int x = 0; x < kHf; ++x) {
    if (x > 0) __syncthreads();  // the columns before are read
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int m = 0; m < kVC; m += 4)
        *(f32x4 *)&part_o[wave][i][kVC * (4 * h + v) + m] = f32x4{acc[x][m][v], acc[x][m + 1][v], acc[x][m + 2][v], acc[x][m + 3][v]};
    __syncthreads();
    for (int at = threadIdx.x; at < heads * 16 * kVC; at += kThreads) {
      const int head = at / (16 * kVC), c = at % (16 * kVC), column = 16 * kVC * x + c;
      if (column >= d) continue;
      float m = part_m[0][head], sum = 0.f, o = 0.f;
#pragma unroll
      for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part_m[w][head]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = part_m[w][head], weight = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - m) * a.scale_log2);
        sum += weight * part_l[w][head];
        o += weight * part_o[w][head][c];
      }
      if (part.parts == 1) {
        ((elem *)a.O)[(first_head + head) * d + column] = (elem)(sum != 0.f ? o / sum : 0.f);
        if (column == 0) a.LSE[(size_t)(g * G + head0 + head) * map.n_seqs + b] = lse_of(m, sum, a.scale);
      } else {
        const size_t to = (size_t)slot * a.hq + g * G + head0 + head;
        a.ws.o[to * d + column] = o;
        if (column == 0) a.ws.ml[to] = make_float2(m, sum);
      }
    }
  }
}

template <class E, class C, Look kLook>
void launch_look(const Args &a, unsigned workgroups, hipStream_t stream) {
  if (kLook != kWholeRows ? a.d <= 64 : a.d == 64) kernel<E, C, 64, kLook><<<workgroups, kThreads, 0, stream>>>(a);
  else if (a.d <= 128) kernel<E, C, 128, kLook><<<workgroups, kThreads, 0, stream>>>(a);
  else kernel<E, C, 256, kLook><<<workgroups, kThreads, 0, stream>>>(a);
}
template <class E, class C> void launch_cache(const Args &a, unsigned workgroups, hipStream_t stream) {
  // whole 16-byte chunks of a row, 8 bytes at its end in an 8-bit cache
  constexpr int kSize = sizeof(typename C::elem), kEven = is_8bit<C>::value ? 8 : 16 / kSize;
  const bool chunks = a.d % kEven == 0 && (((uintptr_t)a.k | (uintptr_t)a.v) & (kEven * kSize - 1)) == 0 && ((uintptr_t)a.Q & 3) == 0;
  const bool dwords = a.d * kSize % 4 == 0 && a.d * kSize >= 16 && (((uintptr_t)a.k | (uintptr_t)a.v) & 3) == 0;
  if (!chunks && dwords) launch_look<E, C, kDwords>(a, workgroups, stream);
  else if (!chunks) launch_look<E, C, kElements>(a, workgroups, stream);
  else if (a.map.page.d % 16 == 0 && (a.d == 64 || a.d == 128 || a.d == 256)) launch_look<E, C, kWholeRows>(a, workgroups, stream);
  else if (a.map.page.d % 16 == 0) launch_look<E, C, kInPage>(a, workgroups, stream);
  else launch_look<E, C, kPerKey>(a, workgroups, stream);
}
template <class E> void launch_queries(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream) {
  if (format == VA_CACHE_I8) launch_cache<E, I8>(a, workgroups, stream);
  else if (format == VA_CACHE_E4M3) launch_cache<E, E4m3>(a, workgroups, stream);
  else launch_cache<E, E>(a, workgroups, stream);
}
void launch_bf16(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream);
void launch_f16(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream);
void launch_f32(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream);

}  // namespace paged
}  // namespace va
