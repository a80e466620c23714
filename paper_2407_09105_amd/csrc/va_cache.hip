// Rows of K and V into the pages of the key-value cache, quantised on the way where the cache holds 8 bits, and back out of them
// as a packed stream.
//
// Quantising a row x of d elements (one token and head): a = max |x_c|, scale = a / m, q_c = round(m x_c / a) with ties to even,
// m = 127 (integers) or 448 (e4m3).  With a = 2^e f, f in [1/2, 1): q_c = round((x_c 2^-e m) / f), where the product is exact
// for 16-bit x (8 or 11 bits times 7 or 3).  The quotient is product * RN(1 / f) corrected once by its remainder, two fused
// multiply-adds: a quotient halfway between two steps comes out exactly, since its remainder is exact, and any other one of
// 16-bit operands lies at least 2^-19 of itself away from halfway (the product has 18 bits at most), farther than the fp32
// quotient is off.  So 16-bit rows are rounded exactly as real numbers would be, without a division per element.
//
// Bound by memory: each element is read once and written once.
#include <algorithm>

#include "va_kv_cache.h"

namespace va {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ long long id_at(const void *ids, va_itype it, int t) {
  return it == VA_I64 ? (long long)((const int64_t *)ids)[t] : (long long)((const int32_t *)ids)[t];
}

// kLanes lanes hold a row, lane l its elements l * kVec .. + kVec - 1, or l, l + kLanes, ... (kVec = 1).  kWhole: d is kVec * kLanes.
// kLanes = 0: d / kVec lanes, whatever that is; no lane idles, but a row cannot be reduced across its lanes (head_dim 96 of 8 heads,
// 8300 e4m3 tokens read 12.5 -> 10.3 us).
// kPast: stores of whole 128-byte lines pass by the caches (non-temporal; lines that two workgroups share would be written twice):
// 65536 bf16 tokens of 8 heads of 128: K's rotary embedding and the write 149 -> 135 us, the read alone 105 -> 95, write and read
// together 205 -> 193; 2 to 3 % slower to 8 % faster together with the next reader of the rows.  Loads do not: the rows to be written have
// often just left another kernel (16384 of those tokens behind the embedding 35 us, with such loads 38).
template <class E, class C, int kVec, int kLanes, bool kWhole>
struct Row {
  typedef typename E::elem elem;
  typedef typename C::elem cached;
  static constexpr int kPer = kVec > 1 || kLanes == 0 ? kVec : 256 / kLanes;   // elements of a lane
  template <class T> using Words = uint32_t __attribute__((ext_vector_type(sizeof(T) * kVec / 4)));
  static __device__ __forceinline__ int column(int lane, int e) { return kVec > 1 || kLanes == 0 ? lane * kVec + e : lane + e * kLanes; }

  template <class T> static __device__ __forceinline__ void load(const T *p, int lane, int d, T (&x)[kPer]) {
    if constexpr (kVec > 1) {
      struct Chunk { T x[kVec]; };
      if (kWhole || lane * kVec < d) {
        const Words<T> *const at = (const Words<T> *)(p + lane * kVec);
        const Chunk c = __builtin_bit_cast(Chunk, *at);
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[e] = c.x[e];
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) x[e] = (T)0;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = column(lane, e) < d ? p[column(lane, e)] : (T)0;
    }
  }
  template <bool kPast, class T> static __device__ __forceinline__ void store(T *p, int lane, int d, const T (&x)[kPer]) {
    if constexpr (kVec > 1) {
      struct Chunk { T x[kVec]; } c;
      if (kWhole || lane * kVec < d) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) c.x[e] = x[e];
        Words<T> *const at = (Words<T> *)(p + lane * kVec);
        if constexpr (kPast) __builtin_nontemporal_store(__builtin_bit_cast(Words<T>, c), at);
        else *at = __builtin_bit_cast(Words<T>, c);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (column(lane, e) < d) p[column(lane, e)] = x[e];
    }
  }

  static __device__ __forceinline__ int8_t rounded(I8, float t) { return (int8_t)(int)rintf(t); }
  static __device__ __forceinline__ uint8_t rounded(E4m3, float t) { return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(t, t, 0, false); }

  // The row in 8 bits; returns its scale, the same in all of its lanes.
  static __device__ __forceinline__ float quantise(const elem (&x)[kPer], cached (&q)[kPer]) {
    uint32_t top = 0;  // magnitudes compare as their bits do; a NaN is above infinity
#pragma unroll
    for (int e = 0; e < kPer; ++e) top = max(top, __float_as_uint((float)x[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, kLanes));
    const bool finite = top < 0x7f800000u;
    const float a = finite ? __uint_as_float(top) : 0.f;
    int ex = 0;
    float f = frexpf(a, &ex);
    if (ex < -100) f = ldexpf(f, ex + 100), ex = -100;  // m 2^-e stays in range; f > 2^-50
    const float pre = ldexpf(C::kTop, -ex), inv = a > 0.f ? 1.f / f : 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const float n = finite ? (float)x[e] * pre : 0.f, t = n * inv;
      q[e] = (cached)rounded(C(), fmaf(fmaf(-t, f, n), inv, t));
    }
    return finite ? fminf(a / C::kTop, C::kMostScale) : __uint_as_float(0x7fc00000u);
  }
};

// What a thread works on: kItems rows of K and of V, their loads and look-ups in flight together, and its place in them.  A group of
// tokens has as many workgroups as there are heads, which take one head each (neighbours in a page, and in K and V where a row is
// whole lines), or, kInOrder, an equal part of the group's rows in the order of K and V, so that lines that rows share are stored
// by one workgroup: int8 rows of 80, 32 heads, 49152 tokens read 245 -> 190 us, e4m3 rows of 96 85 -> 81.  kTogether: the workgroups of a
// group on one XCD, whose L2 then serves both that share a line (60000 tokens of 32 heads of 80 written: bf16 into pages of 16 252 ->
// 240 us, pages of one 363 -> 248, int8 there 336 -> 291; 8300 e4m3 rows of 8 heads of 96 read 10.4 -> 9.4, fp32 rows of 33 110 -> 103),
// also where few groups leave XCDs out (32 heads of 80 quantised: 400 tokens 6.4 -> 5.5, 200 of 4 heads 4.0 and 4.0).
template <int kLanes, int kItems, bool kInOrder, bool kTogether> struct Work {
  int lane, t[kItems], g[kItems];  // token, head
  bool there[kItems];
  __device__ __forceinline__ Work(int first, int N, const FastDiv &heads, const FastDiv &lanes) {
    const int H = heads.d, tid = threadIdx.x, per_row = kLanes ? kLanes : (int)lanes.d, rows = kThreads / per_row;
    const int mine = kLanes ? tid / (kLanes ? kLanes : 1) : tid / lanes;  // row of this thread
    int group = (int)blockIdx.x / heads, head = (blockIdx.x - group * H + group) % heads;  // heads in turn across XCDs
    if constexpr (kTogether) {
      const int turn = blockIdx.x >> 3, eighth = turn / heads;
      group = eighth * 8 + (blockIdx.x & 7), head = turn - eighth * H;
    }
    lane = tid - mine * per_row;
    const long long tokens = N - first, begin = (long long)group * (rows * kItems);
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      long long at = begin + u * rows + mine;
      g[u] = head;
      if constexpr (kInOrder) {  // the head-th part of the rows of the group's tokens
        const int row = (head * kItems + u) * rows + mine, token = row / heads;
        at = begin + token, g[u] = row - token * H;
      }
      there[u] = mine < rows && at < tokens;
      t[u] = first + (there[u] ? (int)at : 0);
    }
  }
};

template <class E, class C, int kVec, int kLanes, bool kWhole, int kItems>
__global__ void __launch_bounds__(kThreads)
write_kernel(const typename E::elem *__restrict__ K, const typename E::elem *__restrict__ V, typename C::elem *__restrict__ Kc,
             typename C::elem *__restrict__ Vc, float *__restrict__ ks, float *__restrict__ vs, PageMap map,
             const int32_t *__restrict__ seq_ids, const void *__restrict__ pos, va_itype it, int first, int N, FastDiv heads, FastDiv lanes, int d) {
  typedef Row<E, C, kVec, kLanes, kWhole> R;
  constexpr bool kPast = kWhole && sizeof(typename C::elem) * kVec * kLanes % 128 == 0;
  const int H = heads.d;
  const Work<kLanes, kItems, false, !kWhole> work(first, N, heads, lanes);
  const int lane = work.lane;
  typename E::elem k[kItems][R::kPer], v[kItems][R::kPer];
  int place[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const size_t from = ((size_t)work.t[u] * H + work.g[u]) * d;
    R::load(K + from, lane, d, k[u]);
    R::load(V + from, lane, d, v[u]);
    place[u] = place_of(map, seq_ids ? seq_ids[work.t[u]] : work.t[u], id_at(pos, it, work.t[u]));
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    if (!work.there[u] || place[u] < 0) continue;
    const size_t row = (size_t)place[u] + (size_t)work.g[u] * map.page.d;
    if constexpr (is_8bit<C>::value) {
      typename C::elem q[R::kPer];
      const float sk = R::quantise(k[u], q);
      R::template store<kPast>(Kc + row * d, lane, d, q);
      const float sv = R::quantise(v[u], q);
      R::template store<kPast>(Vc + row * d, lane, d, q);
      if (lane == 0) {
        ks[row] = sk;
        vs[row] = sv;
      }
    } else {
      R::template store<kPast>(Kc + row * d, lane, d, k[u]);
      R::template store<kPast>(Vc + row * d, lane, d, v[u]);
    }
  }
}

template <class E, class C, int kVec, int kLanes, bool kWhole, int kItems>
__global__ void __launch_bounds__(kThreads)
read_kernel(typename E::elem *__restrict__ K, typename E::elem *__restrict__ V, const typename C::elem *__restrict__ Kc,
            const typename C::elem *__restrict__ Vc, const float *__restrict__ ks, const float *__restrict__ vs, PageMap map,
            const int32_t *__restrict__ seq_ids, const void *__restrict__ pos, va_itype it, int first, int N, FastDiv heads, FastDiv lanes, int d) {
  typedef Row<E, C, kVec, kLanes, kWhole> R;
  constexpr bool kInOrder = kLanes == 0, kPast = kInOrder ? kVec > 1 : sizeof(typename E::elem) * kVec * kLanes % 128 == 0;
  const int H = heads.d;
  const Work<kLanes, kItems, kInOrder, !kWhole> work(first, N, heads, lanes);
  const int lane = work.lane;
  typename C::elem k[kItems][R::kPer], v[kItems][R::kPer];
  float sk[kItems], sv[kItems];
  int place[kItems];
#pragma unroll
  for (int u = 0; u < kItems; ++u)
    place[u] = place_of(map, seq_ids ? seq_ids[work.t[u]] : work.t[u], id_at(pos, it, work.t[u]));
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const size_t row = (size_t)max(place[u], 0) + (size_t)work.g[u] * map.page.d;  // of page 0 where there is none
    R::load(Kc + row * d, lane, d, k[u]);
    R::load(Vc + row * d, lane, d, v[u]);
    if constexpr (is_8bit<C>::value) sk[u] = ks[row], sv[u] = vs[row];
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    if (!work.there[u]) continue;
    typename E::elem x[R::kPer], y[R::kPer];
#pragma unroll
    for (int e = 0; e < R::kPer; ++e) {
      x[e] = y[e] = (typename E::elem)0.f;
      if (place[u] >= 0) {
        if constexpr (is_8bit<C>::value) {
          x[e] = (typename E::elem)(cached_to_f32(C(), k[u][e]) * sk[u]);
          y[e] = (typename E::elem)(cached_to_f32(C(), v[u][e]) * sv[u]);
        } else {
          x[e] = k[u][e], y[e] = v[u][e];
        }
      }
    }
    const size_t to = ((size_t)work.t[u] * H + work.g[u]) * d;
    R::template store<kPast>(K + to, lane, d, x);
    R::template store<kPast>(V + to, lane, d, y);
  }
}

struct Call {
  const void *K, *V;  // written to by a read
  const va_kv_cache &c;
  const int32_t *seq_ids;
  const void *pos;
  va_itype it;
  int N;
  bool write;
  hipStream_t stream;
};

template <class E, class C, int kVec, int kLanes, bool kWhole, int kItems> hipError_t launch_rows(const Call &a) {
  typedef typename E::elem elem;
  typedef typename C::elem cached;
  constexpr bool kWrites = kLanes > 0 || !is_8bit<C>::value, kReads = kLanes == 0 || kWhole;  // see launch_ec
  const FastDiv heads = fast_div(a.c.hkv), lanes = fast_div(kLanes ? kLanes : a.c.d / kVec);
  const PageMap map = page_map(a.c);
  const int rows = kThreads / (int)lanes.d * kItems;                                   // of a workgroup
  // tokens of a launch: its workgroups (rounded up, see below), and its rows in 31 bits
  const long long most = std::min((kMostWorkgroups / a.c.hkv - 7) * rows, 0x7fffffffll / a.c.hkv);
  for (long long first = 0; first < a.N; first += most) {
    const long long end = std::min(first + most, (long long)a.N);
    long long groups = (end - first + rows - 1) / rows;
    if (!kWhole) groups = (groups + 7) / 8 * 8;  // a group of each XCD at a time
    const unsigned workgroups = (unsigned)(groups * a.c.hkv);
    if constexpr (kWrites)
      if (a.write)
        write_kernel<E, C, kVec, kLanes, kWhole, kItems><<<workgroups, kThreads, 0, a.stream>>>(
            (const elem *)a.K, (const elem *)a.V, (cached *)a.c.k, (cached *)a.c.v, a.c.k_scale, a.c.v_scale, map, a.seq_ids, a.pos, a.it,
            (int)first, (int)end, heads, lanes, a.c.d);
    if constexpr (kReads)
      if (!a.write)
        read_kernel<E, C, kVec, kLanes, kWhole, kItems><<<workgroups, kThreads, 0, a.stream>>>(
            (elem *)a.K, (elem *)a.V, (const cached *)a.c.k, (const cached *)a.c.v, a.c.k_scale, a.c.v_scale, map, a.seq_ids, a.pos, a.it,
            (int)first, (int)end, heads, lanes, a.c.d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Rows of 8 bits are short enough for two in flight, once there are workgroups for several rounds: 65536 tokens of 32 heads read back
// 412 -> 390 us; 8300 of 8 heads 11.5, with two 12.7, 20 of 4 heads 3.5 and 4.1.
template <class E, class C, int kVec, int kLanes, bool kWhole> hipError_t launch(const Call &a) {
  constexpr long long kFill = 1 << 18;
  if constexpr (is_8bit<C>::value && kVec > 1)
    if ((long long)a.N * a.c.hkv >= kFill) return launch_rows<E, C, kVec, kLanes, kWhole, 2>(a);
  return launch_rows<E, C, kVec, kLanes, kWhole, 1>(a);
}

// Chunks of 16 bytes of K and V where the rows of both sides consist of whole aligned ones, else single elements.  Lanes of a row: 8, 16,
// 32 or 64 where that is all of it; otherwise as many as it has chunks, unless it is quantised.
template <class E, class C> hipError_t launch_ec(const Call &a) {
  constexpr int kVec = 16 / sizeof(typename E::elem);
  constexpr bool k64 = kVec == 4;  // rows of 64 chunks: d <= 256
  const uintptr_t cached_at = (uintptr_t)a.c.k | (uintptr_t)a.c.v, rows_at = (uintptr_t)a.K | (uintptr_t)a.V;
  const bool wide = a.c.d % kVec == 0 && rows_at % 16 == 0 && cached_at % (kVec * sizeof(typename C::elem)) == 0;
  const int chunks = a.c.d / kVec;
  if (wide) {
    if (chunks == 8) return launch<E, C, kVec, 8, true>(a);
    if (chunks == 16) return launch<E, C, kVec, 16, true>(a);
    if (chunks == 32) return launch<E, C, kVec, 32, true>(a);
    if constexpr (k64)
      if (chunks == 64) return launch<E, C, kVec, 64, true>(a);
  }
  if constexpr (is_8bit<C>::value) {
    if (a.write && !wide) return launch<E, C, 1, 64, false>(a);
    if (a.write && chunks < 8) return launch<E, C, kVec, 8, false>(a);
    if (a.write && chunks < 16) return launch<E, C, kVec, 16, false>(a);
    if (a.write && (!k64 || chunks < 32)) return launch<E, C, kVec, 32, false>(a);
    if constexpr (k64)
      if (a.write) return launch<E, C, kVec, 64, false>(a);
  }
  return wide ? launch<E, C, kVec, 0, false>(a) : launch<E, C, 1, 0, false>(a);
}
template <class E> hipError_t launch_e(const Call &a) {
  if (a.c.format == VA_CACHE_I8) return launch_ec<E, I8>(a);
  if (a.c.format == VA_CACHE_E4M3) return launch_ec<E, E4m3>(a);
  return launch_ec<E, E>(a);
}
hipError_t launch_dt(va_dtype dt, const Call &a) {
  return dt == VA_BF16 ? launch_e<Bf16>(a) : dt == VA_F16 ? launch_e<F16>(a) : launch_e<F32>(a);
}

}  // namespace

hipError_t launch_cache_write(const void *K, const void *V, va_dtype dt, const va_kv_cache &cache, const int32_t *seq_ids,
                              const void *pos, va_itype it, int N, hipStream_t stream) {
  return launch_dt(dt, {K, V, cache, seq_ids, pos, it, N, true, stream});
}
hipError_t launch_cache_read(void *K, void *V, va_dtype dt, const va_kv_cache &cache, const int32_t *seq_ids, const void *pos,
                             va_itype it, int N, hipStream_t stream) {
  return launch_dt(dt, {K, V, cache, seq_ids, pos, it, N, false, stream});
}

}  // namespace va
