// Attention of one new token of every sequence over the paged key-value cache: how the work is cut, and the parts of cut sequences
// joined.  The kernel that does the work is in va_paged.h.
#include <algorithm>

#include "va_paged.h"

namespace va {
namespace paged {

// Workgroups that the cuts should add, where the lengths allow it, to the one that every sequence has for each KV head.  A few
// sequences have equal parts, and two workgroups per CU of them are as fast as four (256 CUs hold 768): 131072 keys of 8 heads of 128
// 85 us with either, but 8.7 or 5.8 for the joining; 4 x 30000 of 2 heads of 256 60 us in all with 1024 and 50 with 512.  Sequences
// of different lengths leave their last parts, which finer ones even out: 128 of 1024 to 8192 tokens, 8 heads, 232 us with 1024 and
// 220 with 2048, 33 of 4096, 32 heads of 64, 227 and 213; 4096 gain nothing more.
// At most kMorePerPair of the additional ones for each sequence and KV head: 8 sequences of 1024 to 16384, 8 heads, 59.5, 56.6, 53.6 and 57.3 us
// with 1, 2, 4 and 8; 48 of about 700 40.3, 38.7, 37.6 and 37.8; 131072 keys, whose parts are equal anyway, 88 with 4 and 103 with 8.
constexpr int kWorkgroups = 512, kMoreWorkgroups = 1536, kMorePerPair = 4;
// Least units of a part (of one, two and four): 1500 keys, 8 heads of 128, 10.1, 11.3 and 14.1 us; 4 sequences of 500 to 2000 12.1, 12.2 and 15.1; 20
// of up to 2500, 4 int8 heads of 80, 18.3, 15.4 and 16.4; 33 of up to 3001, one int8 head of 64, 13.7, 14 and 16.8.
constexpr int kLeastUnits = 2;
constexpr int kUncut = 512;    // sequences times KV heads that fill the chip in one piece each
// Up to this much room for more parts than one of each sequence (the host does not know how many there are), parts are joined by one wave
// for each head: 128 sequences, 40 heads, two parts 10.9 -> 4.8 us, 3 sequences of up to eight 3.9 -> 3.4; with 128 parts (one
// sequence) a workgroup takes 9 us.
constexpr int kFewParts = 8;   // a sequence

Split split_of(int n_seqs, long long capacity, int hq, int hkv) {
  const int groups = ceil_div(hq / hkv, kHeads);
  const long long least = kLeastUnits * kUnit, most = n_seqs * ((capacity + least - 1) / least);  // parts that there can be
  const long long each = (long long)hkv * groups, more = std::min<long long>(kMoreWorkgroups, kMorePerPair * n_seqs * each);
  const long long room = (kWorkgroups + more + each - 1) / each;
  // Short contexts are not cut, which saves the joining: 480 keys, 32/8 heads of 128, one sequence 9.8 -> 8.0 us, 64 of them 27 -> 21;
  // 900 keys, one sequence 10.1 (uncut 12), 64 of them 45 -> 38: there workgroups are enough without.
  if (capacity <= (n_seqs * each >= kUncut ? 8 : 4) * kUnit) return {n_seqs, kLeastUnits, fast_div(1)};
  const int extra = (int)std::min(room, most);
  return {n_seqs + extra, kLeastUnits, fast_div(extra)};
}

namespace {

// One workgroup per (sequence, query head) adds up the parts' sums, weighted relative to the largest reference score: every
// kJoinRows-th part one group of threads', a column each, and then the groups' sums in order.
constexpr int kMostParts = kWorkgroups + kMoreWorkgroups + 1;  // of one sequence

template <class E, int kCols>  // kCols: threads of a group, d rounded up to 64, 128 or 256
__global__ void __launch_bounds__(kThreads)
join_kernel(typename E::elem *__restrict__ O, float *__restrict__ LSE, Workspace ws, int n_seqs, int hq, int d, float scale, float scale_log2) {
  constexpr int kJoinRows = kThreads / kCols, kFly = 8;  // parts in flight
  __shared__ float weight[kMostParts], some[2][kThreads];
  const int b = blockIdx.x, head = blockIdx.y, t = threadIdx.x;
  const int2 of = ws.parts[b];
  const int first = of.x, parts = of.y;
  if (parts == 1) return;  // its only workgroup has written the result
  const float2 *const ml = ws.ml + (size_t)first * hq + head;
  const int c = t % kCols, x1 = t / kCols;  // this thread's column and first part
  const float *const o = ws.o + ((size_t)first * hq + head) * d + min(c, d - 1);
  float v[kFly];
  auto load = [&](int x0) {
#pragma unroll
    for (int k = 0; k < kFly; ++k) v[k] = o[(size_t)min(x0 + k * kJoinRows, parts - 1) * hq * d];
  };
  load(x1);  // on their way before the weights are known
  float2 mine[(kMostParts + kThreads - 1) / kThreads];
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k * kThreads < kMostParts; ++k) {
    const int x = t + k * kThreads;
    mine[k] = x < parts ? ml[(size_t)x * hq] : make_float2(-INFINITY, 0.f);
    top = fmaxf(top, mine[k].x);
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  if (t % 64 == 0) some[0][t / 64] = top;
  __syncthreads();
  top = fmaxf(fmaxf(some[0][0], some[0][1]), fmaxf(some[0][2], some[0][3]));
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k * kThreads < kMostParts; ++k) {
    const int x = t + k * kThreads;
    const float w = mine[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine[k].x - top) * scale_log2);
    if (x < parts) weight[x] = w;
    sum += w * mine[k].y;
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o);
  if (t % 64 == 0) some[1][t / 64] = sum;
  __syncthreads();
  sum = some[1][0] + some[1][1] + some[1][2] + some[1][3];
  float y = 0.f;
  for (int x0 = x1; x0 < parts; x0 += kJoinRows * kFly) {
#pragma unroll
    for (int k = 0; k < kFly; ++k)
      if (x0 + k * kJoinRows < parts) y += weight[x0 + k * kJoinRows] * v[k];
    load(x0 + kJoinRows * kFly);
  }
  if constexpr (kJoinRows > 1) {
    __syncthreads();  // both of `some` are read
    some[0][t] = y;
    __syncthreads();
    y = 0.f;
#pragma unroll
    for (int k = 0; k < kJoinRows; ++k) y += some[0][k * kCols + c];
  }
  if (t < d) O[((size_t)b * hq + head) * d + t] = (typename E::elem)(sum != 0.f ? y / sum : 0.f);
  if (t == 0) LSE[(size_t)head * n_seqs + b] = lse_of(top, sum, scale);
}

// The same by one wave per (sequence, query head), four of them in a workgroup, for batches in which there is room for few parts a sequence: a
// column per lane and 64 of d, the weights of 64 parts at a time in the lanes.
template <class E, int kCols>
__global__ void __launch_bounds__(kThreads)
join_few_kernel(typename E::elem *__restrict__ O, float *__restrict__ LSE, Workspace ws, int n_seqs, int hq, int d, float scale, float scale_log2) {
  constexpr int kOwn = kCols / 64, kFly = 4;
  const int b = blockIdx.x, head = blockIdx.y * kWaves + uniform(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (head >= hq) return;
  const int2 of = ws.parts[b];
  const int first = uniform(of.x), parts = uniform(of.y);
  if (parts == 1) return;
  const float2 *const ml = ws.ml + (size_t)first * hq + head;
  const float *const o = ws.o + ((size_t)first * hq + head) * d;
  float top = -INFINITY;
  for (int x = lane; x < parts; x += 64) top = fmaxf(top, ml[(size_t)x * hq].x);
#pragma unroll
  for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
  float sum = 0.f, y[kOwn] = {};
  for (int x0 = 0; x0 < parts; x0 += 64) {
    const int x = x0 + lane;
    const float2 one = x < parts ? ml[(size_t)x * hq] : make_float2(-INFINITY, 0.f);
    const float weight = one.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((one.x - top) * scale_log2);
    sum += weight * one.y;
    const int many = min(parts - x0, 64);
    for (int k0 = 0; k0 < many; k0 += kFly) {
      float v[kFly][kOwn];
#pragma unroll
      for (int k = 0; k < kFly; ++k)
#pragma unroll
        for (int e = 0; e < kOwn; ++e) v[k][e] = o[(size_t)(x0 + min(k0 + k, many - 1)) * hq * d + min(lane + 64 * e, d - 1)];
#pragma unroll
      for (int k = 0; k < kFly; ++k) {
        if (k0 + k >= many) continue;
        const float w = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(weight), k0 + k));
#pragma unroll
        for (int e = 0; e < kOwn; ++e) y[e] += w * v[k][e];
      }
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
#pragma unroll
  for (int e = 0; e < kOwn; ++e)
    if (lane + 64 * e < d) O[((size_t)b * hq + head) * d + lane + 64 * e] = (typename E::elem)(sum != 0.f ? y[e] / sum : 0.f);
  if (lane == 0) LSE[(size_t)head * n_seqs + b] = lse_of(top, sum, scale);
}

template <class E> void launch_join(void *O, float *LSE, const Workspace &ws, const Split &split, int n_seqs, int hq, int d, float scale,
                                    float scale_log2, hipStream_t stream) {
  const dim3 grid((unsigned)n_seqs, (unsigned)hq);
  typename E::elem *const o = (typename E::elem *)O;
  if ((int)split.extra.d <= kFewParts * n_seqs) {
    const dim3 few((unsigned)n_seqs, (unsigned)ceil_div(hq, kWaves));
    if (d <= 64) join_few_kernel<E, 64><<<few, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
    else if (d <= 128) join_few_kernel<E, 128><<<few, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
    else join_few_kernel<E, 256><<<few, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
    return;
  }
  if (d <= 64) join_kernel<E, 64><<<grid, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
  else if (d <= 128) join_kernel<E, 128><<<grid, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
  else join_kernel<E, 256><<<grid, kThreads, 0, stream>>>(o, LSE, ws, n_seqs, hq, d, scale, scale_log2);
}

}  // namespace
}  // namespace paged

size_t paged_workspace_bytes(int n_seqs, long long capacity, int hq, int hkv, int d) {
  return paged::workspace_bytes(paged::split_of(n_seqs, capacity, hq, hkv), n_seqs, hq, d);
}

hipError_t launch_paged(const void *Q, void *O, float *LSE, va_dtype dt, const va_kv_cache &c, int hq, const int32_t *lens, float scale,
                        float *work, hipStream_t stream) {
  using namespace paged;
  const Split split = split_of(c.n_seqs, (long long)c.max_pages * c.page_size, hq, c.hkv);
  const Workspace ws = workspace(work, split, c.n_seqs, hq);
  const int G = hq / c.hkv, groups = ceil_div(G, kHeads);
  const Args a = {Q, O, LSE, c.k, c.v, c.k_scale, c.v_scale, page_map(c), lens, split, ws, fast_div(c.hkv), fast_div(groups), hq, G, c.d, scale,
                  scale * 1.4426950408889634f};
  const long long workgroups = ((long long)split.slots * c.hkv + 7) / 8 * 8 * groups;
  if (workgroups > kMostWorkgroups) return hipErrorInvalidValue;
  (dt == VA_BF16 ? launch_bf16 : dt == VA_F16 ? launch_f16 : launch_f32)(a, c.format, (unsigned)workgroups, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || split.slots == c.n_seqs) return e;
  (dt == VA_BF16 ? launch_join<Bf16> : dt == VA_F16 ? launch_join<F16> : launch_join<F32>)(O, LSE, ws, split, c.n_seqs, hq, c.d, scale,
                                                                                            a.scale_log2, stream);
  return hipGetLastError();
}

}  // namespace va
