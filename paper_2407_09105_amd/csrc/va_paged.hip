// Attention of one new token of every sequence over the paged key-value cache: how the work is cut, and the parts of cut sequences
// joined.  The kernel that does the work is in va_paged.h.
#include <algorithm>

#include "va_paged.h"

namespace va {
namespace paged {

// Workgroups that the parts should make where the lengths allow it: 256 CUs hold 768.
constexpr int kWorkgroups = 1024;
constexpr int kLeastUnits = 2;

Split split_of(int n_seqs, long long capacity, int hq, int hkv) {
  const int groups = ceil_div(hq / hkv, kHeads);
  const long long least = kLeastUnits * kUnit, most = n_seqs * ((capacity + least - 1) / least);  // parts that there can be
  const long long room = (kWorkgroups + (long long)hkv * groups - 1) / ((long long)hkv * groups);
  if (capacity <= least) return {n_seqs, kLeastUnits};
  return {n_seqs + (int)std::min(room, most), kLeastUnits};
}

namespace {

// One workgroup per (sequence, query head): the parts' sums, relative to the largest reference exponent, added in order.
template <class E>
__global__ void __launch_bounds__(kThreads)
join_kernel(typename E::elem *__restrict__ O, float *__restrict__ LSE, Workspace ws, const int32_t *__restrict__ lens, PageMap map,
            Split split, int hq, int d) {
  const int b = blockIdx.x, head = blockIdx.y;
  Part part;
  if (!find_part(lens, map, split, -1, b, part) || part.parts == 1) return;
  const float2 *const ml = ws.ml + (size_t)part.first * hq + head;
  const float *const o = ws.o + ((size_t)part.first * hq + head) * d;
  float top = -INFINITY;
  for (int x = 0; x < part.parts; ++x) top = fmaxf(top, ml[(size_t)x * hq].x);
  float sum = 0.f, y = 0.f;
  const int c = threadIdx.x;
  for (int x = 0; x < part.parts; ++x) {
    const float2 one = ml[(size_t)x * hq];
    const float weight = one.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(one.x - top);
    sum += weight * one.y;
    if (c < d) y += weight * o[(size_t)x * hq * d + c];
  }
  if (c < d) O[((size_t)b * hq + head) * d + c] = (typename E::elem)(sum != 0.f ? y / sum : 0.f);
  if (c == 0) LSE[(size_t)head * map.n_seqs + b] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace
}  // namespace paged

size_t paged_workspace_bytes(int n_seqs, long long capacity, int hq, int hkv, int d) {
  const paged::Split s = paged::split_of(n_seqs, capacity, hq, hkv);
  return s.slots == n_seqs ? 0 : ((size_t)s.slots * hq * d + 1) / 2 * 2 * sizeof(float) + (size_t)s.slots * hq * sizeof(float2);
}

hipError_t launch_paged(const void *Q, void *O, float *LSE, va_dtype dt, const va_kv_cache &c, int hq, const int32_t *lens, float scale,
                        float *work, hipStream_t stream) {
  using namespace paged;
  const Split split = split_of(c.n_seqs, (long long)c.max_pages * c.page_size, hq, c.hkv);
  const Workspace ws = workspace(work, split, hq, c.d);
  const Args a = {Q, O, LSE, c.k, c.v, c.k_scale, c.v_scale, page_map(c), lens, split, ws, hq, c.d, scale * 1.4426950408889634f};
  const long long groups = ceil_div(hq / c.hkv, kHeads), workgroups = ((long long)split.slots * c.hkv + 7) / 8 * 8 * groups;
  if (workgroups > 0x7fffffffll) return hipErrorInvalidValue;
  (dt == VA_BF16 ? launch_bf16 : dt == VA_F16 ? launch_f16 : launch_f32)(a, c.format, (unsigned)workgroups, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || split.slots == c.n_seqs) return e;
  const dim3 grid((unsigned)c.n_seqs, (unsigned)hq);
  if (dt == VA_BF16) join_kernel<Bf16><<<grid, kThreads, 0, stream>>>((__bf16 *)O, LSE, ws, lens, a.map, split, hq, c.d);
  else if (dt == VA_F16) join_kernel<F16><<<grid, kThreads, 0, stream>>>((_Float16 *)O, LSE, ws, lens, a.map, split, hq, c.d);
  else join_kernel<F32><<<grid, kThreads, 0, stream>>>((float *)O, LSE, ws, lens, a.map, split, hq, c.d);
  return hipGetLastError();
}

}  // namespace va
