// Attention of one new token of every sequence over the paged key-value cache.
//
// One workgroup per (sequence, query head): 16 groups of 16 lanes take a key each, every 16th key one group's; a lane holds up to
// 16 columns of q, of the key and of the sum.  Every group keeps the running maximum and sum of its softmax in fp32; they are
// joined at the end.
#include "va_kv_cache.h"

namespace va {
namespace {

constexpr int kThreads = 256, kLanes = 16, kGroups = kThreads / kLanes, kPer = 256 / kLanes;

template <class E, class C>
__global__ void __launch_bounds__(kThreads)
paged_kernel(const typename E::elem *__restrict__ Q, typename E::elem *__restrict__ O, float *__restrict__ LSE,
             const typename C::elem *__restrict__ Kc, const typename C::elem *__restrict__ Vc, const float *__restrict__ ks,
             const float *__restrict__ vs, PageMap map, const int32_t *__restrict__ lens, int hq, int d, float scale) {
  __shared__ float all_m[kGroups], all_l[kGroups], all_o[kGroups][256];
  const int b = blockIdx.x, h = blockIdx.y, g = h / (hq / map.hkv);
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int n = min(max(lens[b], 0), map.capacity);
  const size_t at = ((size_t)b * hq + h) * d;
  float q[kPer], o[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int c = lane + e * kLanes;
    q[e] = c < d ? (float)Q[at + c] : 0.f;
    o[e] = 0.f;
  }
  for (int j = group; j < n; j += kGroups) {
    const int place = place_of(map, b, j);
    if (place < 0) continue;
    const size_t row = (size_t)place + (size_t)g * map.page.d;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int c = lane + e * kLanes;
      if (c < d) s = fmaf(q[e], cached_to_f32(C(), Kc[row * d + c]), s);
    }
#pragma unroll
    for (int x = 1; x < kLanes; x *= 2) s += __shfl_xor(s, x, kLanes);
    float vscale = 1.f;
    if constexpr (is_8bit<C>::value) s *= ks[row], vscale = vs[row];
    s *= scale;
    const float m_new = fmaxf(m, s), alpha = m == -INFINITY ? 0.f : __expf(m - m_new);
    const float p = s == -INFINITY ? 0.f : __expf(s - m_new);  // a NaN stays one
    m = m_new;
    l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int c = lane + e * kLanes;
      if (c < d) o[e] = fmaf(p * vscale, cached_to_f32(C(), Vc[row * d + c]), o[e] * alpha);
    }
  }
  if (lane == 0) all_m[group] = m, all_l[group] = l;
#pragma unroll
  for (int e = 0; e < kPer; ++e) all_o[group][lane + e * kLanes] = o[e];
  __syncthreads();
  float top = -INFINITY, sum = 0.f, x = 0.f;
  for (int i = 0; i < kGroups; ++i) top = fmaxf(top, all_m[i]);
  for (int i = 0; i < kGroups; ++i) {
    const float w = all_m[i] == -INFINITY ? 0.f : __expf(all_m[i] - top);
    sum += w * all_l[i];
    x += w * all_o[i][threadIdx.x];
  }
  if ((int)threadIdx.x < d) O[at + threadIdx.x] = (typename E::elem)(sum != 0.f ? x / sum : 0.f);
  if (threadIdx.x == 0) LSE[(size_t)h * map.n_seqs + b] = sum != 0.f ? top + __logf(sum) : -INFINITY;
}

template <class E, class C>
hipError_t launch(const void *Q, void *O, float *LSE, const va_kv_cache &c, int hq, const int32_t *lens, float scale, hipStream_t stream) {
  paged_kernel<E, C><<<dim3((unsigned)c.n_seqs, (unsigned)hq), kThreads, 0, stream>>>(
      (const typename E::elem *)Q, (typename E::elem *)O, LSE, (const typename C::elem *)c.k, (const typename C::elem *)c.v, c.k_scale,
      c.v_scale, page_map(c), lens, hq, c.d, scale);
  return hipGetLastError();
}
template <class E>
hipError_t launch_e(const void *Q, void *O, float *LSE, const va_kv_cache &c, int hq, const int32_t *lens, float scale, hipStream_t stream) {
  if (c.format == VA_CACHE_I8) return launch<E, I8>(Q, O, LSE, c, hq, lens, scale, stream);
  if (c.format == VA_CACHE_E4M3) return launch<E, E4m3>(Q, O, LSE, c, hq, lens, scale, stream);
  return launch<E, E>(Q, O, LSE, c, hq, lens, scale, stream);
}

}  // namespace

size_t paged_workspace_bytes(int, long long, int, int, int) { return 0; }

hipError_t launch_paged(const void *Q, void *O, float *LSE, va_dtype dt, const va_kv_cache &c, int hq, const int32_t *lens,
                        float scale, float *, hipStream_t stream) {
  return dt == VA_BF16 ? launch_e<Bf16>(Q, O, LSE, c, hq, lens, scale, stream)
         : dt == VA_F16 ? launch_e<F16>(Q, O, LSE, c, hq, lens, scale, stream)
                        : launch_e<F32>(Q, O, LSE, c, hq, lens, scale, stream);
}

}  // namespace va
