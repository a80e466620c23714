// Attention of one token over the key-value cache, queries in f32 (va_paged.h).
#include "va_paged.h"

void va::paged::launch_f32(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream) {
  launch_queries<F32>(a, format, workgroups, stream);
}
