// Attention of one token over the key-value cache, queries in bf16 (va_paged.h).
#include "va_paged.h"

void va::paged::launch_bf16(const Args &a, va_cache_format format, unsigned workgroups, hipStream_t stream) {
  launch_queries<Bf16>(a, format, workgroups, stream);
}
