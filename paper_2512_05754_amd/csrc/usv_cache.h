// The quantised key/value cache: layout, arguments.
//
// cache[page][head]: K codes [page_size][d * bits / 8], V codes, K scales [page_size][d / 32], V scales, one behind the other.  32
// neighbouring channels of a row share the scale 2^(byte - 127), byte 255: the group held an infinity or a NaN.  Codes: e2m1, two to
// a byte, the even channel in the low half; or e4m3.
#pragma once

#include "usv_window.h"

namespace usv {

struct CacheShape {
  int B, H, d, bits, page_size, pages, table_pages;
  const int32_t* table;  // [B, table_pages]
  Div by_page, by_groups;  // page_size; page_size / 16
  __host__ __device__ int code_bytes() const { return d * bits / 8; }
  __host__ __device__ int scale_bytes() const { return d / 32; }
  __host__ __device__ long long head_bytes() const { return 2LL * page_size * (code_bytes() + scale_bytes()); }
};

struct CacheRowsArgs {  // cache_write, cache_read
  CacheShape c;
  unsigned char* cache;
  const int32_t *starts, *counts;  // position of row 0 of each sequence; rows that count (NULL: all)
  int rows;
  void *k, *v;
  Strides3 sk, sv;
};

struct CacheAttnArgs {
  CacheShape c;
  const unsigned char* cache;
  WindowArgs f;  // q, out, lse, pieces; k, v unused
};

constexpr int kCacheGroup = 16;  // keys of a page that are looked up together; page_size is a multiple

hipError_t launch_cache_write(const CacheRowsArgs& a, bool bf16, hipStream_t st);
hipError_t launch_cache_read(const CacheRowsArgs& a, bool bf16, hipStream_t st);
// query rows (tokens x the heads that share a key head) of a workgroup: 16, or 64 where that many are at hand
inline int cache_attn_rows(const WindowShape& w) { return (long long)w.Lq * w.group > 32 ? 64 : 16; }
// the keys that some query row sees (window_all_keys), in bf16, to k, v [B, heads, rows, d] of a
hipError_t launch_cache_expand(const CacheRowsArgs& a, const WindowShape& w, hipStream_t st);
hipError_t launch_cache_attn(const CacheAttnArgs& a, hipStream_t st);

}  // namespace usv
