// Host-side launchers of the windowed-attention and cache kernels; each enqueues on `s` and returns hipGetLastError().
#pragma once
#include "window_common.h"

namespace vsa {

constexpr int kPage = 64;           // tokens of a cache page
constexpr int kLowestScale = -60;   // exponent of the smallest scale a page gets

// The 8-bit cache.  Page p, key head h: keys [64][d], values [d][64], one scale each.
struct CacheArgs {
  uint8_t *k, *v;
  float *ks, *vs;
  const int32_t* table;  // [B, max_pages]: pages of a sequence; entries outside [0, pages) name nothing
  const int32_t* lens;   // [B]
  int max_pages, pages;
};

struct AppendArgs {
  CacheArgs c;
  int B, Hkv, d, f16;
  WinRows rows;  // of the new tokens
  RowView k, v;
};

// `parts`: row_parts(a, longest keys, d) floats
hipError_t launch_window_fwd(const WinArgs& a, int d, bool f16, float* parts, hipStream_t s);
size_t row_parts(const WinArgs& a, long long max_k, int d);
// `parts`: window_parts(a, d) floats
hipError_t launch_window_bwd(const WinArgs& a, int d, bool f16, float* parts, hipStream_t s);
size_t window_parts(const WinArgs& a, int d);
hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s);
// many rows a key head: the walk of launch_window_fwd over pages; `parts`: row_parts(a, max_pages * kPage, d) floats
hipError_t launch_cache_chunk(const WinArgs& a, const CacheArgs& c, int d, bool f16, float* parts, hipStream_t s);
// few rows (16 at a time): the keys split over workgroups, joined behind them.  `parts`: cache_parts(...) floats
hipError_t launch_cache_token(const WinArgs& a, const CacheArgs& c, int d, bool f16, float* parts, hipStream_t s);
size_t cache_parts(int B, int H, int Hkv, int d, int max_q, int max_pages);

}  // namespace vsa
