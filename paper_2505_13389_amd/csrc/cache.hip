// The 8-bit cache: new tokens into its pages, and attention of few query rows over them.
#include "window_kernels.h"
#include "window_tile.h"

namespace vsa {

// ---------------------------------------------------------------------------------------------------------------
// Append.  One workgroup per (sequence, page the new tokens touch, key head): it has the page to itself, so the scale is a
// maximum over a workgroup and nothing is ordered by atomics.  Scales are powers of two: e4m3 is a floating format, so a
// finer scale would not make its values any more precise (only the smallest ones), dividing by a power of two is exact, and
// so is moving a page that holds tokens to a larger scale, but for values that become subnormal.
// A thread holds 4 tokens x 8 elements: K goes out as 8 bytes a token, V is transposed through LDS, 4 tokens to a dword.
// Bound by HBM: 2 bytes in and 1 out a value.  75600 tokens, 40 heads, d = 128: 410 us, 5.7 TB/s of both ways; a frame of 1560
// tokens for two sequences, 12 heads: 8.2 us in the kernel; a token for 16 sequences: 5.7, start, one trip to memory, the maximum and the stores.

// the smallest power of two that brings `top` (finite, not negative) to 448 = 0.875 * 2^9 or less
__device__ __forceinline__ float page_scale(float top) {
  const uint32_t u = __float_as_uint(top);
  int e = (int)(u >> 23) - 126;  // top = m * 2^e with m in [0.5, 1); subnormals of fp32 end below the smallest scale
  e += (u & 0x7fffffu) > 0x600000u ? 1 : 0;
  return __uint_as_float((uint32_t)(max(e - 9, kLowestScale) + 127) << 23);
}
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  uint32_t r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// four e4m3 values times a power of two
__device__ __forceinline__ uint32_t rescaled(uint32_t u, float f) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
  return to_e4m3(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float finite_or_nan(float x) { return x - x == 0.f ? x : __uint_as_float(0x7fc00000u); }

// LARGE: every XCD takes a contiguous run of the launch (pages and heads whose rows lie side by side), and what is written goes past the
// caches: 75600 tokens, 40 heads, d = 128 454 -> 412 us.
template <int D, bool F16, bool LARGE>
__global__ __launch_bounds__(2 * D) void k_cache_append(AppendArgs a, int most_pages) {
  constexpr int CPR = D / 8, NT = 2 * D, NWV = NT / 64;
  __shared__ float top_of[2][NWV];
  __shared__ uint32_t tile[D * 16];  // V: [dv][16 dwords of 4 tokens], 16-byte chunks swizzled
  const unsigned block = LARGE ? xcd_chunked_id(blockIdx.x, gridDim.x) : blockIdx.x;
  const int head = (int)(block % (unsigned)a.Hkv), rest = (int)(block / (unsigned)a.Hkv);  // (rows of all heads lie side by side)
  const int slot_page = rest % most_pages, b = rest / most_pages;
  const WinSeq seq = win_seq(a.rows, b);
  const int start = max(0, min(a.c.lens[b], a.c.max_pages * kPage));
  const int page = start / kPage + slot_page;
  if (seq.n == 0 || page >= a.c.max_pages || page * kPage - start >= seq.n) return;
  const int lo = max(0, start - page * kPage), hi = min(kPage, start + seq.n - page * kPage);
  const long long first = seq.row0 + page * kPage - start;  // row of slot 0
  const int tid = threadIdx.x, c = tid % CPR, r4 = tid / CPR * 4;
  uint4 raw[2][4];
  float x[2][4][8];
  float top[2] = {0.f, 0.f};
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int slot = r4 + i;
      uint4 u = {0, 0, 0, 0};
      if (slot >= lo && slot < hi) u = *((const uint4*)(t ? a.v : a.k).row(b, first + slot, head) + c);
      raw[t][i] = u;
    }
  const int id = a.c.table[(long long)b * a.c.max_pages + page];  // (on its way together with the rows)
  if ((unsigned)id >= (unsigned)a.c.pages) return;
  const long long ph = (long long)id * a.Hkv + head;
  uint8_t* const kp = a.c.k + ph * (kPage * D);
  uint8_t* const vp = a.c.v + ph * (kPage * D);

#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      widen8<F16>(raw[t][i], x[t][i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[t][i][e] = finite_or_nan(x[t][i][e]);  // (fmaxf takes the other operand where one is NaN)
        top[t] = fmaxf(top[t], fabsf(x[t][i][e]));
      }
    }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) top[t] = fmaxf(top[t], __shfl_xor(top[t], m));
    if ((tid & 63) == 0) top_of[t][tid >> 6] = top[t];
  }
  __syncthreads();
  float scale[2], ratio[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int w = 0; w < NWV; ++w) top[t] = fmaxf(top[t], top_of[t][w]);
    scale[t] = page_scale(top[t]);
    ratio[t] = 1.f;
    float* const at = (t ? a.c.vs : a.c.ks) + ph;
    if (lo > 0) {  // tokens are there: their scale stays unless the new ones need a larger one
      const float was = *at;
      if (was >= scale[t]) scale[t] = was;
      else ratio[t] = was / scale[t];
    }
  }
  __syncthreads();  // (every thread has read the old scales)
  if (tid < 2) (tid ? a.c.vs : a.c.ks)[ph] = scale[tid];

  const float ik = 1.f / scale[0], iv = 1.f / scale[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = r4 + i;
    uint2* const p = (uint2*)(kp + slot * D) + c;
    if (slot >= lo && slot < hi) {
      const float* f = x[0][i];
      const u32x2 u = {to_e4m3(f[0] * ik, f[1] * ik, f[2] * ik, f[3] * ik), to_e4m3(f[4] * ik, f[5] * ik, f[6] * ik, f[7] * ik)};
      if (LARGE) __builtin_nontemporal_store(u, (u32x2*)p);
      else *(u32x2*)p = u;
    } else if (slot < lo && ratio[0] != 1.f) {
      const uint2 u = *p;
      *p = make_uint2(rescaled(u.x, ratio[0]), rescaled(u.y, ratio[0]));
    }
  }
  auto place = [](int dv, int chunk) { return dv * 16 + ((chunk ^ ((dv >> 3) & 3)) << 2); };
#pragma unroll
  for (int e = 0; e < 8; ++e)
    tile[place(8 * c + e, r4 >> 4) + ((r4 >> 2) & 3)] = to_e4m3(x[1][0][e] * iv, x[1][1][e] * iv, x[1][2][e] * iv, x[1][3][e] * iv);
  __syncthreads();
  for (int i = tid; i < D * 4; i += NT) {
    const int dv = i >> 2, chunk = i & 3, s0 = chunk * 16;
    if (s0 >= hi || (s0 + 16 <= lo && ratio[1] == 1.f)) continue;
    uint4 u = *(const uint4*)&tile[place(dv, chunk)];
    uint4* const p = (uint4*)(vp + dv * kPage) + chunk;
    if (s0 < lo || s0 + 16 > hi) {  // what is not new stays: as it is, or at the larger scale
      const uint4 was = *p;
      uint32_t n[4] = {u.x, u.y, u.z, u.w}, o[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t held = ratio[1] == 1.f ? o[w] : rescaled(o[w], ratio[1]);
        uint32_t r = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int slot = s0 + 4 * w + y;
          r |= ((slot < lo ? held : slot < hi ? n[w] : o[w])) & (0xffu << (8 * y));
        }
        n[w] = r;
      }
      u = make_uint4(n[0], n[1], n[2], n[3]);
    }
    store16<LARGE>(p, u);
  }
}

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
  const int most_pages = (a.rows.most + kPage - 1) / kPage + 1;
  const unsigned grid = (unsigned)a.B * (unsigned)most_pages * (unsigned)a.Hkv;
  const bool large = (a.rows.cu ? a.rows.total : (long long)a.B * a.rows.most) * a.Hkv * a.d * 4 > kStreamBytes;
#define VSA_APPEND(D_, F16_)                                                            \
  do {                                                                                  \
    if (large) k_cache_append<D_, F16_, true><<<grid, 2 * D_, 0, s>>>(a, most_pages);   \
    else k_cache_append<D_, F16_, false><<<grid, 2 * D_, 0, s>>>(a, most_pages);        \
  } while (0)
  if (a.d == 128) {
    if (a.f16) VSA_APPEND(128, true);
    else VSA_APPEND(128, false);
  } else {
    if (a.f16) VSA_APPEND(64, true);
    else VSA_APPEND(64, false);
  }
#undef VSA_APPEND
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------------------------
// Attention of few rows.  16 rows at a time (the heads of a group, then the next queries), the pages they walk cut into
// parts of a workgroup each; a wavefront takes whole pages, straight into registers: the tile's rows are keys in the order
// that puts a lane's 16 values of S^T at consecutive keys, so K and V are 16-byte loads, V's contiguous over the wavefront.
// The scales are factors of the softmax: K's of its argument, V's is an addend of the exponent, P' = exp2(x + log2(scale) - ref)
// with the running maximum of x + log2(scale) as reference, so that P' stays within [0, 1] and 16 bits of either type hold it
// as well as they would hold P; the sum of the row takes it out again, a page at a time.
// The next page is on its way while one is multiplied.  Partial results (O, reference, sum) are joined in order by a second
// launch where there is more than one part.  P' is rounded to 16 bits, half a step of each term; all else is fp32 up to O.
// Bound by HBM: 2 d bytes a token and head.  16 sequences of 1000 to 131072 tokens, 16 heads on 4, d = 128: 103 us and 5 for the
// join, 5.7 TB/s; four of up to 2011 tokens: 8.8 and 3.8, chains of trips to memory (lengths, table, scales, page).
constexpr float kNoRow = -1e30f;

// How the pages are dealt to workgroups.  The host knows bounds only, so the kernels work it out from the lengths: all pages that the
// sequences walk (times key heads and row tiles) over `target` workgroups give the pages of a part, a multiple of 4 (a workgroup's
// wavefronts) and the same for all sequences; a sequence has as many parts as it needs.  Then all workgroups run side by side, take
// about as long as each other, and none is launched for pages that are not there.
struct TokenPlan {
  int tiles;                 // row tiles of the longest sequence
  int target, groups, grid;  // workgroups aimed at; (sequence, key head, row tile) triples; workgroups needed at most
  int one;                   // every group is one workgroup's, whatever its length: nothing is joined
};
static TokenPlan token_plan(int B, int H, int Hkv, int d, int max_q, int max_pages) {
  const int G = H / Hkv;
  const long long groups = (long long)B * Hkv * (((long long)max_q * G + 15) / 16);
  TokenPlan p;
  // one generation (two workgroups a compute unit) where that is enough for all, else several
  p.target = (int)(groups <= 256 ? 512 - groups : 4 * groups);
  p.tiles = (int)(((long long)max_q * G + 15) / 16);
  p.groups = (int)groups;
  // A workgroup's eight wavefronts take 8 pages in 2.3 us (d = 128; d = 64: 1), parts of their own and the join cost 3 to 5 us whatever
  // the lengths: 16 heads, 4 sequences, d = 128: 16 pages 11.5 us by one workgroup, 14.0 in parts, 32 pages 16.9 and 14.2.  Where the
  // groups fill the chip by themselves one workgroup is better for longer (64 sequences, 8 key heads, 32 pages: 46 us, in parts 60),
  // but a long sequence among short ones would be alone at the end: no further than 32.
  p.one = (long long)max_pages * d <= (groups >= 128 ? 32 : 16) * 128;
  p.grid = p.one ? p.groups : p.target + p.groups;
  return p;
}
size_t cache_parts(int B, int H, int Hkv, int d, int max_q, int max_pages) {
  const TokenPlan p = token_plan(B, H, Hkv, d, max_q, max_pages);
  return p.one ? 0 : (size_t)p.grid * 16 * (d + 2) + (size_t)p.groups * 4;
}
// Which sequence a workgroup works for, and what of it.
struct TokenItem {
  int b, hk, rt, part, parts, per;  // its part of `parts`, of `per` pages
  int first;                        // slot of part 0 of its (sequence, key head, row tile); further parts: `step` slots on
  int step;
};
__device__ __forceinline__ int token_pages(const WinArgs& a, const CacheArgs& c, int b, int nq) {
  if (nq == 0) return 0;
  const int nk = max(0, min(c.lens[b], c.max_pages * kPage));
  return max(1, WinWalk(a.mask, nk - nq, nk - 1, nk, kPage, kPage).n);
}
// item number `item` of all; false: there are fewer.  (All lanes of a wavefront.)
__device__ __forceinline__ bool token_item(const WinArgs& a, const CacheArgs& c, const TokenPlan& plan, unsigned item, TokenItem& t) {
  const int lane = threadIdx.x & 63;
  auto of = [&](int b, int& pages, int& groups) {  // of sequence b: pages, (key head, row tile) pairs
    const int nq = b < a.B ? win_seq(a.rq, b).n : 0;
    groups = a.Hkv * ((nq * a.G + 15) / 16);
    pages = b < a.B ? token_pages(a, c, b, nq) : 0;
  };
  auto sum = [](long long x) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m);
    return x;
  };
  int pages, groups;
  of(lane, pages, groups);
  long long total = (long long)pages * groups;
  for (int b = 64 + lane; b - lane < a.B; b += 64) {
    int p, g;
    of(b, p, g);
    total += (long long)p * g;
  }
  total = sum(total);
  t.per = (int)max(4ll, (total / plan.target + 4) / 4 * 4);
  unsigned before = 0;  // items of the sequences ahead
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (b0) of(b0 + lane, pages, groups);
    const int parts = (pages + t.per - 1) / t.per;
    const unsigned mine = (unsigned)(parts * groups);
    unsigned upto = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const unsigned x = __shfl_up(upto, m);
      if (lane >= m) upto += x;
    }
    const unsigned long long past = __ballot(before + upto > item);
    if (past) {
      const int l = __builtin_ctzll(past);
      t.b = b0 + l;
      const unsigned at = before + (unsigned)__builtin_amdgcn_readlane((int)(upto - mine), l);
      const int g = __builtin_amdgcn_readlane(groups, l), k = (int)(item - at);
      t.parts = __builtin_amdgcn_readlane(parts, l);
      t.part = k / g;
      const int r = k - t.part * g, tiles = g / a.Hkv;
      t.hk = r / tiles;
      t.rt = r - t.hk * tiles;
      t.first = (int)at + r;
      t.step = g;
      t.b = __builtin_amdgcn_readfirstlane(t.b);
      t.per = __builtin_amdgcn_readfirstlane(t.per);
      t.part = __builtin_amdgcn_readfirstlane(t.part);
      t.hk = __builtin_amdgcn_readfirstlane(t.hk);
      t.rt = __builtin_amdgcn_readfirstlane(t.rt);
      return true;
    }
    before += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
  }
  return false;
}

// ONE: a workgroup takes all pages of its rows.
template <int D, bool F16, bool ONE>
__global__ __launch_bounds__(ONE ? 512 : 256, ONE ? 1 : 2) void k_cache_token(WinArgs a, CacheArgs cache, float* __restrict__ parts, TokenPlan plan) {
  constexpr int KL = D / 64, VT = D / 16, NW = ONE ? 8 : 4;  // 16-byte loads a row of K, tiles of 16 dv, wavefronts
  __shared__ float lds_o[NW][16 * D];
  __shared__ float lds_ml[NW][16][2];
  TokenItem at = {};
  if (ONE) {
    at.rt = (int)blockIdx.x % plan.tiles;
    at.hk = (int)blockIdx.x / plan.tiles % a.Hkv;
    at.b = (int)blockIdx.x / plan.tiles / a.Hkv;
    at.parts = 1, at.per = cache.max_pages;
  } else if (!token_item(a, cache, plan, blockIdx.x, at)) {
    return;
  }
  const int rt = at.rt, hk = at.hk, b = at.b;
  const WinSeq sq = win_seq(a.rq, b);
  const int rows = min(16, sq.n * a.G - rt * 16);
  if (ONE && rows <= 0) return;
  const int nk = __builtin_amdgcn_readfirstlane(max(0, min(cache.lens[b], cache.max_pages * kPage))), shift = nk - sq.n;
  WinWalk walk(a.mask, rt * 16 / a.G + shift, (rt * 16 + rows - 1) / a.G + shift, nk, kPage, kPage);
  walk.uniform();
  // (a tile may walk fewer pages than the sequence: parts behind them are empty)
  const int p0 = min(walk.n, at.part * at.per), p1 = min(walk.n, p0 + at.per);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int row = rt * 16 + min(m, rows - 1), qi = row / a.G, hq = hk * a.G + row % a.G;
  const WinSpan span = win_span(a.mask, qi + shift, nk);
  // the wavefront's pages, 64 at a time, one a lane
  const int np = p1 - p0 > wave ? (p1 - p0 - wave + NW - 1) / NW : 0;
  int id = -1, chunk = -1;
  float sks = 1.f, svs = 1.f;
  auto want = [&](int i) {
    if (i >> 6 == chunk) return;
    chunk = i >> 6;
    const int mine = chunk * 64 + lane;
    id = -1, sks = 1.f, svs = 1.f;
    if (mine < np) {
      id = cache.table[(long long)b * cache.max_pages + walk.begin(p0 + wave + NW * mine) / kPage];
      if ((unsigned)id >= (unsigned)cache.pages) id = -1;
      if (id >= 0) {
        sks = cache.ks[(long long)id * a.Hkv + hk];
        svs = cache.vs[(long long)id * a.Hkv + hk];
      }
    }
  };
  // of page i
  struct Scales {
    float f, lv;
    bool there;
  };
  bf16x8 qreg[2 * KL];
  {
    const uint4* p = (const uint4*)a.q.row(b, sq.row0 + qi, hq);
#pragma unroll
    for (int s = 0; s < 2 * KL; ++s) qreg[s] = __builtin_bit_cast(bf16x8, p[8 * (s >> 1) + 2 * g + (s & 1)]);
  }
  f32x4 o[VT];
#pragma unroll
  for (int x = 0; x < VT; ++x) o[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref = kNoRow, sum = 0.f;
  const float sl2 = a.scale * kLog2e;
  struct Page {
    uint4 k[4][KL], v[VT];
  };
  auto fetch = [&](int i, Page& p, Scales& sc) {
    want(i);
    sc.there = __builtin_amdgcn_readlane(id, i & 63) >= 0;
    sc.f = sl2 * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sks), i & 63));
    sc.lv = fast_log2(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(svs), i & 63)));
    const int page = max(__builtin_amdgcn_readlane(id, i & 63), 0);
    const uint8_t* kp = cache.k + ((long long)page * a.Hkv + hk) * (kPage * D);
    const uint8_t* vp = cache.v + ((long long)page * a.Hkv + hk) * (kPage * D);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < KL; ++c) p.k[t][c] = *(const uint4*)(kp + (16 * (m >> 2) + 4 * t + (m & 3)) * D + 64 * c + 16 * g);
#pragma unroll
    for (int x = 0; x < VT; ++x) p.v[x] = *(const uint4*)(vp + (16 * x + m) * kPage + 16 * g);
  };
  auto multiply = [&](int i, Page& p, const Scales& sc) {
    const int piece = p0 + wave + NW * i, key0 = walk.begin(piece);
    if (!sc.there) return;  // (the entry names no page: hidden)
    const float f = sc.f, lv = sc.lv;
    f32x4 s[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        s[t] = mm16<F16>(from_e4m3<F16>(p.k[t][c].x, p.k[t][c].y), qreg[2 * c], s[t]);
        s[t] = mm16<F16>(from_e4m3<F16>(p.k[t][c].z, p.k[t][c].w), qreg[2 * c + 1], s[t]);
      }
    }
    if (walk.masked(piece)) {
      const WinSpan w = walk.span_in(piece, span);
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = key0 + 16 * g + 4 * t + r;
          s[t][r] = key < w.hi && (key >= w.lo || key < w.se) ? s[t][r] : -INFINITY;
        }
      if (key0 + kPage > nk) {  // values behind the last token may be anything: zero
        const int live = nk - key0 - 16 * g;
#pragma unroll
        for (int x = 0; x < VT; ++x) {
          uint32_t* const u = &p.v[x].x;
#pragma unroll
          for (int w4 = 0; w4 < 4; ++w4) {
            const int keep = min(4, max(0, live - 4 * w4));
            u[w4] &= keep == 4 ? 0xffffffffu : (1u << (8 * keep)) - 1u;
          }
        }
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, s[t][r]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float mnew = fmaxf(fmaf(top, f, lv), ref);
    if (__any(mnew > ref)) {
      const float alpha = fast_exp2(ref - mnew);
      sum *= alpha;
#pragma unroll
      for (int x = 0; x < VT; ++x) o[x] *= alpha;
      ref = mnew;
    }
    float e[4][4], page_sum = 0.f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[t][r] = fast_exp2(fmaf(s[t][r], f, lv - ref));
        page_sum += e[t][r];
      }
    sum = fmaf(page_sum, fast_exp2(-lv), sum);
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const uint4 u = {pack16<F16>(e[2 * s2][0], e[2 * s2][1]), pack16<F16>(e[2 * s2][2], e[2 * s2][3]),
                       pack16<F16>(e[2 * s2 + 1][0], e[2 * s2 + 1][1]), pack16<F16>(e[2 * s2 + 1][2], e[2 * s2 + 1][3])};
#pragma unroll
      for (int x = 0; x < VT; ++x)
        o[x] = mm16<F16>(s2 ? from_e4m3<F16>(p.v[x].z, p.v[x].w) : from_e4m3<F16>(p.v[x].x, p.v[x].y), __builtin_bit_cast(bf16x8, u), o[x]);
    }
  };
  if (np > 0) {
    Page pa, pb;
    Scales sa, sb;
    fetch(0, pa, sa);
    int i = 0;
    for (; i + 2 < np; i += 2) {
      fetch(i + 1, pb, sb);
      multiply(i, pa, sa);
      fetch(i + 2, pa, sa);
      multiply(i + 1, pb, sb);
    }
    if (i + 1 < np) {
      fetch(i + 1, pb, sb);
      multiply(i, pa, sa);
      multiply(i + 1, pb, sb);
    } else {
      multiply(i, pa, sa);
    }
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (g == 0) *(float2*)lds_ml[wave][m] = make_float2(ref, sum);
#pragma unroll
  for (int x = 0; x < VT; ++x) *(f32x4*)&lds_o[wave][m * D + (((4 * x + g) ^ m) << 2)] = o[x];
  __syncthreads();
  if (!ONE && tid == 0 && at.part == 0)  // for the join: where the parts are
    ((int4*)(parts + (long long)plan.grid * (16 * (D + 2))))[(b * a.Hkv + hk) * plan.tiles + rt] = make_int4(at.first, at.parts, at.step, 0);
  // rows of the tile, 8 elements a thread
  for (int it = tid; it < rows * (D / 8); it += 64 * NW) {
    const int r = it / (D / 8), ch = it % (D / 8);
    float M = lds_ml[0][r][0], L = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, lds_ml[w][r][0]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = fast_exp2(lds_ml[w][r][0] - M);
      L += f * lds_ml[w][r][1];
      const f32x4 y0 = *(const f32x4*)&lds_o[w][r * D + (((2 * ch) ^ r) << 2)], y1 = *(const f32x4*)&lds_o[w][r * D + (((2 * ch + 1) ^ r) << 2)];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += f * y0[e], v[4 + e] += f * y1[e];
    }
    const int row_of = rt * 16 + r, q_of = row_of / a.G, h_of = hk * a.G + row_of % a.G;
    if (ONE || at.parts == 1) {
      const bool none = M <= kNoRow;
      const float inv = none ? 0.f : 1.f / L;
      const uint4 u = {pack16<F16>(v[0] * inv, v[1] * inv), pack16<F16>(v[2] * inv, v[3] * inv), pack16<F16>(v[4] * inv, v[5] * inv),
                       pack16<F16>(v[6] * inv, v[7] * inv)};
      *((uint4*)a.o.out(b, sq.row0 + q_of, h_of) + ch) = u;
      if (a.lse && ch == 0) a.lse[a.stat(h_of, b, sq.row0, q_of)] = none ? -INFINITY : (M + fast_log2(L)) * kLn2;
    } else {
      float* const to = parts + (long long)blockIdx.x * (16 * (D + 2));
      *(float4*)&to[r * D + ch * 8] = make_float4(v[0], v[1], v[2], v[3]);
      *(float4*)&to[r * D + ch * 8 + 4] = make_float4(v[4], v[5], v[6], v[7]);
      if (ch == 0) *(float2*)&to[16 * D + 2 * r] = make_float2(M, L);
    }
  }
}

// one workgroup a row: 256 / (D / 8) threads share its parts
template <int D, bool F16>
__global__ __launch_bounds__(256) void k_cache_join(WinArgs a, CacheArgs cache, const float* __restrict__ parts, TokenPlan plan) {
  constexpr int CH = D / 8, PG = 256 / CH;
  __shared__ float so[PG][D + 4], sm[PG], sl[PG];
  const int r = blockIdx.x % 16, group = blockIdx.x / 16, rt = group % plan.tiles, hk = group / plan.tiles % a.Hkv, b = group / plan.tiles / a.Hkv;
  const WinSeq sq = win_seq(a.rq, b);
  if (r >= min(16, sq.n * a.G - rt * 16)) return;
  const int4 at = ((const int4*)(parts + (long long)plan.grid * (16 * (D + 2))))[group];  // first slot, parts, slots from one to the next
  const int tid = threadIdx.x, ch = tid % CH, pg = tid / CH, live = at.y;
  if (live == 1) return;
  const float* from = parts + (long long)at.x * (16 * (D + 2));
  const long long step = (long long)at.z * (16 * (D + 2));
  float M = kNoRow, L = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int p = pg; p < live; p += PG) {
    const float* x = from + p * step;
    const float2 ml = *(const float2*)&x[16 * D + 2 * r];
    const float4 y0 = *(const float4*)&x[r * D + ch * 8], y1 = *(const float4*)&x[r * D + ch * 8 + 4];
    const float mn = fmaxf(M, ml.x), fa = fast_exp2(M - mn), fb = fast_exp2(ml.x - mn);
    M = mn;
    L = L * fa + ml.y * fb;
    const float y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * fa + y[e] * fb;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) so[pg][ch * 8 + e] = v[e];
  if (ch == 0) sm[pg] = M, sl[pg] = L;
  __syncthreads();
  if (tid >= CH) return;
  M = sm[0];
#pragma unroll
  for (int w = 1; w < PG; ++w) M = fmaxf(M, sm[w]);
  L = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  for (int w = 0; w < PG; ++w) {
    const float f = fast_exp2(sm[w] - M);
    L += f * sl[w];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += f * so[w][tid * 8 + e];
  }
  const bool none = M <= kNoRow;
  const float inv = none ? 0.f : 1.f / L;
  const int row_of = rt * 16 + r, q_of = row_of / a.G, h_of = hk * a.G + row_of % a.G;
  const uint4 u = {pack16<F16>(v[0] * inv, v[1] * inv), pack16<F16>(v[2] * inv, v[3] * inv), pack16<F16>(v[4] * inv, v[5] * inv),
                   pack16<F16>(v[6] * inv, v[7] * inv)};
  *((uint4*)a.o.out(b, sq.row0 + q_of, h_of) + tid) = u;
  if (a.lse && tid == 0) a.lse[a.stat(h_of, b, sq.row0, q_of)] = none ? -INFINITY : (M + fast_log2(L)) * kLn2;
}

namespace {
template <int D, bool F16>
hipError_t token(const WinArgs& a, const CacheArgs& c, float* parts, hipStream_t s) {
  const TokenPlan plan = token_plan(a.B, a.H, a.Hkv, D, a.rq.most, c.max_pages);
  if (plan.one) k_cache_token<D, F16, true><<<(unsigned)plan.grid, 512, 0, s>>>(a, c, parts, plan);
  else k_cache_token<D, F16, false><<<(unsigned)plan.grid, 256, 0, s>>>(a, c, parts, plan);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.one) return e;
  k_cache_join<D, F16><<<(unsigned)plan.groups * 16u, 256, 0, s>>>(a, c, parts, plan);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_cache_token(const WinArgs& a, const CacheArgs& c, int d, bool f16, float* parts, hipStream_t s) {
  if (d == 128) return f16 ? token<128, true>(a, c, parts, s) : token<128, false>(a, c, parts, s);
  return f16 ? token<64, true>(a, c, parts, s) : token<64, false>(a, c, parts, s);
}

}  // namespace vsa
