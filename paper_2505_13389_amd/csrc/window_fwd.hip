// Windowed attention, forward: O = softmax over the visible keys, one pass with a running reference and sum.
//
// A wavefront multiplies units of 32 keys with the 64 query rows of its block, everything transposed as in the fine forward:
//   S^T[key, q] = K (A operand) x Q^T (B operand, registers),   O^T[dv, q] += V^T (A) x P^T (B, the registers of S^T in 16 bits)
// so that a lane owns two query columns.  Its units are copied to LDS stages of its own (K two units, V two), without a
// barrier in the walk: S of unit u + 1 is multiplied while P of unit u is formed, PV of u behind it.  NW wavefronts share a
// block where a launch has few of them and merge at the end.
//
// PAGED: K and V come from the pages of the 8-bit cache, as bytes, and are widened as operands.  Rows of the tile are keys in an
// order that puts a lane's 16 values of S^T at consecutive keys, and a contraction step pair of K at 16 consecutive bytes:
// every LDS read is 16 bytes.  K's scale goes into the softmax's factor, V's into its exponent and reference: see k_cache_token.
//
// Roundings: P goes to 16 bits before the product with V, half a step of each term, as in the fine kernels (a product of 32-bit
// operands would take 16 times the matrix instructions); S, sums, references, O and log-sum-exps are fp32, and O is rounded once,
// when it is stored.  Against 64 bits 2.3e-3 of the norm in bf16, 2.6e-4 in fp16 (rounding the exact result: 1.7e-3 and 2.0e-4).
//
// Bound by matrix instructions and the power they take, in small launches by start-up (about 10000 cycles from launch to the first
// product, and the way of O out).  A unit is 1600 cycles (1024 of them the matrix pipe's; d = 64: half), PAGED 2060, 64 conversions
// more.  32760 tokens, 12 heads, d = 128, a window of 7 frames of 1560: 2000 to 2050 us, 1.02 to 1.05 PFLOP/s on the visible pairs, the
// pipe busy 58 % at 1.48 GHz; 16384 tokens, 5 frames of 1024: 460 us; packed texts of 13385 tokens, 16 heads, fp16: 131 to 135;
// 1560 queries on the cache of 32760 tokens: 139.
#include <type_traits>

#include "ticks.h"
#include "unit_stream.h"
#include "window_kernels.h"
#include "window_tile.h"

namespace vsa {

constexpr float kUnset = -1e30f;      // a column without a visible key so far
constexpr float kMostSum = 8192.f;    // a lane's sum of 16 values above this moves the reference (fp16 ends at 65504)

// Pages of a sequence, 64 entries of its table at a time, an entry a lane.
struct PageList {
  const int32_t* table;
  const float *ks, *vs;
  int n, pages, Hkv, hk, lane, chunk, id;
  float sk, sv;
  __device__ __forceinline__ void load(int c) {
    chunk = c;
    const int e = c * 64 + lane;
    id = e < n ? table[e] : -1;
    if ((unsigned)id >= (unsigned)pages) id = -1;
    sk = id < 0 ? 1.f : ks[(long long)id * Hkv + hk];
    sv = id < 0 ? 1.f : vs[(long long)id * Hkv + hk];
    asm volatile("" : "+v"(id), "+v"(sk), "+v"(sv));  // (the waits for the loads lie here)
  }
  __device__ __forceinline__ void want(int page) {
    if (__builtin_expect(page >> 6 != chunk, 0)) load(page >> 6);
  }
  __device__ __forceinline__ int page_id(int page) const { return __builtin_amdgcn_readlane(id, page & 63); }
  __device__ __forceinline__ float scale_k(int page) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sk), page & 63)); }
  __device__ __forceinline__ float scale_v(int page) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(sv), page & 63)); }
};

// A unit of a page: 32 keys.  K: LDS row m holds key 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3), D bytes; V: row dv, 32 bytes.
template <int D>
struct PageCopy {
  static constexpr int NC = D / 32, CPR = D / 16;
  unsigned ko[NC], vo[NC];
  __device__ static __forceinline__ int swz(int m) { return (m >> (D == 128 ? 1 : 2)) & (CPR - 1); }
  __device__ __forceinline__ void init(int lane) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int m = c * (1024 / D) + lane / CPR, pc = lane % CPR;
      ko[c] = (unsigned)((16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3)) * D + ((pc ^ swz(m)) << 4));
      const int dv = c * 32 + (lane >> 1);
      vo[c] = (unsigned)(dv * kPage + (((lane & 1) ^ ((dv >> 3) & 1)) << 4));
    }
  }
  // bytes of K: contraction steps 2 sp, 2 sp + 1 (elements 32 sp + 16 h + ..) of row l32
  __device__ static __forceinline__ uint4 k_at(const unsigned char* stage, int lane, int sp) {
    const int m = lane & 31;
    return *(const uint4*)(stage + m * D + (((2 * sp + (lane >> 5)) ^ swz(m)) << 4));
  }
  // bytes of V: keys 16 h .. 16 h + 15 of dv = 32 x + l32
  __device__ static __forceinline__ uint4 v_at(const unsigned char* stage, int lane, int x) {
    const int dv = 32 * x + (lane & 31);
    return *(const uint4*)(stage + dv * 32 + (((lane >> 5) ^ ((dv >> 3) & 1)) << 4));
  }
};

// What lies behind which matrix instruction of a unit (see ticks.h): S of the next unit, then PV.  The softmax of a unit, in
// operations, is done from the second instruction of the PV phase before it to the last but one of the next S phase.
template <int D, bool PAGED>
struct WinTicks : TickCycles<D / 2> {  // (two units)
  using Table = TickCycles<D / 2>;
  using typename Table::Work;
  using Table::cycles;
  using Table::T;
  static constexpr int KS = D / 16, PH = 2 * KS, U = T / 2;  // contraction steps of S (and operands of V); matrix instructions of a phase, of a unit
  static constexpr int NC = PAGED ? D / 32 : KS;             // copies of a unit's K, or V
  static constexpr int kEvery = PH / NC < 4 ? PH / NC : 4;   // a copy behind every so many
  static constexpr int kAhead = D == 128 ? 4 : 2;            // operands are read so many steps ahead
  static constexpr int kOps = 112;
  Work w[kOps] = {};
  int ahead[T + 1] = {};
  static constexpr int in_pv(int j) { return PH + j; }
  static constexpr int in_s(int j) { return U + j; }
  constexpr WinTicks() {
    for (int t = 0; t < T; ++t) {
      const int u = t % U, j = u % PH;
      if (j % kEvery == 0 && j / kEvery < NC) cycles[t] += Table::kCopy + (j == 0 ? 5 * Table::kScalar : 0);
      if (j % 2 == 0) cycles[t] += Table::kRead;               // (operands: two reads of V's, one of K's, of either one in pages)
      if (j % 2 == 1 && u >= PH && !PAGED) cycles[t] += Table::kRead;
      if (PAGED) cycles[t] += 2 * 5;                           // widening
      if (u < PH && j == PH - 2) cycles[t] += 38;              // the check of the references
      if (u < PH && (j == 1 || j == 3)) cycles[t] += 5 * Table::kScalar;  // where the next unit lies
    }
    int n = 0;
    w[n++] = {Table::MUL, 0, 0};
    w[n++] = {Table::MUL, 0, 1};
    for (int g = 0; g < 17; ++g) {
      if (g < 16) w[n++] = {Table::EXP, g, 0};
      if (g < 15) w[n++] = {Table::MUL, g + 1, 0};
      if (g < 15) w[n++] = {Table::MUL, g + 1, 1};
      if (g < 16) w[n++] = {Table::EXP, g, 1};
      if (g > 0) w[n++] = {Table::ADD, g - 1, 0};
      if (g > 0) w[n++] = {Table::CVT, g - 1, 0};
      if (g > 0) w[n++] = {Table::ADD, g - 1, 1};
    }
    this->deal(ahead, w, kOps, in_pv(1), in_s(PH - 1));
  }
  constexpr bool in_order() const { return ahead[in_pv(1)] == 0 && ahead[in_s(PH - 1)] == kOps && this->ordered(w, kOps); }
};
static_assert(WinTicks<128, false>().in_order() && WinTicks<64, false>().in_order() && WinTicks<128, true>().in_order() && WinTicks<64, true>().in_order(),
              "operations of the softmax");

// O of d = 128 lives in the accumulation registers (256 + 256 registers a wavefront, see mfma_a)
template <int D, bool F16>
__device__ __forceinline__ void mm_o(f32x16& acc, bf16x8 a, bf16x8 b) {
  if constexpr (D == 64) acc = mm32<F16>(a, b, acc);
  else if constexpr (F16) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  else mfma_a(acc, a, b);
}

template <int D, bool F16, int NW, bool PAGED>
__global__ __launch_bounds__(64 * NW, 1) void k_window_fwd(WinArgs a, CacheArgs cache, RowPlan plan, float* __restrict__ parts) {
  using TL = Tile<D>;
  using TK = WinTicks<D, PAGED>;
  constexpr TK ticks;
  constexpr int KS = D / 16, DVB = D / 32, PH = 2 * KS, HALF = 32 * D * 2, STAGE = PAGED ? HALF / 2 : HALF, NC = TK::NC, kAhead = TK::kAhead, kEvery = TK::kEvery;
  static_assert(NC == (PAGED ? PageCopy<D>::NC : RowCopy<D>::NC) && (NC - 1) * kEvery < PH, "copies of a phase");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * 4 * HALF];
  __shared__ float ml[NW * 64 * 2];

  RowItem at;
  if (!win_rows(a, plan, blockIdx.x, PAGED, at)) return;
  const int b = at.b, hk = at.hk, qb = at.qb, hq = hk * a.G + at.g;
  const WinSeq sq = at.q;
  const int r0 = qb * 64, rows = min(64, sq.n - r0);
  if (rows <= 0) return;
  WinSeq sk = at.k;
  if constexpr (PAGED) sk = {0, max(0, min(cache.lens[b], cache.max_pages * kPage))};
  const int nk = __builtin_amdgcn_readfirstlane(sk.n), shift = nk - sq.n;
  WinWalk walk(a.mask, r0 + shift, r0 + rows - 1 + shift, nk, 32, PAGED ? 32 : 1);
  walk.uniform();
  // this workgroup's part of the walk
  const int want = (walk.n + plan.per - 1) / plan.per, live = plan.parts == 1 || want <= 1 ? 1 : want < plan.parts ? want : plan.parts;
  if (at.part >= live) return;
  const int begin = (int)((long long)walk.n * at.part / live), end = (int)((long long)walk.n * (at.part + 1) / live);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int nu = end - begin > wave ? (end - begin - wave + NW - 1) / NW : 0;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * (4 * HALF);
  unsigned char* const mine = smem + wave * (4 * HALF);
  const unsigned char *kb = nullptr, *vb = nullptr;
  RowCopy<D> kc, vc;
  PageCopy<D> pc;
  PageList pages;
  if constexpr (PAGED) {
    pc.init(lane);
    pages = {cache.table + (long long)b * cache.max_pages, cache.ks, cache.vs, (nk + kPage - 1) / kPage, cache.pages, a.Hkv, hk, lane, -1, 0, 1.f, 1.f};
  } else {
    kb = (const unsigned char*)uniform_ptr(a.k.row(b, sk.row0, hk));
    vb = (const unsigned char*)uniform_ptr(a.v.row(b, sk.row0, hk));
    kc.init(lane, (unsigned)a.k.token);
    vc.init(lane, (unsigned)a.v.token);
  }
  // A unit of the wavefront's walk, and where its rows lie.  (Units behind the last one are that one again: their copies are
  // made, so that the waits can count, and not used.)
  struct U {
    int a;                           // first key
    bool masked;
    const unsigned char *k, *v;
    float f, lv;                     // of the softmax: P' = exp2(f S + lv - ref)
  };
  const float sl2 = a.scale * kLog2e;
  auto unit = [&](int u) {
    const int i = begin + wave + NW * min(u, nu - 1);
    U x;
    x.a = walk.begin(i);
    x.masked = walk.masked(i);
    x.f = sl2, x.lv = 0.f;
    if constexpr (PAGED) {
      const int e = x.a / kPage;
      pages.want(e);
      const int id = pages.page_id(e);
      x.masked |= id < 0;
      x.f = sl2 * pages.scale_k(e);
      x.lv = fast_log2(pages.scale_v(e));
      const long long at = ((long long)max(id, 0) * a.Hkv + hk) * (kPage * D);
      x.k = cache.k + at + (x.a & 32) * D;
      x.v = cache.v + at + (x.a & 32);
      x.a = id < 0 ? nk : x.a;  // (no key of it is visible)
    } else {
      x.k = kb + (long long)x.a * kc.stride;
      x.v = vb + (long long)x.a * vc.stride;
    }
    return x;
  };
  // copies of a unit's K into stage 0 or 1, V into 2 or 3
  auto copy_all = [&](const U& x, bool of_v, int stage) {
    const unsigned lds = lds0 + stage * STAGE;
    if constexpr (PAGED) {
#pragma unroll
      for (int c = 0; c < NC; ++c) win_copy16(of_v ? x.v : x.k, of_v ? pc.vo[c] : pc.ko[c], lds + c * 1024);
    } else {
      if (of_v) vc.all(x.v, lds, lane, nk - x.a);
      else kc.all(x.k, lds, lane, nk - x.a);
    }
  };
  auto copy_aim = [&](bool of_v, int stage, int c) {
    if constexpr (PAGED) set_m0_ahead(lds0 + stage * STAGE + c * 1024);
    else (of_v ? vc : kc).aim(lds0 + stage * STAGE, c);
    __builtin_amdgcn_sched_barrier(0);  // (the matrix instruction between this and the copy stays between them)
  };
  auto copy_piece = [&](const U& x, bool of_v, int c) {
    if constexpr (PAGED) lds_dma16_at<0>(of_v ? x.v : x.k, of_v ? pc.vo[c] : pc.ko[c]);
    else if (of_v) vc.piece(x.v, c);
    else kc.piece(x.k, c);
  };

  // The first copies and Q are requested as early as can be; what follows up to their wait is done while they are on their way.
  U cur = {}, n1 = {}, n2 = {};
  if (nu > 0) {
    cur = unit(0), n1 = unit(1), n2 = unit(2);
    copy_all(cur, false, 0);
    copy_all(n1, false, 1);
    copy_all(cur, true, 2);
  }
  // Q: of a page's operands, contraction step 2 sp + e holds elements 32 sp + 16 h + 8 e ..
  bf16x8 qreg[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint4* p = (const uint4*)a.q.row(b, sq.row0 + min(r0 + 32 * t + l32, sq.n - 1), hq);
#pragma unroll
    for (int s = 0; s < KS; ++s) qreg[t][s] = __builtin_bit_cast(bf16x8, p[PAGED ? 4 * (s >> 1) + 2 * h + (s & 1) : 2 * s + h]);
  }
  WinSpan span[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) span[t] = win_span(a.mask, min(r0 + 32 * t + l32, sq.n - 1) + shift, nk);

  f32x16 o[DVB][2];
  float nil = 0.f;
  asm volatile("" : "+v"(nil));
#pragma unroll
  for (int x = 0; x < DVB; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[x][t][i] = nil;
  auto pin_o = [](f32x16& acc) {
    if (D == 128) asm volatile("" : "+a"(acc));
    else asm volatile("" : "+v"(acc));
  };
#pragma unroll
  for (int x = 0; x < DVB; ++x) pin_o(o[x][0]), pin_o(o[x][1]);

  float ref[2] = {kUnset, kUnset}, lsum[2] = {0.f, 0.f};
  float ta[2] = {0.f, 0.f}, tb[2] = {0.f, 0.f};  // a lane's sums of a unit, even and odd values
  uint4 pb[2][2];                                // P^T as operands: [query half][contraction step]
  f32x16 zero16;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero16[i] = 0.f;

  auto put = [](uint4& u4, int w, uint32_t x) {
    if (w == 0) u4.x = x;
    if (w == 1) u4.y = x;
    if (w == 2) u4.z = x;
    if (w == 3) u4.w = x;
  };
  // Item `it` of 16 of a unit's softmax: two values of one query half, the first eight of contraction step 0
  float xf[2][2] = {}, xe[2][2] = {};
  auto p_fma = [&](const f32x16 (&S)[2], int it, int i, float f, const float* sub) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    xf[it & 1][i] = fmaf(S[t][e + i], f, -sub[t]);
    asm volatile("" : : "v"(xf[it & 1][i]));  // (pure arithmetic has no place of its own in the order: tie it to this one)
  };
  auto p_exp = [&](int it, int i) {
    xe[it & 1][i] = fast_exp2(xf[it & 1][i]);
    asm volatile("" : : "v"(xe[it & 1][i]));
  };
  auto p_sum = [&](int it, int i) {
    float& t = (i ? tb : ta)[(it >> 2) & 1];
    const float x = xe[it & 1][i];
    t = (it & 11) == 0 ? x : t + x;
    asm volatile("" : : "v"(t));
  };
  auto p_convert = [&](int it) {
    const uint32_t pp = pack16<F16>(xe[it & 1][0], xe[it & 1][1]);
    put(pb[(it >> 2) & 1][it >> 3], it & 3, pp);
    asm volatile("" : : "v"(pp));
  };
  auto p_ops = [&](const f32x16 (&S)[2], auto from, auto to, float f, const float* sub) {
    in_steps<decltype(to)::value - decltype(from)::value>([&](auto number) {
      constexpr typename TK::Work w = ticks.w[decltype(from)::value + decltype(number)::value];
      if constexpr (w.op == TK::MUL) p_fma(S, w.item, w.i, f, sub);
      if constexpr (w.op == TK::EXP) p_exp(w.item, w.i);
      if constexpr (w.op == TK::ADD) p_sum(w.item, w.i);
      if constexpr (w.op == TK::CVT) p_convert(w.item);
    });
  };
  auto unit_max = [&](const f32x16& S) {
    float m = fmaxf(fmaxf(S[0], S[1]), S[2]);
#pragma unroll
    for (int i = 3; i < 15; i += 2) m = fmaxf(fmaxf(m, S[i]), S[i + 1]);
    return max_across_halves(fmaxf(m, S[15]));
  };
  auto hide = [&](f32x16 (&S)[2], const U& x, int u) {  // what a query does not see
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const WinSpan w = walk.span_in(begin + wave + NW * u, span[t]);
      int first = x.a + (PAGED ? 16 * h : 4 * h);
      asm volatile("" : "+v"(first));  // (nothing of this is kept in registers through the walk)
      if (w.se <= x.a) {  // (no sinks among these keys)
        const unsigned from = (unsigned)(first - w.lo), many = (unsigned)(w.hi - w.lo);
#pragma unroll
        for (int i = 0; i < 16; ++i) S[t][i] = from + (unsigned)(PAGED ? i : 8 * (i >> 2) + (i & 3)) < many ? S[t][i] : -INFINITY;
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = first + (PAGED ? i : 8 * (i >> 2) + (i & 3));
          S[t][i] = key < w.hi && (key >= w.lo || key < w.se) ? S[t][i] : -INFINITY;
        }
      }
    }
  };
  auto clear_tail = [&](const U& x, int stage) {  // values behind the last token may be anything: zero
    const int live = nk - x.a;
    for (int dv = lane; dv < D; dv += 64) {
      unsigned* p = (unsigned*)(mine + stage * STAGE + dv * 32);
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const int key = ((w >> 2) ^ ((dv >> 3) & 1)) * 16 + (w & 3) * 4, keep = min(4, max(0, live - key));
        p[w] = keep == 4 ? p[w] : p[w] & ((1u << (8 * keep)) - 1u);
      }
    }
    __builtin_amdgcn_wave_barrier();
  };

  const int lane_a = TL::rowmajor_lane(0, lane);
  int lane_b0, lane_b1;
  TL::transposed_lane(0, lane, lane_b0, lane_b1);
  // operand reads.  K: step s; of pages two steps a read.  V: operand i = (contraction step i / DVB, tile i % DVB), two reads; of
  // pages one for both steps of a tile.
  constexpr int NK = PAGED ? KS / 2 : KS, NV = PAGED ? DVB : KS;  // reads (V of rows: pairs of them)
  struct Row8 {
    bf16x8 x;
  };
  using KRaw = std::conditional_t<PAGED, uint4, bf16x8>;
  using VRaw = std::conditional_t<PAGED, uint4, bf16x8>;
  auto read_k = [&](int stage, int i) -> KRaw {
    if constexpr (PAGED) return PageCopy<D>::k_at(mine + stage * STAGE, lane, i);
    else return TL::rowmajor_at(mine + stage * STAGE, lane_a, i);
  };
  auto read_v = [&](int stage, int i) -> VRaw {
    if constexpr (PAGED) return PageCopy<D>::v_at(mine + stage * STAGE, lane, i);
    else return TL::transposed_at(mine + stage * STAGE, lane_b0, lane_b1, i / DVB, i % DVB);
  };
  auto k_op = [&](const KRaw& r, int s) -> bf16x8 {
    if constexpr (PAGED) return s & 1 ? from_e4m3<F16>(r.z, r.w) : from_e4m3<F16>(r.x, r.y);
    else return r;
  };
  auto v_op = [&](const VRaw& r, int st) -> bf16x8 {
    if constexpr (PAGED) return st ? from_e4m3<F16>(r.z, r.w) : from_e4m3<F16>(r.x, r.y);
    else return r;
  };

  f32x16 s0[2], s1[2];
  constexpr int kKeep = PAGED ? kAhead / 2 : kAhead;  // K reads of a unit's first steps, made during the phase before
  KRaw kcur[kKeep];
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qreg[0][s]), "+v"(qreg[1][s]));  // (requested behind the first copies, and waited for with them)
  if (nu > 0) {
    win_wait<2 * NC>();  // K of the first unit
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bf16x8 ka = k_op(read_k(0, PAGED ? s / 2 : s), s);
      s0[0] = mm32<F16>(ka, qreg[0][s], s == 0 ? zero16 : s0[0]);
      s0[1] = mm32<F16>(ka, qreg[1][s], s == 0 ? zero16 : s0[1]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    copy_all(n2, false, 0);
    if (cur.masked) hide(s0, cur, 0);
    win_wait<2 * NC>();  // K of the second (newer: V of the first, K of the third)
#pragma unroll
    for (int i = 0; i < kKeep; ++i) kcur[i] = read_k(1, i);
    // the first reference; a column of which nothing is visible yet has none, and any sum of it is above the bound
#pragma unroll
    for (int t = 0; t < 2; ++t) ref[t] = fmaxf(fmaf(unit_max(s0[t]), cur.f, cur.lv), kUnset);
    const float sub[2] = {ref[0] - cur.lv, ref[1] - cur.lv};
    p_ops(s0, std::integral_constant<int, 0>{}, std::integral_constant<int, ticks.ahead[TK::U]>{}, cur.f, sub);
  }

  // Unit u, whose S is there: P(u) while S(u + 1) is multiplied into T, then PV(u) while P(u + 1) begins.  K(u + 1) has landed, K(u + 2) and
  // V(u) are on their way; V(u + 1) is requested during the first phase, K(u + 3) during the second.
  // STEADY: copies piece by piece, of rows that are there; else at once, and u may be the last unit (then what is made of the one behind
  // it is not used).  `par` = u & 1 (a constant in the unrolled loop).
  auto body = [&](auto steady_tag, int par, f32x16 (&S)[2], f32x16 (&T)[2], int u) {
    constexpr bool STEADY = decltype(steady_tag)::value;
    const int kn = 1 - par, vn = 3 - par, vc_ = 2 + par;  // stages: K(u + 1) and then K(u + 3), V(u + 1), V(u)
    KRaw kr[NK];
    VRaw vr[NV];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) kr[i] = kcur[i];
    const float sub[2] = {ref[0] - cur.lv, ref[1] - cur.lv};
    U n3 = {};
    if (!STEADY) copy_all(n1, true, vn);
    bf16x8 kop;
    __builtin_amdgcn_sched_barrier(0);
    in_steps<PH>([&](auto number) {
      constexpr int j = decltype(number)::value, s = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0 && j / kEvery < NC;
      if (copies) copy_aim(true, vn, j / kEvery);
      if (j % 2 == 0) kop = k_op(kr[PAGED ? s / 2 : s], s);
      T[j & 1] = mm32<F16>(kop, qreg[j & 1][s], s == 0 ? zero16 : T[j & 1]);
      __builtin_amdgcn_sched_barrier(0);
      if (copies) copy_piece(n1, true, j / kEvery);
      if (j == PH - 2 * kAhead) {  // V(u) has landed; newer: K(u + 2) and what has been requested of V(u + 1)
        constexpr int part = (PH - 2 * kAhead) / kEvery + 1 < NC ? (PH - 2 * kAhead) / kEvery + 1 : NC;
        win_wait<NC + (STEADY ? part : NC)>();
        if (PAGED && cur.a + 32 > nk) clear_tail(cur, vc_);
      }
      // operands kAhead steps further on
      if constexpr (j % 2 == 0) {
        constexpr int to = s + kAhead;
        if constexpr (to < KS) {
          if constexpr (!(PAGED && to % 2)) kr[PAGED ? to / 2 : to] = read_k(kn, PAGED ? to / 2 : to);
        } else if constexpr (to - KS < NV) {
          vr[to - KS] = read_v(vc_, to - KS);
        }
      }
      if (j == 1) n3 = unit(u + 3);
      p_ops(S, std::integral_constant<int, ticks.ahead[TK::in_s(j)]>{}, std::integral_constant<int, ticks.ahead[TK::in_s(j + 1)]>{}, cur.f, sub);
      __builtin_amdgcn_sched_barrier(0);
      if (j == PH - 2) {
        // A column's reference stays unless one of its two lanes sums 16 values to more than kMostSum (infinity: it has none yet).
        const float tsum[2] = {ta[0] + tb[0], ta[1] + tb[1]};
        const float out = PAGED ? fast_exp2(-cur.lv) : 1.f;
        float add[2] = {tsum[0], tsum[1]};
        if (__builtin_expect(__any(!(fmaxf(tsum[0], tsum[1]) <= kMostSum)), 0)) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const bool moves = !(max_across_halves(tsum[t]) <= kMostSum);
            if (!__any(moves)) continue;
            const float to = fmaxf(fmaf(unit_max(S[t]), cur.f, cur.lv), ref[t]), next = moves ? to : ref[t];
            const float alpha = fast_exp2(ref[t] - next);
            lsum[t] *= alpha;
#pragma unroll
            for (int x = 0; x < DVB; ++x) {
              pin_o(o[x][t]);  // (moved to ordinary registers from here on and not before the branch)
#pragma unroll
              for (int i = 0; i < 16; ++i) o[x][t][i] *= alpha;
              pin_o(o[x][t]);
              __builtin_amdgcn_sched_barrier(0);  // (one block of O in ordinary registers at a time)
            }
            ref[t] = next;
            const float now[2] = {ref[0] - cur.lv, ref[1] - cur.lv};
#pragma unroll
            for (int st = 0; st < 2; ++st)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const int it = 8 * st + 4 * t + w;
                for (int i = 0; i < 2; ++i) {
                  p_fma(S, it, i, cur.f, now);
                  p_exp(it, i);
                  p_sum(it, i);
                }
                p_convert(it);
              }
            add[t] = ta[t] + tb[t];
          }
        }
        lsum[0] = fmaf(add[0], out, lsum[0]);
        lsum[1] = fmaf(add[1], out, lsum[1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    if (__builtin_expect(n1.masked, 0)) hide(T, n1, u + 1);
    const uint4 p[2][2] = {{pb[0][0], pb[0][1]}, {pb[1][0], pb[1][1]}};
    const float sub1[2] = {ref[0] - n1.lv, ref[1] - n1.lv};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (K(u + 1) has been read: its stage may be filled; of V only what is used next is waited for early)
    if (!STEADY) copy_all(n3, false, kn);
    bf16x8 vop = v_op(vr[0], 0), vop1;
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 1");  // (two wait states between the operands and the first matrix instruction)
    in_steps<PH>([&](auto number) {
      constexpr int j = decltype(number)::value, i = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0 && j / kEvery < NC;
      if (copies) copy_aim(false, kn, j / kEvery);
      mm_o<D, F16>(o[i % DVB][j & 1], vop, __builtin_bit_cast(bf16x8, p[j & 1][i / DVB]));
      __builtin_amdgcn_sched_barrier(0);
      if (copies) copy_piece(n3, false, j / kEvery);
      if (j == PH - 2 * kAhead) {  // K(u + 2) has landed; newer: V(u + 1) and what has been requested of K(u + 3)
        constexpr int part = (PH - 2 * kAhead) / kEvery + 1 < NC ? (PH - 2 * kAhead) / kEvery + 1 : NC;
        win_wait<NC + (STEADY ? part : NC)>();
      }
      if constexpr (j % 2 == 0) {
        constexpr int to = i + kAhead;
        if constexpr (to < KS) {
          if constexpr (to < NV) vr[to] = read_v(vc_, to);
        } else if constexpr (!(PAGED && (to - KS) % 2)) {
          kcur[PAGED ? (to - KS) / 2 : to - KS] = read_k(par, PAGED ? (to - KS) / 2 : to - KS);
        }
        if constexpr (i + 1 < KS) {
          vop1 = v_op(vr[(i + 1) % NV], (i + 1) / DVB);
          if (PAGED) asm volatile("" : "+v"(vop1));  // (made here, two instructions and more ahead of its use)
        }
      } else {
        vop = vop1;
      }
      p_ops(T, std::integral_constant<int, ticks.ahead[TK::in_pv(j)]>{}, std::integral_constant<int, ticks.ahead[TK::in_pv(j + 1)]>{}, n1.f, sub1);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (D == 128 && !STEADY) mfma_fence();  // (O may be moved to other registers between one form of this and another)
    cur = n1;
    n1 = n2;
    n2 = n3;
  };
  if (nu > 0) {
    // units whose copies (of the next one's V and of K three on) are of 32 rows that are there: all, or not the last of either run of keys
    int whole = PAGED ? nu : 0;
    if (!PAGED && kc.plain(nk - 32 * (walk.n_sink - 1)) && vc.plain(32))
      whole = nk - walk.begin(walk.n - 1) >= 32 ? nu : (min(end, walk.n - 1) - begin - wave + NW - 1) / NW - 3;
    int u = 0;
    for (; u + 1 < whole; u += 2) {
      body(std::true_type{}, 0, s0, s1, u);
      body(std::true_type{}, 1, s1, s0, u + 1);
    }
    if (D == 128) mfma_fence();
    for (; u < nu; ++u) {
      body(std::false_type{}, u & 1, s0, s1, u);
      s0[0] = s1[0];
      s0[1] = s1[1];
    }
    win_wait<0>();  // (the copies made for units behind the last one land before their place is used again)
  }
  mfma_fence();  // the last matrix results land before they are read
#pragma unroll
  for (int x = 0; x < DVB; ++x) pin_o(o[x][0]), pin_o(o[x][1]);
  __builtin_amdgcn_sched_barrier(0);

  // merge: reference and sum of a column by way of LDS, O normalised by its own wavefront
  float M[2], L[2], fac[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    M[t] = ref[t];
    L[t] = lsum[t] + __shfl_xor(lsum[t], 32);
    if (NW > 1 && h == 0) *(float2*)&ml[(wave * 64 + t * 32 + l32) * 2] = make_float2(M[t], L[t]);
  }
  if (NW > 1) __syncthreads();
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const float own = M[t];
    if (NW > 1) {
      float m[NW], l[NW];
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        m[w] = ml[(w * 64 + t * 32 + l32) * 2];
        l[w] = ml[(w * 64 + t * 32 + l32) * 2 + 1];
        M[t] = fmaxf(M[t], m[w]);
      }
      L[t] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) L[t] += l[w] * fast_exp2(m[w] - M[t]);
    }
    const bool none = M[t] <= kUnset;
    fac[t] = none ? 0.f : live > 1 ? fast_exp2(own - M[t]) : fast_exp2(own - M[t]) / L[t];  // (parts: normalised when they are joined)
    const int r = t * 32 + l32;
    if (live > 1) {
      if (h == 0 && wave == 0) *(float2*)&parts[(long long)blockIdx.x * (64 * (D + 2)) + 64 * D + 2 * r] = make_float2(M[t], L[t]);
    } else if (a.lse && h == 0 && wave == 0 && r < rows)
      a.lse[a.stat(hq, b, sq.row0, r0 + r)] = none ? -INFINITY : (M[t] + fast_log2(L[t])) * kLn2;
  }
  float* const part = (float*)mine;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int x = 0; x < DVB; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4*)&part[merge_offset(t * 32 + l32, x * 32 + 8 * i + 4 * h, D)] =
            make_float4(o[x][t][4 * i] * fac[t], o[x][t][4 * i + 1] * fac[t], o[x][t][4 * i + 2] * fac[t], o[x][t][4 * i + 3] * fac[t]);
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  float* const slot = parts + (long long)blockIdx.x * (64 * (D + 2));
  const unsigned ostride = (unsigned)a.o.token;
  unsigned char* const orow = a.o.out(b, sq.row0 + r0, hq);
  win_rows_out<D, NW>((const float*)smem, 64 * D, tid, rows, [&](int r, int ch, const float* v) {
    if (live > 1) {
      *(float4*)&slot[r * D + ch * 8] = make_float4(v[0], v[1], v[2], v[3]);
      *(float4*)&slot[r * D + ch * 8 + 4] = make_float4(v[4], v[5], v[6], v[7]);
      return;
    }
    const uint4 u = {pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7])};
    *((uint4*)(orow + (size_t)((unsigned)r * ostride)) + ch) = u;
  });
}

// The parts of a block joined in order: one workgroup a block, 8 elements a thread and turn.
template <int D, bool F16, bool PAGED>
__global__ __launch_bounds__(256) void k_window_merge(WinArgs a, CacheArgs cache, RowPlan plan, const float* __restrict__ parts) {
  // (the number of the first part's workgroup: parts of a block are neighbours among the items of a head)
  __shared__ float weight[16][64];
  int head, item;
  const bool packed = a.rq.cu != nullptr;
  const unsigned heads = (unsigned)(packed ? a.Hkv : a.B * a.Hkv), per_head = (unsigned)(plan.blocks * a.G);
  if (!win_item(blockIdx.x, heads, per_head, head, item)) return;
  const int g = item % a.G, block = plan.blocks - 1 - item / a.G;
  int b, hk, qb;
  WinSeq sq = {0, a.rq.most}, sk = {0, a.rk.most};
  if (packed) {
    hk = head;
    if (!win_find(a.rq, PAGED ? nullptr : &a.rk, a.B, (unsigned)block, b, qb, sq, sk)) return;
  } else {
    b = head / a.Hkv, hk = head - b * a.Hkv, qb = block;
  }
  const int hq = hk * a.G + g, r0 = qb * 64, rows = min(64, sq.n - r0);
  if (rows <= 0) return;
  const int nk = PAGED ? max(0, min(cache.lens[b], cache.max_pages * kPage)) : sk.n, shift = nk - sq.n;
  const WinWalk walk(a.mask, r0 + shift, r0 + rows - 1 + shift, nk, 32, PAGED ? 32 : 1);
  const int want = (walk.n + plan.per - 1) / plan.per, live = want <= 1 ? 1 : want < plan.parts ? want : plan.parts;
  if (live == 1) return;
  // workgroup number of part p: the inverse of win_item
  auto place = [&](int p) {
    const unsigned n = (unsigned)(item * plan.parts + p), full = per_head * (unsigned)plan.parts, whole = heads >> 3, rest = heads & 7u;
    if ((unsigned)head < 8u * whole) return ((unsigned)head >> 3) * full * 8u + n * 8u + ((unsigned)head & 7u);
    const unsigned j = n * rest + ((unsigned)head - 8u * whole);
    return (whole * full + (j >> 3)) * 8u + (j & 7u);
  };
  auto part = [&](int p) { return parts + (long long)place(p) * (64 * (D + 2)); };
  if (threadIdx.x < (unsigned)rows) {
    const int r = threadIdx.x;
    float M = kUnset, L = 0.f;
    for (int p = 0; p < live; ++p) M = fmaxf(M, part(p)[64 * D + 2 * r]);
    for (int p = 0; p < live; ++p) {
      const float2 ml = *(const float2*)&part(p)[64 * D + 2 * r];
      const float w = fast_exp2(ml.x - M);
      weight[p][r] = w;
      L += w * ml.y;
    }
    const bool none = M <= kUnset;
    for (int p = 0; p < live; ++p) weight[p][r] = none ? 0.f : weight[p][r] / L;
    if (a.lse) a.lse[a.stat(hq, b, sq.row0, r0 + r)] = none ? -INFINITY : (M + fast_log2(L)) * kLn2;
  }
  __syncthreads();
  for (int it = threadIdx.x; it < rows * (D / 8); it += 256) {
    const int r = it / (D / 8), ch = it % (D / 8);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < live; ++p) {
      const float* x = part(p) + r * D + ch * 8;
      const float4 y0 = *(const float4*)x, y1 = *(const float4*)(x + 4);
      const float w = weight[p][r];
      v[0] = fmaf(w, y0.x, v[0]), v[1] = fmaf(w, y0.y, v[1]), v[2] = fmaf(w, y0.z, v[2]), v[3] = fmaf(w, y0.w, v[3]);
      v[4] = fmaf(w, y1.x, v[4]), v[5] = fmaf(w, y1.y, v[5]), v[6] = fmaf(w, y1.z, v[6]), v[7] = fmaf(w, y1.w, v[7]);
    }
    const uint4 u = {pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7])};
    *((uint4*)a.o.out(b, sq.row0 + r0 + r, hq) + ch) = u;
  }
}

// Wavefronts a block and parts of its walk, by the time they would take: generations of the workgroups that fit at once (a wavefront
// takes a SIMD, 1024 in all; d = 64: half of one) times the units of one, kStart units' worth of start-up and stores each, and where
// there are parts what writing and joining them takes.  (A unit is about 0.7 us.  2048 tokens, two heads, d = 64: one wavefront a
// block 21 us, four 10; 1560 queries on a cache of 32760 tokens, 12 heads, d = 128: unsplit 188 us, in parts 140.  Of 38 shapes of 64
// to 8192 queries on up to 32760 keys the plan is within 10 % of the best of one or four wavefronts, one, two or four parts.)
static RowPlan row_plan(const WinArgs& a, long long max_k, int d) {
  constexpr long long kStart = 6, kJoin = 10;
  RowPlan best = {};
  const long long n = win_blocks(a.rq, a.B) * a.H, units = win_units(a.mask, max_k);
  long long least = -1;
  for (int nw = 1; nw <= 4; nw *= 4)
    for (int p = 1; p <= 16; ++p) {
      const long long places = (d == 64 ? 2048 : 1024) / nw, each = (units + nw * p - 1) / (nw * p);
      if (p > 1 && each < 4) break;
      const long long gens = (n * p + places - 1) / places;
      const long long time = gens * (each + kStart + (nw > 1 ? 2 : 0)) + (p > 1 ? kJoin + n * p / 64 + p : 0);
      if (least < 0 || time < least) {
        least = time;
        best.nw = nw, best.parts = p, best.per = (int)((units + p - 1) / p);
      }
    }
  best.blocks = (int)(a.rq.cu ? win_blocks(a.rq, a.B) : (a.rq.most + 63) / 64);
  return best;
}
size_t row_parts(const WinArgs& a, long long max_k, int d) {
  const RowPlan p = row_plan(a, max_k, d);
  return p.parts > 1 ? (size_t)win_grid(win_workgroups(a, p)) * (64 * (d + 2)) : 0;
}

namespace {
template <int D, bool F16, bool PAGED>
hipError_t launch(const WinArgs& a, const CacheArgs& c, float* parts, hipStream_t s) {
  const RowPlan plan = row_plan(a, PAGED ? (long long)c.max_pages * kPage : a.rk.most, D);
  const unsigned grid = win_grid(win_workgroups(a, plan));
  if (plan.nw == 4) k_window_fwd<D, F16, 4, PAGED><<<grid, 256, 0, s>>>(a, c, plan, parts);
  else k_window_fwd<D, F16, 1, PAGED><<<grid, 64, 0, s>>>(a, c, plan, parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || plan.parts == 1) return e;
  k_window_merge<D, F16, PAGED><<<win_grid(win_workgroups(a, plan) / plan.parts), 256, 0, s>>>(a, c, plan, parts);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_window_fwd(const WinArgs& a, int d, bool f16, float* parts, hipStream_t s) {
  const CacheArgs none = {};
  if (d == 128) return f16 ? launch<128, true, false>(a, none, parts, s) : launch<128, false, false>(a, none, parts, s);
  return f16 ? launch<64, true, false>(a, none, parts, s) : launch<64, false, false>(a, none, parts, s);
}

hipError_t launch_cache_chunk(const WinArgs& a, const CacheArgs& c, int d, bool f16, float* parts, hipStream_t s) {
  if (d == 128) return f16 ? launch<128, true, true>(a, c, parts, s) : launch<128, false, true>(a, c, parts, s);
  return f16 ? launch<64, true, true>(a, c, parts, s) : launch<64, false, true>(a, c, parts, s);
}

}  // namespace vsa
