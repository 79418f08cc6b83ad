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

template <int D, bool F16, int NW, bool PAGED>
__global__ __launch_bounds__(64 * NW, D == 128 ? 1 : 2) void k_window_fwd(WinArgs a, CacheArgs cache, unsigned items, int nqb, int chunked) {
  using TL = Tile<D>;
  constexpr int KS = D / 16, DVB = D / 32, HALF = 32 * D * 2, STAGE = PAGED ? HALF / 2 : HALF;
  constexpr int NC = PAGED ? PageCopy<D>::NC : RowCopy<D>::NC;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * 4 * HALF];
  __shared__ float ml[NW * 64 * 2];

  int b;
  unsigned item;
  if (!win_item(blockIdx.x, items, chunked != 0, b, item)) return;
  const int g = (int)(item % (unsigned)a.G), rest = (int)(item / (unsigned)a.G);
  const int hk = rest / nqb, qb = chunked ? rest % nqb : nqb - 1 - rest % nqb, hq = hk * a.G + g;
  const WinSeq sq = win_seq(a.rq, b);
  const int r0 = qb * 64, rows = min(64, sq.n - r0);
  if (rows <= 0) return;
  WinSeq sk = {0, 0};
  if constexpr (PAGED) sk.n = max(0, min(cache.lens[b], cache.max_pages * kPage));
  else sk = win_seq(a.rk, b);
  const int nk = sk.n, shift = nk - sq.n;
  const WinWalk walk(a.mask, r0 + shift, r0 + rows - 1 + shift, nk, 32, PAGED ? 32 : 1);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int nu = walk.n > wave ? (walk.n - wave + NW - 1) / NW : 0;
  WinSpan span[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) span[t] = win_span(a.mask, min(r0 + 32 * t + l32, sq.n - 1) + shift, nk);

  // Q: of a page's operands, contraction step 2 sp + e holds elements 32 sp + 16 h + 8 e ..
  bf16x8 qreg[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint4* p = (const uint4*)a.q.row(b, sq.row0 + min(r0 + 32 * t + l32, sq.n - 1), hq);
#pragma unroll
    for (int s = 0; s < KS; ++s) qreg[t][s] = __builtin_bit_cast(bf16x8, p[PAGED ? 4 * (s >> 1) + 2 * h + (s & 1) : 2 * s + h]);
  }
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qreg[0][s]), "+v"(qreg[1][s]));  // (waited for here, ahead of the copies)

  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * (4 * HALF);
  unsigned char* const mine = smem + wave * (4 * HALF);
  const unsigned kstride = (unsigned)a.k.token, vstride = (unsigned)a.v.token;
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
    kc.init(lane, kstride);
    vc.init(lane, vstride);
  }
  struct U {
    int a;            // first key
    bool masked;
    int page;         // PAGED: its page, or -1
    float sk, lv;     // PAGED: scale of K, log2 of the scale of V
  };
  auto unit = [&](int u) {
    const int i = wave + NW * min(u, nu - 1);
    U x = {walk.begin(i), walk.masked(i), 0, 1.f, 0.f};
    if constexpr (PAGED) {
      const int e = x.a / kPage;
      pages.want(e);
      x.page = pages.page_id(e);
      x.masked |= x.page < 0;
      x.sk = pages.scale_k(e);
      x.lv = fast_log2(pages.scale_v(e));
    }
    return x;
  };
  auto page_base = [&](const uint8_t* pool, const U& x, int bytes) {
    return (const unsigned char*)uniform_ptr(pool + ((long long)max(x.page, 0) * a.Hkv + hk) * (kPage * D) + bytes);
  };
  auto copy_k = [&](const U& x, int stage) {
    if constexpr (PAGED) {
      const unsigned char* base = page_base(cache.k, x, (x.a & 32) * D);
#pragma unroll
      for (int c = 0; c < NC; ++c) win_copy16(base, pc.ko[c], lds0 + stage * STAGE + c * 1024);
    } else {
      kc.all(kb + (long long)x.a * kstride, lds0 + stage * STAGE, lane, kstride, nk - x.a);
    }
  };
  auto copy_v = [&](const U& x, int stage) {
    if constexpr (PAGED) {
      const unsigned char* base = page_base(cache.v, x, x.a & 32);
#pragma unroll
      for (int c = 0; c < NC; ++c) win_copy16(base, pc.vo[c], lds0 + (2 + stage) * STAGE + c * 1024);
    } else {
      vc.all(vb + (long long)x.a * vstride, lds0 + (2 + stage) * STAGE, lane, vstride, nk - x.a);
    }
  };

  f32x16 o[DVB][2], s[2];
#pragma unroll
  for (int x = 0; x < DVB; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[x][t][i] = 0.f;
  float ref[2] = {kUnset, kUnset}, lsum[2] = {0.f, 0.f};
  bool have = false;  // every column has a reference
  const float sl2 = a.scale * kLog2e;
  f32x16 zero16;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero16[i] = 0.f;

  if (nu > 0) {
    U cur = unit(0);
    copy_k(cur, 0);
    copy_v(cur, 0);
    for (int u = 0; u < nu; ++u) {
      const int par = u & 1;
      const U next = unit(u + 1);
      if (u + 1 < nu) {
        copy_k(next, 1 - par);
        copy_v(next, 1 - par);
        win_wait<2 * NC>();
      } else {
        win_wait<0>();
      }
      const unsigned char *ks = mine + par * STAGE, *vs = mine + (2 + par) * STAGE;
      if (PAGED && cur.a + 32 > nk) {  // values behind the last token may be anything: zero
        const int live = nk - cur.a;
#pragma unroll
        for (int dv = lane; dv < D; dv += 64) {
          unsigned* p = (unsigned*)(vs + dv * 32);
          for (int w = 0; w < 8; ++w) {
            const int key = ((w >> 2) ^ ((dv >> 3) & 1)) * 16 + (w & 3) * 4, keep = min(4, max(0, live - key));
            p[w] = keep == 4 ? p[w] : p[w] & ((1u << (8 * keep)) - 1u);
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
      // S^T
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        bf16x8 ka;
        if constexpr (PAGED) {
          const uint4 raw = PageCopy<D>::k_at(ks, lane, st >> 1);
          ka = st & 1 ? from_e4m3<F16>(raw.z, raw.w) : from_e4m3<F16>(raw.x, raw.y);
        } else {
          ka = TL::rowmajor_at(ks, TL::rowmajor_lane(0, lane), st);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mm32<F16>(ka, qreg[t][st], st == 0 ? zero16 : s[t]);
      }
      const float f = sl2 * cur.sk;
      if (cur.masked) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const WinSpan w = walk.span_in(wave + NW * u, span[t]);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = cur.a + (PAGED ? 16 * h + i : 8 * (i >> 2) + 4 * h + (i & 3));
            const bool see = key < w.hi && (key >= w.lo || key < w.se) && (!PAGED || cur.page >= 0);
            s[t][i] = see ? s[t][i] : -INFINITY;
          }
        }
      }
      // P^T: the reference is the running maximum
      uint32_t p[2][8];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float m = s[t][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, s[t][i]);
        m = fmaxf(fmaf(max_across_halves(m), f, cur.lv), ref[t]);
        if (__any(m > ref[t])) {
          const float alpha = fast_exp2(ref[t] - m);
          lsum[t] *= alpha;
#pragma unroll
          for (int x = 0; x < DVB; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][t][i] *= alpha;
          ref[t] = m;
        }
        float e[16], sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          e[i] = fast_exp2(fmaf(s[t][i], f, cur.lv - ref[t]));
          sum += e[i];
        }
        lsum[t] += PAGED ? sum * fast_exp2(-cur.lv) : sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[t][i] = pack16<F16>(e[2 * i], e[2 * i + 1]);
      }
      // O^T
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        bf16x8 pop[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) pop[t] = __builtin_bit_cast(bf16x8, make_uint4(p[t][4 * st], p[t][4 * st + 1], p[t][4 * st + 2], p[t][4 * st + 3]));
#pragma unroll
        for (int x = 0; x < DVB; ++x) {
          bf16x8 va;
          if constexpr (PAGED) {
            const uint4 raw = PageCopy<D>::v_at(vs, lane, x);
            va = st ? from_e4m3<F16>(raw.z, raw.w) : from_e4m3<F16>(raw.x, raw.y);
          } else {
            int b0, b1;
            TL::transposed_lane(0, lane, b0, b1);
            va = TL::transposed_at(vs, b0, b1, st, x);
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) o[x][t] = mm32<F16>(va, pop[t], o[x][t]);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // every read of the stages is over: they may be filled again
      __builtin_amdgcn_sched_barrier(0);
      cur = next;
    }
  }
  (void)have;

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
    fac[t] = none ? 0.f : fast_exp2(own - M[t]) / L[t];
    const int r = t * 32 + l32;
    if (a.lse && h == 0 && wave == 0 && r < rows)
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
  for (int it = tid; it < 64 * TL::CPR; it += 64 * NW) {
    const int r = it / TL::CPR, ch = it % TL::CPR;
    if (r >= rows) break;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float* q = (const float*)smem + w * 64 * D;
      const float4 x = *(const float4*)&q[merge_offset(r, ch * 8, D)], y = *(const float4*)&q[merge_offset(r, ch * 8 + 4, D)];
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
    }
    uint4 u = {pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7])};
    *((uint4*)a.o.out(b, sq.row0 + r0 + r, hq) + ch) = u;
  }
}

namespace {
template <int D, bool F16, bool PAGED>
hipError_t launch(const WinArgs& a, const CacheArgs& c, hipStream_t s) {
  const int nqb = (a.rq.most + 63) / 64;
  const unsigned items = (unsigned)nqb * (unsigned)a.H, grid = win_grid(a.B, items);
  const int chunked = a.mask.left >= 0;
  const long long blocks = (long long)items * a.B;
  if (blocks <= 512) k_window_fwd<D, F16, 4, PAGED><<<grid, 256, 0, s>>>(a, c, items, nqb, chunked);
  else k_window_fwd<D, F16, 1, PAGED><<<grid, 64, 0, s>>>(a, c, items, nqb, chunked);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_window_fwd(const WinArgs& a, int d, bool f16, hipStream_t s) {
  const CacheArgs none = {};
  if (d == 128) return f16 ? launch<128, true, false>(a, none, s) : launch<128, false, false>(a, none, s);
  return f16 ? launch<64, true, false>(a, none, s) : launch<64, false, false>(a, none, s);
}

hipError_t launch_cache_chunk(const WinArgs& a, const CacheArgs& c, int d, bool f16, hipStream_t s) {
  if (d == 128) return f16 ? launch<128, true, true>(a, c, s) : launch<128, false, true>(a, c, s);
  return f16 ? launch<64, true, true>(a, c, s) : launch<64, false, true>(a, c, s);
}

}  // namespace vsa
