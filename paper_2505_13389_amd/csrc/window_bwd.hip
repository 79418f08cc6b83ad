// Windowed attention, backward: two passes over the visible pairs, with P formed again from the saved log-sum-exp.
//
//   P = exp(scale q.k - lse),  D = rowsum(dO * O),  dS = P * (dO V^T - D)
//   k_window_dq:  a wavefront has 64 queries, walks units of 32 keys      dQ = scale dS K
//   k_window_dkv: a wavefront has 64 keys, walks units of 32 queries of all heads of its group      dV = P^T dO, dK = scale dS^T Q
// The second sums shared heads on the way, in order: no atomics, the same bits every time.  S and dP are formed twice (7 products
// for 5), which costs less than passing P and dS through memory.  As in the forward a lane owns columns of 32 (queries, keys), the
// other index runs through its registers, and what has been formed in them is the operand of the product over that index.
#include "window_kernels.h"
#include "window_tile.h"

namespace vsa {

// D and the log-sum-exp in log2 units, a float2 a row: 8 elements a lane
template <int D, bool F16>
__global__ __launch_bounds__(256) void k_window_stats(WinArgs a) {
  constexpr int CPR = D / 8;
  const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) / CPR;
  const int ch = threadIdx.x % CPR;
  const long long n = a.lse_rows * a.H;
  const long long row = (at < n ? at : n - 1) / a.H;  // heads of a row side by side
  const int h = (int)((at < n ? at : n - 1) % a.H);
  const int b = a.rq.cu ? 0 : (int)(row / a.rq.most);
  const long long t = a.rq.cu ? row : row % a.rq.most;
  float o[8], d[8], sum = 0.f;
  widen8<F16>(*((const uint4*)a.o.row(b, t, h) + ch), o);
  widen8<F16>(*((const uint4*)a.dout.row(b, t, h) + ch), d);
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(o[e], d[e], sum);
#pragma unroll
  for (int m = CPR / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
  if (at >= n || ch) return;
  const float lse = a.lse[h * a.lse_rows + row];
  a.stats[h * a.lse_rows + row] = make_float2(lse == -INFINITY ? INFINITY : lse * kLog2e, sum);
}

// accumulator tiles [32 x ..][64 columns] of NW wavefronts -> rows of 16 bits, scaled; `buf`: 64 * D floats a wavefront
template <int D, bool F16, int NW, int CT, class ROW>
__device__ __forceinline__ void store_columns(const f32x16 (&acc)[D / 32][CT], float scale, float* buf, int tid, int rows, const ROW& row_of) {
  const int lane = tid & 63, wave = tid >> 6, l32 = lane & 31, h = lane >> 5;
  float* const mine = buf + wave * 32 * CT * D;
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4*)&mine[merge_offset(t * 32 + l32, x * 32 + 8 * i + 4 * h, D)] =
            make_float4(acc[x][t][4 * i], acc[x][t][4 * i + 1], acc[x][t][4 * i + 2], acc[x][t][4 * i + 3]);
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  for (int it = tid; it < rows * (D / 8); it += 64 * NW) {
    const int r = it / (D / 8), ch = it % (D / 8);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float* q = buf + w * 32 * CT * D;
      const float4 x = *(const float4*)&q[merge_offset(r, ch * 8, D)], y = *(const float4*)&q[merge_offset(r, ch * 8 + 4, D)];
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= scale;
    const uint4 u = {pack16<F16>(v[0], v[1]), pack16<F16>(v[2], v[3]), pack16<F16>(v[4], v[5]), pack16<F16>(v[6], v[7])};
    *((uint4*)row_of(r) + ch) = u;
  }
}

template <int D, bool F16, int NW>
__global__ __launch_bounds__(64 * NW, 1) void k_window_dq(WinArgs a, unsigned items, int nqb, int chunked) {
  using TL = Tile<D>;
  constexpr int KS = D / 16, DVB = D / 32, HALF = 32 * D * 2, NC = RowCopy<D>::NC;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * 4 * HALF];
  int b;
  unsigned item;
  if (!win_item(blockIdx.x, items, chunked != 0, b, item)) return;
  const int g = (int)(item % (unsigned)a.G), rest = (int)(item / (unsigned)a.G);
  const int hk = rest / nqb, qb = chunked ? rest % nqb : nqb - 1 - rest % nqb, hq = hk * a.G + g;
  const WinSeq sq = win_seq(a.rq, b), sk = win_seq(a.rk, b);
  const int r0 = qb * 64, rows = min(64, sq.n - r0);
  if (rows <= 0) return;
  const int nk = __builtin_amdgcn_readfirstlane(sk.n), shift = nk - sq.n;
  WinWalk walk(a.mask, r0 + shift, r0 + rows - 1 + shift, nk, 32, 1);
  walk.uniform();
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int nu = walk.n > wave ? (walk.n - wave + NW - 1) / NW : 0;

  WinSpan span[2];
  float lse2[2], delta[2];
  bf16x8 qreg[2][KS], dreg[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = min(r0 + 32 * t + l32, sq.n - 1);
    span[t] = win_span(a.mask, r + shift, nk);
    const float2 st = a.stats[a.stat(hq, b, sq.row0, r)];
    lse2[t] = st.x, delta[t] = st.y;
    const uint4 *p = (const uint4*)a.q.row(b, sq.row0 + r, hq), *pd = (const uint4*)a.dout.row(b, sq.row0 + r, hq);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qreg[t][s] = __builtin_bit_cast(bf16x8, p[2 * s + h]);
      dreg[t][s] = __builtin_bit_cast(bf16x8, pd[2 * s + h]);
    }
  }
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qreg[0][s]), "+v"(qreg[1][s]), "+v"(dreg[0][s]), "+v"(dreg[1][s]));
  asm volatile("" : "+v"(lse2[0]), "+v"(lse2[1]), "+v"(delta[0]), "+v"(delta[1]));

  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * (4 * HALF);
  unsigned char* const mine = smem + wave * (4 * HALF);
  const unsigned kstride = (unsigned)a.k.token, vstride = (unsigned)a.v.token;
  const unsigned char* kb = (const unsigned char*)uniform_ptr(a.k.row(b, sk.row0, hk));
  const unsigned char* vb = (const unsigned char*)uniform_ptr(a.v.row(b, sk.row0, hk));
  RowCopy<D> kc, vc;
  kc.init(lane, kstride);
  vc.init(lane, vstride);
  auto copy = [&](int u, int stage) {
    const int at = walk.begin(wave + NW * u);
    kc.all(kb + (long long)at * kstride, lds0 + stage * HALF, lane, nk - at);
    vc.all(vb + (long long)at * vstride, lds0 + (2 + stage) * HALF, lane, nk - at);
  };
  f32x16 acc[DVB][2], zero16;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero16[i] = 0.f;
#pragma unroll
  for (int x = 0; x < DVB; ++x) acc[x][0] = acc[x][1] = zero16;
  const float sl2 = a.scale * kLog2e;
  const int lane_a = TL::rowmajor_lane(0, lane);
  int b0, b1;
  TL::transposed_lane(0, lane, b0, b1);

  if (nu > 0) copy(0, 0);
  for (int u = 0; u < nu; ++u) {
    const int par = u & 1, piece = wave + NW * u;
    if (u + 1 < nu) {
      copy(u + 1, 1 - par);
      win_wait<2 * NC>();
    } else {
      win_wait<0>();
    }
    const unsigned char *ks = mine + par * HALF, *vs = mine + (2 + par) * HALF;
    f32x16 s[2], p[2];
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      const bf16x8 ka = TL::rowmajor_at(ks, lane_a, st), va = TL::rowmajor_at(vs, lane_a, st);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s[t] = mm32<F16>(ka, qreg[t][st], st == 0 ? zero16 : s[t]);
        p[t] = mm32<F16>(va, dreg[t][st], st == 0 ? zero16 : p[t]);
      }
    }
    const int key0 = walk.begin(piece);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = fast_exp2(fmaf(s[t][i], sl2, -lse2[t])) * (p[t][i] - delta[t]);
    if (walk.masked(piece)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const WinSpan w = walk.span_in(piece, span[t]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 8 * (i >> 2) + 4 * h + (i & 3);
          s[t][i] = key < w.hi && (key >= w.lo || key < w.se) ? s[t][i] : 0.f;
        }
      }
    }
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      bf16x8 ds[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint4 w = {pack16<F16>(s[t][8 * st], s[t][8 * st + 1]), pack16<F16>(s[t][8 * st + 2], s[t][8 * st + 3]),
                   pack16<F16>(s[t][8 * st + 4], s[t][8 * st + 5]), pack16<F16>(s[t][8 * st + 6], s[t][8 * st + 7])};
        ds[t] = __builtin_bit_cast(bf16x8, w);
      }
#pragma unroll
      for (int x = 0; x < DVB; ++x) {
        const bf16x8 ka = TL::transposed_at(ks, b0, b1, st, x);
#pragma unroll
        for (int t = 0; t < 2; ++t) acc[x][t] = mm32<F16>(ka, ds[t], acc[x][t]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  if (NW > 1) __syncthreads();
  store_columns<D, F16, NW, 2>(acc, a.scale, (float*)smem, tid, rows, [&](int r) { return a.dq.out(b, sq.row0 + r0 + r, hq); });
}

// columns of 32 keys of a wavefront: at d = 128 two need more than 512 registers
template <int D>
constexpr int dkv_tiles() { return D == 128 ? 1 : 2; }

template <int D, bool F16, int NW>
__global__ __launch_bounds__(64 * NW, 1) void k_window_dkv(WinArgs a, unsigned items, int nkb, int chunked) {
  using TL = Tile<D>;
  constexpr int KT = dkv_tiles<D>(), KS = D / 16, DVB = D / 32, HALF = 32 * D * 2, NC = RowCopy<D>::NC;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[NW * 4 * HALF];
  __shared__ __attribute__((aligned(256))) float2 stat_stage[NW][2][32];
  int b;
  unsigned item;
  if (!win_item(blockIdx.x, items, chunked != 0, b, item)) return;
  const int hk = (int)(item / (unsigned)nkb), kblk = (int)(item % (unsigned)nkb);
  const WinSeq sq = win_seq(a.rq, b), sk = win_seq(a.rk, b);
  const int k0 = kblk * (32 * KT), keys = min(32 * KT, sk.n - k0);
  if (keys <= 0) return;
  const int shift = sk.n - sq.n;
  const KeyWalk walk(a.mask, k0, k0 + keys, sq.n, shift, 32);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int all = walk.n * a.G, nu = all > wave ? (all - wave + NW - 1) / NW : 0;

  int from[KT], to[KT];  // queries that see the lane's keys
  bf16x8 kreg[KT][KS], vreg[KT][KS];
#pragma unroll
  for (int t = 0; t < KT; ++t) {
    const int j = min(k0 + 32 * t + l32, sk.n - 1);
    const KeySpan w = key_span(a.mask, j);
    auto clamp = [&](long long x) { return (int)(x < 0 ? 0 : x > sq.n ? sq.n : x); };
    from[t] = clamp(w.lo - shift);
    to[t] = clamp(w.hi - shift);
    const uint4 *p = (const uint4*)a.k.row(b, sk.row0 + j, hk), *pv = (const uint4*)a.v.row(b, sk.row0 + j, hk);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kreg[t][s] = __builtin_bit_cast(bf16x8, p[2 * s + h]);
      vreg[t][s] = __builtin_bit_cast(bf16x8, pv[2 * s + h]);
    }
  }
#pragma unroll
  for (int t = 0; t < KT; ++t)
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(kreg[t][s]), "+v"(vreg[t][s]));

  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * (4 * HALF);
  const unsigned stat0 = __builtin_amdgcn_readfirstlane(lds_address(stat_stage)) + (unsigned)wave * 512u;
  unsigned char* const mine = smem + wave * (4 * HALF);
  const unsigned qstride = (unsigned)a.q.token, dstride = (unsigned)a.dout.token;
  RowCopy<D> qc, dc;
  qc.init(lane, qstride);
  dc.init(lane, dstride);
  auto copy = [&](int u, int stage) {
    const int i = wave + NW * u, g = i / walk.n, at = walk.from + (i - g * walk.n) * 32, hq = hk * a.G + g, have = sq.n - at;
    const unsigned char* qb = (const unsigned char*)uniform_ptr(a.q.row(b, sq.row0 + at, hq));
    const unsigned char* db = (const unsigned char*)uniform_ptr(a.dout.row(b, sq.row0 + at, hq));
    const void* sb = uniform_ptr(a.stats + a.stat(hq, b, sq.row0, at));
    qc.all(qb, lds0 + stage * HALF, lane, have);
    dc.all(db, lds0 + (2 + stage) * HALF, lane, have);
    lds_dma4<4>(sb, (unsigned)min(lane >> 1, have - 1) * 8u + (lane & 1) * 4u, stat0 + stage * 256u);
  };
  f32x16 dk[DVB][KT], dv[DVB][KT], zero16;
#pragma unroll
  for (int i = 0; i < 16; ++i) zero16[i] = 0.f;
#pragma unroll
  for (int x = 0; x < DVB; ++x)
#pragma unroll
    for (int t = 0; t < KT; ++t) dk[x][t] = dv[x][t] = zero16;
  const float sl2 = a.scale * kLog2e;
  const int lane_a = TL::rowmajor_lane(0, lane);
  int b0, b1;
  TL::transposed_lane(0, lane, b0, b1);

  if (nu > 0) copy(0, 0);
  for (int u = 0; u < nu; ++u) {
    const int par = u & 1;
    if (u + 1 < nu) {
      copy(u + 1, 1 - par);
      win_wait<2 * NC + 1>();
    } else {
      win_wait<0>();
    }
    const unsigned char *qs = mine + par * HALF, *ds = mine + (2 + par) * HALF;
    const int i0 = wave + NW * u, q0 = walk.from + (i0 % walk.n) * 32;
    const long long pos = (long long)q0 + shift;
    const bool masked = pos < walk.seen_from || pos + 32 > walk.seen_to || q0 + 32 > sq.n;
    uint32_t pw[KT][8], sw[KT][8];
    f32x16 s[KT], p[KT];
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      const bf16x8 qa = TL::rowmajor_at(qs, lane_a, st), da = TL::rowmajor_at(ds, lane_a, st);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        s[t] = mm32<F16>(qa, kreg[t][st], st == 0 ? zero16 : s[t]);
        p[t] = mm32<F16>(da, vreg[t][st], st == 0 ? zero16 : p[t]);
      }
    }
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const float4 x = *(const float4*)&stat_stage[wave][par][8 * r4 + 4 * h], y = *(const float4*)&stat_stage[wave][par][8 * r4 + 4 * h + 2];
      const float lse2[4] = {x.x, x.z, y.x, y.z}, delta[4] = {x.y, x.w, y.y, y.w};
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * r4 + e;
          s[t][i] = fast_exp2(fmaf(s[t][i], sl2, -lse2[e]));
          p[t][i] = s[t][i] * (p[t][i] - delta[e]);
        }
    }
    if (masked) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int q = q0 + 8 * (i >> 2) + 4 * h + (i & 3);
          const bool see = q >= from[t] && q < to[t];
          s[t][i] = see ? s[t][i] : 0.f;
          p[t][i] = see ? p[t][i] : 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pw[t][i] = pack16<F16>(s[t][2 * i], s[t][2 * i + 1]);
        sw[t][i] = pack16<F16>(p[t][2 * i], p[t][2 * i + 1]);
      }
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      bf16x8 po[KT], so[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        po[t] = __builtin_bit_cast(bf16x8, make_uint4(pw[t][4 * st], pw[t][4 * st + 1], pw[t][4 * st + 2], pw[t][4 * st + 3]));
        so[t] = __builtin_bit_cast(bf16x8, make_uint4(sw[t][4 * st], sw[t][4 * st + 1], sw[t][4 * st + 2], sw[t][4 * st + 3]));
      }
#pragma unroll
      for (int x = 0; x < DVB; ++x) {
        const bf16x8 da = TL::transposed_at(ds, b0, b1, st, x), qa = TL::transposed_at(qs, b0, b1, st, x);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          dv[x][t] = mm32<F16>(da, po[t], dv[x][t]);
          dk[x][t] = mm32<F16>(qa, so[t], dk[x][t]);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  if (NW > 1) __syncthreads();
  store_columns<D, F16, NW, KT>(dv, 1.f, (float*)smem, tid, keys, [&](int r) { return a.dv.out(b, sk.row0 + k0 + r, hk); });
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  store_columns<D, F16, NW, KT>(dk, a.scale, (float*)smem, tid, keys, [&](int r) { return a.dk.out(b, sk.row0 + k0 + r, hk); });
}

namespace {
template <int D, bool F16>
hipError_t launch(const WinArgs& a, hipStream_t s) {
  const long long lanes = a.lse_rows * a.H * (D / 8);
  if (lanes > 0) k_window_stats<D, F16><<<(unsigned)((lanes + 255) / 256), 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int nqb = (a.rq.most + 63) / 64, per = 32 * dkv_tiles<D>(), nkb = (a.rk.most + per - 1) / per;
  const int chunked = a.mask.left >= 0;
  if (nqb > 0) {
    const unsigned items = (unsigned)nqb * a.H, grid = win_grid(a.B, items);
    if ((long long)items * a.B <= 512) k_window_dq<D, F16, 4><<<grid, 256, 0, s>>>(a, items, nqb, chunked);
    else k_window_dq<D, F16, 1><<<grid, 64, 0, s>>>(a, items, nqb, chunked);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (nkb > 0) {
    const unsigned items = (unsigned)nkb * a.Hkv, grid = win_grid(a.B, items);
    if ((long long)items * a.B <= 512) k_window_dkv<D, F16, 4><<<grid, 256, 0, s>>>(a, items, nkb, chunked);
    else k_window_dkv<D, F16, 1><<<grid, 64, 0, s>>>(a, items, nkb, chunked);
    e = hipGetLastError();
  }
  return e;
}
}  // namespace

hipError_t launch_window_bwd(const WinArgs& a, int d, bool f16, hipStream_t s) {
  if (d == 128) return f16 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return f16 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace vsa
