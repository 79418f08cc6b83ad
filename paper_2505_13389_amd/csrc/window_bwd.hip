// Windowed attention, backward: two passes over the visible pairs, with P formed again from the saved log-sum-exp.
//
//   P = exp(scale q.k - lse),  D = rowsum(dO * O),  dS = P * (dO V^T - D)
//   k_window_dq:  a wavefront has 64 queries, walks units of 32 keys      dQ = scale dS K
//   k_window_dkv: a wavefront has 64 keys, walks units of 32 queries of all heads of its group      dV = P^T dO, dK = scale dS^T Q
// The second sums shared heads on the way, in order: no atomics, the same bits every time.  S and dP are formed twice (7 products
// for 5), which costs less than passing P and dS through memory.  As in the forward a lane owns columns of 32 (queries, keys), the
// other index runs through its registers, and what has been formed in them is the operand of the product over that index.
//
// Roundings: P and dS go to 16 bits before their products, half a step of each term, as in the fine kernels; D is formed of the O
// that was stored, all sums and the partial results of cut walks are fp32, and a gradient is rounded once.  Against 64 bits 2.7e-3 of
// the norm in bf16 (rounding the exact gradient: 1.7e-3).
//
// Bound by matrix instructions and power at d = 128 (a unit 2340 cycles in dQ, 3050 in dK/dV, of which the matrix pipe 1536 and 2048);
// at d = 64, where P and dS take half of a unit's issue slots, by instruction issue and by start and end of walks.  16384 tokens, 12 heads,
// d = 128, 5 frames of 1024: rows' terms 23 us, both passes 1403, 0.80 PFLOP/s on the visible pairs, the pipe busy 58 % at 1.7 GHz; packed
// texts of 10332 tokens, 16 heads on 4, d = 64, 511 tokens back: 11, 136 and 5 for the join.
#include <type_traits>

#include "unit_stream.h"
#include "window_kernels.h"
#include "window_tile.h"

namespace vsa {

// -lse / scale (-inf for a row that sees nothing) and -D, a plane each: what S and dP start from.  8 elements a lane.
template <int D, bool F16>
__global__ __launch_bounds__(256) void k_window_stats(WinArgs a) {
  constexpr int CPR = D / 8;
  const unsigned at = (blockIdx.x * 256u + threadIdx.x) / CPR, ch = threadIdx.x % CPR;  // (fewer than 2^32 lanes)
  const unsigned n = (unsigned)(a.lse_rows * a.H), here = at < n ? at : n - 1, row = here / (unsigned)a.H;  // heads of a row side by side
  const int h = (int)(here - row * (unsigned)a.H);
  const int b = a.rq.cu || a.B == 1 ? 0 : (int)(row / (unsigned)a.rq.most);
  const long long t = (long long)row - (long long)b * a.rq.most;
  float o[8], d[8], sum = 0.f;
  widen8<F16>(*((const uint4*)a.o.row(b, t, h) + ch), o);
  widen8<F16>(*((const uint4*)a.dout.row(b, t, h) + ch), d);
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(o[e], d[e], sum);
#pragma unroll
  for (int m = CPR / 2; m > 0; m >>= 1) sum += __shfl_xor(sum, m);
  if (at >= n || ch) return;
  const float lse = a.lse[h * a.lse_rows + row];
  a.stats[h * a.lse_rows + row] = lse == -INFINITY ? -INFINITY : -lse / a.scale;
  a.stats[n + h * a.lse_rows + row] = -sum;
}

// dQ, dK, dV lie in the accumulation registers (256 + 256 registers a wavefront, see mfma_a): at d = 64, left to the compiler, parts of
// them were moved there and back in every unit (packed training 188 us, 183 so).
template <int D, bool F16>
__device__ __forceinline__ void mm_acc(f32x16& acc, bf16x8 a, bf16x8 b) {
  if constexpr (F16) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  else mfma_a(acc, a, b);
}
template <int D>
__device__ __forceinline__ void pin_acc(f32x16& acc) {
  asm volatile("" : "+a"(acc));
}
// accumulators in ordinary registers, from the values of c (INIT), or on
template <int D, bool F16, bool INIT>
__device__ __forceinline__ void mm_v(f32x16& d, bf16x8 a, bf16x8 b, const f32x16& c) {
  if constexpr (D == 64) d = mm32<F16>(a, b, INIT ? c : d);
  else if constexpr (F16) {
    if constexpr (INIT) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %3" : "=&v"(d) : "v"(a), "v"(b), "v"(c));
    else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "v"(b));
  } else {
    if constexpr (INIT) mfma_v_from(d, a, b, c);
    else mfma_v(d, a, b);
  }
}
template <int D, bool F16>
__device__ __forceinline__ void mm_v_zero(f32x16& d, bf16x8 a, bf16x8 b) {
  if constexpr (D == 64) {
    f32x16 zero;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.f;
    d = mm32<F16>(a, b, zero);
  } else if constexpr (F16) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
}
// products whose second operand (Q, which is read by these alone) is in the accumulation registers at d = 128; FIRST: from zero
template <int D, bool F16, bool FIRST>
__device__ __forceinline__ void mm_q(f32x16& d, bf16x8 a, bf16x8 q) {
  if constexpr (D == 64) {
    f32x16 zero;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.f;
    d = mm32<F16>(a, q, FIRST ? zero : d);
  } else if constexpr (F16) {
    if constexpr (FIRST) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "a"(q));
    else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "a"(q));
  } else {
    if constexpr (FIRST) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "a"(q));
    else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "a"(q));
  }
}

// accumulator tiles [32 x ..][64 columns] of NW wavefronts -> rows of 16 bits, scaled; `buf`: 64 * D floats a wavefront
template <int D, bool F16, int NW, class ROW>
__device__ __forceinline__ void store_columns(f32x16 (&acc)[D / 32][2], float scale, float* buf, int pitch, int tid, int rows, const ROW& row_of) {
  const int lane = tid & 63, wave = tid >> 6, l32 = lane & 31, h = lane >> 5;
  float* const mine = buf + wave * pitch;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      pin_acc<D>(acc[x][t]);  // (a tile at a time in ordinary registers)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4*)&mine[merge_offset(t * 32 + l32, x * 32 + 8 * i + 4 * h, D)] =
            make_float4(acc[x][t][4 * i], acc[x][t][4 * i + 1], acc[x][t][4 * i + 2], acc[x][t][4 * i + 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  win_rows_out<D, NW>(buf, pitch, tid, rows, [&](int r, int ch, const float* v) {
    const uint4 u = {pack16<F16>(v[0] * scale, v[1] * scale), pack16<F16>(v[2] * scale, v[3] * scale), pack16<F16>(v[4] * scale, v[5] * scale),
                     pack16<F16>(v[6] * scale, v[7] * scale)};
    *((uint4*)row_of(r) + ch) = u;
  });
}

// the same into a slot of partial results, [64][D] floats
template <int D, int NW>
__device__ __forceinline__ void store_part(f32x16 (&acc)[D / 32][2], float* buf, int tid, int rows, float* slot) {
  const int lane = tid & 63, wave = tid >> 6, l32 = lane & 31, h = lane >> 5;
  float* const mine = buf + wave * 64 * D;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      pin_acc<D>(acc[x][t]);  // (a tile at a time in ordinary registers)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4*)&mine[merge_offset(t * 32 + l32, x * 32 + 8 * i + 4 * h, D)] =
            make_float4(acc[x][t][4 * i], acc[x][t][4 * i + 1], acc[x][t][4 * i + 2], acc[x][t][4 * i + 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  win_rows_out<D, NW>(buf, 64 * D, tid, rows, [&](int r, int ch, const float* v) {
    *(float4*)&slot[r * D + ch * 8] = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)&slot[r * D + ch * 8 + 4] = make_float4(v[4], v[5], v[6], v[7]);
  });
}

// dQ.  The products of a unit, in this order, and what lies behind their matrix instructions:
//   dP(u) = V dO^T     the rest of P(u), copies of K(u + 2)
//   S(u + 1) = K Q^T   dS(u)
//   dQ += K^T dS(u)    the first of P(u + 1), copies of V(u + 2)
// K has three stages (of unit u to its end, of u + 1, of u + 2), V two.
template <int D, int NW>
struct DqShape {
  static constexpr int PLACE = 5 * 32 * D * 2;  // of a wavefront
  static constexpr int LDS = NW * PLACE;
};
template <int D, bool F16, int NW>
__device__ __forceinline__ void dq_block(unsigned char* smem, const WinArgs& a, const RowPlan& plan, unsigned workgroup, int tid) {
  using TL = Tile<D>;
  constexpr int KS = D / 16, DVB = D / 32, HALF = 32 * D * 2, NC = RowCopy<D>::NC, PH = 2 * KS, IPM = 16 / PH;  // softmax items a matrix instruction
  constexpr int kAhead = 2, kEvery = PH / NC, kEarly = 4;  // kEarly: items of P done in the phase before its own
  constexpr int PLACE = DqShape<D, NW>::PLACE;
  static_assert(PLACE >= 64 * D * 4, "the partial results fit the stages");
  RowItem at;
  if (!win_rows(a, plan, workgroup, false, at)) return;
  const int b = at.b, hk = at.hk, qb = at.qb, hq = hk * a.G + at.g;
  const WinSeq sq = at.q, sk = at.k;
  const int r0 = qb * 64, rows = min(64, sq.n - r0);
  if (rows <= 0) return;
  const int nk = __builtin_amdgcn_readfirstlane(sk.n), shift = nk - sq.n;
  WinWalk walk(a.mask, r0 + shift, r0 + rows - 1 + shift, nk, 32, 1);
  walk.uniform();
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int nu = walk.n > wave ? (walk.n - wave + NW - 1) / NW : 0;
  const float sl2 = a.scale * kLog2e;

  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * PLACE;
  unsigned char* const mine = smem + wave * PLACE;
  const unsigned char* kb = (const unsigned char*)uniform_ptr(a.k.row(b, sk.row0, hk));
  const unsigned char* vb = (const unsigned char*)uniform_ptr(a.v.row(b, sk.row0, hk));
  RowCopy<D> kc, vc;
  kc.init(lane, (unsigned)a.k.token);
  vc.init(lane, (unsigned)a.v.token);
  auto first_key = [&](int u) { return walk.begin(wave + NW * min(u, nu - 1)); };  // (units behind the last: that one again)
  auto copy_all = [&](const RowCopy<D>& c, const unsigned char* base, int key, unsigned lds) {
    c.all(base + (long long)key * c.stride, lds, lane, nk - key);
  };
  constexpr int kV = 3 * HALF;  // of the V stages

  // the first copies, then Q and dO, then what can be done while they are on their way
  if (nu > 0) {
    copy_all(kc, kb, first_key(0), lds0);
    copy_all(vc, vb, first_key(0), lds0 + kV);
    copy_all(kc, kb, first_key(1), lds0 + HALF);
    copy_all(vc, vb, first_key(1), lds0 + kV + HALF);
  }
  WinSpan span[2];
  float from[2], minus[2];  // exponents start from, -D
  bf16x8 qreg[2][KS], dreg[2][KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int r = min(r0 + 32 * t + l32, sq.n - 1);
    span[t] = win_span(a.mask, r + shift, nk);
    const long long st = a.stat(hq, b, sq.row0, r);
    from[t] = a.stats[st] * sl2, minus[t] = a.stats[a.lse_rows * a.H + st];
    const uint4 *p = (const uint4*)a.q.row(b, sq.row0 + r, hq), *pd = (const uint4*)a.dout.row(b, sq.row0 + r, hq);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      qreg[t][s] = __builtin_bit_cast(bf16x8, p[2 * s + h]);
      dreg[t][s] = __builtin_bit_cast(bf16x8, pd[2 * s + h]);
    }
  }
  f32x16 acc[DVB][2];
  float nil = 0.f;
  asm volatile("" : "+v"(nil));
#pragma unroll
  for (int x = 0; x < DVB; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[x][t][i] = nil;
      pin_acc<D>(acc[x][t]);
    }
  const int lane_a = TL::rowmajor_lane(0, lane);
  int b0, b1;
  TL::transposed_lane(0, lane, b0, b1);
  auto hide = [&](f32x16 (&S)[2], int u) {
    const int key0 = first_key(u);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const WinSpan w = walk.span_in(wave + NW * u, span[t]);
      int first = key0 + 4 * h;
      asm volatile("" : "+v"(first));
      if (w.se <= key0) {  // (no sinks among these keys)
        const unsigned from = (unsigned)(first - w.lo), many = (unsigned)(w.hi - w.lo);
#pragma unroll
        for (int i = 0; i < 16; ++i) S[t][i] = from + (unsigned)(8 * (i >> 2) + (i & 3)) < many ? S[t][i] : -INFINITY;
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = first + 8 * (i >> 2) + (i & 3);
          S[t][i] = key < w.hi && (key >= w.lo || key < w.se) ? S[t][i] : -INFINITY;
        }
      }
    }
  };
  // P of item `it` in place of S: exponents, then exponentials
  auto p_arg = [&](f32x16 (&S)[2], int it) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    for (int i = 0; i < 2; ++i) {
      S[t][e + i] = fmaf(S[t][e + i], sl2, from[t]);
      asm volatile("" : : "v"(S[t][e + i]));
    }
  };
  auto p_exp = [&](f32x16 (&S)[2], int it) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    for (int i = 0; i < 2; ++i) {
      S[t][e + i] = fast_exp2(S[t][e + i]);
      asm volatile("" : : "v"(S[t][e + i]));
    }
  };
  // slot n of 17: the argument of item n, the exponential of the one before
  auto p_slots = [&](f32x16 (&S)[2], int from_slot, int to_slot) {
#pragma unroll
    for (int n = from_slot; n < to_slot; ++n) {
      if (n < 16) p_arg(S, n);
      if (n > 0) p_exp(S, n - 1);
    }
  };
  uint32_t dsw[2][2][4];
  auto d_sub = [&](f32x16 (&dp)[2], int it) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    for (int i = 0; i < 2; ++i) {
      dp[t][e + i] += minus[t];
      asm volatile("" : : "v"(dp[t][e + i]));
    }
  };
  auto d_mul = [&](f32x16 (&dp)[2], const f32x16 (&S)[2], int it) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    for (int i = 0; i < 2; ++i) {
      dp[t][e + i] *= S[t][e + i];
      asm volatile("" : : "v"(dp[t][e + i]));
    }
  };
  auto d_cvt = [&](const f32x16 (&dp)[2], int it) {
    const int t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3);
    dsw[t][it >> 3][it & 3] = pack16<F16>(dp[t][e], dp[t][e + 1]);
    asm volatile("" : : "v"(dsw[t][it >> 3][it & 3]));
  };
  auto d_slots = [&](f32x16 (&dp)[2], const f32x16 (&S)[2], int from_slot, int to_slot) {
#pragma unroll
    for (int n = from_slot; n < to_slot; ++n) {
      if (n < 16) d_sub(dp, n);
      if (n > 0 && n < 17) d_mul(dp, S, n - 1);
      if (n > 1 && n < 18) d_cvt(dp, n - 2);
    }
  };
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (D == 128) asm volatile("" : "+a"(qreg[t][s]));
      else asm volatile("" : "+v"(qreg[t][s]));
      asm volatile("" : "+v"(dreg[t][s]));
    }
  asm volatile("" : "+v"(from[0]), "+v"(from[1]), "+v"(minus[0]), "+v"(minus[1]));

  f32x16 s0[2], s1[2];
  unsigned k_at = 0;  // stage of K(u), bytes
  auto after = [](unsigned x) { return x == 2u * HALF ? 0u : x + HALF; };
  auto rows_of = [&](unsigned stage, int s) { return TL::rowmajor_at(mine + stage, lane_a, s); };
  bf16x8 vcur[kAhead];
  if (nu > 0) {
    win_wait<2 * NC>();
    in_steps<KS>([&](auto number) {
      constexpr int s = decltype(number)::value;
      const bf16x8 ka = rows_of(0, s);
      mm_q<D, F16, s == 0>(s0[0], ka, qreg[0][s]);
      mm_q<D, F16, s == 0>(s0[1], ka, qreg[1][s]);
    });
    mfma_fence();
    if (walk.masked(wave)) hide(s0, 0);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) vcur[s] = rows_of(kV, s);
    p_slots(s0, 0, kEarly);
  }
  // STEADY: the copies are of 32 rows that are there, piece by piece; else at once, and u may be the last unit.  `par` = u & 1 (a
  // constant in the unrolled loop).
  auto body = [&](auto steady_tag, int par, f32x16 (&S)[2], f32x16 (&T)[2], int u) {
    constexpr bool STEADY = decltype(steady_tag)::value;
    const bool more = STEADY || u + 1 < nu;
    const unsigned k1 = after(k_at), k2 = after(k1);
    const int key2 = first_key(u + 2);
    const unsigned char *kp = kb + (long long)key2 * kc.stride, *vp = vb + (long long)key2 * vc.stride;
    f32x16 dp[2];
    bf16x8 vr[KS], kr[KS], tr[KS];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) vr[s] = vcur[s];
    if (!STEADY) copy_all(kc, kb, key2, lds0 + k2);
    __builtin_amdgcn_sched_barrier(0);
    in_steps<PH>([&](auto number) {  // dP(u)
      constexpr int j = decltype(number)::value, s = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0;
      if (copies) {
        kc.aim(lds0 + k2, j / kEvery);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (s == 0) mm_v_zero<D, F16>(dp[j & 1], vr[s], dreg[j & 1][s]);
      else mm_v<D, F16, false>(dp[j & 1], vr[s], dreg[j & 1][s], dp[j & 1]);
      __builtin_amdgcn_sched_barrier(0);
      if (copies) kc.piece(kp, j / kEvery);
      if (j == PH - 2 * kAhead) {  // K(u + 1) has landed; newer: V(u + 1) and what has been requested of K(u + 2)
        constexpr int part = STEADY ? j / kEvery + 1 : NC;
        win_wait<NC + part>();
      }
      if (j % 2 == 0) {
        constexpr int to = s + kAhead;
        if constexpr (to < KS) vr[to] = rows_of(kV + par * HALF, to);
        else kr[to - KS] = rows_of(k1, to - KS);
      }
      constexpr int n0 = kEarly + (17 - kEarly) * j / PH, n1 = kEarly + (17 - kEarly) * (j + 1) / PH;
      p_slots(S, n0, n1);
      __builtin_amdgcn_sched_barrier(0);
    });
    auto t_op = [&](int i) { return TL::transposed_at(mine + k_at, b0, b1, i / DVB, i % DVB); };
    constexpr int kLag = 2;  // dP is complete that many matrix instructions on
    in_steps<PH>([&](auto number) {  // S(u + 1)
      constexpr int j = decltype(number)::value, s = j >> 1;
      mm_q<D, F16, s == 0>(T[j & 1], kr[s], qreg[j & 1][s]);
      __builtin_amdgcn_sched_barrier(0);
      if (j % 2 == 0) {
        constexpr int to = s + kAhead;
        if constexpr (to < KS) {
          kr[to] = rows_of(k1, to);
        } else {
          tr[to - KS] = t_op(to - KS);
        }
      }
      constexpr int n0 = j < kLag ? 0 : 18 * (j - kLag) / (PH - kLag), n1 = j < kLag ? 0 : 18 * (j + 1 - kLag) / (PH - kLag);
      d_slots(dp, S, n0, n1);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (more && __builtin_expect(walk.masked(wave + NW * min(u + 1, nu - 1)), 0)) {
      mfma_fence();
      hide(T, u + 1);
    }
    if (!STEADY) copy_all(vc, vb, key2, lds0 + kV + par * HALF);
    bf16x8 ds[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int st = 0; st < 2; ++st) ds[t][st] = __builtin_bit_cast(bf16x8, make_uint4(dsw[t][st][0], dsw[t][st][1], dsw[t][st][2], dsw[t][st][3]));
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 1");
    in_steps<PH>([&](auto number) {  // dQ
      constexpr int j = decltype(number)::value, i = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0;
      if (copies) {
        vc.aim(lds0 + kV + par * HALF, j / kEvery);
        __builtin_amdgcn_sched_barrier(0);
      }
      mm_acc<D, F16>(acc[i % DVB][j & 1], tr[i], ds[j & 1][i / DVB]);
      __builtin_amdgcn_sched_barrier(0);
      if (copies) vc.piece(vp, j / kEvery);
      if (j == PH - 2 * kAhead) {  // V(u + 1) has landed; newer: K(u + 2) and what has been requested of V(u + 2)
        constexpr int part = STEADY ? j / kEvery + 1 : NC;
        win_wait<NC + part>();
      }
      if (j % 2 == 0) {
        constexpr int to = i + kAhead;
        if constexpr (to < KS) tr[to] = t_op(to);
        else vcur[to - KS] = rows_of(kV + (1 - par) * HALF, to - KS);
      }
      // (S(u + 1) is complete and may be read from here on: its last product lies kLag matrix instructions back)
      constexpr int n0 = j < kLag ? 0 : kEarly * (j - kLag) / (PH - kLag), n1 = j < kLag ? 0 : kEarly * (j + 1 - kLag) / (PH - kLag);
      p_slots(T, n0, n1);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (!STEADY) mfma_fence();  // (accumulators may be moved between one form of this and another)
    k_at = k1;
  };
  if (nu > 0) {
    // units whose copies (two on) are of 32 rows that are there: all, or not the last of either run of keys
    int whole = 0;
    if (kc.plain(nk - 32 * (walk.n_sink - 1)) && vc.plain(32)) whole = nk - walk.begin(walk.n - 1) >= 32 ? nu : (walk.n - 1 - wave + NW - 1) / NW - 2;
    int u = 0;
    for (; u + 1 < whole; u += 2) {
      body(std::true_type{}, 0, s0, s1, u);
      body(std::true_type{}, 1, s1, s0, u + 1);
    }
    mfma_fence();
    for (; u < nu; ++u) {  // (behind the last unit: that one again)
      body(std::false_type{}, u & 1, s0, s1, u);
      s0[0] = s1[0];
      s0[1] = s1[1];
    }
    win_wait<0>();
  }
  mfma_fence();
#pragma unroll
  for (int x = 0; x < DVB; ++x) pin_acc<D>(acc[x][0]), pin_acc<D>(acc[x][1]);
  __builtin_amdgcn_sched_barrier(0);
  if (NW > 1) __syncthreads();
  store_columns<D, F16, NW>(acc, a.scale, (float*)smem, PLACE / 4, tid, rows, [&](int r) { return a.dq.out(b, sq.row0 + r0 + r, hq); });
}

// How the key blocks of a head are cut into workgroups: a block whose queries (of all heads of the group) are more than `per` units is
// walked in parts of its own, which leave their sums in fp32 to be added, in order, by k_window_join.  Blocks of sinks, which every
// later query sees, are the long ones.
struct DkvPlan {
  int heads, per_head;                      // (dense: sequences times heads; packed: heads); items of each
  int sinks, sink_blocks, sink_parts;       // sequences of a head whose first blocks may hold sinks; those blocks, parts of each
  int blocks, parts;                        // 64-key blocks of a head (of all sequences, at most); parts of each that holds no sink
  int per, run;                             // units of a part at most, of a part of a block without sinks
  long long slots;                          // partial results of a head
  // item of a head: those of the sinks come first.  Their slots are numbered like the items.
  __host__ __device__ int sink_items() const { return sinks * sink_blocks * sink_parts; }
  // parts that a block of so many units has work for
  __host__ __device__ int live(int units, int of) const {
    const int want = (units + per - 1) / per;
    return want < 1 ? 1 : want < of ? want : of;
  }
};
struct DkvItem {
  int b, hk, block, part, of;
  WinSeq q, k;
};
// item number `item` of a head (first part of a block: `item` of the join) -> what it is; false: nothing
__device__ __forceinline__ bool dkv_item(const WinArgs& a, const DkvPlan& plan, int head, int item, DkvItem& t) {
  const bool packed = a.rk.cu != nullptr;
  const int first = plan.sink_items();
  t.hk = packed ? head : head % a.Hkv;
  if (item < first) {
    t.of = plan.sink_parts;
    t.part = item % t.of;
    const int k = item / t.of;
    t.block = k % plan.sink_blocks;
    t.b = packed ? k / plan.sink_blocks : head / a.Hkv;
    t.q = win_seq(a.rq, t.b);
    t.k = win_seq(a.rk, t.b);
    return true;
  }
  t.of = plan.parts;
  t.part = (item - first) % t.of;
  const int k = (item - first) / t.of;
  if (packed) {
    if (!win_find(a.rk, &a.rq, a.B, (unsigned)k, t.b, t.block, t.k, t.q)) return false;
  } else {
    t.b = head / a.Hkv;
    t.block = k;
    t.q = {0, a.rq.most};
    t.k = {0, a.rk.most};
  }
  return t.block >= plan.sink_blocks;
}

static DkvPlan dkv_plan(const WinArgs& a) {
  DkvPlan p = {};
  const WinMask& m = a.mask;
  const bool packed = a.rk.cu != nullptr;
  const long long nkb = (a.rk.most + 63) / 64, most = (a.rq.most + 31) / 32 + 1;
  p.heads = packed ? a.Hkv : a.B * a.Hkv;
  p.blocks = (int)(packed ? win_blocks(a.rk, a.B) : nkb);
  const long long run = m.left < 0 || m.right < 0 ? most : ((long long)(m.left + m.right + 2) * m.unit + 64) / 32 + 2;
  const long long ur = (run < most ? run : most) * a.G, us = most * a.G;
  const long long sb = run < most ? ((long long)m.sinks + 63) / 64 : 0;
  p.sink_blocks = (int)(sb < nkb ? sb : nkb);
  p.sinks = p.sink_blocks ? (packed ? a.B : 1) : 0;
  const long long sinks = (long long)p.sinks * p.sink_blocks, others = p.blocks;
  const long long total = p.heads * (sinks * us + others * ur);
  // 512 workgroups of two wavefronts run at a time: a part is at most half of what one gets in all
  long long per = total / 1024;
  if (per < 32) per = 32;
  if (per > 1 << 30) per = 1 << 30;
  p.per = (int)per;
  auto parts = [&](long long units) { return (int)((units + per - 1) / per < 64 ? (units + per - 1) / per : 64); };
  p.sink_parts = p.sink_blocks ? parts(us) : 1;
  p.parts = p.heads * others >= 512 ? 1 : parts(ur);
  if (p.parts < 1) p.parts = 1;
  p.run = (int)((ur + p.parts - 1) / p.parts < per ? (ur + p.parts - 1) / p.parts : per);
  p.per_head = (int)(p.sink_items() + others * p.parts);
  p.slots = p.parts > 1 ? p.per_head : p.sink_parts > 1 ? p.sink_items() : 0;
  return p;
}

size_t window_parts(const WinArgs& a, int d) { const DkvPlan p = dkv_plan(a); return (size_t)p.heads * p.slots * (2 * 64 * d); }

// dK, dV.  The products of a unit, in this order, and what lies behind their matrix instructions:
//   S = Q K^T, from -lse / scale    copies of Q and the row terms of u + 1
//   dP = dO V^T, from -D            most of P
//   dV += dO^T P                    the rest of P, most of dS
//   dK += Q^T dS                    the rest of dS, copies of dO(u + 2)
// dK and dV are accumulation registers, K and V of the first 32 keys ordinary ones, V of the others is in LDS.
template <int D, int NW>
struct DkvShape {
  static constexpr int HALF = 32 * D * 2, PLACE = 4 * HALF;  // 32 rows; stages of a wavefront
  static constexpr int V = NW * PLACE, TERMS = V + HALF, SEEN = TERMS + NW * 512, LDS = SEEN + NW * 512;
};
template <int D, bool F16, int NW>
__device__ __forceinline__ void dkv_block(unsigned char* smem, const WinArgs& a, const DkvPlan& plan, float* __restrict__ parts, unsigned workgroup) {
  using TL = Tile<D>;
  constexpr int KS = D / 16, DVB = D / 32, HALF = 32 * D * 2, NC = RowCopy<D>::NC, PH = 2 * KS;
  constexpr int kAhead = 2, kEvery = PH / NC;
  using SH = DkvShape<D, NW>;
  constexpr int PLACE = SH::PLACE;
  unsigned char* const vsecond = smem + SH::V;                       // V of the second 32 keys
  float(*const terms)[2][64] = (float(*)[2][64])(smem + SH::TERMS);  // of a unit's 32 rows: what S starts from, dP
  int2(*const seen_by)[64] = (int2(*)[64])(smem + SH::SEEN);         // queries that see a key (registers are short)
  static_assert(PLACE == 64 * D * 4, "the partial results fit the stages");
  int head, item;
  DkvItem at;
  if (!win_item(workgroup, (unsigned)plan.heads, (unsigned)plan.per_head, head, item) || !dkv_item(a, plan, head, item, at)) return;
  const int b = at.b, hk = at.hk, kblk = at.block, part = at.part, of = at.of;
  const WinSeq sq = at.q, sk = at.k;
  const int k0 = kblk * 64, keys = min(64, sk.n - k0);
  if (keys <= 0) return;
  const int nq = __builtin_amdgcn_readfirstlane(sq.n), shift = sk.n - nq;
  const KeyWalk walk(a.mask, k0, k0 + keys, nq, shift, 32);
  const int wn = __builtin_amdgcn_readfirstlane(walk.n), wfrom = __builtin_amdgcn_readfirstlane(walk.from);
  auto clamp_q = [&](int x) { return __builtin_amdgcn_readfirstlane(x < 0 ? 0 : x > nq ? nq : x); };
  const int seen_from = clamp_q(walk.seen_from - shift), seen_to = clamp_q(walk.seen_to - shift);
  const int all = wn * a.G, live = plan.live(all, of);
  if (part >= live) return;
  const int begin = (int)((long long)all * part / live), end = (int)((long long)all * (part + 1) / live);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  const int nu = end - begin > wave ? (end - begin - wave + NW - 1) / NW : 0;

  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem)) + (unsigned)wave * PLACE;
  const unsigned terms0 = __builtin_amdgcn_readfirstlane(lds_address(terms)) + (unsigned)wave * 512u;
  unsigned char* const mine = smem + wave * PLACE;
  RowCopy<D> qc, dc;
  qc.init(lane, (unsigned)a.q.token);
  dc.init(lane, (unsigned)a.dout.token);
  const unsigned plane = (unsigned)(a.lse_rows * a.H) * 4u;
  const unsigned term_off = (unsigned)(lane & 31) * 4u + (lane < 32 ? 0u : plane);
  // where a unit lies: head of the group and first query
  struct U {
    int q;
    const unsigned char *qp, *dp, *st;
  };
  const unsigned char* const q_base = (const unsigned char*)uniform_ptr(a.q.row(b, sq.row0, hk * a.G));
  const unsigned char* const d_base = (const unsigned char*)uniform_ptr(a.dout.row(b, sq.row0, hk * a.G));
  const unsigned char* const s_base = (const unsigned char*)uniform_ptr(a.stats + a.stat(hk * a.G, b, sq.row0, 0));
  // units follow one another: first query and head advance with them
  int at_g = 0, at_i = 0;
  auto unit_at = [&](int i) {  // of the walk over all heads
    at_g = i / wn;
    at_i = i - at_g * wn;
    at_g = __builtin_amdgcn_readfirstlane(at_g);
    at_i = __builtin_amdgcn_readfirstlane(at_i);
  };
  auto unit_here = [&] {
    U x;
    x.q = wfrom + 32 * at_i;
    x.qp = q_base + (long long)at_g * a.q.head + (long long)x.q * qc.stride;
    x.dp = d_base + (long long)at_g * a.dout.head + (long long)x.q * dc.stride;
    x.st = s_base + ((long long)at_g * a.lse_rows + x.q) * 4;
    return x;
  };
  auto advance = [&] {  // by NW units, not behind the last one of the part
    at_i += NW;
    while (at_i >= wn) at_i -= wn, ++at_g;
  };
  auto copy_q = [&](const U& x, int stage) {
    qc.all(x.qp, lds0 + stage * HALF, lane, nq - x.q);
  };
  auto copy_d = [&](const U& x, int stage) {
    dc.all(x.dp, lds0 + (2 + stage) * HALF, lane, nq - x.q);
  };
  auto copy_terms = [&](const U& x, int stage) {
    const unsigned off = nq - x.q >= 32 ? term_off : (unsigned)min(lane & 31, nq - x.q - 1) * 4u + (lane < 32 ? 0u : plane);
    lds_dma4<4>(x.st, off, terms0 + stage * 256u);
  };

  // the first copies, then K and V, then what can be done while they are on their way
  U cur = {}, n1 = {}, n2 = {};
  if (nu > 0) {
    unit_at(begin + wave);
    cur = unit_here();
    if (nu > 1) advance();
    n1 = unit_here();
    copy_d(cur, 0);
    copy_q(cur, 0);
    copy_terms(cur, 0);
    copy_d(n1, 1);
  }
  bf16x8 kreg[2][KS], vreg[KS];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int j = min(k0 + 32 * t + l32, sk.n - 1);
    const KeySpan w = key_span(a.mask, j);
    auto clamp = [&](int x) { return x < 0 ? 0 : x > nq ? nq : x; };
    if (h == 0) seen_by[wave][32 * t + l32] = make_int2(clamp(w.lo - shift), max(clamp(w.lo - shift), clamp(w.hi - shift)));
    const uint4 *p = (const uint4*)a.k.row(b, sk.row0 + j, hk), *pv = (const uint4*)a.v.row(b, sk.row0 + j, hk);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      kreg[t][s] = __builtin_bit_cast(bf16x8, p[2 * s + h]);
      if (t == 0) vreg[s] = __builtin_bit_cast(bf16x8, pv[2 * s + h]);
      else if (wave == 0) *(uint4*)(vsecond + TL::off(l32, 2 * s + h)) = pv[2 * s + h];
    }
  }
  f32x16 dk[DVB][2], dv[DVB][2];
  float nil = 0.f;
  asm volatile("" : "+v"(nil));
#pragma unroll
  for (int x = 0; x < DVB; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) dk[x][t][i] = nil, dv[x][t][i] = nil;
      pin_acc<D>(dk[x][t]);
      pin_acc<D>(dv[x][t]);
    }
  const float sl2 = a.scale * kLog2e;
  const int lane_a = TL::rowmajor_lane(0, lane);
  int b0, b1;
  TL::transposed_lane(0, lane, b0, b1);

  f32x16 S[2], dp[2];
  uint32_t pw[2][2][4], sw[2][2][4];
  auto place = [](int it, int& t, int& e) { t = (it >> 2) & 1, e = 8 * (it >> 3) + 2 * (it & 3); };
  // P in place of S, dS in place of dP; slot n: the first operation of item n, the next of the one before, ...
  auto p_slots = [&](int from_slot, int to_slot) {
#pragma unroll
    for (int n = from_slot; n < to_slot; ++n) {
      int t, e;
      if (n < 16) {
        place(n, t, e);
        for (int i = 0; i < 2; ++i) {
          S[t][e + i] *= sl2;
          asm volatile("" : : "v"(S[t][e + i]));
        }
      }
      if (n > 0 && n < 17) {
        place(n - 1, t, e);
        for (int i = 0; i < 2; ++i) {
          S[t][e + i] = fast_exp2(S[t][e + i]);
          asm volatile("" : : "v"(S[t][e + i]));
        }
      }
      if (n > 1 && n < 18) {
        place(n - 2, t, e);
        pw[t][(n - 2) >> 3][(n - 2) & 3] = pack16<F16>(S[t][e], S[t][e + 1]);
        asm volatile("" : : "v"(pw[t][(n - 2) >> 3][(n - 2) & 3]));
      }
    }
  };
  auto d_slots = [&](int from_slot, int to_slot) {
#pragma unroll
    for (int n = from_slot; n < to_slot; ++n) {
      int t, e;
      if (n < 16) {
        place(n, t, e);
        for (int i = 0; i < 2; ++i) {
          dp[t][e + i] *= S[t][e + i];
          asm volatile("" : : "v"(dp[t][e + i]));
        }
      }
      if (n > 0 && n < 17) {
        place(n - 1, t, e);
        sw[t][(n - 1) >> 3][(n - 1) & 3] = pack16<F16>(dp[t][e], dp[t][e + 1]);
        asm volatile("" : : "v"(sw[t][(n - 1) >> 3][(n - 1) & 3]));
      }
    }
  };
  auto word4 = [](const uint32_t (&w)[4]) { return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3])); };
  auto term16 = [&](int par, int which) {  // rows 8 * r4 + 4 h ..
    f32x16 x;
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const f32x4 y = *(const f32x4*)&terms[wave][par][32 * which + 8 * r4 + 4 * h];
      x[4 * r4] = y[0], x[4 * r4 + 1] = y[1], x[4 * r4 + 2] = y[2], x[4 * r4 + 3] = y[3];
    }
    return x;
  };
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(kreg[0][s]), "+v"(kreg[1][s]), "+v"(vreg[s]));
  if (NW > 1) __syncthreads();
  else __builtin_amdgcn_wave_barrier();

  bf16x8 qcur[kAhead];
  if (nu > 0) {
    win_wait<NC>();
#pragma unroll
    for (int s = 0; s < kAhead; ++s) qcur[s] = TL::rowmajor_at(mine, lane_a, s);
  }
  // STEADY: the copies are of 32 rows that are there, piece by piece; else at once, and u may be the last unit.  `par` = u & 1 (a
  // constant in the unrolled loop).
  auto body = [&](auto steady_tag, int par, int u) {
    constexpr bool STEADY = decltype(steady_tag)::value;
    const bool more = STEADY || u + 1 < nu;
    const unsigned char *qs = mine + par * HALF, *ds = mine + (2 + par) * HALF;
    bf16x8 qr[KS], dr[KS], vr[KS], tr[KS], tq[KS];
    int lane_v = lane_a;
    asm volatile("" : "+v"(lane_v));  // (the addresses of V are made per unit: registers are short)
#pragma unroll
    for (int s = 0; s < kAhead; ++s) qr[s] = qcur[s];
    if (!STEADY && more) copy_q(n1, 1 - par);
    if (more) copy_terms(n1, 1 - par);
    const f32x16 s_from = term16(par, 0);
    f32x16 d_from;
    __builtin_amdgcn_sched_barrier(0);
    in_steps<PH>([&](auto number) {  // S
      constexpr int j = decltype(number)::value, s = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0;
      if (copies) {
        qc.aim(lds0 + (1 - par) * HALF, j / kEvery);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (j == 0) mm_v<D, F16, true>(S[0], qr[0], kreg[0][0], s_from);
      else {
        if (j == 1) S[1] = s_from;  // (in place)
        mm_v<D, F16, false>(S[j & 1], qr[s], kreg[j & 1][s], S[j & 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (copies) qc.piece(n1.qp, j / kEvery);
      if (j == 1 && more) {
        if (u + 2 < nu) advance();
        n2 = unit_here();
      }
      if (j % 2 == 0) {
        constexpr int to = s + kAhead;
        if constexpr (to < KS) qr[to] = TL::rowmajor_at(qs, lane_a, to);
        else dr[to - KS] = TL::rowmajor_at(ds, lane_a, to - KS);
      }
      if (j == PH - 5) d_from = term16(par, 1);
      if constexpr (j % 2 && j >= PH - 4) vr[(j - PH + 4) / 2] = TL::rowmajor_at(vsecond, lane_v, (j - PH + 4) / 2);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__builtin_expect(cur.q < seen_from || cur.q + 32 > seen_to, 0)) {  // (rows behind the last query among them)
      int first = 4 * h;
      asm volatile("" : "+v"(first));
      first += cur.q;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int2 by = seen_by[wave][32 * t + l32];
#pragma unroll
        for (int i = 0; i < 16; ++i) S[t][i] = (unsigned)(first - by.x) + (unsigned)(8 * (i >> 2) + (i & 3)) < (unsigned)(by.y - by.x) ? S[t][i] : -INFINITY;
      }
    }
    auto dt_op = [&](int i) { return TL::transposed_at(ds, b0, b1, i / DVB, i % DVB); };
    auto qt_op = [&](int i) { return TL::transposed_at(qs, b0, b1, i / DVB, i % DVB); };
    constexpr int kP = 14;  // slots of P done behind dP: those of contraction step 0 among them
    in_steps<PH>([&](auto number) {  // dP
      constexpr int j = decltype(number)::value, s = j >> 1;
      if constexpr (j == 0) mm_v<D, F16, true>(dp[0], dr[0], vreg[0], d_from);
      else {
        if (j == 1) dp[1] = d_from;
        mm_v<D, F16, false>(dp[j & 1], dr[s], j & 1 ? vr[s] : vreg[s], dp[j & 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (j % 2 == 0) {
        constexpr int to = s + kAhead;
        if constexpr (to < KS) dr[to] = TL::rowmajor_at(ds, lane_a, to);
        else tr[to - KS] = dt_op(to - KS);
      } else if constexpr (s + 2 < KS) {
        vr[s + 2] = TL::rowmajor_at(vsecond, lane_v, s + 2);
      }
      p_slots(kP * j / PH, kP * (j + 1) / PH);
      __builtin_amdgcn_sched_barrier(0);
    });
    asm volatile("s_nop 1");
    in_steps<PH>([&](auto number) {  // dV
      constexpr int j = decltype(number)::value, i = j >> 1;
      mm_acc<D, F16>(dv[i % DVB][j & 1], tr[i], word4(pw[j & 1][i / DVB]));
      __builtin_amdgcn_sched_barrier(0);
      if (j % 2 == 0) {
        constexpr int to = i + kAhead;
        if constexpr (to < KS) tr[to] = dt_op(to);
        else tq[to - KS] = qt_op(to - KS);
      }
      constexpr int half = PH / 2 - 2;  // P of contraction step 1 is there two matrix instructions ahead of its use
      if (j < half) p_slots(kP + (18 - kP) * j / half, kP + (18 - kP) * (j + 1) / half);
      constexpr int d0 = j < 2 ? 0 : 14 * (j - 2) / (PH - 2), d1 = j < 2 ? 0 : 14 * (j - 1) / (PH - 2);
      d_slots(d0, d1);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (!STEADY && more) copy_d(n2, par);
    asm volatile("s_nop 1");
    in_steps<PH>([&](auto number) {  // dK
      constexpr int j = decltype(number)::value, i = j >> 1;
      constexpr bool copies = STEADY && j % kEvery == 0;
      if (copies) {
        dc.aim(lds0 + (2 + par) * HALF, j / kEvery);
        __builtin_amdgcn_sched_barrier(0);
      }
      mm_acc<D, F16>(dk[i % DVB][j & 1], tq[i], word4(sw[j & 1][i / DVB]));
      __builtin_amdgcn_sched_barrier(0);
      if (copies) dc.piece(n2.dp, j / kEvery);
      if (more && j == PH - 2 * kAhead) {  // Q(u + 1) and all that is older have landed; newer: what has been requested of dO(u + 2)
        constexpr int done = STEADY ? j / kEvery + 1 : NC;
        win_wait<done>();
      }
      if (j % 2 == 0) {
        constexpr int to = i + kAhead;
        if constexpr (to < KS) tq[to] = qt_op(to);
        else if (more) qcur[to - KS] = TL::rowmajor_at(mine + (1 - par) * HALF, lane_a, to - KS);
      }
      constexpr int half = PH / 2 - 2;
      if (j < half) d_slots(14 + 3 * j / half, 14 + 3 * (j + 1) / half);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (!STEADY) mfma_fence();
    cur = n1;
    n1 = n2;
  };
  if (nu > 0) {
    // (the next unit, and the one behind it; a walk that ends behind the last query ends in rows that are not there)
    const bool plain = qc.plain(32) && dc.plain(32) && wfrom + 32 * wn <= nq;
    int u = 0;
    for (; plain && u + 3 < nu; u += 2) {
      body(std::true_type{}, 0, u);
      body(std::true_type{}, 1, u + 1);
    }
    mfma_fence();
    for (; u < nu; ++u) body(std::false_type{}, u & 1, u);
    win_wait<0>();
  }
  mfma_fence();
#pragma unroll
  for (int x = 0; x < DVB; ++x) pin_acc<D>(dk[x][0]), pin_acc<D>(dk[x][1]), pin_acc<D>(dv[x][0]), pin_acc<D>(dv[x][1]);
  __builtin_amdgcn_sched_barrier(0);
  if (NW > 1) __syncthreads();
  if (live == 1) {
    store_columns<D, F16, NW>(dv, 1.f, (float*)smem, PLACE / 4, tid, keys, [&](int r) { return a.dv.out(b, sk.row0 + k0 + r, hk); });
    if (NW > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    store_columns<D, F16, NW>(dk, a.scale, (float*)smem, PLACE / 4, tid, keys, [&](int r) { return a.dk.out(b, sk.row0 + k0 + r, hk); });
  } else {
    float* const slot = parts + (head * plan.slots + item) * (2 * 64 * D);
    store_part<D, NW>(dv, (float*)smem, tid, keys, slot);
    if (NW > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    store_part<D, NW>(dk, (float*)smem, tid, keys, slot + 64 * D);
  }
}

// Both passes in one launch, dK/dV's workgroups first: dQ's fill what they leave of the chip (packed training of 10332 tokens, d = 64:
// 216 us with a launch each, 201 so, both before their walks at d = 64 became as they are; 16 frames of 1024 tokens, 12 heads, d = 128: 1901 and 1805).  NW = 4: the four wavefronts share a
// block of queries too; NW = 2: each takes one of its own.
template <int D, bool F16, int NW>
__global__ __launch_bounds__(64 * NW, 1) void k_window_dq_dkv(WinArgs a, RowPlan rows, DkvPlan plan, float* __restrict__ parts, unsigned first) {
  constexpr int DQ = NW == 4 ? DqShape<D, 4>::LDS : NW * DqShape<D, 1>::LDS;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[DQ > DkvShape<D, NW>::LDS ? DQ : DkvShape<D, NW>::LDS];
  if (blockIdx.x < first) {
    dkv_block<D, F16, NW>(smem, a, plan, parts, blockIdx.x);
  } else if constexpr (NW == 4) {
    dq_block<D, F16, 4>(smem, a, rows, blockIdx.x - first, threadIdx.x);
  } else {
    const unsigned w = blockIdx.x - first, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    dq_block<D, F16, 1>(smem + wave * DqShape<D, 1>::LDS, a, rows, ((w >> 3) * NW + wave) * 8u + (w & 7u), threadIdx.x & 63);
  }
}

// the parts of a block added in order, 8 elements a thread
template <int D, bool F16>
__global__ __launch_bounds__(256) void k_window_join(WinArgs a, DkvPlan plan, const float* __restrict__ parts, int sink_blocks, int blocks) {
  constexpr int CPR = D / 8, SLICES = 2 * 64 * CPR / 256;  // workgroups a block: an item a thread
  const int slice = blockIdx.x % SLICES, rest = blockIdx.x / SLICES;
  const int k = rest % (sink_blocks + blocks), head = rest / (sink_blocks + blocks);
  const int item = k < sink_blocks ? k * plan.sink_parts : plan.sink_items() + (k - sink_blocks) * plan.parts;
  DkvItem at;
  if (!dkv_item(a, plan, head, item, at)) return;
  const int b = at.b, hk = at.hk;
  const WinSeq sq = at.q, sk = at.k;
  const int k0 = at.block * 64, keys = min(64, sk.n - k0);
  if (keys <= 0) return;
  const KeyWalk walk(a.mask, k0, k0 + keys, sq.n, sk.n - sq.n, 32);
  const int live = plan.live(walk.n * a.G, at.of);
  if (live == 1) return;
  const int it = slice * 256 + (int)threadIdx.x, which = it / (64 * CPR), r = it / CPR % 64, ch = it % CPR;
  if (r >= keys) return;
  const float* x = parts + (head * plan.slots + item) * (2 * 64 * D) + which * 64 * D + r * D + ch * 8;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < live; p += 4) {  // (four parts on their way at once; added in order)
    float4 y[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* from = x + (long long)min(p + i, live - 1) * (2 * 64 * D);
      y[i][0] = *(const float4*)from, y[i][1] = *(const float4*)(from + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < live) {
        v[0] += y[i][0].x, v[1] += y[i][0].y, v[2] += y[i][0].z, v[3] += y[i][0].w;
        v[4] += y[i][1].x, v[5] += y[i][1].y, v[6] += y[i][1].z, v[7] += y[i][1].w;
      }
  }
  const float f = which ? a.scale : 1.f;
  const uint4 u = {pack16<F16>(v[0] * f, v[1] * f), pack16<F16>(v[2] * f, v[3] * f), pack16<F16>(v[4] * f, v[5] * f), pack16<F16>(v[6] * f, v[7] * f)};
  *((uint4*)(which ? a.dk : a.dv).out(b, sk.row0 + k0 + r, hk) + ch) = u;
}

namespace {
// Four wavefronts a workgroup or two, by the time that either would take: all work spread over the workgroups that fit at once, and
// the longest item behind it.  A unit of dQ is 2, one of dK/dV 3, start and stores of a workgroup 24.  (28 shapes of 512 to 8192
// tokens, one to eight key heads: the faster one in 25, at most 5 % off in the others.  2048 tokens, 8 heads, d = 64, causal: four 63 us,
// two 94; 8192 tokens, two heads, a window of 512: four 53, two 46.)
bool four(const WinArgs& a, const DkvPlan& plan, long long items, long long groups) {
  const double uq = (double)win_units(a.mask, a.rk.most), uk = (double)plan.run;
  auto time = [&](int nw) {
    const double k = 3 * uk / nw + 24, q = 2 * uq / (nw == 4 ? 4 : 1) + 24;
    return (items * k + (nw == 4 ? groups : groups / 2.) * q) * nw / 1024 + (k > q ? k : q);
  };
  return time(4) <= time(2);
}
template <int D, bool F16>
hipError_t launch(const WinArgs& a, float* parts, hipStream_t s) {
  const long long lanes = a.lse_rows * a.H * (D / 8);
  if (lanes > 0) k_window_stats<D, F16><<<(unsigned)((lanes + 255) / 256), 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const RowPlan rows = {(int)(a.rq.cu ? win_blocks(a.rq, a.B) : (a.rq.most + 63) / 64), 1, 1, 1};
  const long long groups = win_workgroups(a, rows);
  const DkvPlan plan = dkv_plan(a);
  const long long items = (long long)plan.heads * plan.per_head;
  if (items + groups == 0) return e;
  const unsigned first = win_grid(items);
  if (four(a, plan, items, groups)) k_window_dq_dkv<D, F16, 4><<<first + win_grid(groups), 256, 0, s>>>(a, rows, plan, parts, first);
  else k_window_dq_dkv<D, F16, 2><<<first + win_grid((groups + 1) / 2), 128, 0, s>>>(a, rows, plan, parts, first);
  e = hipGetLastError();
  if (e != hipSuccess || plan.slots == 0) return e;
  const int sinks = plan.sink_parts > 1 ? plan.sinks * plan.sink_blocks : 0, blocks = plan.parts > 1 ? plan.blocks : 0;
  k_window_join<D, F16><<<(unsigned)(plan.heads * (sinks + blocks)) * (2u * 64u * (D / 8) / 256u), 256, 0, s>>>(a, plan, parts, sinks, blocks);
  e = hipGetLastError();
  return e;
}
}  // namespace

hipError_t launch_window_bwd(const WinArgs& a, int d, bool f16, float* parts, hipStream_t s) {
  if (d == 128) return f16 ? launch<128, true>(a, parts, s) : launch<128, false>(a, parts, s);
  return f16 ? launch<64, true>(a, parts, s) : launch<64, false>(a, parts, s);
}

}  // namespace vsa
