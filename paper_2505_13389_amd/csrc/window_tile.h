// Operands and copies of the windowed-attention kernels: both 16-bit types, rows with any stride, and pages of the 8-bit cache.
#pragma once
#include "fine_tile.h"
#include "window_common.h"

namespace vsa {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Operands are carried as bf16x8 whatever their type: 16 bytes.
template <bool F16>
__device__ __forceinline__ f32x16 mm32(bf16x8 a, bf16x8 b, f32x16 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
template <bool F16>
__device__ __forceinline__ f32x4 mm16(bf16x8 a, bf16x8 b, f32x4 c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// two floats to 16 bits, to the nearest even
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (F16) {
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
  } else {
    return pack_bf16(a, b);
  }
}
template <bool F16>
__device__ __forceinline__ void widen16(uint32_t u, float& a, float& b) {
  if constexpr (F16) {
    const f16x2 x = __builtin_bit_cast(f16x2, u);
    a = (float)x[0], b = (float)x[1];
  } else {
    a = bf_lo(u), b = bf_hi(u);
  }
}
template <bool F16>
__device__ __forceinline__ void widen8(const uint4& u, float* f) {
  widen16<F16>(u.x, f[0], f[1]);
  widen16<F16>(u.y, f[2], f[3]);
  widen16<F16>(u.z, f[4], f[5]);
  widen16<F16>(u.w, f[6], f[7]);
}

// eight e4m3 values (8 bytes) to 16 bits: exact, e4m3's values are all bf16 and fp16 values
template <bool F16>
__device__ __forceinline__ bf16x8 from_e4m3(uint32_t lo, uint32_t hi) {
  uint4 u;
  if constexpr (F16) {
    u.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
    u.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
    u.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
    u.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
  } else {
    u.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    u.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    u.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    u.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  }
  return __builtin_bit_cast(bf16x8, u);
}

// 64 lanes x 16 bytes, global -> 1 KiB of LDS at `lds`.  The base may have come out of a vector register right before, which
// takes 5 wait states; M0 takes one.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void win_copy16(const void* base, unsigned voff, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff), "s"(base), "s"(lds) : "memory", "m0");
}
// the same waits, ahead of a run of copies
__device__ __forceinline__ void win_aim(unsigned lds) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 4" : : "s"(lds) : "m0", "memory"); }
#pragma clang diagnostic pop
template <int N>
__device__ __forceinline__ void win_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Copies of 32 rows with any stride by one wavefront: instruction c fills LDS rows c*RPI .., swizzled on the source side.  Four
// of them share a value of M0 (their immediate offsets are added to both addresses, the lane offsets make up for the global one, which
// takes rows that are at least as far apart as in LDS) and their lane offsets: the swizzle repeats after 16 rows.
template <int D>
struct RowCopy {
  using TL = Tile<D>;
  static constexpr int NC = 32 / TL::RPI;
  unsigned off[4];
  unsigned stride;
  __device__ __forceinline__ unsigned at(int c, int lane, int last) const {
    const int x = c * TL::RPI + lane / TL::CPR, pc = lane % TL::CPR;
    return (unsigned)min(x, last) * stride + ((pc ^ TL::swz(x)) << 4);
  }
  __device__ __forceinline__ void init(int lane, unsigned stride_) {
    stride = stride_;
#pragma unroll
    for (int c = 0; c < 4; ++c) off[c] = at(c, lane, 31) - (unsigned)c * 1024u;
  }
  // 32 rows are there, far enough apart: piece by piece
  __device__ __forceinline__ bool plain(int have) const { return have >= 32 && stride >= TL::ROW_BYTES; }
  __device__ __forceinline__ void aim(unsigned lds, int c) const {
    if (c % 4 == 0) set_m0_ahead(lds + (unsigned)c * 1024u);
  }
  // (aim(lds, c) and another instruction came before it)
  __device__ __forceinline__ void piece(const unsigned char* base, int c) const {
    const unsigned char* g = c < 4 ? base : base + 4 * TL::RPI * (long long)stride;
    if (c % 4 == 0) lds_dma16_at<0>(g, off[c % 4]);
    if (c % 4 == 1) lds_dma16_at<1 * 1024>(g, off[c % 4]);
    if (c % 4 == 2) lds_dma16_at<2 * 1024>(g, off[c % 4]);
    if (c % 4 == 3) lds_dma16_at<3 * 1024>(g, off[c % 4]);
  }
  // all of it; `have` rows are there: the last of them stands for those behind it
  __device__ __forceinline__ void all(const unsigned char* base, unsigned lds, int lane, int have) const {
    if (__builtin_expect(plain(have), 1)) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        if (c % 4 == 0) win_aim(lds + (unsigned)c * 1024u);
        piece(base, c);
      }
    } else {
      asm volatile("" : "+v"(lane));  // (nothing of this is kept in registers)
#pragma unroll
      for (int c = 0; c < NC; ++c) win_copy16(base, at(c, lane, min(have, 32) - 1), lds + (unsigned)c * 1024u);
    }
  }
};

// Rows of results out of LDS, 8 elements a thread and turn: fp32 partial results [64][D] of NW wavefronts (XOR-swizzled, see merge_offset),
// `pitch` floats apart, added.  Reads of several turns are in flight at once: read one after the other, the rows of a block of 64 took a
// lone wavefront 9000 cycles of the 80000 of a walk of 1100 keys.  use(row, chunk, values).
template <int D, int NW, class USE>
__device__ __forceinline__ void win_rows_out(const float* buf, int pitch, int tid, int rows, const USE& use) {
  constexpr int CPR = D / 8, NT = 64 * NW, TURNS = 64 * CPR / NT, AT_ONCE = TURNS < 4 ? TURNS : 4;
  static_assert(NT % CPR == 0, "a thread keeps its column chunk");
  const int ch = tid % CPR, r0 = tid / CPR;
#pragma unroll
  for (int t0 = 0; t0 < TURNS; t0 += AT_ONCE) {
    if (t0 * (NT / CPR) >= rows) break;
    float4 x[AT_ONCE][NW][2];
#pragma unroll
    for (int t = 0; t < AT_ONCE; ++t)
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const int r = (t0 + t) * (NT / CPR) + r0;
        x[t][w][0] = *(const float4*)&buf[w * pitch + merge_offset(r, ch * 8, D)];
        x[t][w][1] = *(const float4*)&buf[w * pitch + merge_offset(r, ch * 8 + 4, D)];
      }
#pragma unroll
    for (int t = 0; t < AT_ONCE; ++t) {
      const int r = (t0 + t) * (NT / CPR) + r0;
      float v[8] = {x[t][0][0].x, x[t][0][0].y, x[t][0][0].z, x[t][0][0].w, x[t][0][1].x, x[t][0][1].y, x[t][0][1].z, x[t][0][1].w};
#pragma unroll
      for (int w = 1; w < NW; ++w) {
        v[0] += x[t][w][0].x, v[1] += x[t][w][0].y, v[2] += x[t][w][0].z, v[3] += x[t][w][0].w;
        v[4] += x[t][w][1].x, v[5] += x[t][w][1].y, v[6] += x[t][w][1].z, v[7] += x[t][w][1].w;
      }
      if (r < rows) use(r, ch, v);
    }
  }
}

}  // namespace vsa
