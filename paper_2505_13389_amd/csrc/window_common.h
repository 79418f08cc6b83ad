// Windowed attention: what a query sees, where sequences and rows lie, and how a block of queries walks its keys.
//
// The last query of a sequence stands at its last key: query i is at position i + nk - nq.  Positions are counted in units
// of `unit` tokens (a frame, or 1).  Key j is visible to position p iff
//     j/unit <= p/unit + right   and   (j/unit >= p/unit - left  or  j/unit < sinks)
// (a negative left or right is no bound), which is j < hi && (j >= lo || j < se) with three numbers a query.  All three
// never fall from one query to the next, so the first and the last query of a block say what a run of keys is to all of it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vsa {

// Numbers of tokens and positions stay below kMostRows, so that everything here fits 32 bits.
constexpr long long kMostRows = 1ll << 28;

struct WinMask {
  int unit, left, right;  // (bounded by what any position can reach: win_mask)
  int sinks;              // in tokens
  uint32_t magic;         // x / unit = x * magic >> 32 + shift for 0 <= x < 2^31, unit > 1
  int shift;
};
inline WinMask win_mask(int unit, int left, int right, int sinks) {
  const long long most = kMostRows;
  WinMask m;
  m.unit = unit < most ? unit : (int)most;
  const int reach = (int)(most / m.unit) + 2;
  m.left = left < reach ? left : reach;
  m.right = right < reach ? right : reach;
  m.sinks = (int)((long long)sinks * unit < most ? (long long)sinks * unit : most);
  int s = 0;
  while ((1ll << s) < m.unit) ++s;
  m.magic = m.unit > 1 ? (uint32_t)(((1ull << (31 + s)) + (uint64_t)m.unit - 1) / (uint64_t)m.unit) : 0;
  m.shift = s - 1;
  return m;
}
__host__ __device__ inline int win_unit(const WinMask& m, int x) {  // floor(x / unit), also of negative x
  if (m.unit == 1) return x;
  const uint32_t y = (uint32_t)(x < 0 ? ~x : x), q = (uint32_t)(((uint64_t)y * m.magic) >> 32) >> m.shift;
  return x < 0 ? ~(int)q : (int)q;
}

struct WinSpan {
  int lo, hi, se;  // lo <= hi, se <= hi <= nk
};

__host__ __device__ inline WinSpan win_span(const WinMask& m, int pos, int nk) {
  const int u = win_unit(m, pos);
  auto clamp = [](int x, int top) { return x < 0 ? 0 : x > top ? top : x; };
  WinSpan s;
  s.hi = m.right < 0 ? nk : clamp((u + m.right + 1) * m.unit, nk);
  s.lo = m.left < 0 ? 0 : clamp((u - m.left) * m.unit, s.hi);
  s.se = m.sinks < s.hi ? m.sinks : s.hi;
  return s;
}

// Keys that queries at positions first .. last walk, in pieces of `piece` keys: [0, sink) and then [from, to).  Keys of the
// second run that a row does not see and of the first behind `sink` are masked.
struct WinWalk {
  WinSpan a, z;  // of the first and the last query
  int sink, from, n_sink, n;  // pieces of the sinks, of both runs
  int piece;
  // `align`: the second run begins at a multiple of it
  __host__ __device__ WinWalk(const WinMask& m, int first, int last, int nk, int piece_, int align) : piece(piece_) {
    a = win_span(m, first, nk);
    z = win_span(m, last, nk);
    from = a.lo / align * align;
    sink = z.se < from ? z.se : from;
    n_sink = (sink + piece - 1) / piece;
    n = n_sink + (z.hi - from + piece - 1) / piece;
  }
  __host__ __device__ int begin(int i) const { return i < n_sink ? i * piece : from + (i - n_sink) * piece; }
#if defined(__HIP_DEVICE_COMPILE__)
  // (equal in all lanes: into scalar registers, where the arithmetic that led here has not put them)
  __device__ __forceinline__ void uniform() {
    int* const all[] = {&a.lo, &a.hi, &a.se, &z.lo, &z.hi, &z.se, &sink, &from, &n_sink, &n};
#pragma unroll
    for (int i = 0; i < 10; ++i) *all[i] = __builtin_amdgcn_readfirstlane(*all[i]);
  }
#else
  __host__ __device__ void uniform() {}
#endif
  // whether piece i holds keys that some query of the block does not see
  __host__ __device__ bool masked(int i) const {
    const int e = begin(i) + piece;
    if (i < n_sink) return e > a.se || e > sink;
    return !(e <= a.hi && (e - piece >= z.lo || e <= a.se));
  }
  // of one query with span s: the visible keys of piece i are those with j < hi && (j >= lo || j < se)
  __host__ __device__ WinSpan span_in(int i, const WinSpan& s) const {
    if (i >= n_sink) return s;
    const int e = s.se < sink ? s.se : sink;
    return {e, e, e};
  }
};

// Queries that see any of the keys k0 .. k1 - 1 are those of [from, to); key j is seen from position lo up to (not with) hi.
struct KeySpan {
  int lo, hi;
};
__host__ __device__ inline KeySpan key_span(const WinMask& m, int j) {
  const int u = win_unit(m, j), far = 1 << 30;
  return {m.right < 0 ? -far : (u - m.right) * m.unit, m.left < 0 || j < m.sinks ? far : (u + m.left + 1) * m.unit};
}
struct KeyWalk {
  int from, to, n;          // queries; pieces of `piece` of them
  int seen_from, seen_to;   // positions that see all of the keys
  __host__ __device__ KeyWalk(const WinMask& m, int k0, int k1, int nq, int shift, int piece) {
    const KeySpan a = key_span(m, k0), z = key_span(m, k1 - 1);
    auto clamp = [&](int x) { return x < 0 ? 0 : x > nq ? nq : x; };
    from = clamp(a.lo - shift);
    // (the first keys may be sinks and the others not)
    to = clamp((a.hi > z.hi ? a.hi : z.hi) - shift);
    if (to < from) to = from;
    n = (to - from + piece - 1) / piece;
    seen_from = z.lo;
    seen_to = z.hi;  // never falls from key to key behind the sinks; the first key behind them has the least
    const int first_other = k0 > m.sinks ? k0 : m.sinks;
    if (first_other < k1) seen_to = key_span(m, first_other).hi;
  }
};

// A tensor of token rows: byte strides of batch, token and head (packed tensors: batch 0).
struct RowView {
  const unsigned char* p;
  long long batch, token, head;
  __host__ __device__ const unsigned char* row(int b, long long t, int h) const { return p + b * batch + t * token + h * head; }
  __host__ __device__ unsigned char* out(int b, long long t, int h) const { return const_cast<unsigned char*>(row(b, t, h)); }
};

// Where the rows of a sequence lie.  Offsets come from device memory and are not trusted: no row leaves [0, total), and no
// sequence is longer than `most`, for which the launch is made.
struct WinRows {
  const int32_t* cu;  // offsets of packed sequences, or null: dense, `most` rows each
  int most;
  long long total;
};
struct WinSeq {
  long long row0;  // first row in the tensor (packed) or 0 (dense)
  int n;
};
__host__ __device__ inline WinSeq win_seq(const WinRows& r, int b) {
  if (!r.cu) return {0, r.most};
  long long s = r.cu[b], e = r.cu[b + 1];
  s = s < 0 ? 0 : s > r.total ? r.total : s;
  const long long top = r.total - s < r.most ? r.total : s + r.most;
  e = e < s ? s : e > top ? top : e;
  return {s, (int)(e - s)};
}

// Item number `block` of a launch -> head (of `heads`) and one of its `per_head` items; false: there are fewer.
// Workgroups are dealt to the 8 XCDs in turn, each of which has an L2.  An XCD takes whole heads, whose items read the same
// keys; those of the heads left over are dealt to all of them, item by item, so that the XCDs get the same amount of work (packed
// prompts of 1 to 6001 tokens, 16 heads on 4: with contiguous runs of a sequence's items 170 us, so 145).
__device__ __forceinline__ bool win_item(unsigned block, unsigned heads, unsigned per_head, int& head, int& item) {
  const unsigned x = block & 7u, n = block >> 3, whole = heads >> 3, rest = heads & 7u;
  if (n < whole * per_head) {
    const unsigned k = n < per_head ? 0u : n / per_head;
    head = (int)(x + 8u * k);
    item = (int)(n - k * per_head);
    return true;
  }
  const unsigned j = (n - whole * per_head) * 8u + x;
  if (j >= rest * per_head) return false;
  item = (int)((rest & (rest - 1u)) == 0u ? j >> __builtin_ctz(rest) : j / rest);
  head = (int)(8u * whole + j - (unsigned)item * rest);
  return true;
}
inline unsigned win_grid(long long items) { return (unsigned)((items + 7) & ~7ll); }

// Blocks of 64 rows of all sequences, one sequence behind the other: at most `win_blocks`.  Dense: the same number each.
inline long long win_blocks(const WinRows& r, int B) {
  const long long each = (r.most + 63) / 64;
  if (!r.cu) return each * B;
  const long long all = r.total / 64 + B;
  return all < each * B ? all : each * B;
}
// Block number t of all -> its sequence, number there and the rows of the sequence in the tensors of r and of `other` (null: not
// asked for); false: there are fewer.  (All lanes of a wavefront: a lane looks at a sequence.)
__device__ __forceinline__ WinSeq win_pick(const WinSeq& s, int lane) {
  return {(long long)(unsigned)__builtin_amdgcn_readlane((int)s.row0, lane), __builtin_amdgcn_readlane(s.n, lane)};  // (rows are below 2^31)
}
__device__ __forceinline__ bool win_find(const WinRows& r, const WinRows* other, int B, unsigned t, int& b, int& block, WinSeq& rows, WinSeq& others) {
  if (!r.cu) {
    const unsigned each = (unsigned)(r.most + 63) / 64u;
    b = (int)(t / each);
    block = (int)(t - (unsigned)b * each);
    rows = {0, r.most};
    if (other) others = win_seq(*other, b);
    return b < B;
  }
  const int lane = threadIdx.x & 63;
  unsigned before = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int at = min(b0 + lane, B - 1);
    const WinSeq here = win_seq(r, at), there = other ? win_seq(*other, at) : WinSeq{0, 0};
    const unsigned mine = b0 + lane < B ? (unsigned)(here.n + 63) / 64u : 0u;
    unsigned upto = mine;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const unsigned x = __shfl_up(upto, m);
      if (lane >= m) upto += x;
    }
    const unsigned long long past = __ballot(before + upto > t);
    if (past) {
      const int l = __builtin_ctzll(past);
      b = __builtin_amdgcn_readfirstlane(b0 + l);
      block = (int)(t - before) - (int)__builtin_amdgcn_readlane((int)(upto - mine), l);
      block = __builtin_amdgcn_readfirstlane(block);
      rows = win_pick(here, l);
      if (other) others = win_pick(there, l);
      return true;
    }
    before += (unsigned)__builtin_amdgcn_readlane((int)upto, 63);
  }
  return false;
}

struct WinArgs {
  WinMask mask;
  int B, H, Hkv, G;  // G = H / Hkv
  WinRows rq, rk;
  RowView q, k, v, o, dout, dq, dk, dv;
  float* lse;    // [H, lse_rows]
  float* stats;  // [2][H, lse_rows], of the backward: -lse / scale (-inf for a row that sees nothing), -rowsum(dO * O)
  long long lse_rows;
  float scale;
  // row of the statistics of query i of sequence b with first row row0
  __device__ long long stat(int h, int b, long long row0, int i) const { return h * lse_rows + (rq.cu ? row0 : (long long)b * rq.most) + i; }
};

// How the blocks of 64 queries are dealt to workgroups of `nw` wavefronts: each head's (dense: each sequence's and head's) `blocks`, in
// `parts` parts of their keys of at least `per` units of 32.
struct RowPlan {
  int blocks, parts, per, nw;
};
struct RowItem {
  int b, hk, g, qb, part;
  WinSeq q, k;
};
// `paged`: the keys are not rows of a tensor
__device__ __forceinline__ bool win_rows(const WinArgs& a, const RowPlan& plan, unsigned workgroup, bool paged, RowItem& t) {
  int head, item;
  const bool packed = a.rq.cu != nullptr;
  if (!win_item(workgroup, (unsigned)(packed ? a.Hkv : a.B * a.Hkv), (unsigned)(plan.blocks * a.G * plan.parts), head, item)) return false;
  t.part = t.g = 0;
  if (plan.parts > 1) t.part = item % plan.parts, item /= plan.parts;
  if (a.G > 1) t.g = item % a.G, item /= a.G;
  const int block = plan.blocks - 1 - item;  // (the last queries have most to walk: they come first)
  if (packed) {
    t.hk = head;
    return win_find(a.rq, paged ? nullptr : &a.rk, a.B, (unsigned)block, t.b, t.qb, t.q, t.k);
  }
  t.b = a.B > 1 ? head / a.Hkv : 0;
  t.hk = head - t.b * a.Hkv;
  t.qb = block;
  t.q = {0, a.rq.most};
  t.k = {0, a.rk.most};
  return true;
}
inline long long win_workgroups(const WinArgs& a, const RowPlan& plan) {
  return (long long)(a.rq.cu ? 1 : a.B) * a.Hkv * plan.blocks * a.G * plan.parts;
}
// units of 32 keys that a block of queries walks at most
inline long long win_units(const WinMask& m, long long max_k) {
  const long long all = max_k / 32 + 1;
  if (m.left < 0 || m.right < 0) return all;
  const long long run = ((long long)(m.left + m.right + 2) * m.unit + 64) / 32 + 1 + (m.sinks + 31) / 32;
  return run < all ? run : all;
}

}  // namespace vsa
