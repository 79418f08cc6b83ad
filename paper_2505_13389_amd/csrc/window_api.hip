// C ABI of windowed attention and the 8-bit cache: checks of the arguments, then the launches.  See include/vsa.h.
#include "../../include/vsa.h"

#include <math.h>

#include <vector>

#include "vsa_kernels.h"
#include "window_kernels.h"

namespace {

using vsa::WinArgs;

static_assert(VSA_PAGE_TOKENS == vsa::kPage, "the page of the header");

using vsa::kMostRows;
constexpr long long kMostBlocks = 1ll << 23;   // workgroups of a launch: 256 threads each stay below 2^32
constexpr int64_t kMostStride = 1 << 24;       // token strides: the byte offsets of 32 rows stay in 32 bits

bool off(const void* p, unsigned bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

int check_common(int B, int H, int Hkv, int d, int unit, int left, int right, int sinks, float scale, int dtype) {
  if (B < 1 || H < 1 || Hkv < 1 || H % Hkv) return VSA_ERR_BAD_ARG;
  if (d != 64 && d != 128) return VSA_ERR_UNSUPPORTED;
  if (unit < 1 || left < -1 || right < -1 || sinks < 0) return VSA_ERR_BAD_ARG;
  if (!(scale <= 3e38f)) return VSA_ERR_BAD_ARG;  // (NaN and infinity)
  if (dtype != VSA_DTYPE_BF16 && dtype != VSA_DTYPE_FP16) return VSA_ERR_BAD_ARG;
  return VSA_OK;
}

// strides of an input (least 0) or an output, whose rows may not overlap (least d), where there is more than one of them
int check_strides(const vsa_strides_t& s, long long batches, long long tokens, long long heads, int64_t least) {
  if (s.batch < 0 || s.token < 0 || s.head < 0) return VSA_ERR_BAD_ARG;
  if (s.batch % 8 || s.token % 8 || s.head % 8) return VSA_ERR_ALIGN;
  if (s.token > kMostStride || s.head > (1ll << 40) || s.batch > (1ll << 40)) return VSA_ERR_UNSUPPORTED;
  if ((batches > 1 && s.batch < least) || (tokens > 1 && s.token < least) || (heads > 1 && s.head < least)) return VSA_ERR_BAD_ARG;
  return VSA_OK;
}

vsa::RowView view(const void* p, const vsa_strides_t& s, bool packed) {
  return {(const unsigned char*)p, packed ? 0 : 2 * s.batch, 2 * s.token, 2 * s.head};
}

float scale_or_default(float scale, int d) { return scale > 0.f ? scale : 1.0f / sqrtf((float)d); }

long long blocks_of(long long B, long long items) { return B * ((items + 7) / 8 * 8); }

int check_window(const vsa_window_t* p) {
  if (!p) return VSA_ERR_NULL;
  const int rc = check_common(p->B, p->H, p->Hkv, p->d, p->unit, p->left, p->right, p->sinks, p->softmax_scale, p->dtype);
  if (rc != VSA_OK) return rc;
  if (p->max_q < 0 || p->max_k < 0 || p->total_q < 0 || p->total_k < 0) return VSA_ERR_BAD_ARG;
  if (p->max_q > kMostRows || p->max_k > kMostRows || p->total_q > kMostRows || p->total_k > kMostRows ||
      (long long)p->B * p->max_q > 2 * kMostRows)
    return VSA_ERR_UNSUPPORTED;
  const long long qb = (p->max_q + 63) / 64, kb = (p->max_k + 31) / 32;
  if (blocks_of(p->B, qb * p->H) > kMostBlocks || blocks_of(p->B, kb * p->Hkv) > kMostBlocks) return VSA_ERR_UNSUPPORTED;
  const long long rows = (long long)p->B * p->max_q > p->total_q ? (long long)p->B * p->max_q : p->total_q;
  if (rows * p->H * (p->d / 8) > (kMostBlocks << 8)) return VSA_ERR_UNSUPPORTED;
  return VSA_OK;
}

// rows of the query tensors; `packed` by whether offsets are given
long long stat_rows(const vsa_window_t* p, bool packed) { return packed ? p->total_q : (long long)p->B * p->max_q; }

WinArgs window_args(const vsa_window_t* p, bool packed, const int32_t* cu_q, const int32_t* cu_k) {
  WinArgs a = {};
  a.mask = vsa::win_mask(p->unit, p->left, p->right, p->sinks);
  a.B = p->B, a.H = p->H, a.Hkv = p->Hkv, a.G = p->H / p->Hkv;
  a.rq = {cu_q, p->max_q, packed ? p->total_q : (long long)p->max_q};
  a.rk = {cu_k, p->max_k, packed ? p->total_k : (long long)p->max_k};
  a.lse_rows = stat_rows(p, packed);
  a.scale = scale_or_default(p->softmax_scale, p->d);
  return a;
}

// of the backward: the rows' terms, then partial results
size_t terms_bytes(const WinArgs& a) { return ((size_t)a.H * a.lse_rows * 8 + 255) / 256 * 256; }
size_t fwd_bytes(const vsa_window_t* p, const WinArgs& a) { return vsa::row_parts(a, p->max_k, p->d) * sizeof(float) + 16; }
size_t bwd_bytes(const vsa_window_t* p, const WinArgs& a) { return terms_bytes(a) + vsa::window_parts(a, p->d) * sizeof(float) + 16; }

int check_window_strides(const vsa_window_t* p, bool packed, bool backward) {
  const long long nb = packed ? 1 : p->B, nq = packed ? p->total_q : p->max_q, nk = packed ? p->total_k : p->max_k;
  int rc = check_strides(p->q, nb, nq, p->H, 0);
  if (rc == VSA_OK) rc = check_strides(p->k, nb, nk, p->Hkv, 0);
  if (rc == VSA_OK) rc = check_strides(p->v, nb, nk, p->Hkv, 0);
  if (rc == VSA_OK) rc = check_strides(p->out, nb, nq, p->H, p->d);
  if (rc != VSA_OK || !backward) return rc;
  rc = check_strides(p->dout, nb, nq, p->H, 0);
  if (rc == VSA_OK) rc = check_strides(p->dq, nb, nq, p->H, p->d);
  if (rc == VSA_OK) rc = check_strides(p->dk, nb, nk, p->Hkv, p->d);
  if (rc == VSA_OK) rc = check_strides(p->dv, nb, nk, p->Hkv, p->d);
  return rc;
}

struct Recorded {
  hipStream_t s;
  int slot;
  Recorded(const char* name, hipStream_t stream) : s(stream), slot(vsa::profile_start(name, stream)) {}
  ~Recorded() { vsa::profile_stop(slot, s); }
};
#define VSA_LAUNCH(name, expr)                    \
  do {                                            \
    Recorded recorded_(name, s);                  \
    if ((expr) != hipSuccess) return VSA_ERR_HIP; \
  } while (0)

// Few rows a key head (the heads of its group times the queries): the pages are split over workgroups.
bool few_rows(const vsa_cache_t* p) { return (long long)p->max_q * (p->H / p->Hkv) <= 128; }

int check_cache(const vsa_cache_t* p, bool attention) {
  if (!p) return VSA_ERR_NULL;
  const int rc = attention ? check_common(p->B, p->H, p->Hkv, p->d, p->unit, p->left, p->right, p->sinks, p->softmax_scale, p->dtype)
                           : check_common(p->B, p->Hkv, p->Hkv, p->d, 1, 0, 0, 0, 0.f, p->dtype);
  if (rc != VSA_OK) return rc;
  if (p->max_q < 0 || p->total_q < 0 || p->pages < 1 || p->max_pages < 1) return VSA_ERR_BAD_ARG;
  if (p->max_q > kMostRows || p->total_q > kMostRows || (long long)p->B * p->max_q > 2 * kMostRows || p->max_pages > kMostRows / vsa::kPage)
    return VSA_ERR_UNSUPPORTED;
  const long long heads = attention ? p->H : p->Hkv;
  if (blocks_of(p->B, ((long long)p->max_q / 64 + 2) * heads) > kMostBlocks) return VSA_ERR_UNSUPPORTED;
  if (attention && few_rows(p) && (long long)p->B * p->Hkv * 8 > kMostBlocks / 16) return VSA_ERR_UNSUPPORTED;  // (row tiles are 8 at most)
  return VSA_OK;
}

WinArgs cache_args(const vsa_cache_t* p, const int32_t* cu) {
  WinArgs a = {};
  a.mask = vsa::win_mask(p->unit, p->left, p->right, p->sinks);
  a.B = p->B, a.H = p->H, a.Hkv = p->Hkv, a.G = p->H / p->Hkv;
  a.rq = {cu, p->max_q, cu ? p->total_q : (long long)p->max_q};
  a.lse_rows = cu ? p->total_q : (long long)p->B * p->max_q;
  a.scale = scale_or_default(p->softmax_scale, p->d);
  return a;
}
size_t cache_bytes(const vsa_cache_t* p, const WinArgs& a) {
  const size_t floats = few_rows(p) ? vsa::cache_parts(p->B, p->H, p->Hkv, p->d, p->max_q, p->max_pages)
                                    : vsa::row_parts(a, (long long)p->max_pages * vsa::kPage, p->d);
  return floats * sizeof(float) + 16;
}

// every visible pair once, no other unmasked: blocks of queries over keys, in pieces
int64_t replay_queries(const vsa_window_t* p, const vsa::WinMask& m, int nq, int nk, int block, int piece, int align) {
  int64_t wrong = 0;
  const int shift = nk - nq;
  std::vector<int> seen(nk);
  for (int r0 = 0; r0 < nq; r0 += block) {
    const int r1 = r0 + block < nq ? r0 + block : nq;
    const vsa::WinWalk walk(m, r0 + shift, r1 - 1 + shift, nk, piece, align);
    for (int r = r0; r < r1; ++r) {
      const vsa::WinSpan span = vsa::win_span(m, r + shift, nk);
      std::fill(seen.begin(), seen.end(), 0);
      for (int i = 0; i < walk.n; ++i) {
        const vsa::WinSpan w = walk.span_in(i, span);
        const int k0 = walk.begin(i);
        if (k0 < 0 || k0 >= nk || (align > 1 && k0 % align)) ++wrong;
        for (int j = k0; j < k0 + piece; ++j) {
          const bool see = j < w.hi && (j >= w.lo || j < w.se);
          if (see && j < nk) ++seen[j];
          if ((see && j >= nk) || (!see && !walk.masked(i))) ++wrong;
        }
      }
      auto unit = [&](long long x) { return x >= 0 ? x / p->unit : -((-x + p->unit - 1) / p->unit); };
      for (int j = 0; j < nk; ++j) {
        const long long uj = unit(j), up = unit((long long)r + shift);
        const bool see = (p->right < 0 || uj <= up + p->right) && (p->left < 0 || uj >= up - p->left || uj < p->sinks);
        wrong += seen[j] != (see ? 1 : 0);
      }
    }
  }
  return wrong;
}
int64_t replay_keys(const vsa::WinMask& m, int nq, int nk, int block) {
  int64_t wrong = 0;
  const int shift = nk - nq;
  std::vector<int> seen(nq);
  for (int k0 = 0; k0 < nk; k0 += block) {
    const int k1 = k0 + block < nk ? k0 + block : nk;
    const vsa::KeyWalk walk(m, k0, k1, nq, shift, 32);
    for (int j = k0; j < k1; ++j) {
      const vsa::KeySpan w = vsa::key_span(m, j);
      std::fill(seen.begin(), seen.end(), 0);
      for (int i = 0; i < walk.n; ++i) {
        const int q0 = walk.from + 32 * i;
        if (q0 < 0 || q0 >= nq) ++wrong;
        const bool masked = q0 + shift < walk.seen_from || q0 + shift + 32 > walk.seen_to || q0 + 32 > nq;
        for (int q = q0; q < q0 + 32; ++q) {
          const bool see = q < nq && q + shift >= w.lo && q + shift < w.hi;
          if (see) ++seen[q];
          if (!see && !masked) ++wrong;
        }
      }
      for (int q = 0; q < nq; ++q) {
        const vsa::WinSpan s = vsa::win_span(m, q + shift, nk);
        const bool see = j < s.hi && (j >= s.lo || j < s.se);
        wrong += seen[q] != (see ? 1 : 0);
      }
    }
  }
  return wrong;
}

}  // namespace

extern "C" {

int vsa_window_forward(const vsa_window_t* p, const void* q, const void* k, const void* v, const int32_t* cu_q,
                       const int32_t* cu_k, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_window(p);
  if (rc != VSA_OK) return rc;
  if (!cu_q != !cu_k) return VSA_ERR_BAD_ARG;
  const bool packed = cu_q != nullptr;
  const long long rows = stat_rows(p, packed), keys = packed ? p->total_k : (long long)p->B * p->max_k;
  if ((rows && (!q || !out)) || (keys && (!k || !v))) return VSA_ERR_NULL;
  if (off(q, 16) || off(k, 16) || off(v, 16) || off(out, 16) || off(lse, 4) || off(cu_q, 4) || off(cu_k, 4) || off(workspace, 16))
    return VSA_ERR_ALIGN;
  if ((rc = check_window_strides(p, packed, false)) != VSA_OK) return rc;
  WinArgs a = window_args(p, packed, cu_q, cu_k);
  if (!workspace || workspace_bytes < fwd_bytes(p, a)) return VSA_ERR_WORKSPACE;
  if (rows == 0 || p->max_q == 0) return VSA_OK;
  a.q = view(q, p->q, packed), a.k = view(k, p->k, packed), a.v = view(v, p->v, packed), a.o = view(out, p->out, packed);
  a.lse = lse;
  hipStream_t s = (hipStream_t)hip_stream;
  VSA_LAUNCH("window_fwd", vsa::launch_window_fwd(a, p->d, p->dtype == VSA_DTYPE_FP16, (float*)workspace, s));
  return VSA_OK;
}

size_t vsa_window_workspace_bytes(const vsa_window_t* p, int backward) {
  if (check_window(p) != VSA_OK) return 0;
  size_t most = 0;
  for (int packed = 0; packed < 2; ++packed) {  // (which of them it is the call says)
    const int32_t* const cu = packed ? (const int32_t*)p : nullptr;  // (never read: not null is all that counts here)
    const WinArgs a = window_args(p, packed != 0, cu, cu);
    const size_t bytes = backward ? bwd_bytes(p, a) : fwd_bytes(p, a);
    most = bytes > most ? bytes : most;
  }
  return most;
}

int vsa_window_backward(const vsa_window_t* p, const void* q, const void* k, const void* v, const int32_t* cu_q,
                        const int32_t* cu_k, const void* out, const void* dout, const float* lse, void* dq, void* dk, void* dv,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_window(p);
  if (rc != VSA_OK) return rc;
  if (!cu_q != !cu_k) return VSA_ERR_BAD_ARG;
  const bool packed = cu_q != nullptr;
  const long long rows = stat_rows(p, packed), keys = packed ? p->total_k : (long long)p->B * p->max_k;
  if ((rows && (!q || !out || !dout || !lse || !dq)) || (keys && (!k || !v || !dk || !dv))) return VSA_ERR_NULL;
  if (off(q, 16) || off(k, 16) || off(v, 16) || off(out, 16) || off(dout, 16) || off(dq, 16) || off(dk, 16) || off(dv, 16) || off(lse, 4) ||
      off(cu_q, 4) || off(cu_k, 4) || off(workspace, 16))
    return VSA_ERR_ALIGN;
  if ((rc = check_window_strides(p, packed, true)) != VSA_OK) return rc;
  WinArgs a = window_args(p, packed, cu_q, cu_k);
  if (!workspace || workspace_bytes < bwd_bytes(p, a)) return VSA_ERR_WORKSPACE;
  a.q = view(q, p->q, packed), a.k = view(k, p->k, packed), a.v = view(v, p->v, packed), a.o = view(out, p->out, packed);
  a.dout = view(dout, p->dout, packed), a.dq = view(dq, p->dq, packed), a.dk = view(dk, p->dk, packed), a.dv = view(dv, p->dv, packed);
  a.lse = const_cast<float*>(lse);
  a.stats = (float*)workspace;
  float* const parts = (float*)((unsigned char*)workspace + terms_bytes(a));
  hipStream_t s = (hipStream_t)hip_stream;
  VSA_LAUNCH("window_bwd", vsa::launch_window_bwd(a, p->d, p->dtype == VSA_DTYPE_FP16, parts, s));
  return VSA_OK;
}

int vsa_cache_append(const vsa_cache_t* p, const void* k, const void* v, const int32_t* cu, const int32_t* lens,
                     const int32_t* table, void* k_pages, void* v_pages, float* k_scale, float* v_scale, void* hip_stream) {
  int rc = check_cache(p, false);
  if (rc != VSA_OK) return rc;
  const bool packed = cu != nullptr;
  const long long rows = packed ? p->total_q : (long long)p->B * p->max_q;
  if ((rows && (!k || !v)) || !lens || !table || !k_pages || !v_pages || !k_scale || !v_scale) return VSA_ERR_NULL;
  if (off(k, 16) || off(v, 16) || off(k_pages, 16) || off(v_pages, 16) || off(k_scale, 4) || off(v_scale, 4) || off(cu, 4) || off(lens, 4) ||
      off(table, 4))
    return VSA_ERR_ALIGN;
  const long long nb = packed ? 1 : p->B, n = packed ? p->total_q : p->max_q;
  if ((rc = check_strides(p->k, nb, n, p->Hkv, 0)) != VSA_OK || (rc = check_strides(p->v, nb, n, p->Hkv, 0)) != VSA_OK) return rc;
  if (rows == 0 || p->max_q == 0) return VSA_OK;
  vsa::AppendArgs a = {};
  a.c = {(uint8_t*)k_pages, (uint8_t*)v_pages, k_scale, v_scale, table, lens, p->max_pages, p->pages};
  a.B = p->B, a.Hkv = p->Hkv, a.d = p->d, a.f16 = p->dtype == VSA_DTYPE_FP16;
  a.rows = {cu, p->max_q, packed ? p->total_q : (long long)p->max_q};
  a.k = view(k, p->k, packed), a.v = view(v, p->v, packed);
  hipStream_t s = (hipStream_t)hip_stream;
  VSA_LAUNCH("cache_append", vsa::launch_cache_append(a, s));
  return VSA_OK;
}

size_t vsa_cache_workspace_bytes(const vsa_cache_t* p) {
  if (check_cache(p, true) != VSA_OK) return 0;
  const size_t dense = cache_bytes(p, cache_args(p, nullptr)), packed = cache_bytes(p, cache_args(p, (const int32_t*)p));  // (not read)
  return dense > packed ? dense : packed;
}

int vsa_cache_attention(const vsa_cache_t* p, const void* q, const int32_t* cu, const int32_t* lens, const int32_t* table,
                        const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale, void* out, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_cache(p, true);
  if (rc != VSA_OK) return rc;
  const bool packed = cu != nullptr;
  const long long rows = packed ? p->total_q : (long long)p->B * p->max_q;
  if ((rows && (!q || !out)) || !lens || !table || !k_pages || !v_pages || !k_scale || !v_scale) return VSA_ERR_NULL;
  if (off(q, 16) || off(out, 16) || off(k_pages, 16) || off(v_pages, 16) || off(k_scale, 4) || off(v_scale, 4) || off(lse, 4) || off(cu, 4) ||
      off(lens, 4) || off(table, 4) || off(workspace, 16))
    return VSA_ERR_ALIGN;
  const long long nb = packed ? 1 : p->B, n = packed ? p->total_q : p->max_q;
  if ((rc = check_strides(p->q, nb, n, p->H, 0)) != VSA_OK || (rc = check_strides(p->out, nb, n, p->H, p->d)) != VSA_OK) return rc;
  WinArgs a = cache_args(p, cu);
  if (!workspace || workspace_bytes < cache_bytes(p, a)) return VSA_ERR_WORKSPACE;
  if (rows == 0 || p->max_q == 0) return VSA_OK;
  a.q = view(q, p->q, packed), a.o = view(out, p->out, packed);
  a.lse = lse;
  const vsa::CacheArgs c = {(uint8_t*)const_cast<void*>(k_pages), (uint8_t*)const_cast<void*>(v_pages), const_cast<float*>(k_scale),
                            const_cast<float*>(v_scale), table, lens, p->max_pages, p->pages};
  hipStream_t s = (hipStream_t)hip_stream;
  const bool f16 = p->dtype == VSA_DTYPE_FP16;
  if (few_rows(p)) VSA_LAUNCH("cache_token", vsa::launch_cache_token(a, c, p->d, f16, (float*)workspace, s));
  else VSA_LAUNCH("cache_chunk", vsa::launch_cache_chunk(a, c, p->d, f16, (float*)workspace, s));
  return VSA_OK;
}

int vsa_host_window_walk(const vsa_window_t* p, int32_t nq, int32_t nk, int64_t* wrong) {
  const int rc = check_window(p);
  if (rc != VSA_OK) return rc;
  if (!wrong) return VSA_ERR_NULL;
  if (nq < 0 || nk < 0 || nq > 1 << 16 || nk > 1 << 16) return VSA_ERR_BAD_ARG;
  const vsa::WinMask m = vsa::win_mask(p->unit, p->left, p->right, p->sinks);
  *wrong = replay_queries(p, m, nq, nk, 64, 32, 1) + replay_queries(p, m, nq, nk, 64, 32, 32) + replay_queries(p, m, nq, nk, 3, 64, 64) +
           replay_keys(m, nq, nk, 32) + replay_keys(m, nq, nk, 64);
  return *wrong ? VSA_ERR_BAD_ARG : VSA_OK;
}

}  // extern "C"
