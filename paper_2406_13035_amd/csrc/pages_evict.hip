// Eviction by accumulated attention over caches in pages: prompts into pages (d2o_pages_fill) and a cache that has outgrown
// its budget back to it, in place (d2o_pages_evict).  Both choose by Eq. 7-8: the first tokens, the last ones, and the
// highest scores among the others.
#include <algorithm>

#include "pages.h"

namespace d2o {
namespace {

constexpr int kSelThreads = 1024;

// Order-preserving integer of a score: larger keys are kept first.  0 is below every score, 0xFFFFFFFF above.
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xFFFFFFFEu;
  if (x == 0.f) x = 0.f;  // -0 and +0 compare equal
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Exclusive prefix sum of v over the workgroup's threads, and the total.
__device__ __forceinline__ void block_scan(int v, int& before, int& total, int* wa) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(inc, o, 64);
    if (lane >= o) inc += t;
  }
  __syncthreads();
  if (lane == 63) wa[w] = inc;
  __syncthreads();
  int off = 0, all = 0;
  for (int i = 0; i < nw; ++i) {
    if (i < w) off += wa[i];
    all += wa[i];
  }
  before = off + inc - v;
  total = all;
}

// The `want`-th largest (1-based) of key(0 .. n-1): its value, and how many keys equal to it belong to the `want`
// largest.  Digits of eight bits from the top: a histogram of the candidates' digits, the bin in which the count from above reaches
// what is still wanted.
template <typename Key, typename F>
__device__ void nth_largest(int n, int want, const F& key, Key& value, int& equal, int* hist, int* sh) {
  const int tid = threadIdx.x;
  Key prefix = 0, mask = 0;
  for (int shift = int(sizeof(Key)) * 8 - 8; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kSelThreads) {
      const Key k = key(j);
      if ((k & mask) == prefix) atomicAdd(&hist[int(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid < 64) {  // lane i: bins 255 - 4 i down to 252 - 4 i
      int h[4], tot = 0;
      for (int u = 0; u < 4; ++u) tot += h[u] = hist[255 - 4 * tid - u];
      int inc = tot;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(inc, o, 64);
        if (tid >= o) inc += t;
      }
      int left = want - (inc - tot);
      if (left > 0 && want <= inc) {
        int u = 0;
        while (h[u] < left) left -= h[u++];
        sh[0] = 255 - 4 * tid - u;
        sh[1] = left;
      }
    }
    __syncthreads();
    prefix |= Key(sh[0]) << shift;
    mask |= Key(0xFF) << shift;
    want = sh[1];
    __syncthreads();
  }
  value = prefix;
  equal = want;
}

struct FillArgs {
  PagePool pool;
  View k, v;
  const int32_t* lens;
  const float* scores;
  int32_t* src;  // [B][Hkv][budget] kept positions, rising (only where something is evicted)
  int32_t n, budget, recent, n_sink;
};

__global__ __launch_bounds__(kSelThreads) void fill_select(FillArgs a) {
  __shared__ int hist[256], wa[16], sh[2];
  const int bh = blockIdx.x, b = bh / a.pool.Hkv, tid = threadIdx.x;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  if (n <= a.budget) return;
  const float* sc = a.scores + int64_t(bh) * a.n;
  const int late = n - a.recent;
  auto key = [&](int j) { return j < a.n_sink || j >= late ? 0xFFFFFFFFu : score_key(sc[j]); };
  uint32_t value;
  int equal;
  nth_largest<uint32_t>(n, a.budget, key, value, equal, hist, sh);
  int32_t* src = a.src + int64_t(bh) * a.budget;
  int kept = 0, same = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const uint32_t k = j < n ? key(j) : 0u;
    const bool eq = j < n && k == value;
    int before, total;
    block_scan(eq, before, total, wa);
    const bool keep = j < n && (k > value || (eq && same + before < equal));
    same += total;
    block_scan(keep, before, total, wa);
    if (keep) src[kept + before] = j;
    kept += total;
  }
}

// 16 bytes of a prompt row per lane, consecutive lanes consecutive chunks.
template <typename T, typename CT, int D>
__global__ __launch_bounds__(256) void fill_rows(FillArgs a) {
  constexpr int kLanes = D * int(sizeof(T)) / 16, kRows = 256 / kLanes, kE = 16 / int(sizeof(T));
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int s = blockIdx.x * kRows + threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  if (s >= min(n, a.budget)) return;
  const int page = a.pool.page_of(b, s);
  if (page < 0) return;
  const int j = n <= a.budget ? s : a.src[int64_t(bh) * a.budget + s];
  const int64_t at = a.pool.at(page, hk, s);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const View& x = which ? a.v : a.k;
    const T* row = static_cast<const T*>(x.ptr) + b * x.sb + hk * x.sh + int64_t(j) * x.sn;
    const u32x4 t = reinterpret_cast<const u32x4*>(row)[c];
    uint8_t* dst = which ? a.pool.v_at(page, hk, s) : a.pool.k_at(page, hk, s);
    if constexpr (sizeof(CT) == 1) {
      float f[kE], m = 0.f;
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        f[i] = __uint_as_float(i & 1 ? t[i / 2] & 0xFFFF0000u : t[i / 2] << 16);
        m = fmaxf(m, fabsf(f[i]));
      }
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      const int e = fp8_row_exponent(m);
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < kE; ++i) w[i / 4] |= uint32_t(fp8_code(f[i], e)) << (8 * (i % 4));
      reinterpret_cast<u32x2*>(dst)[c] = u32x2{w[0], w[1]};
      if (c == 0) (which ? a.pool.v_exp : a.pool.k_exp)[at] = int8_t(e);
    } else {
      reinterpret_cast<u32x4*>(dst)[c] = t;
    }
  }
  if (c == 0) {
    if (a.pool.score) a.pool.score[at] = a.scores ? a.scores[int64_t(bh) * a.n + j] : 0.f;
    if (a.pool.pos) a.pool.pos[at] = j;
  }
}

struct EvictArgs {
  PagePool pool;
  const int32_t* lens;
  int32_t* moves;  // [B][Hkv][2][most] entries below the budget that are given up, kept entries behind it, rising
  int32_t* count;  // [B][Hkv] pairs
  int32_t max_len, budget, recent, n_sink, most;
};

__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a) {
  __shared__ int hist[256], wa[16], sh[2];
  const int bh = blockIdx.x, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv, tid = threadIdx.x;
  const int n = min(a.lens[b], a.max_len), S = a.budget;
  if (n <= S) {
    if (tid == 0) a.count[bh] = 0;
    return;
  }
  int newest = INT32_MIN;
  for (int j = tid; j < n; j += kSelThreads) {
    const int page = a.pool.page_of(b, j);
    if (page >= 0) newest = max(newest, a.pool.pos[a.pool.at(page, hk, j)]);
  }
  newest = -wave_min(newest == INT32_MIN ? INT32_MAX : -newest);
  if ((tid & 63) == 0) wa[tid >> 6] = newest;
  __syncthreads();
  for (int i = 0; i < 16; ++i) newest = max(newest, wa[i]);
  __syncthreads();
  const int64_t late = int64_t(newest) - a.recent;
  // protected entries first, then by score, then by position; entries without a page last
  auto key = [&](int j) -> uint64_t {
    const int page = a.pool.page_of(b, j);
    if (page < 0) return 0;
    const int64_t at = a.pool.at(page, hk, j);
    const int32_t p = a.pool.pos[at];
    const uint32_t hi = p < a.n_sink || p > late ? 0xFFFFFFFFu : score_key(a.pool.score[at]);
    return uint64_t(hi) << 32 | ~(uint32_t(p) ^ 0x80000000u);
  };
  uint64_t value;
  int equal;
  nth_largest<uint64_t>(n, S, key, value, equal, hist, sh);
  int32_t* hole = a.moves + int64_t(bh) * 2 * a.most;
  int32_t* from = hole + a.most;
  int holes = 0, rows = 0, same = 0;
  for (int j0 = 0; j0 < n; j0 += kSelThreads) {
    const int j = j0 + tid;
    const uint64_t k = j < n ? key(j) : 0u;
    const bool eq = j < n && k == value;
    int before, total;
    block_scan(eq, before, total, wa);
    const bool keep = j < n && (k > value || (eq && same + before < equal));
    same += total;
    const bool is_hole = j < S && !keep && a.pool.page_of(b, j) >= 0, is_row = j >= S && keep && k != 0;
    block_scan(is_hole, before, total, wa);
    if (is_hole && holes + before < a.most) hole[holes + before] = j;
    holes += total;
    block_scan(is_row, before, total, wa);
    if (is_row && rows + before < a.most) from[rows + before] = j;
    rows += total;
  }
  if (tid == 0) a.count[bh] = min(min(holes, rows), a.most);
}

// Kept rows into the holes: sources lie at or behind the budget, targets below it.
template <int ROW>  // bytes of a row
__global__ __launch_bounds__(256) void evict_move(EvictArgs a) {
  constexpr int kLanes = ROW / 16, kRows = 256 / kLanes;
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv;
  const int i = blockIdx.x * kRows + threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  if (i >= a.count[bh]) return;
  const int32_t* hole = a.moves + int64_t(bh) * 2 * a.most;
  const int to = hole[i], from = hole[a.most + i];
  const int pt = a.pool.page_of(b, to), pf = a.pool.page_of(b, from);
  if (pt < 0 || pf < 0) return;
  const u32x4 k = reinterpret_cast<const u32x4*>(a.pool.k_at(pf, hk, from))[c];
  const u32x4 v = reinterpret_cast<const u32x4*>(a.pool.v_at(pf, hk, from))[c];
  reinterpret_cast<u32x4*>(a.pool.k_at(pt, hk, to))[c] = k;
  reinterpret_cast<u32x4*>(a.pool.v_at(pt, hk, to))[c] = v;
  if (c == 0) {
    const int64_t t = a.pool.at(pt, hk, to), f = a.pool.at(pf, hk, from);
    a.pool.score[t] = a.pool.score[f];
    a.pool.pos[t] = a.pool.pos[f];
    if (a.pool.k_exp) {
      a.pool.k_exp[t] = a.pool.k_exp[f];
      a.pool.v_exp[t] = a.pool.v_exp[f];
    }
  }
}

}  // namespace

size_t pages_evict_bytes(const d2o_pages* p, int32_t max_len) {
  const size_t bh = size_t(p->batch) * p->n_kv_heads;
  return round256(bh * 2 * max_len * sizeof(int32_t)) + round256(bh * sizeof(int32_t));
}

}  // namespace d2o

using namespace d2o;

extern "C" int d2o_pages_fill(const d2o_pages* pages, d2o_view K, d2o_view V, int32_t n, const int32_t* lens,
                              const float* scores, int32_t budget, int32_t recent, int32_t n_sink, void* workspace,
                              size_t workspace_bytes, void* stream) {
  FillArgs a;
  const int rc = check_pages(pages, &a.pool);
  if (rc != D2O_OK) return rc;
  const int es = pages->dtype == D2O_BF16 ? 2 : 4, D = pages->head_dim;
  if (n < 1 || budget < 1 || recent < 0 || n_sink < 0 || int64_t(recent) + n_sink > budget) return D2O_ERR_INVALID_ARG;
  if (!scores && budget < n) return D2O_ERR_INVALID_ARG;
  if (!dense_view_ok(K, es, true) || !dense_view_ok(V, es, true)) return D2O_ERR_INVALID_ARG;
  const int most = std::min(n, budget);
  if (most > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < pages_evict_bytes(pages, n)) return D2O_ERR_CAPACITY;
  const int64_t bh = int64_t(pages->batch) * pages->n_kv_heads;
  if (bh > 65535) return D2O_ERR_UNSUPPORTED;
  a.k = to_view(K);
  a.v = to_view(V);
  a.lens = lens;
  a.scores = scores;
  a.src = static_cast<int32_t*>(workspace);
  a.n = n;
  a.budget = std::min(budget, n);
  a.recent = recent;
  a.n_sink = n_sink;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (budget < n) fill_select<<<dim3(unsigned(bh)), kSelThreads, 0, s>>>(a);
  auto rows = [&](auto kernel, int per) { kernel<<<dim3((most + per - 1) / per, unsigned(bh)), 256, 0, s>>>(a); };
  if (pages->cache_fp8)
    D == 64 ? rows(fill_rows<uint16_t, uint8_t, 64>, 32) : rows(fill_rows<uint16_t, uint8_t, 128>, 16);
  else if (pages->dtype == D2O_BF16)
    D == 64 ? rows(fill_rows<uint16_t, uint16_t, 64>, 32) : rows(fill_rows<uint16_t, uint16_t, 128>, 16);
  else
    D == 64 ? rows(fill_rows<float, float, 64>, 16) : rows(fill_rows<float, float, 128>, 8);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}

extern "C" int d2o_pages_evict(const d2o_pages* pages, const int32_t* lens, int32_t max_len, int32_t budget,
                               int32_t recent, int32_t n_sink, void* workspace, size_t workspace_bytes, void* stream) {
  EvictArgs a;
  const int rc = check_pages(pages, &a.pool);
  if (rc != D2O_OK) return rc;
  if (!lens || !pages->score || !pages->pos || max_len < 1) return D2O_ERR_INVALID_ARG;
  if (budget < 1 || recent < 0 || n_sink < 0 || int64_t(recent) + n_sink > budget) return D2O_ERR_INVALID_ARG;
  if (max_len > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < pages_evict_bytes(pages, max_len)) return D2O_ERR_CAPACITY;
  const int64_t bh = int64_t(pages->batch) * pages->n_kv_heads;
  if (bh > 65535) return D2O_ERR_UNSUPPORTED;
  if (max_len <= budget) return D2O_OK;  // no sequence can have more than it keeps
  a.lens = lens;
  a.max_len = max_len;
  a.budget = budget;
  a.recent = recent;
  a.n_sink = n_sink;
  a.most = std::min(budget, max_len - budget);
  a.moves = static_cast<int32_t*>(workspace);
  a.count = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + round256(size_t(bh) * 2 * max_len * sizeof(int32_t)));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  evict_select<<<dim3(unsigned(bh)), kSelThreads, 0, s>>>(a);
  const int row = pages->head_dim * (pages->cache_fp8 ? 1 : pages->dtype == D2O_BF16 ? 2 : 4);
  auto move = [&](auto kernel) {
    const int per = 256 / (row / 16);
    kernel<<<dim3((a.most + per - 1) / per, unsigned(bh)), 256, 0, s>>>(a);
  };
  switch (row) {
    case 64: move(evict_move<64>); break;
    case 128: move(evict_move<128>); break;
    case 256: move(evict_move<256>); break;
    default: move(evict_move<512>); break;
  }
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
