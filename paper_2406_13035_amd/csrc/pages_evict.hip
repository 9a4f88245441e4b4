// Eviction by accumulated attention over caches in pages: prompts into pages (d2o_pages_fill) and a cache that has outgrown
// its budget back to it, in place (d2o_pages_evict).  Both choose by Eq. 7-8: the first tokens, the last ones, and the
// highest scores among the others.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace d2o {
namespace {

// Order-preserving integer of a score: larger keys are kept first.  0 is below every score, kProtected above.
constexpr uint32_t kProtected = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t score_key(float x) {
  if (x != x) return 0xFFFFFFFEu;
  if (x == 0.f) x = 0.f;  // -0 and +0 compare equal
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// ---- selection of one head by one workgroup.  Radix select from the top: a histogram of 2048 bins of the candidates' next eleven
// bits, then the bin in which the count from above reaches what is still wanted.  (Eleven bits: sign, exponent and two bits of the
// fraction spread accumulated attention over a few dozen bins, so that the lanes of a wavefront seldom meet in one; with eight, the
// exponent alone, they queue.)
constexpr int kBins = 2048;

struct SelectShared {
  int hist[kBins];
  int wave[16];
  int bin, left, above;
};

// One digit: of the n candidates counted into sh.hist, the bin that holds the `want`-th largest (1-based), and how many are wanted of
// that bin.  All threads; sh.hist is free again when it returns.
template <int NT>
__device__ __forceinline__ void pick_bin(SelectShared& sh, int want) {
  constexpr int kPer = kBins / NT;  // bins per thread, from the top: thread 0 has the largest
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  __syncthreads();
  int h[kPer], tot = 0;
#pragma unroll
  for (int u = 0; u < kPer; ++u) tot += h[u] = sh.hist[kBins - 1 - tid * kPer - u];
  int inc = tot;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(inc, o, 64);
    if (lane >= o) inc += t;
  }
  if (lane == 63) sh.wave[w] = inc;
  __syncthreads();
  for (int i = 0; i < w; ++i) inc += sh.wave[i];
  int left = want - (inc - tot);
  if (left > 0 && want <= inc) {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      if (left > 0 && h[u] >= left) {
        sh.bin = kBins - 1 - tid * kPer - u;
        sh.left = left;
        sh.above = h[u];
        left = 0;
      }
      left -= h[u];
    }
  }
  __syncthreads();
}
template <int NT>
__device__ __forceinline__ void clear_bins(SelectShared& sh) {
  for (int i = threadIdx.x; i < kBins; i += NT) sh.hist[i] = 0;
  __syncthreads();
}

// One of a bin for every active lane; lanes that all have the same bin (scores that are all zero, or equal) add once.
__device__ __forceinline__ void count_bin(int* hist, int bin) {
  const int first = __builtin_amdgcn_readfirstlane(bin);
  const uint64_t all = __ballot(true);
  if (__ballot(bin == first) != all)
    atomicAdd(&hist[bin], 1);
  else if (__builtin_amdgcn_mbcnt_hi(uint32_t(all >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(all), 0)) == 0)
    atomicAdd(&hist[bin], __popcll(all));
}

// The `want`-th largest of the 32-bit values that `each_value(f)` hands to f(value) on all threads together; `equal` becomes how many of
// those equal to it are wanted, `same` how many there are.  FIRST = 1: values of 21 bits.
template <int NT, int FIRST = 0, typename F>
__device__ __forceinline__ uint32_t nth_largest(SelectShared& sh, int want, int& equal, int& same, const F& each_value) {
  uint32_t prefix = 0;
#pragma unroll
  for (int pass = FIRST; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digit = pass == 2 ? 1023u : 2047u;
    clear_bins<NT>(sh);
    each_value([&](uint32_t v) {
      const bool in = pass == 0 || (v >> (pass == 1 ? 21 : 10)) == (prefix >> (pass == 1 ? 21 : 10));
      if (in) count_bin(sh.hist, int((v >> shift) & digit));
    });
    pick_bin<NT>(sh, want);
    prefix |= uint32_t(sh.bin) << shift;
    want = sh.left;
    same = sh.above;
  }
  __syncthreads();
  equal = want;
  return prefix;
}

// Ranks in entry order for entries u * NT + thread: counts of two predicates per (u, wavefront) in `cnt` (16 bits each, at most 65535
// entries), turned into the counts before.
template <int NT, int PT>
__device__ __forceinline__ void prefix_counts(uint32_t* cnt) {
  constexpr int kN = PT * (NT / 64), kPer = (kN + 63) / 64;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    uint32_t v[kPer], tot = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      v[i] = lane * kPer + i < kN ? cnt[lane * kPer + i] : 0;
      tot += v[i];
    }
    uint32_t inc = tot;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t t = __shfl_up(int(inc), o, 64);
      if (lane >= o) inc += t;
    }
    uint32_t run = inc - tot;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (lane * kPer + i < kN) cnt[lane * kPer + i] = run;
      run += v[i];
    }
    if (lane == 63) cnt[kN] = run;
  }
  __syncthreads();
}
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

struct FillArgs {
  PagePool pool;
  View k, v;
  const int32_t* lens;
  const float* scores;
  int32_t* src;    // [B][Hkv][budget] kept positions, rising (where some are evicted)
  // longer prompts, by slices:
  uint16_t* hist;  // [B][Hkv][slices][kBins] of a slice's keys
  uint32_t* cand;  // [B][Hkv][n] the tokens in the threshold's bin: slice and lower 21 bits of the key, slice by slice in any order
  int32_t* above;  // [B][Hkv][slices] keys above that bin
  int32_t* head;   // [B][Hkv][4] candidates, the bin, how many of it are kept
  int32_t n, budget, recent, n_sink, slices;

  __device__ __forceinline__ int length(int b) const { return lens ? min(max(lens[b], 0), n) : n; }
  // keys of tokens j0, j0 + step, ..: all loads on their way before the first is used (tokens behind the last: key 0)
  template <int N>
  __device__ __forceinline__ void keys(const float* sc, int len, int j0, int step, uint32_t* key) const {
    float x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = sc[min(j0 + u * step, len - 1)];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int j = j0 + u * step;
      key[u] = j >= len ? 0 : j < n_sink || j >= len - recent ? kProtected : score_key(x[u]);
    }
  }
};
constexpr int kFillSelect = 16384;  // tokens of a prompt that one workgroup holds in registers

// Prompts of at most NT * PT tokens: keys in registers, the kept positions to a list.
template <int NT, int PT>
__global__ __launch_bounds__(NT) void fill_select(FillArgs a) {
  __shared__ SelectShared sh;
  __shared__ uint32_t cnt[PT * (NT / 64) + 1];
  const int bh = blockIdx.x, b = bh / a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = a.length(b);
  if (n <= a.budget) return;
  const float* sc = a.scores + int64_t(bh) * a.n;
  uint32_t key[PT];
  a.keys<PT>(sc, n, tid, NT, key);
  // among those that are not protected (these share one key, at whose bin thousands would queue): n_sink + recent are
  int equal = a.n_sink + a.recent, same;
  uint32_t t = kProtected;
  if (a.budget > equal)
    t = nth_largest<NT>(sh, a.budget - equal, equal, same, [&](auto f) {
#pragma unroll
      for (int u = 0; u < PT; ++u)
        if (u * NT + tid < n && key[u] != kProtected) f(key[u]);
    });
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const uint32_t c = uint32_t(__popcll(__ballot(key[u] > t))) | uint32_t(__popcll(__ballot(key[u] == t))) << 16;
    if (lane == 0) cnt[u * (NT / 64) + w] = c;
  }
  prefix_counts<NT, PT>(cnt);
  int32_t* src = a.src + int64_t(bh) * a.budget;
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const uint32_t c = cnt[u * (NT / 64) + w];
    const bool gt = key[u] > t, eq = key[u] == t;
    const int above = int(c & 0xFFFF) + lanes_before(__ballot(gt)), rank = int(c >> 16) + lanes_before(__ballot(eq));
    if (gt || (eq && rank < equal)) src[above + min(rank, equal)] = u * NT + tid;
  }
}

// Longer prompts, in slices of kSlice tokens.  First a histogram of every slice's top digits ...
constexpr int kSlice = 4096, kSliceThreads = 256, kSlicePer = kSlice / kSliceThreads;
__global__ __launch_bounds__(kSliceThreads) void fill_hist(FillArgs a) {
  __shared__ int hist[kBins];
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, tid = threadIdx.x, j0 = blockIdx.x * kSlice;
  const int n = a.length(b);
  if (n <= a.budget || j0 >= n) return;
  const float* sc = a.scores + int64_t(bh) * a.n;
  uint32_t key[kSlicePer];
  a.keys<kSlicePer>(sc, n, j0 + tid, kSliceThreads, key);
  for (int i = tid; i < kBins; i += kSliceThreads) hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u)
    if (j0 + u * kSliceThreads + tid < n) count_bin(hist, int(key[u] >> 21));
  __syncthreads();
  uint32_t* out = reinterpret_cast<uint32_t*>(a.hist + (int64_t(bh) * a.slices + blockIdx.x) * kBins);
  for (int i = tid; i < kBins / 2; i += kSliceThreads) out[i] = uint32_t(hist[2 * i]) | uint32_t(hist[2 * i + 1]) << 16;
  if (blockIdx.x == 0 && tid == 0) a.head[bh * 4] = 0;
}

// ... then the bin that holds the threshold (found by every slice for itself from all histograms: a workgroup that did it for
// the head, and then read all its scores, took 48 us at 131072 tokens), and the tokens in it to the head's list ...
constexpr int kMaxSlices = 2048;
__global__ __launch_bounds__(kSliceThreads) void fill_candidates(FillArgs a) {
  __shared__ SelectShared sh;
  __shared__ uint32_t cnt[kSlicePer * (kSliceThreads / 64) + 1];
  __shared__ int at;
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, j0 = blockIdx.x * kSlice;
  const int n = a.length(b);
  if (n <= a.budget || j0 >= n) return;
  uint32_t key[kSlicePer];
  a.keys<kSlicePer>(a.scores + int64_t(bh) * a.n, n, j0 + tid, kSliceThreads, key);
  const int slices = (n + kSlice - 1) / kSlice;
  constexpr int kWords = kBins / 2 / kSliceThreads;  // pairs of bins per thread
  static_assert(kWords == 4, "a load of 16 bytes");
  const u32x4* hist = reinterpret_cast<const u32x4*>(a.hist + int64_t(bh) * a.slices * kBins) + tid;
  int sum[2 * kWords] = {};
#pragma unroll 8
  for (int s = 0; s < slices; ++s) {
    const u32x4 v = hist[int64_t(s) * (kBins / 8)];
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      sum[2 * i] += v[i] & 0xFFFF;
      sum[2 * i + 1] += v[i] >> 16;
    }
  }
#pragma unroll
  for (int i = 0; i < 2 * kWords; ++i) sh.hist[tid * 2 * kWords + i] = sum[i];
  pick_bin<kSliceThreads>(sh, a.budget);
  const uint32_t top = sh.bin;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const bool in = j0 + u * kSliceThreads + tid < n;
    const uint32_t v = uint32_t(__popcll(__ballot(in && key[u] >> 21 > top))) | uint32_t(__popcll(__ballot(in && key[u] >> 21 == top))) << 16;
    if (lane == 0) cnt[u * (kSliceThreads / 64) + w] = v;
  }
  prefix_counts<kSliceThreads, kSlicePer>(cnt);
  const uint32_t all = cnt[kSlicePer * (kSliceThreads / 64)];
  if (tid == 0) {
    a.above[int64_t(bh) * a.slices + blockIdx.x] = int(all & 0xFFFF);
    at = atomicAdd(&a.head[bh * 4], int(all >> 16));
    if (blockIdx.x == 0) {
      a.head[bh * 4 + 1] = int(top);
      a.head[bh * 4 + 2] = sh.left;
    }
  }
  __syncthreads();
  uint32_t* cand = a.cand + int64_t(bh) * a.n + at;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const bool is = j0 + u * kSliceThreads + tid < n && key[u] >> 21 == top;
    const uint64_t m = __ballot(is);
    if (is) cand[int(cnt[u * (kSliceThreads / 64) + w] >> 16) + lanes_before(m)] = (key[u] & 0x1FFFFF) | uint32_t(blockIdx.x) << 21;
  }
}

// ... and every slice finds the threshold among the candidates, counts what the slices before it keep, and lists its kept positions
// behind those.  (Their rows are copied by a launch of their own: the slice with the recent tokens has more than all others.)
constexpr int kCand = 8192;  // candidates held in LDS
__global__ __launch_bounds__(kSliceThreads) void fill_list(FillArgs a) {
  __shared__ SelectShared sh;
  __shared__ uint32_t held[kCand];
  __shared__ uint32_t cnt[kSlicePer * (kSliceThreads / 64) + 1];
  __shared__ int before[2];
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = a.length(b), j0 = blockIdx.x * kSlice, me = blockIdx.x;
  if (n <= a.budget || j0 >= n) return;
  uint32_t key[kSlicePer];
  a.keys<kSlicePer>(a.scores + int64_t(bh) * a.n, n, j0 + tid, kSliceThreads, key);
  const int total = a.head[bh * 4];
  const uint32_t top = a.head[bh * 4 + 1];
  const uint32_t* list = a.cand + int64_t(bh) * a.n;
  const bool fits = total <= kCand;
  if (fits)
    for (int i = tid; i < total; i += kSliceThreads) held[i] = list[i];
  if (tid < 2) before[tid] = 0;
  __syncthreads();
  auto each_candidate = [&](auto f) {
    if (fits) {
      for (int i = tid; i < total; i += kSliceThreads) f(held[i]);
    } else {
#pragma unroll 8
      for (int i = tid; i < total; i += kSliceThreads) f(list[i]);
    }
  };
  int equal, same;
  const uint32_t low = nth_largest<kSliceThreads, 1>(sh, a.head[bh * 4 + 2], equal, same,
                                                     [&](auto f) { each_candidate([&](uint32_t v) { f(v & 0x1FFFFF); }); });
  int gt0 = 0, eq0 = 0;  // kept by the slices before: above the threshold, level with it
  for (int s = tid; s < me; s += kSliceThreads) gt0 += a.above[int64_t(bh) * a.slices + s];
  each_candidate([&](uint32_t v) {
    if (int(v >> 21) < me) {
      gt0 += (v & 0x1FFFFF) > low;
      eq0 += (v & 0x1FFFFF) == low;
    }
  });
  if (gt0) atomicAdd(&before[0], gt0);
  if (eq0) atomicAdd(&before[1], eq0);
  const uint32_t t = top << 21 | low;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const uint32_t v = uint32_t(__popcll(__ballot(key[u] > t))) | uint32_t(__popcll(__ballot(key[u] == t))) << 16;
    if (lane == 0) cnt[u * (kSliceThreads / 64) + w] = v;
  }
  prefix_counts<kSliceThreads, kSlicePer>(cnt);
  gt0 = before[0];
  eq0 = before[1];
  const int quota = max(0, equal - eq0);  // of the equal ones of this slice
  int32_t* src = a.src + int64_t(bh) * a.budget + gt0 + min(eq0, equal);
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const uint32_t v = cnt[u * (kSliceThreads / 64) + w];
    const bool gt = key[u] > t, eq = key[u] == t;
    const int above = int(v & 0xFFFF) + lanes_before(__ballot(gt)), rank = int(v >> 16) + lanes_before(__ballot(eq));
    if (gt || (eq && rank < quota)) src[above + min(rank, quota)] = j0 + u * kSliceThreads + tid;
  }
}

// Token j of the prompt to entry s: 16 bytes of the row per lane, consecutive lanes consecutive chunks.  PAST: read past the caches.
template <typename T, typename CT, int D, bool PAST>
__device__ __forceinline__ void put_row(const FillArgs& a, int bh, int b, int hk, int s, int j, int c) {
  constexpr int kLanes = D * int(sizeof(T)) / 16, kE = 16 / int(sizeof(T));
  const int page = a.pool.page_of(b, s);
  if (page < 0) return;
  const int64_t at = a.pool.at(page, hk, s);
  u32x4 t[2];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const View& x = which ? a.v : a.k;
    const u32x4* row = reinterpret_cast<const u32x4*>(static_cast<const T*>(x.ptr) + b * x.sb + hk * x.sh + int64_t(j) * x.sn) + c;
    if constexpr (PAST)
      t[which] = __builtin_nontemporal_load(row);
    else
      t[which] = *row;
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    uint8_t* dst = which ? a.pool.v_at(page, hk, s) : a.pool.k_at(page, hk, s);
    if constexpr (sizeof(CT) == 1) {
      float f[kE], m = 0.f;
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        f[i] = __uint_as_float(i & 1 ? t[which][i / 2] & 0xFFFF0000u : t[which][i / 2] << 16);
        m = fmaxf(m, fp8_magnitude(f[i]));
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
      reinterpret_cast<u32x4*>(dst)[c] = t[which];
    }
  }
  if (c == 0) {
    if (a.pool.score) a.pool.score[at] = a.scores ? a.scores[int64_t(bh) * a.n + j] : 0.f;
    if (a.pool.pos) a.pool.pos[at] = j;
  }
}

template <typename T, typename CT, int D, bool PAST>
__global__ __launch_bounds__(256) void fill_rows(FillArgs a) {
  constexpr int kLanes = D * int(sizeof(T)) / 16, kRows = 256 / kLanes;
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv;
  const int n = a.length(b);
  const int s = blockIdx.x * kRows + threadIdx.x / kLanes;
  if (s >= min(n, a.budget)) return;
  put_row<T, CT, D, PAST>(a, bh, b, hk, s, n <= a.budget ? s : a.src[int64_t(bh) * a.budget + s], threadIdx.x % kLanes);
}

struct EvictArgs {
  PagePool pool;
  const int32_t* lens;
  int32_t* moves;  // [B][Hkv][2][most] entries below the budget that are given up, kept entries behind it, rising
  int32_t* count;  // [B][Hkv] pairs
  // long caches, by slices:
  int32_t* newest;   // [B][Hkv][slices] largest position of a slice
  int32_t* guarded;  // [B][Hkv][slices] its protected entries
  uint32_t* cand;    // [B][Hkv][slices * extra][3] its lowest entries, as many as the sequence gives up: score's key, position's, entry | protected << 31
  int32_t max_len, budget, recent, n_sink, most, slices, extra;
};
constexpr int kInline = 512;  // moves of a head that the workgroup which chose them makes itself (256 rows of 32 heads: 15.7 us,
                              // in a launch of their own 18)

// Kept rows into holes, `lanes` lanes of 16 bytes per row: pairs i0, i0 + step, .. below `pairs`, a few at a time on their way.  Sources lie
// at or behind the budget, targets below it: moves never meet.
template <int N>
__device__ __forceinline__ void move_rows(const EvictArgs& a, int b, int hk, const int32_t* from, const int32_t* hole, int i0, int step,
                                          int pairs, int c) {
  for (int i = i0; i < pairs; i += N * step) {
    u32x4 k[N], v[N];
    float score[N];
    int32_t pos[N], to[N], pt[N];
    int8_t ke[N], ve[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const bool is = i + u * step < pairs;
      const int src = is ? from[i + u * step] : 0;
      to[u] = is ? hole[i + u * step] : 0;
      pt[u] = is ? a.pool.page_of(b, to[u]) : -1;
      const int pf = is ? a.pool.page_of(b, src) : -1;
      if (pf < 0) pt[u] = -1;
      const int page = max(pf, 0);
      const int64_t at = a.pool.at(page, hk, src);
      k[u] = reinterpret_cast<const u32x4*>(a.pool.k_at(page, hk, src))[c];
      v[u] = reinterpret_cast<const u32x4*>(a.pool.v_at(page, hk, src))[c];
      score[u] = a.pool.score[at];
      pos[u] = a.pool.pos[at];
      ke[u] = a.pool.k_exp ? a.pool.k_exp[at] : 0;
      ve[u] = a.pool.k_exp ? a.pool.v_exp[at] : 0;
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (pt[u] < 0) continue;
      reinterpret_cast<u32x4*>(a.pool.k_at(pt[u], hk, to[u]))[c] = k[u];
      reinterpret_cast<u32x4*>(a.pool.v_at(pt[u], hk, to[u]))[c] = v[u];
      if (c == 0) {
        const int64_t at = a.pool.at(pt[u], hk, to[u]);
        a.pool.score[at] = score[u];
        a.pool.pos[at] = pos[u];
        if (a.pool.k_exp) {
          a.pool.k_exp[at] = ke[u];
          a.pool.v_exp[at] = ve[u];
        }
      }
    }
  }
}

// What decides about an entry: protected ones first, then by score, then by position; without a page last.  `crowded`: more are protected than
// stay (positions that occur more than once): these go by score too, and the others are below all of them.
struct Rank {
  uint32_t key, low;
};
__device__ __forceinline__ bool is_guarded(const EvictArgs& a, int32_t p, int64_t late) { return p < a.n_sink || p > late; }
__device__ __forceinline__ Rank rank_of(const EvictArgs& a, float score, int32_t p, int64_t late, bool crowded) {
  const bool guarded = is_guarded(a, p, late);
  const uint32_t k = score_key(score);
  return {crowded ? (guarded ? k : 1u) : (guarded ? kProtected : k), ~(uint32_t(p) ^ 0x80000000u)};
}
template <int NT>
__device__ __forceinline__ int block_total(int v, int* buf) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < NT / 64; ++i) v += buf[i];
  __syncthreads();
  return v;
}
template <int NT>
__device__ __forceinline__ int block_max(int v, int* buf) {
  v = -wave_min(-max(v, -INT32_MAX));
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int i = 0; i < NT / 64; ++i) v = max(v, buf[i]);
  __syncthreads();
  return v;
}

// The lowest of the entries that each_rank(f) hands to f(entry, rank) on all threads together; of equals the last.
struct Lowest {
  uint32_t key, low;
  int at;
  __device__ __forceinline__ void take(uint32_t k, uint32_t l, int j) {
    if (k < key || (k == key && (l < low || (l == low && j > at)))) key = k, low = l, at = j;
  }
};
template <int NT, typename F>
__device__ __forceinline__ Lowest lowest_entry(SelectShared& sh, const F& each_rank) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Lowest x{0xFFFFFFFFu, 0xFFFFFFFFu, -1};
  each_rank([&](int j, const Rank& r) __attribute__((always_inline)) { x.take(r.key, r.low, j); });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    x.take(uint32_t(__shfl_xor(int(x.key), o, 64)), uint32_t(__shfl_xor(int(x.low), o, 64)), __shfl_xor(x.at, o, 64));
  if (lane == 0) {
    sh.hist[w] = int(x.key);
    sh.hist[16 + w] = int(x.low);
    sh.hist[32 + w] = x.at;
  }
  __syncthreads();
  for (int i = 0; i < NT / 64; ++i) x.take(uint32_t(sh.hist[i]), uint32_t(sh.hist[16 + i]), sh.hist[32 + i]);
  __syncthreads();
  return x;
}

// Which of the entries that each_rank(f) hands to f(entry, rank) are the `keep` highest; `guarded` of them have the key kProtected.
// few: LDS of kFew words.
struct Threshold {
  uint32_t t, tl;
  int ts;
  __device__ __forceinline__ bool stays(const Rank& x, int j) const { return x.key > t || (x.key == t && (x.low > tl || (x.low == tl && j <= ts))); }
};
constexpr int kFew = 256;
template <int NT, typename F>
__device__ __forceinline__ Threshold threshold(SelectShared& sh, uint64_t* few, int keep, int guarded, const F& each_rank) {
  static_assert(kFew <= NT, "a thread each");
  const int tid = threadIdx.x;
  // among the entries that are not protected (which share one key, at whose bin thousands would queue)
  int equal = keep, same = guarded;
  uint32_t t = kProtected;
  if (guarded != keep)
    t = nth_largest<NT>(sh, keep - guarded, equal, same, [&](auto f) __attribute__((always_inline)) {
      each_rank([&](int, const Rank& x) {
        if (x.key != kProtected) f(x.key);
      });
    });
  // Of several entries with the threshold's key only some stay: those with the lowest positions, of equal positions the first entries; (tl, ts)
  // are the last one's.  A few are ranked against each other, many selected digit by digit.
  uint32_t tl = 0;
  int ts = INT32_MAX;
  if (equal < same && same <= kFew) {
    if (tid == 0) sh.bin = 0;
    __syncthreads();
    each_rank([&](int j, const Rank& x) {
      if (x.key == t) few[atomicAdd(&sh.bin, 1)] = uint64_t(x.low) << 32 | ~uint32_t(j);  // larger: kept before
    });
    __syncthreads();
    if (tid < same) {
      const uint64_t mine = few[tid];
      int before = 0;
#pragma unroll 8
      for (int i = 0; i < same; ++i) before += few[i] > mine;
      if (before == equal - 1) {
        sh.left = int(mine >> 32);
        sh.above = int(~uint32_t(mine));
      }
    }
    __syncthreads();
    tl = sh.left;
    ts = sh.above;
  } else if (equal < same) {
    tl = nth_largest<NT>(sh, equal, equal, same, [&](auto f) __attribute__((always_inline)) {
      each_rank([&](int, const Rank& x) {
        if (x.key == t) f(x.low);
      });
    });
    if (equal < same)
      ts = ~int(nth_largest<NT>(sh, equal, equal, same, [&](auto f) __attribute__((always_inline)) {
        each_rank([&](int j, const Rank& x) {
          if (x.key == t && x.low == tl) f(~uint32_t(j));
        });
      }));
  }
  return {t, tl, ts};
}

// One workgroup per head, entries u * NT + thread: in registers (PT of them per thread) or, PT = 0, read again for every use.
template <int NT, int PT>
__global__ __launch_bounds__(NT) void evict_select(EvictArgs a, int lanes) {
  __shared__ SelectShared sh;
  __shared__ uint32_t cnt[(PT ? PT : 16) * (NT / 64) + 1];
  __shared__ __attribute__((aligned(8))) int lists[2 * kInline];
  const int bh = blockIdx.x, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = min(a.lens[b], a.max_len), S = a.budget;
  const bool here = a.most <= kInline;
  if (n <= S) {
    if (tid == 0 && !here) a.count[bh] = 0;
    return;
  }
  constexpr int kKeep = PT ? PT : 1;
  float score[kKeep];
  int32_t pos[kKeep];
  uint32_t present = 0;  // bit u
  int newest = -INT32_MAX;
  // score and position of entry j, false where it has no page or is none (then of the pool's first row)
  auto look = [&](int j, float& sc, int32_t& p) __attribute__((always_inline)) {
    const int page = a.pool.page_of(b, min(j, n - 1));
    const bool there = j < n && page >= 0;
    const int64_t at = there ? a.pool.at(page, hk, j) : 0;
    sc = a.pool.score[at];
    p = a.pool.pos[at];
    return there;
  };
  if constexpr (PT > 0) {
    int page[kKeep];
#pragma unroll
    for (int u = 0; u < PT; ++u) page[u] = a.pool.page_of(b, min(u * NT + tid, n - 1));
#pragma unroll
    for (int u = 0; u < PT; ++u) {
      const bool there = u * NT + tid < n && page[u] >= 0;
      const int64_t at = there ? a.pool.at(page[u], hk, u * NT + tid) : 0;
      score[u] = a.pool.score[at];
      pos[u] = a.pool.pos[at];
      present |= uint32_t(there) << u;
    }
#pragma unroll
    for (int u = 0; u < PT; ++u)
      if (present >> u & 1) newest = max(newest, pos[u]);
  } else {
#pragma unroll 4
    for (int j = tid; j < n; j += NT) {
      float sc;
      int32_t p;
      if (look(j, sc, p)) newest = max(newest, p);
    }
  }
  newest = block_max<NT>(newest, sh.wave);
  const int64_t late = int64_t(newest) - a.recent;
  // the protected entries: more than stay?
  int guarded = 0;
  if constexpr (PT > 0) {
#pragma unroll
    for (int u = 0; u < PT; ++u) guarded += (present >> u & 1) && is_guarded(a, pos[u], late);
  } else {
#pragma unroll 4
    for (int j = tid; j < n; j += NT) {
      float sc;
      int32_t p;
      guarded += look(j, sc, p) && is_guarded(a, p, late);
    }
  }
  guarded = block_total<NT>(guarded, sh.wave);
  const bool crowded = guarded > S;
  Rank r[kKeep];
  if constexpr (PT > 0) {
#pragma unroll
    for (int u = 0; u < PT; ++u) {
      r[u] = rank_of(a, score[u], pos[u], late, crowded);
      if (!(present >> u & 1)) r[u] = {0, 0};
    }
  }
  auto rank_at = [&](int j) __attribute__((always_inline)) {
    float sc;
    int32_t p;
    return look(j, sc, p) ? rank_of(a, sc, p, late, crowded) : Rank{0, 0};
  };
  auto each_rank = [&](auto f) __attribute__((always_inline)) {  // f(entry, rank)
    if constexpr (PT > 0) {
#pragma unroll
      for (int u = 0; u < PT; ++u)
        if (u * NT + tid < n) f(u * NT + tid, r[u]);
    } else {
#pragma unroll 4
      for (int j = tid; j < n; j += NT) f(j, rank_at(j));
    }
  };

  if (n == S + 1) {  // one entry goes: the lowest, of equals the last
    const int at = lowest_entry<NT>(sh, each_rank).at;
    if (!here) {
      if (tid == 0) {
        int32_t* hole = a.moves + int64_t(bh) * 2 * a.most;
        hole[0] = at;
        hole[a.most] = S;
        a.count[bh] = at < S ? 1 : 0;
      }
    } else if (at < S && tid < lanes) {
      move_rows<1>(a, b, hk, &S, &at, 0, 1, 1, tid);  // (no move if either has no page)
    }
    return;
  }

  static_assert(2 * kFew <= 2 * kInline, "two words each");
  const Threshold kept = threshold<NT>(sh, reinterpret_cast<uint64_t*>(lists), S, crowded ? 0 : guarded, each_rank);
  int32_t *hole = lists, *from = lists + kInline;
  if (!here) {
    hole = a.moves + int64_t(bh) * 2 * a.most;
    from = hole + a.most;
  }
  constexpr int kU = PT ? PT : 16;  // rounds of NT entries ranked together
  int holes = 0, rows = 0;
  for (int j0 = 0; j0 < n; j0 += kU * NT) {
    Rank x[kU];
    uint32_t keep = 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int j = j0 + u * NT + tid;
      if constexpr (PT > 0)
        x[u] = r[u];
      else
        x[u] = rank_at(j);
      keep |= uint32_t(j < n && kept.stays(x[u], j)) << u;
    }
    __syncthreads();
    // holes below the budget and kept rows behind it
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int j = j0 + u * NT + tid;
      const bool there = x[u].key != 0, k = keep >> u & 1;
      const uint64_t mh = __ballot(j < n && j < S && !k && there), mr = __ballot(j < n && j >= S && k && there);
      if (lane == 0) cnt[u * (NT / 64) + w] = uint32_t(__popcll(mh)) | uint32_t(__popcll(mr)) << 16;
    }
    prefix_counts<NT, kU>(cnt);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int j = j0 + u * NT + tid;
      const bool there = x[u].key != 0, k = keep >> u & 1;
      const bool is_hole = j < n && j < S && !k && there, is_row = j < n && j >= S && k && there;
      const uint32_t c = cnt[u * (NT / 64) + w];
      const int ih = holes + int(c & 0xFFFF) + lanes_before(__ballot(is_hole)), ir = rows + int(c >> 16) + lanes_before(__ballot(is_row));
      if (is_hole && ih < a.most) hole[ih] = j;
      if (is_row && ir < a.most) from[ir] = j;
    }
    const uint32_t all = cnt[kU * (NT / 64)];
    holes += int(all & 0xFFFF);
    rows += int(all >> 16);
  }
  const int pairs = min(min(holes, rows), a.most);
  if (!here) {
    if (tid == 0) a.count[bh] = pairs;
    return;
  }
  __syncthreads();
  move_rows<4>(a, b, hk, from, hole, tid / lanes, NT / lanes, pairs, tid % lanes);
}

// The moves of heads that have many: `lanes` lanes of 16 bytes per row, again and again where a grid (below 2^32 threads) does not hold them.
__global__ __launch_bounds__(256) void evict_move(EvictArgs a, int lanes) {
  const int bh = blockIdx.y, per = 256 / lanes;
  const int32_t* hole = a.moves + int64_t(bh) * 2 * a.most;
  move_rows<1>(a, bh / a.pool.Hkv, bh % a.pool.Hkv, hole + a.most, hole, blockIdx.x * per + threadIdx.x / lanes, gridDim.x * per,
               a.count[bh], threadIdx.x % lanes);
}

// Caches that a workgroup does not hold in registers and that give up few entries, in slices of kSlice entries.  The entries that go are among
// the lowest of each slice, as many as go in all: the largest position of each slice, ...
__global__ __launch_bounds__(kSliceThreads) void evict_newest(EvictArgs a) {
  __shared__ int buf[kSliceThreads / 64];
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv, j0 = blockIdx.x * kSlice + threadIdx.x;
  const int n = min(a.lens[b], a.max_len);
  if (n <= a.budget || int(blockIdx.x) * kSlice >= n) return;
  int page[kSlicePer], pos[kSlicePer], newest = -INT32_MAX;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) page[u] = a.pool.page_of(b, min(j0 + u * kSliceThreads, n - 1));
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) pos[u] = a.pool.pos[page[u] >= 0 ? a.pool.at(page[u], hk, min(j0 + u * kSliceThreads, n - 1)) : 0];
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u)
    if (page[u] >= 0) newest = max(newest, pos[u]);
  newest = block_max<kSliceThreads>(newest, buf);
  if (threadIdx.x == 0) a.newest[int64_t(bh) * a.slices + blockIdx.x] = newest;
}

// ... the lowest entries of each slice in the order (protected, score, position, entry), which both orders of Rank agree with on what
// goes: protected entries that go at all go by score, and then every other entry goes ...
__global__ __launch_bounds__(kSliceThreads) void evict_lowest(EvictArgs a) {
  __shared__ SelectShared sh;
  __shared__ uint64_t few[kFew];
  __shared__ uint32_t cnt[kSlicePer * (kSliceThreads / 64) + 1];
  const int bh = blockIdx.y, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, j0 = blockIdx.x * kSlice;
  const int n = min(a.lens[b], a.max_len), have = min(kSlice, n - j0), goes = min(n - a.budget, have);
  if (n <= a.budget || j0 >= n) return;
  int page[kSlicePer], pos[kSlicePer], newest = -INT32_MAX;
  float score[kSlicePer];
  uint32_t present = 0, guard = 0;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) page[u] = a.pool.page_of(b, min(j0 + u * kSliceThreads + tid, n - 1));
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const int j = j0 + u * kSliceThreads + tid;
    const bool there = j < n && page[u] >= 0;
    const int64_t at = there ? a.pool.at(page[u], hk, j) : 0;
    score[u] = a.pool.score[at];
    pos[u] = a.pool.pos[at];
    present |= uint32_t(there) << u;
  }
  for (int i = tid; i * kSlice < n; i += kSliceThreads) newest = max(newest, a.newest[int64_t(bh) * a.slices + i]);
  const int64_t late = int64_t(block_max<kSliceThreads>(newest, sh.wave)) - a.recent;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) guard |= uint32_t((present >> u & 1) && is_guarded(a, pos[u], late)) << u;
  const int guarded = block_total<kSliceThreads>(__popc(guard), sh.wave);
  const bool crowded = have - guarded < goes;
  Rank r[kSlicePer];
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    r[u] = rank_of(a, score[u], pos[u], late, crowded);
    if (!(present >> u & 1)) r[u] = {0, 0};
  }
  auto each_rank = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kSlicePer; ++u)
      if (u * kSliceThreads + tid < have) f(u * kSliceThreads + tid, r[u]);
  };
  Threshold kept{0xFFFFFFFFu, 0xFFFFFFFFu, -1};  // none
  if (goes == 1) {
    const Lowest x = lowest_entry<kSliceThreads>(sh, each_rank);
    kept = {x.key, x.low, x.at - 1};
  } else if (goes < have) {
    kept = threshold<kSliceThreads>(sh, few, have - goes, crowded ? 0 : guarded, each_rank);
  }
  uint32_t gone = 0;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const int j = u * kSliceThreads + tid;
    gone |= uint32_t(j < have && !kept.stays(r[u], j)) << u;
    const uint64_t m = __ballot(gone >> u & 1);
    if (lane == 0) cnt[u * (kSliceThreads / 64) + w] = __popcll(m);
  }
  prefix_counts<kSliceThreads, kSlicePer>(cnt);
  uint32_t* out = a.cand + (int64_t(bh) * a.slices + blockIdx.x) * a.extra * 3;
#pragma unroll
  for (int u = 0; u < kSlicePer; ++u) {
    const bool is = gone >> u & 1;
    const int at = cnt[u * (kSliceThreads / 64) + w] + lanes_before(__ballot(is));
    if (is && at < a.extra) {
      const bool there = present >> u & 1;
      out[at * 3] = there ? score_key(score[u]) : 0;
      out[at * 3 + 1] = r[u].low;
      out[at * 3 + 2] = uint32_t(j0 + u * kSliceThreads + tid) | (guard >> u & 1) << 31;
    }
  }
  if (tid == 0) a.guarded[int64_t(bh) * a.slices + blockIdx.x] = guarded;
}

// ... and the lowest of those, with the moves that follow: a workgroup per head, at most NT * PT candidates.
constexpr int kPick = 16384;
template <int NT, int PT>
__global__ __launch_bounds__(NT) void evict_pick(EvictArgs a, int lanes) {
  __shared__ SelectShared sh;
  __shared__ uint64_t few[kFew];
  __shared__ uint32_t cnt[PT * (NT / 64) + 1];
  __shared__ int hole[kInline], from[kInline], gone[kInline];
  static_assert(kInline <= NT, "a thread per entry behind the budget");
  const int bh = blockIdx.x, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n = min(a.lens[b], a.max_len), S = a.budget, goes = n - S;
  if (goes <= 0) return;
  const int slices = (n + kSlice - 1) / kSlice, count = (slices - 1) * goes + min(goes, n - (slices - 1) * kSlice);
  uint32_t key[PT], entry[PT];
  Rank r[PT];
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const int i = min(u * NT + tid, count - 1);
    const uint32_t* c = a.cand + ((int64_t(bh) * a.slices + i / goes) * a.extra + i % goes) * 3;
    key[u] = c[0];
    r[u].low = c[1];
    entry[u] = c[2];
  }
  int guarded = 0, mine = 0;  // in all; of the candidates
  for (int i = tid; i < slices; i += NT) guarded += a.guarded[int64_t(bh) * a.slices + i];
  if (tid < goes) gone[tid] = 0;
  const bool crowded = block_total<NT>(guarded, sh.wave) > S;
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const bool guard = entry[u] >> 31;
    r[u].key = key[u] == 0 ? 0 : crowded ? (guard ? key[u] : 1u) : guard ? kProtected : key[u];
    mine += u * NT + tid < count && r[u].key == kProtected;
  }
  mine = block_total<NT>(mine, sh.wave);
  auto each_rank = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < PT; ++u)
      if (u * NT + tid < count) f(u * NT + tid, r[u]);
  };
  Threshold kept{0xFFFFFFFFu, 0xFFFFFFFFu, -1};  // none
  if (goes == 1) {
    const Lowest x = lowest_entry<NT>(sh, each_rank);
    kept = {x.key, x.low, x.at - 1};
  } else if (goes < count) {
    kept = threshold<NT>(sh, few, count - goes, mine, each_rank);
  }
  uint32_t is_hole = 0;
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const int i = u * NT + tid, j = int(entry[u] & 0x7FFFFFFFu);
    const bool goner = i < count && !kept.stays(r[u], i);
    if (goner && j >= S) gone[j - S] = 1;
    is_hole |= uint32_t(goner && j < S && key[u] != 0) << u;
    const uint64_t m = __ballot(is_hole >> u & 1);
    if (lane == 0) cnt[u * (NT / 64) + w] = __popcll(m);
  }
  prefix_counts<NT, PT>(cnt);
#pragma unroll
  for (int u = 0; u < PT; ++u) {
    const bool is = is_hole >> u & 1;
    const int at = cnt[u * (NT / 64) + w] + lanes_before(__ballot(is));
    if (is && at < kInline) hole[at] = int(entry[u] & 0x7FFFFFFFu);
  }
  const int holes = cnt[PT * (NT / 64)];
  // the entries behind the budget that stay
  const bool row = tid < goes && !gone[tid] && a.pool.page_of(b, S + tid) >= 0;
  const uint64_t m = __ballot(row);
  if (lane == 0) sh.wave[w] = __popcll(m);
  __syncthreads();
  int at = lanes_before(m), rows = 0;
  for (int i = 0; i < NT / 64; ++i) {
    if (i < w) at += sh.wave[i];
    rows += sh.wave[i];
  }
  if (row) from[at] = S + tid;
  __syncthreads();
  move_rows<4>(a, b, hk, from, hole, tid / lanes, NT / lanes, min(min(holes, rows), kInline), tid % lanes);
}

// Workspace of a fill: a list of kept positions; of a long prompt also the slices' histograms and counts, and the candidates.
size_t fill_bytes(size_t bh, size_t n) {
  const size_t list = round256(bh * n * sizeof(int32_t)), slices = (n + kSlice - 1) / kSlice;
  if (n <= kFillSelect) return list;
  return 2 * list + round256(bh * slices * kBins * sizeof(uint16_t)) + round256(bh * slices * sizeof(int32_t)) + round256(bh * 4 * sizeof(int32_t));
}
// Of an eviction: the moves, or what the slices leave.
size_t moves_bytes(size_t bh, size_t n) {
  const size_t moves = round256(bh * 2 * n * sizeof(int32_t)) + round256(bh * sizeof(int32_t)), slices = (n + kSlice - 1) / kSlice;
  if (n <= kFillSelect) return moves;
  return std::max(moves, 2 * round256(bh * slices * sizeof(int32_t)) + bh * std::min<size_t>(kPick, slices * kInline) * 3 * sizeof(uint32_t));
}
}  // namespace

size_t pages_evict_bytes(const d2o_pages* p, int32_t max_len) {
  const size_t bh = size_t(p->batch) * p->n_kv_heads;
  return std::max(fill_bytes(bh, max_len), moves_bytes(bh, max_len));
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
  if (!pages_apart(pages)) return D2O_ERR_INVALID_ARG;
  const int most = std::min(n, budget);
  if (most > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  const int64_t bh = int64_t(pages->batch) * pages->n_kv_heads;
  if (workspace_bytes < fill_bytes(bh, n)) return D2O_ERR_CAPACITY;
  if (bh > 65535 || n > kSlice * kMaxSlices) return D2O_ERR_UNSUPPORTED;
  a.k = to_view(K);
  a.v = to_view(V);
  a.lens = lens;
  a.scores = scores;
  a.n = n;
  a.budget = most;
  a.recent = recent;
  a.n_sink = n_sink;
  a.slices = (n + kSlice - 1) / kSlice;
  // Rows read and written that exceed half the 256 MB memory-side cache would only push each other out of it (16 x 8 heads, 1638 rows of
  // 8192: 56 -> 48 us); fewer may be there still from the prompt's attention (8 heads, 6553 of 131072: 39 instead of 37.5).
  const bool past = bh * most * 4 * D * es > 128ll << 20;
  char* ws = static_cast<char*>(workspace);
  a.src = reinterpret_cast<int32_t*>(ws);
  ws += round256(size_t(bh) * n * sizeof(int32_t));
  a.cand = reinterpret_cast<uint32_t*>(ws);
  ws += round256(size_t(bh) * n * sizeof(int32_t));
  a.hist = reinterpret_cast<uint16_t*>(ws);
  ws += round256(size_t(bh) * a.slices * kBins * sizeof(uint16_t));
  a.above = reinterpret_cast<int32_t*>(ws);
  ws += round256(size_t(bh) * a.slices * sizeof(int32_t));
  a.head = reinterpret_cast<int32_t*>(ws);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 heads{unsigned(bh)};
  if (most < n && n > kFillSelect) {
    fill_hist<<<dim3(a.slices, unsigned(bh)), kSliceThreads, 0, s>>>(a);
    fill_candidates<<<dim3(a.slices, unsigned(bh)), kSliceThreads, 0, s>>>(a);
    fill_list<<<dim3(a.slices, unsigned(bh)), kSliceThreads, 0, s>>>(a);
  } else if (most < n) {
    if (n <= 2048)
      fill_select<256, 8><<<heads, 256, 0, s>>>(a);
    else if (n <= 8192)
      fill_select<1024, 8><<<heads, 1024, 0, s>>>(a);
    else
      fill_select<1024, 16><<<heads, 1024, 0, s>>>(a);
  }
  auto write = [&](auto t, auto ct, auto d) {
    typedef decltype(t) T;
    typedef decltype(ct) CT;
    constexpr int kD = decltype(d)::value, kRows = 256 / (kD * int(sizeof(T)) / 16);
    const auto kernel = past ? fill_rows<T, CT, kD, true> : fill_rows<T, CT, kD, false>;
    kernel<<<dim3((most + kRows - 1) / kRows, unsigned(bh)), 256, 0, s>>>(a);
  };
  auto rows = [&](auto t, auto ct) {
    if (D == 64)
      write(t, ct, std::integral_constant<int, 64>{});
    else
      write(t, ct, std::integral_constant<int, 128>{});
  };
  if (pages->cache_fp8)
    rows(uint16_t{}, uint8_t{});
  else if (pages->dtype == D2O_BF16)
    rows(uint16_t{}, uint16_t{});
  else
    rows(float{}, float{});
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}

extern "C" int d2o_pages_evict(const d2o_pages* pages, const int32_t* lens, int32_t max_len, int32_t budget,
                               int32_t recent, int32_t n_sink, void* workspace, size_t workspace_bytes, void* stream) {
  EvictArgs a;
  const int rc = check_pages(pages, &a.pool);
  if (rc != D2O_OK) return rc;
  if (!lens || !pages->score || !pages->pos || max_len < 1 || !pages_apart(pages)) return D2O_ERR_INVALID_ARG;
  if (budget < 1 || recent < 0 || n_sink < 0 || int64_t(recent) + n_sink > budget) return D2O_ERR_INVALID_ARG;
  if (max_len > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  const int64_t bh = int64_t(pages->batch) * pages->n_kv_heads;
  if (workspace_bytes < moves_bytes(bh, max_len)) return D2O_ERR_CAPACITY;
  if (bh > 65535) return D2O_ERR_UNSUPPORTED;
  if (max_len <= budget) return D2O_OK;  // no sequence can have more than it keeps
  a.lens = lens;
  a.max_len = max_len;
  a.budget = budget;
  a.recent = recent;
  a.n_sink = n_sink;
  a.most = std::min(budget, max_len - budget);
  a.extra = max_len - budget;
  a.slices = (max_len + kSlice - 1) / kSlice;
  a.moves = static_cast<int32_t*>(workspace);
  a.count = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + round256(size_t(bh) * 2 * max_len * sizeof(int32_t)));
  a.newest = a.moves;
  a.guarded = a.newest + round256(size_t(bh) * a.slices * sizeof(int32_t)) / sizeof(int32_t);
  a.cand = reinterpret_cast<uint32_t*>(a.guarded + round256(size_t(bh) * a.slices * sizeof(int32_t)) / sizeof(int32_t));
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int lanes = pages->head_dim * (pages->cache_fp8 ? 1 : pages->dtype == D2O_BF16 ? 2 : 4) / 16;
  const dim3 heads{unsigned(bh)};
  // More than the registers of a workgroup hold: in slices where few go (one of 8 x 26214 entries 24 us, by a workgroup per head that reads them
  // again for every use 44; of 8 x 131072 25 and 184; 256 of 8 x 26214 42 and 100), by that workgroup where slices would leave as many candidates.
  const bool by_slices = max_len > 16384 && a.extra <= kInline && int64_t(a.slices) * a.extra <= kPick && a.slices <= kMaxSlices;
  if (max_len <= 2048)
    evict_select<256, 8><<<heads, 256, 0, s>>>(a, lanes);
  else if (max_len <= 4096)
    evict_select<1024, 4><<<heads, 1024, 0, s>>>(a, lanes);
  else if (max_len <= 16384)
    evict_select<1024, 16><<<heads, 1024, 0, s>>>(a, lanes);
  else if (by_slices) {
    const dim3 grid(a.slices, unsigned(bh));
    evict_newest<<<grid, kSliceThreads, 0, s>>>(a);
    evict_lowest<<<grid, kSliceThreads, 0, s>>>(a);
    if (a.slices * a.extra <= 1024)
      evict_pick<1024, 1><<<heads, 1024, 0, s>>>(a, lanes);
    else
      evict_pick<1024, 16><<<heads, 1024, 0, s>>>(a, lanes);
  } else
    evict_select<1024, 0><<<heads, 1024, 0, s>>>(a, lanes);
  if (a.most > kInline) {  // (by slices: never)
    const int per = 256 / lanes;
    evict_move<<<dim3(std::min((a.most + per - 1) / per, 65536), unsigned(bh)), 256, 0, s>>>(a, lanes);
  }
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
