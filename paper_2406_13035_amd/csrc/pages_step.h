// Generation steps over pages: what the kernels for rows of 32, 16 and 8 bits (pages_step.hip) and of 4 bits (pages_fp4.hip) share.
#pragma once

#include <algorithm>

#include "fp4.h"
#include "pages.h"
#include "pages_columns.h"

namespace d2o {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;       // wavefronts of a workgroup
constexpr int kTile = 16;       // entries of a tile: the rows of one matrix operand
constexpr int kRowBcast = 0x150;  // lane i of each row of 16 lanes to all of the row (data-parallel primitive, + i)

// (4-bit rows) a maximum that grew by less than 2^kSlack stays what weights are relative to.
constexpr int kSlack = 8;

struct StepArgs {
  PagePool pool;
  View q, kn, vn, out;
  const int32_t* lens;
  const int32_t* positions;
  float* logits;   // [B][Hq][pad] base-2 logits of the entries that are seen (scores kept)
  float* part_o;   // [B * Hkv][splits][G][D] outputs of a share, not normalised
  float* part_ml;  // [B * Hkv][splits][G][2] its softmax maximum and sum (outputs and sums: times 2^-TileList::bias)
  int32_t Hq, G, max_len, window, n_sink, pad, splits, joins;  // joins: workgroups of step_finish that join outputs
  int32_t pairs;  // 1: tiles are looked at in pairs, entries 32 i .. 32 i + 31
  int32_t share;  // tiles of a workgroup at least (0: a sequence's tiles are spread over all shares)
};

// The tiles of a sequence that hold what a step sees: those of the first tokens, then those from the window's start.  (Where the
// pages keep positions, entries lie in any order and all tiles are looked at.)
struct TileList {
  int n, sink_tiles, rest0, tiles, share;  // entries, tiles of the first tokens, first tile behind them, tiles in all, tiles per workgroup
  int64_t last;                            // the new token's position
  int bias;                                // n < 2^bias (weights may be as large as 2^kSlack: n < 2^(bias - kSlack))
  __device__ __forceinline__ TileList() {}
  __device__ __forceinline__ TileList(const StepArgs& a, int b, int least) {
    n = min(a.lens[b], a.max_len);
    if (n <= 0) {
      n = tiles = share = sink_tiles = rest0 = bias = 0;
      last = 0;
      return;
    }
    last = a.positions ? a.positions[b] : n - 1;
    choose(a, last - a.window + 1, least);
  }
  // The tiles of the n entries (n > 0) for windows that start at entry `lo` or later.
  __device__ __forceinline__ void choose(const StepArgs& a, int64_t lo, int least) {
    bias = 32 - __clz(n) + (a.pairs ? kSlack : 0);
    const int all = (n + kTile - 1) / kTile;
    sink_tiles = rest0 = 0;
    if (a.window != 0 && !a.pool.pos) {
      sink_tiles = min(((min(a.n_sink, n) + kTile - 1) / kTile + a.pairs) & ~a.pairs, all);
      rest0 = int(min(max(lo / kTile & ~int64_t(a.pairs), int64_t(sink_tiles)), int64_t(all)));
      if (lo < 0) rest0 = sink_tiles;
    }
    tiles = sink_tiles + all - rest0;
    if (tiles == 0) {  // nothing is seen: the last tile, whose entries are all masked
      rest0 = all - 1;
      tiles = 1;
    }
    share = max(((tiles + a.splits - 1) / a.splits + least - 1) / least * least, a.share);  // whole rounds of the wavefronts
  }
  __device__ __forceinline__ int slot(int t) const { return (t < sink_tiles ? t : rest0 + t - sink_tiles) * kTile; }
  __device__ __forceinline__ int shares() const { return tiles ? (tiles + share - 1) / share : 0; }
  // Whether the window shows entry s, whose position is `pos` where the pages keep positions.
  __device__ __forceinline__ bool sees(const StepArgs& a, int s, int32_t pos) const {
    const int p = a.pool.pos ? pos : s;
    return a.window == 0 || p > last - a.window || p < a.n_sink;
  }
};

namespace {

template <int L>
__device__ __forceinline__ float row_bcast(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kRowBcast + L, 0xF, 0xF, true));
}
// v + the same of the lanes 16 and 32 away: every lane gets the sum over the four rows of 16.
__device__ __forceinline__ float sum_rows(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  v = __int_as_float(a[0]) + __int_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(b[0]) + __int_as_float(b[1]);
}

__device__ __forceinline__ float max_rows(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
  v = fmaxf(__int_as_float(a[0]), __int_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return fmaxf(__int_as_float(b[0]), __int_as_float(b[1]));
}

// out[h] of a (sequence, KV head) from joined partials.
template <typename T>
__device__ __forceinline__ void store_out(const StepArgs& a, int b, int hq, int col, float o) {
  (static_cast<T*>(a.out.ptr) + b * a.out.sb + hq * a.out.sh)[col] = Elem<T>::from_f32(o);
}

// The new token's row into its page: two wavefronts, one for K and one for V.
template <typename T, typename CT, int D>
__device__ __forceinline__ void store_new(const StepArgs& a, int b, int hk, int page, int s, int64_t position) {
  const int tid = threadIdx.x;
  const int64_t at = a.pool.at(page, hk, s);
  if (tid < 128) {
    const int which = tid >> 6, lane = tid & 63;
    const View& x = which ? a.vn : a.kn;
    const T* src = static_cast<const T*>(x.ptr) + b * x.sb + hk * x.sh;
    CT* dst = reinterpret_cast<CT*>(which ? a.pool.v_at(page, hk, s) : a.pool.k_at(page, hk, s));
    if constexpr (std::is_same_v<CT, Code4>) {
      if (lane < D / 8) {
        int e;
        const uint32_t codes = fp4_encode_block(reinterpret_cast<const u32x4*>(src)[lane], e);
        reinterpret_cast<uint32_t*>(dst)[lane] = codes;
        if (lane % 4 == 0) (which ? a.pool.v_exp : a.pool.k_exp)[at * (D / kBlock4) + lane / 4] = int8_t(e);
      }
    } else if constexpr (sizeof(CT) == 1) {
      float m = 0.f;
      for (int i = lane; i < D; i += 64) m = fmaxf(m, fp8_magnitude(Elem<T>::to_f32(src[i])));
      const int e = fp8_row_exponent(wave_max(m));
      for (int i = lane; i < D; i += 64) dst[i] = fp8_code(Elem<T>::to_f32(src[i]), e);
      if (lane == 0) (which ? a.pool.v_exp : a.pool.k_exp)[at] = int8_t(e);
    } else {
      for (int i = lane; i < D; i += 64) dst[i] = src[i];
    }
  }
  if (tid == 0) {
    if (a.pool.score) a.pool.score[at] = 0.f;
    if (a.pool.pos) a.pool.pos[at] = int32_t(position);
  }
}

// Adds the softmax rows of a (sequence, KV head) to the scores of entries i0, i0 + step, .. (in the order of the tiles) below `end`, N of them
// (Eq. 6); the group's query heads in rising order.  What is read - logits, pages, old scores - is on its way before `totals` forms M and
// inv, maximum and reciprocal sum (of exp2(x - M)) of each head.
template <int N, int GM, typename F>
__device__ __forceinline__ void add_scores(const StepArgs& a, const TileList& list, int b, int hk, int i0, int step, int end,
                                           const float* M, const float* inv, const F& totals) {
  const float* lg = a.logits + (int64_t(b) * a.Hq + hk * a.G) * a.pad;
  int s[N], page[N];
  float x[GM][N], old[N];
  int64_t at[N];
  int32_t pos[N] = {};
  const bool by_pos = a.window != 0 && a.pool.pos;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int i = i0 + u * step;
    s[u] = i < end ? list.slot(i / kTile) + i % kTile : list.n;
    page[u] = s[u] < list.n ? a.pool.page_of(b, s[u]) : -1;
  }
#pragma unroll
  for (int h = 0; h < GM; ++h)
    if (h < a.G) {
#pragma unroll
      for (int u = 0; u < N; ++u) x[h][u] = lg[int64_t(h) * a.pad + min(s[u], list.n - 1)];
    }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    at[u] = page[u] >= 0 ? a.pool.at(page[u], hk, s[u]) : 0;
    old[u] = a.pool.score[at[u]];
    if (by_pos) pos[u] = a.pool.pos[at[u]];
  }
  totals();
  float add[N] = {};
#pragma unroll
  for (int h = 0; h < GM; ++h)
    if (h < a.G) {
#pragma unroll
      for (int u = 0; u < N; ++u) add[u] += __builtin_amdgcn_exp2f(x[h][u] - M[h]) * inv[h];
    }
  // (only what is seen: the logit of -infinity of an entry that is not would become NaN beside a NaN or an infinity of its head)
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (page[u] >= 0 && list.sees(a, s[u], pos[u]) && add[u] != 0.f) a.pool.score[at[u]] = old[u] + add[u];
}

// Joins the shares of the heads that have several: the first `joins` workgroups the outputs, one query head each, the others the scores.
constexpr int kFinish = 256, kFinishEntries = 1024;  // threads; entries of a workgroup that adds scores
template <typename T, int D, int GM>
__global__ __launch_bounds__(kFinish) void step_finish(StepArgs a, int least) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  // maximum and sum of a query head over the shares: a wavefront, a lane per share
  auto total = [&](const float* ml, int ns, float& M, float& L) __attribute__((always_inline)) {
    M = -3.402823466e38f;
    for (int i = lane; i < ns; i += 64) M = fmaxf(M, ml[int64_t(i) * a.G * 2]);
    M = wave_max(M);
    L = 0.f;
    for (int i = lane; i < ns; i += 64) L = fmaf(ml[int64_t(i) * a.G * 2 + 1], __builtin_amdgcn_exp2f(ml[int64_t(i) * a.G * 2] - M), L);
    L = wave_sum(L);
  };
  if (int(blockIdx.x) < a.joins) {
    constexpr int kCols = D / 4, kParts = kFinish / kCols;  // four columns per thread, the shares among kParts groups of threads
    __shared__ f32x4 so[kParts][kCols];
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, bh = b * a.pool.Hkv + hq / a.G, h = hq % a.G;
    const TileList list(a, b, least);
    const int ns = list.shares();
    if (ns <= 1) return;
    const float* ml = a.part_ml + (int64_t(bh) * a.splits * a.G + h) * 2;
    float M, L;
    total(ml, ns, M, L);
    const int col = tid % kCols, part = tid / kCols;
    const f32x4* po = reinterpret_cast<const f32x4*>(a.part_o + (int64_t(bh) * a.splits * a.G + h) * D) + col;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = part; i < ns; i += kParts) o += po[int64_t(i) * a.G * kCols] * __builtin_amdgcn_exp2f(ml[int64_t(i) * a.G * 2] - M);
    so[part][col] = o;
    __syncthreads();
    if (tid < D) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kParts; ++i) sum += so[i][tid / 4][tid % 4];
      store_out<T>(a, b, hq, tid, L == 0.f ? 0.f : sum / L);
    }
    return;
  }
  __shared__ float sM[16], sinv[16];
  const int per = (a.pad + kFinishEntries - 1) / kFinishEntries, x = blockIdx.x - a.joins, bh = x / per, b = bh / a.pool.Hkv, hk = bh % a.pool.Hkv;
  const TileList list(a, b, least);
  const int first = x % per * kFinishEntries, ns = list.shares();
  if (first >= list.tiles * kTile || ns <= 1) return;
  const int end = min(first + kFinishEntries, list.tiles * kTile);
  add_scores<kFinishEntries / kFinish, GM>(a, list, b, hk, first + tid, kFinish, end, sM, sinv, [&]() __attribute__((always_inline)) {
    for (int h = w; h < a.G; h += kFinish / 64) {
      float M, L;
      total(a.part_ml + (int64_t(bh) * a.splits * a.G + h) * 2, ns, M, L);
      if (lane == 0) {
        sM[h] = M;
        sinv[h] = L == 0.f ? 0.f : ldexpf(1.f / L, -list.bias);
      }
    }
    __syncthreads();
  });
}

// Shares per head, for at most `tiles` tiles each: workgroups of 64 tiles, about four per CU (a workgroup's ends cost as much as a dozen
// tiles: 128 heads of 258 tiles of 8-bit rows 36 us in eight shares, 30 in four), but for two per CU shares as small as two rounds of a workgroup.
int step_splits(int64_t bh, int64_t tiles) {
  const int64_t large = std::min<int64_t>(1024 / bh, tiles / 64), small = std::min<int64_t>(512 / bh, tiles / (2 * kWaves));
  return int(std::max<int64_t>(1, std::max(large, small)));
}
// Tiles that a sequence of max_len entries shows at most, to `columns` neighbouring tokens.
int64_t most_tiles(const d2o_pages* p, int32_t max_len, int32_t window, int32_t n_sink, int32_t columns = 0) {
  if (window == 0 || p->pos) return (int64_t(max_len) + kTile - 1) / kTile;
  return shown_tiles(max_len, window, n_sink, columns, kTile);
}

}  // namespace

// The step over 4-bit rows (pages_fp4.hip).
void launch_step4(StepArgs& a, int batch, int D, hipStream_t s);

}  // namespace d2o
