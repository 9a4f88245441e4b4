// One generation step over a cache in pages (d2o_pages_step): the new token's row is stored, every query head attends
// over the entries that its window shows, and the softmax rows are added to the entries' scores.
#include <algorithm>

#include "pages.h"

namespace d2o {

bool dense_view_ok(const d2o_view& v, int esize, bool rows) {
  const int64_t al = 16 / esize;
  if (!v.ptr || (reinterpret_cast<uintptr_t>(v.ptr) & 15)) return false;
  if (v.stride_b < 0 || v.stride_h < 0 || (rows && v.stride_n < 0)) return false;
  return v.stride_b % al == 0 && v.stride_h % al == 0 && (!rows || v.stride_n % al == 0);
}

bool rows_apart(const d2o_view& v, const int32_t (&counts)[3], int d) {
  const int64_t strides[3] = {v.stride_b, v.stride_h, v.stride_n};
  for (int i = 0; i < 3; ++i)
    if (counts[i] > 1 && strides[i] < d) return false;
  return true;
}
bool pages_apart(const d2o_pages* p) {
  const int32_t counts[3] = {p->n_pages, p->n_kv_heads, p->page_size};
  return rows_apart(p->K, counts, p->head_dim) && rows_apart(p->V, counts, p->head_dim);
}

int check_pages(const d2o_pages* p, PagePool* out) {
  if (!p) return D2O_ERR_INVALID_ARG;
  if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->max_pages < 1) return D2O_ERR_INVALID_ARG;
  if (p->n_q_heads % p->n_kv_heads) return D2O_ERR_INVALID_ARG;
  if (p->dtype != D2O_F32 && p->dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return D2O_ERR_UNSUPPORTED;
  if (p->n_q_heads / p->n_kv_heads > 16) return D2O_ERR_UNSUPPORTED;
  if (p->cache_fp8 != 0 && p->cache_fp8 != 1) return D2O_ERR_INVALID_ARG;
  if (p->cache_fp8 && p->dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (p->page_size < 1 || p->page_size > 1024 || (p->page_size & (p->page_size - 1))) return D2O_ERR_INVALID_ARG;
  if (int64_t(p->max_pages) * p->page_size > 0x7FFF0000) return D2O_ERR_INVALID_ARG;
  if (int64_t(p->batch) * p->n_q_heads > 0x3FFFFFFF) return D2O_ERR_INVALID_ARG;
  const int es = p->cache_fp8 ? 1 : p->dtype == D2O_BF16 ? 2 : 4;
  if (!dense_view_ok(p->K, es, true) || !dense_view_ok(p->V, es, true)) return D2O_ERR_INVALID_ARG;
  if (p->cache_fp8 && (!p->K_exp || !p->V_exp)) return D2O_ERR_INVALID_ARG;
  if (!p->page_table || (reinterpret_cast<uintptr_t>(p->page_table) | reinterpret_cast<uintptr_t>(p->score) |
                         reinterpret_cast<uintptr_t>(p->pos)) & 3)
    return D2O_ERR_INVALID_ARG;
  if (!out) return D2O_OK;
  out->K = static_cast<uint8_t*>(p->K.ptr);
  out->V = static_cast<uint8_t*>(p->V.ptr);
  out->k_page = p->K.stride_b * es;
  out->k_head = p->K.stride_h * es;
  out->k_row = p->K.stride_n * es;
  out->v_page = p->V.stride_b * es;
  out->v_head = p->V.stride_h * es;
  out->v_row = p->V.stride_n * es;
  out->k_exp = p->cache_fp8 ? p->K_exp : nullptr;
  out->v_exp = p->cache_fp8 ? p->V_exp : nullptr;
  out->score = p->score;
  out->pos = p->pos;
  out->table = p->page_table;
  out->shift = __builtin_ctz(unsigned(p->page_size));
  out->n_pages = p->n_pages;
  out->max_pages = p->max_pages;
  out->Hkv = p->n_kv_heads;
  return D2O_OK;
}

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;       // wavefronts of a workgroup
constexpr int kTile = 16;       // entries of a tile: the rows of one matrix operand
constexpr int kRowBcast = 0x150;  // lane i of each row of 16 lanes to all of the row (data-parallel primitive, + i)

struct StepArgs {
  PagePool pool;
  View q, kn, vn, out;
  const int32_t* lens;
  const int32_t* positions;
  float* logits;   // [B][Hq][pad] base-2 logits of the entries that are seen (scores kept)
  float* part_o;   // [B * Hkv][splits][G][D] outputs of a share, not normalised
  float* part_ml;  // [B * Hkv][splits][G][2] its softmax maximum and sum (outputs and sums: times 2^-TileList::bias)
  int32_t Hq, G, max_len, window, n_sink, pad, splits, joins;  // joins: workgroups of step_finish that join outputs
};

// The tiles of a sequence that hold what a step sees: those of the first tokens, then those from the window's start.  (Where the
// pages keep positions, entries lie in any order and all tiles are looked at.)
struct TileList {
  int n, sink_tiles, rest0, tiles, share;  // entries, tiles of the first tokens, first tile behind them, tiles in all, tiles per workgroup
  int64_t last;                            // the new token's position
  int bias;                                // n < 2^bias
  __device__ __forceinline__ TileList(const StepArgs& a, int b, int least) {
    n = min(a.lens[b], a.max_len);
    if (n <= 0) {
      n = tiles = share = sink_tiles = rest0 = bias = 0;
      last = 0;
      return;
    }
    last = a.positions ? a.positions[b] : n - 1;
    bias = 32 - __clz(n);
    const int all = (n + kTile - 1) / kTile;
    sink_tiles = rest0 = 0;
    if (a.window != 0 && !a.pool.pos) {
      const int64_t lo = last - a.window + 1;  // first entry of the window
      sink_tiles = (min(a.n_sink, n) + kTile - 1) / kTile;
      rest0 = int(min(max(lo / kTile, int64_t(sink_tiles)), int64_t(all)));
      if (lo < 0) rest0 = sink_tiles;
    }
    tiles = sink_tiles + all - rest0;
    if (tiles == 0) {  // nothing is seen: the last tile, whose entries are all masked
      rest0 = all - 1;
      tiles = 1;
    }
    share = ((tiles + a.splits - 1) / a.splits + least - 1) / least * least;  // whole rounds of the wavefronts
  }
  __device__ __forceinline__ int slot(int t) const { return (t < sink_tiles ? t : rest0 + t - sink_tiles) * kTile; }
  __device__ __forceinline__ int shares() const { return tiles ? (tiles + share - 1) / share : 0; }
  // Whether the window shows entry s, whose position is `pos` where the pages keep positions.
  __device__ __forceinline__ bool sees(const StepArgs& a, int s, int32_t pos) const {
    const int p = a.pool.pos ? pos : s;
    return a.window == 0 || p > last - a.window || p < a.n_sink;
  }
};

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

// What a lane holds of rows of type CT with D elements.  K: lane l has row l % 16 of a tile, chunks of 16 bytes that the four rows of
// lanes take in turn; V: the 16 lanes of a row of lanes share a row of V, D / 16 elements each.
template <typename CT, int D>
struct Rows;
template <int D>
struct Rows<uint16_t, D> {
  static constexpr int kK = D / 32, kE = D / 16;  // 16-byte chunks of K per lane; elements of V per lane
  typedef std::conditional_t<D == 128, u32x4, u32x2> VReg;
  bf16x8 q[kK];
  __device__ __forceinline__ void load_q(const uint16_t* row, int g) {
#pragma unroll
    for (int i = 0; i < kK; ++i)
      q[i] = row ? *reinterpret_cast<const bf16x8*>(row + i * 32 + g * 8) : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  }
  __device__ __forceinline__ f32x4 logits(const u32x4* k, float) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kK; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i]), q[i], s, 0, 0, 0);
    return s;
  }
  static __device__ __forceinline__ VReg load_v(const uint8_t* row, int c) { return __builtin_nontemporal_load(reinterpret_cast<const VReg*>(row) + c); }
  static __device__ __forceinline__ int column(int c, int e) { return c * kE + e; }
  static __device__ __forceinline__ void values(const VReg& v, float, float* f) {
#pragma unroll
    for (int i = 0; i < kE / 2; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
};
template <int D>
struct Rows<float, D> {
  static constexpr int kK = D / 16, kE = D / 16;
  struct VReg {
    f32x4 x[D / 64];
  };
  f32x4 q[kK];
  __device__ __forceinline__ void load_q(const float* row, int g) {
#pragma unroll
    for (int i = 0; i < kK; ++i) q[i] = row ? *reinterpret_cast<const f32x4*>(row + i * 16 + g * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ f32x4 logits(const u32x4* k, float) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kK; ++i) {
      const f32x4 x = __builtin_bit_cast(f32x4, k[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], q[i][j], s, 0, 0, 0);
    }
    return s;
  }
  static __device__ __forceinline__ VReg load_v(const uint8_t* row, int c) {
    VReg v;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) v.x[i] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row) + i * 16 + c);
    return v;
  }
  static __device__ __forceinline__ int column(int c, int e) { return (e / 4) * 64 + c * 4 + e % 4; }
  static __device__ __forceinline__ void values(const VReg& v, float, float* f) {
#pragma unroll
    for (int e = 0; e < kE; ++e) f[e] = v.x[e / 4][e % 4];
  }
};
// 8-bit codes: K as bf16 with the row's power of two (exact: four significant bits), V in fp32.
template <int D>
struct Rows<uint8_t, D> {
  static constexpr int kK = D / 64, kE = D / 16;
  typedef std::conditional_t<D == 128, u32x2, uint32_t> VReg;
  bf16x8 q[2 * kK];
  __device__ __forceinline__ void load_q(const uint16_t* row, int g) {
#pragma unroll
    for (int i = 0; i < 2 * kK; ++i)
      q[i] = row ? *reinterpret_cast<const bf16x8*>(row + i / 2 * 64 + g * 16 + i % 2 * 8)
                 : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  }
  __device__ __forceinline__ f32x4 logits(const u32x4* k, float scale) const {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2 * kK; ++i) {
      u32x4 x;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t w = k[i / 2][i % 2 * 2 + j];
        x[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
        x[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
      }
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), q[i], s, 0, 0, 0);
    }
    return s;
  }
  static __device__ __forceinline__ VReg load_v(const uint8_t* row, int c) { return __builtin_nontemporal_load(reinterpret_cast<const VReg*>(row) + c); }
  static __device__ __forceinline__ int column(int c, int e) { return c * kE + e; }
  static __device__ __forceinline__ void values(const VReg& v, float scale, float* f) {
#pragma unroll
    for (int i = 0; i < kE / 4; ++i) {
      uint32_t w;
      if constexpr (D == 128)
        w = v[i];
      else
        w = v;
      const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
      const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
      f[4 * i] = lo[0];
      f[4 * i + 1] = lo[1];
      f[4 * i + 2] = hi[0];
      f[4 * i + 3] = hi[1];
    }
  }
};

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
    if constexpr (sizeof(CT) == 1) {
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

// One workgroup per (sequence, KV head, share of its tiles).  U tiles of 16 entries per wavefront and round: the logits of all
// query heads of the group come from the matrix core (heads are its columns, padded to 16), straight from rows in registers: lane l
// holds 16 bytes of row l % 16 at a time, and the order of the products' terms is free.  A lane of the result has head
// l % 16 and four entries of its row of lanes, and that row of lanes reads the rows of V of just these entries: every row of lanes keeps a
// softmax of its own over the entries it meets, with nothing exchanged in the loop; a probability reaches the lanes of
// its row by a register broadcast, and P V runs on the vector ALU.  More than four heads per group: P V on the fp32 matrix instruction (16 x 16 x 4), of
// which a lane's probability (head l % 16, one entry per row of lanes) and value are the operands as they are; the four rows of lanes then
// share a maximum.  (8 x 16384 entries of 8 heads, 16 per group: 8-bit rows 143 -> 88 us, bf16 157 -> 137; 8 per group 93 -> 77, 122 -> 117; but 16 x 8192 with
// four 79 -> 83, and one per group, whose fifteen idle rows cost as much, 29 -> 43 for 4 x 32 heads x 4100.)  Both in fp32: a rounding of P would cost more bits.
// WIDE: a tile lies in one page, whose number and address are the same for all lanes and live in scalar registers; a lane adds a
// displacement of 32 bits that never changes.  Rows of V are read once and past the caches (16 lanes take whole lines; 131072 entries
// 104 -> 98 us), K's are not: an instruction takes half lines, and with the hint the other half came from memory again.  Two wavefronts per
// SIMD at least (three: 65 -> 71 us for four heads per group).  (With an address per lane and row, computed for every tile, the vector ALU was as busy
// with addresses as with sums: 4 x 32 heads x 4100 entries of 8-bit rows took 71 us, now 25.)
template <typename T, typename CT, int D, int GM, int U, bool WIDE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void step_part(StepArgs a) {
  typedef Rows<CT, D> R;
  constexpr int E = R::kE;
  constexpr bool kMatrix = GM > 4;
  __shared__ float so[kWaves][GM][D];
  __shared__ float sml[kWaves][GM][2];
  __shared__ float sM[GM], sinv[GM];
  const int Hkv = a.pool.Hkv, bh = blockIdx.y, b = bh / Hkv, hk = bh % Hkv;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  const TileList list(a, b, kWaves * U);
  const int t0 = blockIdx.x * list.share, t1 = min(t0 + list.share, list.tiles);
  if (list.n == 0) {
    if (blockIdx.x == 0)
      for (int i = tid; i < a.G * D; i += 64 * kWaves) store_out<T>(a, b, hk * a.G + i / D, i % D, 0.f);
    return;
  }
  if (t0 >= t1) return;
  const int n = list.n;
  // the workgroup of the last tile stores the new token; it reads it where it came from, not to wait for the store
  int fresh = -1;
  if (a.kn.ptr && t1 == list.tiles && a.lens[b] <= a.max_len) {
    const int page = a.pool.page_of(b, n - 1);
    if (page >= 0) {
      store_new<T, CT, D>(a, b, hk, page, n - 1, list.last);
      fresh = n - 1;
    }
    if constexpr (sizeof(CT) == 1) {  // read back, as it was encoded
      __threadfence_block();
      __syncthreads();
    }
  }
  R rows;
  rows.load_q(c < a.G ? static_cast<const T*>(a.q.ptr) + b * a.q.sb + (hk * a.G + c) * a.q.sh : nullptr, g);
  const float scale2 = kLog2e / sqrtf(float(D));
  const bool ordered = a.window != 0 && !a.pool.pos, by_pos = a.window != 0 && a.pool.pos;
  const int64_t lo64 = a.window == 0 ? INT64_MIN : list.last - a.window + 1;  // first position of the window
  const int lo = int(min(max(lo64, int64_t(0)), int64_t(n)));                 // (entries in order of position)
  // Probabilities are formed as 2^-bias * p, so that no sum of them is above one and P V never above the largest value.  (What is 2^(126 - bias)
  // below a head's highest entry is zero.)
  const float bias = list.bias;
  float m = -3.402823466e38f, l = 0.f, acc[kMatrix ? 1 : GM][E] = {};
  f32x4 om[kMatrix ? E : 1] = {};  // (kMatrix) register i: head 4 g + i, column R::column(c, e)
  float* lg = a.pool.score ? a.logits + (int64_t(b) * a.Hq + hk * a.G + c) * a.pad : nullptr;
  // (the page table: what an earlier launch or copy wrote, read through the scalar cache)
  const auto table = (const __attribute__((address_space(4))) int32_t*)(a.pool.table + int64_t(b) * a.pool.max_pages);
  const int rmask = (1 << a.pool.shift) - 1;
  const uint32_t koff = uint32_t(c) * uint32_t(a.pool.k_row) + g * 16, voff = uint32_t(4 * g) * uint32_t(a.pool.v_row);
  for (int t = t0 + w * U; t < t1; t += kWaves * U) {
    u32x4 k[U][R::kK];
    typename R::VReg v[U][4];
    float ke[U], ve[U][4];
    uint32_t seen[U];  // bit i: entry i of the tile is seen
    if constexpr (WIDE) {
      int page[U], s0[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s0[u] = list.slot(min(t + u, t1 - 1));
        page[u] = table[s0[u] >> a.pool.shift];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = uint32_t(page[u]) < uint32_t(a.pool.n_pages);
        const int p = there ? page[u] : 0;  // (no page: the pool's first, whose values are not used; rows behind the end lie in the page)
        const int64_t at = ((int64_t(p) * Hkv + hk) << a.pool.shift) + (s0[u] & rmask);
        const uint8_t* kp = a.pool.K + p * a.pool.k_page + hk * a.pool.k_head + (s0[u] & rmask) * a.pool.k_row;
        const uint8_t* vp = a.pool.V + p * a.pool.v_page + hk * a.pool.v_head + (s0[u] & rmask) * a.pool.v_row;
#pragma unroll
        for (int i = 0; i < R::kK; ++i) k[u][i] = *reinterpret_cast<const u32x4*>(kp + (koff + i * 64));
#pragma unroll
        for (int r = 0; r < 4; ++r) v[u][r] = R::load_v(vp + r * a.pool.v_row + voff, c);
        if constexpr (sizeof(CT) == 1) {
          ke[u] = pow2_f32((a.pool.k_exp + at)[uint32_t(c)]);
          const uint32_t four = *reinterpret_cast<const uint32_t*>(a.pool.v_exp + at + uint32_t(4 * g));
#pragma unroll
          for (int r = 0; r < 4; ++r) ve[u][r] = pow2_f32(int8_t(four >> (8 * r)));
        }
        seen[u] = 0;
        if (there && t + u < t1) {
          if (s0[u] + kTile <= n && !by_pos && (!ordered || s0[u] >= lo || s0[u] + kTile <= a.n_sink)) {
            seen[u] = 0xFFFFu;
          } else {
            const int s = s0[u] + c;
            bool ok = s < n;
            if (ordered) ok = ok && (s >= lo || s < a.n_sink);
            if (by_pos) {
              const int ps = (a.pool.pos + at)[uint32_t(c)];
              ok = ok && (ps >= lo64 || ps < a.n_sink);
            }
            seen[u] = uint32_t(__ballot(ok)) & 0xFFFFu;
          }
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int s0 = t + u < t1 ? list.slot(t + u) : n;  // (a tile behind the share: no entry)
        const int s = s0 + c;
        const int pk = s < n ? a.pool.page_of(b, s) : -1;
        bool ok = s < n && pk >= 0;
        if (ordered) ok = ok && (s >= lo || s < a.n_sink);
        if (by_pos && ok) {
          const int p = a.pool.pos[a.pool.at(pk, hk, s)];
          ok = p >= lo64 || p < a.n_sink;
        }
        seen[u] = uint32_t(__ballot(ok)) & 0xFFFFu;
        // (rows that are not seen: the first row of the pool instead, whose values are not used)
        const uint8_t* kr = ok ? a.pool.k_at(pk, hk, s) : a.pool.K;
#pragma unroll
        for (int i = 0; i < R::kK; ++i) k[u][i] = reinterpret_cast<const u32x4*>(kr)[i * 4 + g];
        if constexpr (sizeof(CT) == 1) ke[u] = ok ? pow2_f32(a.pool.k_exp[a.pool.at(pk, hk, s)]) : 1.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sv = s0 + 4 * g + r, pv = __shfl(pk, 4 * g + r, 64);
          const bool okv = seen[u] >> (4 * g + r) & 1;
          v[u][r] = R::load_v(okv ? a.pool.v_at(pv, hk, sv) : a.pool.V, c);
          if constexpr (sizeof(CT) == 1) ve[u][r] = okv ? pow2_f32(a.pool.v_exp[a.pool.at(pv, hk, sv)]) : 1.f;
        }
      }
    }
    if constexpr (sizeof(CT) > 1) {
      if (fresh >= 0) {
        const uint8_t* kn = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.kn.ptr) + b * a.kn.sb + hk * a.kn.sh);
        const uint8_t* vn = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.vn.ptr) + b * a.vn.sb + hk * a.vn.sh);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = fresh - (t + u < t1 ? list.slot(t + u) : n);
          if (at < 0 || at >= kTile) continue;
          if (c == at) {
#pragma unroll
            for (int i = 0; i < R::kK; ++i) k[u][i] = *reinterpret_cast<const u32x4*>(kn + (i * 4 + g) * 16);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * g + r == at) v[u][r] = R::load_v(vn, c);
          if (by_pos) seen[u] |= 1u << at;  // (its position is being written)
        }
      }
    }
    f32x4 s[U];
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = rows.logits(k[u], ke[u]) * scale2;
      if (seen[u] != 0xFFFFu) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!(seen[u] >> (4 * g + r) & 1)) s[u][r] = -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[u][r]);
      if (lg && c < a.G && t + u < t1) *reinterpret_cast<f32x4*>(lg + list.slot(t + u) + 4 * g) = s[u];
    }
    if constexpr (kMatrix) mx = max_rows(mx);  // one maximum per head
    if (__any(mx > m)) {
      const float f = __builtin_amdgcn_exp2f(m - mx);
      m = mx;
      l *= f;
      if constexpr (kMatrix) {
        const f32x4 fh = {__shfl(f, 4 * g, 64), __shfl(f, 4 * g + 1, 64), __shfl(f, 4 * g + 2, 64), __shfl(f, 4 * g + 3, 64)};
#pragma unroll
        for (int e = 0; e < E; ++e) om[e] *= fh;
      } else {
        each<GM>([&](auto h) {
          const float fh = row_bcast<h>(f);
#pragma unroll
          for (int e = 0; e < E; ++e) acc[h][e] *= fh;
        });
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f((s[u][r] - m) - bias);
        l += p;
        float f[E];
        R::values(v[u][r], ve[u][r], f);
        if (seen[u] != 0xFFFFu) {
          const bool okv = seen[u] >> (4 * g + r) & 1;
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = okv ? f[e] : 0.f;
        }
        if constexpr (kMatrix) {
#pragma unroll
          for (int e = 0; e < E; ++e) om[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(p, f[e], om[e], 0, 0, 0);
        } else {
          each<GM>([&](auto h) {
            const float ph = row_bcast<h>(p);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[h][e] = fmaf(ph, f[e], acc[h][e]);
          });
        }
      }
    }
  }
  // join the four rows of lanes, then the wavefronts
  const float mw = max_rows(m), f = __builtin_amdgcn_exp2f(m - mw);
  l = sum_rows(l * f);
  if constexpr (kMatrix) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * g + i < GM) so[w][4 * g + i][R::column(c, e)] = om[e][i];
  } else {
    each<GM>([&](auto h) {
      const float fh = row_bcast<h>(f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float o = sum_rows(acc[h][e] * fh);
        if (g == h % 4) so[w][h][R::column(c, e)] = o;
      }
    });
  }
  if (lane < GM) {
    sml[w][lane][0] = mw;
    sml[w][lane][1] = l;
  }
  __threadfence_block();  // (the logits, which the whole workgroup reads where it is a head's only one)
  __syncthreads();
  const bool single = list.shares() == 1;
  for (int i = tid; i < a.G * D; i += 64 * kWaves) {
    const int h = i / D, col = i % D;
    float M = sml[0][h][0];
#pragma unroll
    for (int x = 1; x < kWaves; ++x) M = fmaxf(M, sml[x][h][0]);
    float L = 0.f, o = 0.f;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float fx = __builtin_amdgcn_exp2f(sml[x][h][0] - M);
      L = fmaf(sml[x][h][1], fx, L);
      o = fmaf(so[x][h][col], fx, o);
    }
    const int64_t at = (int64_t(bh) * a.splits + blockIdx.x) * a.G + h;
    if (single)
      store_out<T>(a, b, hk * a.G + h, col, L == 0.f ? 0.f : o / L);
    else
      a.part_o[at * D + col] = o;
    if (col == 0) {
      if (single) {
        sM[h] = M;
        sinv[h] = L == 0.f ? 0.f : ldexpf(1.f / L, -list.bias);
      } else {
        a.part_ml[at * 2] = M;
        a.part_ml[at * 2 + 1] = L;
      }
    }
  }
  if (lg && single) {
    __syncthreads();
    for (int i = tid; i < list.tiles * kTile; i += 64 * kWaves)
      add_scores<1, GM>(a, list, b, hk, i, 0, list.tiles * kTile, sM, sinv, [] {});
  }
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

// Tiles per wavefront and round: two, where their rows take 16 KB at most.
// (8-bit rows in fours: 39 instead of 36 us for 4 x 32 heads x 4100 entries; bf16 rows of 128 singly: 109 instead of 105 us for 8 heads of 131072.)
template <typename CT, int D, int GM>
constexpr int tiles_per_round() {
  return 2 * kTile * 2 * D * int(sizeof(CT)) <= 16384 ? 2 : 1;
}

template <typename T, typename CT, int D, int GM>
void launch_step(StepArgs& a, int batch, hipStream_t s) {
  constexpr int U = tiles_per_round<CT, D, GM>();
  const int bh = batch * a.pool.Hkv;
  // pages that hold whole tiles, displacements that fit, exponents that can be read four at a time
  const bool wide = a.pool.shift >= 4 && a.pool.k_row < (1 << 24) && a.pool.v_row < (1 << 24) &&
                    !(reinterpret_cast<uintptr_t>(a.pool.v_exp) & 3);
  const auto part = wide ? step_part<T, CT, D, GM, U, true> : step_part<T, CT, D, GM, U, false>;
  part<<<dim3(a.splits, bh), 64 * kWaves, 0, s>>>(a);
  if (a.splits == 1) return;
  a.joins = batch * a.Hq;
  const int64_t scores = a.pool.score ? int64_t((a.pad + kFinishEntries - 1) / kFinishEntries) * bh : 0;
  step_finish<T, D, GM><<<dim3(unsigned(a.joins + scores)), kFinish, 0, s>>>(a, kWaves * U);
}

template <typename T, typename CT, int D>
void launch_step(StepArgs& a, int batch, hipStream_t s) {
  if (a.G == 1) launch_step<T, CT, D, 1>(a, batch, s);
  else if (a.G == 2) launch_step<T, CT, D, 2>(a, batch, s);
  else if (a.G <= 4) launch_step<T, CT, D, 4>(a, batch, s);
  else if (a.G <= 8) launch_step<T, CT, D, 8>(a, batch, s);
  else launch_step<T, CT, D, 16>(a, batch, s);
}

template <typename T, typename CT>
void launch_step(StepArgs& a, int batch, int D, hipStream_t s) {
  if (D == 64) launch_step<T, CT, 64>(a, batch, s);
  else launch_step<T, CT, 128>(a, batch, s);
}

// Shares per head, for at most `tiles` tiles each: workgroups of 64 tiles, about four per CU (a workgroup's ends cost as much as a dozen
// tiles: 128 heads of 258 tiles of 8-bit rows 36 us in eight shares, 30 in four), but for two per CU shares as small as two rounds of a workgroup.
int step_splits(int64_t bh, int64_t tiles) {
  const int64_t large = std::min<int64_t>(1024 / bh, tiles / 64), small = std::min<int64_t>(512 / bh, tiles / (2 * kWaves));
  return int(std::max<int64_t>(1, std::max(large, small)));
}
// Tiles that a sequence of max_len entries shows at most.
int64_t most_tiles(const d2o_pages* p, int32_t max_len, int32_t window, int32_t n_sink) {
  const int64_t all = (int64_t(max_len) + kTile - 1) / kTile;
  if (window == 0 || p->pos) return all;
  return std::min(all, (int64_t(window) + n_sink) / kTile + 3);
}

}  // namespace

size_t pages_step_bytes(const d2o_pages* p, int32_t max_len) {
  const size_t bh = size_t(p->batch) * p->n_kv_heads, hq = size_t(p->batch) * p->n_q_heads, pad = (size_t(max_len) + kTile - 1) / kTile * kTile;
  const size_t splits = step_splits(bh, most_tiles(p, max_len, 0, 0));  // (a window has no more tiles, so no more shares)
  return round256(p->score ? hq * pad * sizeof(float) : 0) + round256(hq * splits * p->head_dim * sizeof(float)) +
         round256(hq * splits * 2 * sizeof(float));
}

}  // namespace d2o

using namespace d2o;

extern "C" int d2o_pages_workspace_bytes(const d2o_pages* pages, int32_t max_len, size_t* bytes) {
  const int rc = check_pages(pages, nullptr);
  if (rc != D2O_OK) return rc;
  if (max_len < 1 || !bytes) return D2O_ERR_INVALID_ARG;
  *bytes = std::max(pages_step_bytes(pages, max_len), pages_evict_bytes(pages, max_len));
  return D2O_OK;
}

extern "C" int d2o_pages_step(const d2o_pages* pages, d2o_view q, d2o_view k_new, d2o_view v_new, const int32_t* lens,
                              const int32_t* positions, int32_t max_len, int32_t window, int32_t n_sink, d2o_view out,
                              void* workspace, size_t workspace_bytes, void* stream) {
  StepArgs a;
  const int rc = check_pages(pages, &a.pool);
  if (rc != D2O_OK) return rc;
  const int es = pages->dtype == D2O_BF16 ? 2 : 4;
  if (!lens || max_len < 1 || window < 0 || n_sink < 0) return D2O_ERR_INVALID_ARG;
  if (!dense_view_ok(q, es, false) || !dense_view_ok(out, es, false)) return D2O_ERR_INVALID_ARG;
  if (!k_new.ptr != !v_new.ptr) return D2O_ERR_INVALID_ARG;
  if (k_new.ptr && (!dense_view_ok(k_new, es, false) || !dense_view_ok(v_new, es, false))) return D2O_ERR_INVALID_ARG;
  if (!rows_apart(out, {pages->batch, pages->n_q_heads, 1}, pages->head_dim) || (k_new.ptr && !pages_apart(pages))) return D2O_ERR_INVALID_ARG;
  if (max_len > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < pages_step_bytes(pages, max_len)) return D2O_ERR_CAPACITY;
  a.q = to_view(q);
  a.kn = to_view(k_new);
  a.vn = to_view(v_new);
  a.out = to_view(out);
  a.lens = lens;
  a.positions = positions;
  const int64_t bh = int64_t(pages->batch) * pages->n_kv_heads, hq = int64_t(pages->batch) * pages->n_q_heads;
  if (bh > 65535) return D2O_ERR_UNSUPPORTED;
  a.pad = (max_len + kTile - 1) / kTile * kTile;
  a.splits = step_splits(bh, most_tiles(pages, max_len, window, n_sink));
  // (step_finish: a grid holds fewer than 2^32 threads)
  if (a.splits > 1 && hq + (pages->score ? bh * ((max_len + kFinishEntries - 1) / kFinishEntries) : 0) > 0xFFFFFF) return D2O_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(workspace);
  a.logits = reinterpret_cast<float*>(ws);
  ws += round256(pages->score ? size_t(hq) * a.pad * sizeof(float) : 0);
  a.part_o = reinterpret_cast<float*>(ws);
  ws += round256(size_t(hq) * a.splits * pages->head_dim * sizeof(float));
  a.part_ml = reinterpret_cast<float*>(ws);
  a.Hq = pages->n_q_heads;
  a.G = pages->n_q_heads / pages->n_kv_heads;
  a.max_len = max_len;
  a.window = window;
  a.n_sink = n_sink;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (pages->cache_fp8)
    launch_step<uint16_t, uint8_t>(a, pages->batch, pages->head_dim, s);
  else if (pages->dtype == D2O_BF16)
    launch_step<uint16_t, uint16_t>(a, pages->batch, pages->head_dim, s);
  else
    launch_step<float, float>(a, pages->batch, pages->head_dim, s);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
