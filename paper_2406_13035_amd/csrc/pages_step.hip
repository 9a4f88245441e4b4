// One generation step over a cache in pages (d2o_pages_step): the new token's row is stored, every query head attends
// over the entries that its window shows, and the softmax rows are added to the entries' scores.
#include <algorithm>

#include "pages_step.h"

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
  const int32_t counts[3] = {p->n_pages, p->n_kv_heads, p->page_size}, row = p->cache_fp4 ? p->head_dim / 2 : p->head_dim;
  return rows_apart(p->K, counts, row) && rows_apart(p->V, counts, row);
}

int check_pages(const d2o_pages* p, PagePool* out) {
  if (!p) return D2O_ERR_INVALID_ARG;
  if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_pages < 1 || p->max_pages < 1) return D2O_ERR_INVALID_ARG;
  if (p->n_q_heads % p->n_kv_heads) return D2O_ERR_INVALID_ARG;
  if (p->dtype != D2O_F32 && p->dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return D2O_ERR_UNSUPPORTED;
  if (p->n_q_heads / p->n_kv_heads > 16) return D2O_ERR_UNSUPPORTED;
  if (p->cache_fp8 != 0 && p->cache_fp8 != 1) return D2O_ERR_INVALID_ARG;
  if ((p->cache_fp4 != 0 && p->cache_fp4 != 1) || (p->cache_fp4 && p->cache_fp8)) return D2O_ERR_INVALID_ARG;
  const bool coded = p->cache_fp8 || p->cache_fp4;
  if (coded && p->dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (p->page_size < 1 || p->page_size > 1024 || (p->page_size & (p->page_size - 1))) return D2O_ERR_INVALID_ARG;
  if (int64_t(p->max_pages) * p->page_size > 0x7FFF0000) return D2O_ERR_INVALID_ARG;
  if (int64_t(p->batch) * p->n_q_heads > 0x3FFFFFFF) return D2O_ERR_INVALID_ARG;
  const int es = coded ? 1 : p->dtype == D2O_BF16 ? 2 : 4;
  if (!dense_view_ok(p->K, es, true) || !dense_view_ok(p->V, es, true)) return D2O_ERR_INVALID_ARG;
  if (coded && (!p->K_exp || !p->V_exp)) return D2O_ERR_INVALID_ARG;
  if (p->cache_fp4 && (reinterpret_cast<uintptr_t>(p->K_exp) | reinterpret_cast<uintptr_t>(p->V_exp)) & 3) return D2O_ERR_INVALID_ARG;
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
  out->k_exp = coded ? p->K_exp : nullptr;
  out->v_exp = coded ? p->V_exp : nullptr;
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
  a.pairs = pages->cache_fp4;
  a.share = 0;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (pages->cache_fp4)
    launch_step4(a, pages->batch, pages->head_dim, s);
  else if (pages->cache_fp8)
    launch_step<uint16_t, uint8_t>(a, pages->batch, pages->head_dim, s);
  else if (pages->dtype == D2O_BF16)
    launch_step<uint16_t, uint16_t>(a, pages->batch, pages->head_dim, s);
  else
    launch_step<float, float>(a, pages->batch, pages->head_dim, s);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
