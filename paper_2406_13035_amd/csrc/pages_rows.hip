// Rows of single tokens into a cache in pages (d2o_pages_put) and out of it (d2o_pages_get), by the slots of a map.
#include <algorithm>

#include "fp4.h"
#include "pages.h"

namespace d2o {
namespace {

struct RowArgs {
  PagePool pool;
  View x[2];             // K, V: [token][head][d]
  const int64_t* slots;  // page * page_size + row
  const int32_t* positions;
  int32_t n;
};

// A slot's page and row of it; page -1 where it names none.
__device__ __forceinline__ int page_of_slot(const PagePool& p, int64_t slot) {
  return uint64_t(slot) < (uint64_t(p.n_pages) << p.shift) ? int(slot >> p.shift) : -1;
}

// D / kE lanes have a row, 16 bytes of the tensors each; the wavefronts of a workgroup take neighbouring tokens of one head, whose rows lie side by side in a
// page.  K and V of kHeads heads are on their way before the first is used.  Bound by memory
// (65536 tokens of 8 heads into 4 bits: 58 us, 5.9 TB/s, back 51; rows of bf16 83 and 80, of fp32 207 and 187), but for putting rows of 8 bits, whose encoding goes through 64 bits
// for every element (120 us, back 60).
template <typename T, typename CT, int D>
__global__ __launch_bounds__(256) void put_rows(RowArgs a) {
  constexpr int kE = 16 / int(sizeof(T)), kLanes = D / kE, kTokens = 256 / kLanes, kHeads = 4;
  const int c = threadIdx.x % kLanes;
  const int64_t t = int64_t(blockIdx.x) * kTokens + threadIdx.x / kLanes;
  const int64_t slot = t < a.n ? a.slots[t] : -1;
  const int page = page_of_slot(a.pool, slot), row = int(slot & ((1 << a.pool.shift) - 1));
  if (page < 0) return;  // (lanes of a row leave together)
  const int h0 = blockIdx.y * kHeads, h1 = min(h0 + kHeads, a.pool.Hkv);
  u32x4 x[kHeads][2];
#pragma unroll
  for (int h = 0; h < kHeads; ++h)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const View& v = a.x[which];
      x[h][which] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(static_cast<const T*>(v.ptr) + t * v.sn + min(h0 + h, h1 - 1) * v.sh) + c);
    }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const int hk = h0 + h;
    if (hk >= h1) break;
    const int64_t at = a.pool.at(page, hk, row);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const u32x4 y = x[h][which];
      uint8_t* dst = which ? a.pool.v_at(page, hk, row) : a.pool.k_at(page, hk, row);
      int8_t* exps = which ? a.pool.v_exp : a.pool.k_exp;
      if constexpr (std::is_same_v<CT, Code4>) {
        int e;
        reinterpret_cast<uint32_t*>(dst)[c] = fp4_encode_block(y, e);
        if (c % 4 == 0) exps[at * (D / kBlock4) + c / 4] = int8_t(e);
      } else if constexpr (std::is_same_v<CT, uint8_t>) {
        float f[8], m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          f[i] = __uint_as_float(i & 1 ? y[i / 2] & 0xFFFF0000u : y[i / 2] << 16);
          m = fmaxf(m, fp8_magnitude(f[i]));
        }
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        const int e = fp8_row_exponent(m);
        uint32_t code[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) code[i / 4] |= uint32_t(fp8_code(f[i], e)) << (8 * (i % 4));
        reinterpret_cast<u32x2*>(dst)[c] = u32x2{code[0], code[1]};
        if (c == 0) exps[at] = int8_t(e);
      } else {
        reinterpret_cast<u32x4*>(dst)[c] = y;
      }
    }
    if (c == 0) {
      if (a.pool.score) a.pool.score[at] = 0.f;
      if (a.pool.pos) a.pool.pos[at] = a.positions[t];
    }
  }
}

template <typename T, typename CT, int D>
__global__ __launch_bounds__(256) void get_rows(RowArgs a) {
  constexpr int kE = 16 / int(sizeof(T)), kLanes = D / kE, kTokens = 256 / kLanes, kHeads = 4;
  const int c = threadIdx.x % kLanes;
  const int64_t t = int64_t(blockIdx.x) * kTokens + threadIdx.x / kLanes;
  const int64_t slot = t < a.n ? a.slots[t] : -1;
  const int page = page_of_slot(a.pool, slot), row = int(slot & ((1 << a.pool.shift) - 1));
  if (page < 0) return;
  typedef std::conditional_t<std::is_same_v<CT, Code4>, uint32_t, std::conditional_t<std::is_same_v<CT, uint8_t>, u32x2, u32x4>> Held;
  const int h0 = blockIdx.y * kHeads, h1 = min(h0 + kHeads, a.pool.Hkv);
  Held x[kHeads][2];
  int e[kHeads][2];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const int hk = min(h0 + h, h1 - 1);
    const int64_t at = a.pool.at(page, hk, row);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      x[h][which] = reinterpret_cast<const Held*>(which ? a.pool.v_at(page, hk, row) : a.pool.k_at(page, hk, row))[c];
      if constexpr (std::is_same_v<CT, Code4>)
        e[h][which] = (which ? a.pool.v_exp : a.pool.k_exp)[at * (D / kBlock4) + c / 4];
      else if constexpr (std::is_same_v<CT, uint8_t>)
        e[h][which] = (which ? a.pool.v_exp : a.pool.k_exp)[at];
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (h0 + h >= h1) break;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const View& v = a.x[which];
      u32x4 y;
      if constexpr (std::is_same_v<CT, Code4>) {
        y = fp4_decode8(x[h][which], fp4_scale(e[h][which]));
      } else if constexpr (std::is_same_v<CT, uint8_t>) {
        const float scale = pow2_f32(e[h][which]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = i % 2 ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[h][which][i / 2], scale, true))
                       : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[h][which][i / 2], scale, false));
      } else {
        y = x[h][which];
      }
      __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(static_cast<T*>(v.ptr) + t * v.sn + (h0 + h) * v.sh) + c);
    }
  }
}

template <bool PUT, typename T, typename CT, int D>
void launch_rows(const RowArgs& a, hipStream_t s) {
  constexpr int kTokens = 256 / (D * int(sizeof(T)) / 16);
  const dim3 grid(unsigned((a.n + kTokens - 1) / kTokens), unsigned((a.pool.Hkv + 3) / 4));
  if constexpr (PUT)
    put_rows<T, CT, D><<<grid, 256, 0, s>>>(a);
  else
    get_rows<T, CT, D><<<grid, 256, 0, s>>>(a);
}
template <bool PUT>
int run_rows(const d2o_pages* pages, d2o_view K, d2o_view V, int32_t n, const int64_t* slots, const int32_t* positions, void* stream) {
  RowArgs a;
  const int rc = check_pages(pages, &a.pool);
  if (rc != D2O_OK) return rc;
  if (n == 0) return D2O_OK;
  if (n < 0 || !slots || (reinterpret_cast<uintptr_t>(slots) & 7) || (reinterpret_cast<uintptr_t>(positions) & 3)) return D2O_ERR_INVALID_ARG;
  const int es = pages->dtype == D2O_BF16 ? 2 : 4, D = pages->head_dim;
  if (!dense_view_ok(K, es, true) || !dense_view_ok(V, es, true)) return D2O_ERR_INVALID_ARG;
  const int32_t counts[3] = {1, pages->n_kv_heads, n};
  if (PUT ? !pages_apart(pages) || (pages->pos && !positions) : !rows_apart(K, counts, D) || !rows_apart(V, counts, D)) return D2O_ERR_INVALID_ARG;
  if (pages->n_kv_heads > 4 * 65535 || n > (1 << 26)) return D2O_ERR_UNSUPPORTED;  // (a grid holds fewer than 2^32 threads)
  a.x[0] = to_view(K);
  a.x[1] = to_view(V);
  a.slots = slots;
  a.positions = positions;
  a.n = n;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  auto of = [&](auto t, auto ct) {
    typedef decltype(t) T;
    typedef decltype(ct) CT;
    D == 64 ? launch_rows<PUT, T, CT, 64>(a, s) : launch_rows<PUT, T, CT, 128>(a, s);
  };
  if (pages->cache_fp4)
    of(uint16_t{}, Code4{});
  else if (pages->cache_fp8)
    of(uint16_t{}, uint8_t{});
  else if (pages->dtype == D2O_BF16)
    of(uint16_t{}, uint16_t{});
  else
    of(float{}, float{});
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}

}  // namespace
}  // namespace d2o

using namespace d2o;

extern "C" int d2o_pages_put(const d2o_pages* pages, d2o_view K, d2o_view V, int32_t n_tokens, const int64_t* slots,
                             const int32_t* positions, void* stream) {
  return run_rows<true>(pages, K, V, n_tokens, slots, positions, stream);
}
extern "C" int d2o_pages_get(const d2o_pages* pages, d2o_view K, d2o_view V, int32_t n_tokens, const int64_t* slots, void* stream) {
  return run_rows<false>(pages, K, V, n_tokens, slots, nullptr, stream);
}
