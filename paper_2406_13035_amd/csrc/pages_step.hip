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
  if (int64_t(p->max_pages) * p->page_size > 0x7FFFFFFF) return D2O_ERR_INVALID_ARG;
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

struct StepArgs {
  PagePool pool;
  View q, kn, vn, out;
  const int32_t* lens;
  const int32_t* positions;
  float* logits;  // [B][Hq][max_len]
  int32_t Hq, G, max_len, window, n_sink;
};

template <typename CT>
__device__ __forceinline__ float value_at(const uint8_t* row, int i) {
  return Elem<CT>::to_f32(reinterpret_cast<const CT*>(row)[i]);
}

// T: type of q, k, v and out; CT: of the cache's rows.  One workgroup per (sequence, KV head).
template <typename T, typename CT, int D>
__global__ __launch_bounds__(256) void step_kernel(StepArgs a) {
  __shared__ float red[4];
  __shared__ float qs[D];
  constexpr float kLog2e = 1.4426950408889634f;
  const int Hkv = a.pool.Hkv, b = blockIdx.x / Hkv, hk = blockIdx.x % Hkv, tid = threadIdx.x;
  const int n = min(a.lens[b], a.max_len);
  T* out = static_cast<T*>(a.out.ptr) + b * a.out.sb;
  if (n <= 0) {
    for (int i = tid; i < a.G * D; i += 256) out[(hk * a.G + i / D) * a.out.sh + i % D] = Elem<T>::from_f32(0.f);
    return;
  }
  const int64_t P = a.positions ? a.positions[b] : n - 1;
  if (a.kn.ptr && a.lens[b] <= a.max_len) {
    const int page = a.pool.page_of(b, n - 1);
    if (page >= 0) {
      const T* src[2] = {static_cast<const T*>(a.kn.ptr) + b * a.kn.sb + hk * a.kn.sh,
                         static_cast<const T*>(a.vn.ptr) + b * a.vn.sb + hk * a.vn.sh};
      const int64_t at = a.pool.at(page, hk, n - 1);
      if (tid < 128) {
        const int which = tid >> 6, lane = tid & 63;
        CT* dst = reinterpret_cast<CT*>(which ? a.pool.v_at(page, hk, n - 1) : a.pool.k_at(page, hk, n - 1));
        if constexpr (sizeof(CT) == 1) {
          float m = 0.f;
          for (int i = lane; i < D; i += 64) m = fmaxf(m, fabsf(Elem<T>::to_f32(src[which][i])));
          const int e = fp8_row_exponent(wave_max(m));
          for (int i = lane; i < D; i += 64) dst[i] = fp8_code(Elem<T>::to_f32(src[which][i]), e);
          if (lane == 0) (which ? a.pool.v_exp : a.pool.k_exp)[at] = int8_t(e);
        } else {
          for (int i = lane; i < D; i += 64) dst[i] = src[which][i];
        }
      }
      if (tid == 0) {
        if (a.pool.score) a.pool.score[at] = 0.f;
        if (a.pool.pos) a.pool.pos[at] = int32_t(P);
      }
    }
    __threadfence_block();
    __syncthreads();
  }
  auto seen = [&](int s, int page) {
    if (page < 0) return false;
    if (a.window == 0) return true;
    const int64_t p = a.pool.pos ? a.pool.pos[a.pool.at(page, hk, s)] : s;
    return p > P - a.window || p < a.n_sink;
  };
  for (int g = 0; g < a.G; ++g) {
    const int hq = hk * a.G + g;
    const T* q = static_cast<const T*>(a.q.ptr) + b * a.q.sb + hq * a.q.sh;
    float* lg = a.logits + (int64_t(b) * a.Hq + hq) * a.max_len;
    __syncthreads();
    if (tid < D) qs[tid] = Elem<T>::to_f32(q[tid]) * (kLog2e / sqrtf(float(D)));
    __syncthreads();
    float m = -INFINITY;
    for (int s = tid; s < n; s += 256) {
      const int page = a.pool.page_of(b, s);
      float x = -INFINITY;
      if (seen(s, page)) {
        const uint8_t* row = a.pool.k_at(page, hk, s);
        x = 0.f;
        for (int i = 0; i < D; ++i) x = fmaf(qs[i], value_at<CT>(row, i), x);
        if constexpr (sizeof(CT) == 1) x = ldexpf(x, a.pool.k_exp[a.pool.at(page, hk, s)]);
      }
      lg[s] = x;
      m = fmaxf(m, x);
    }
    m = wave_max(m);
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    __syncthreads();
    float l = 0.f;
    for (int s = tid; s < n; s += 256) {
      const float p = seen(s, a.pool.page_of(b, s)) ? exp2f(lg[s] - m) : 0.f;
      lg[s] = p;
      l += p;
    }
    l = wave_sum(l);
    if ((tid & 63) == 0) red[tid >> 6] = l;
    __threadfence_block();
    __syncthreads();
    l = (red[0] + red[1]) + (red[2] + red[3]);
    bool any = false;
    if (tid < D) {
      float o = 0.f;
      for (int s = 0; s < n; ++s) {
        const int page = a.pool.page_of(b, s);
        if (!seen(s, page)) continue;
        any = true;
        float v = value_at<CT>(a.pool.v_at(page, hk, s), tid);
        if constexpr (sizeof(CT) == 1) v = ldexpf(v, a.pool.v_exp[a.pool.at(page, hk, s)]);
        o = fmaf(lg[s], v, o);
      }
      out[hq * a.out.sh + tid] = Elem<T>::from_f32(any ? o / l : 0.f);
    }
    if (a.pool.score)
      for (int s = tid; s < n; s += 256) {
        const int page = a.pool.page_of(b, s);
        if (seen(s, page)) a.pool.score[a.pool.at(page, hk, s)] += lg[s] / l;
      }
  }
}

template <typename T, typename CT>
void launch_step(const StepArgs& a, int batch, int D, hipStream_t s) {
  const dim3 grid(batch * a.pool.Hkv);
  if (D == 64)
    step_kernel<T, CT, 64><<<grid, 256, 0, s>>>(a);
  else
    step_kernel<T, CT, 128><<<grid, 256, 0, s>>>(a);
}

}  // namespace

size_t pages_step_bytes(const d2o_pages* p, int32_t max_len) {
  return round256(size_t(p->batch) * p->n_q_heads * max_len * sizeof(float));
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
  if (max_len > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < pages_step_bytes(pages, max_len)) return D2O_ERR_CAPACITY;
  a.q = to_view(q);
  a.kn = to_view(k_new);
  a.vn = to_view(v_new);
  a.out = to_view(out);
  a.lens = lens;
  a.positions = positions;
  a.logits = static_cast<float*>(workspace);
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
