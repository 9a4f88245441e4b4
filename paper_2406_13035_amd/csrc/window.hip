// Causal prompt attention over a window of recent tokens and a few first ones (d2o_window_attend).
#include <algorithm>

#include "pages.h"

namespace d2o {
namespace {

struct WindowArgs {
  View q, k, v, o;
  const int32_t* lens;
  int32_t n, Hq, G, window, n_sink;  // window: at least 1, INT32_MAX without one
};

// One wavefront per query: 64 keys at a time, a key per lane for the logits, D / 64 columns per lane for the output.
template <typename T, int D>
__global__ __launch_bounds__(64) void window_row(WindowArgs a) {
  constexpr float kLog2e = 1.4426950408889634f;
  __shared__ float qs[D];
  const int i = blockIdx.x, hq = blockIdx.y % a.Hq, b = blockIdx.y / a.Hq, hk = hq / a.G, lane = threadIdx.x;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  if (i >= n) return;
  const T* q = static_cast<const T*>(a.q.ptr) + b * a.q.sb + hq * a.q.sh + i * a.q.sn;
  const T* k = static_cast<const T*>(a.k.ptr) + b * a.k.sb + hk * a.k.sh;
  const T* v = static_cast<const T*>(a.v.ptr) + b * a.v.sb + hk * a.v.sh;
  for (int c = lane; c < D; c += 64) qs[c] = Elem<T>::to_f32(q[c]) * (kLog2e / sqrtf(float(D)));
  __syncthreads();
  const int lo = max(0, int(int64_t(i) + 1 - a.window)), sinks = min(a.n_sink, lo), seen = sinks + i + 1 - lo;
  float m = -1e30f, l = 0.f, o[D / 64] = {};
  for (int t0 = 0; t0 < seen; t0 += 64) {
    const int t = t0 + lane, j = t < sinks ? t : lo + t - sinks;
    float s = -INFINITY;
    if (t < seen) {
      s = 0.f;
      for (int c = 0; c < D; ++c) s = fmaf(qs[c], Elem<T>::to_f32(k[j * a.k.sn + c]), s);
    }
    const float mn = fmaxf(m, wave_max(s)), p = t < seen ? exp2f(s - mn) : 0.f, f = exp2f(m - mn);
    m = mn;
    l = l * f + wave_sum(p);
    for (int c = 0; c < D / 64; ++c) o[c] *= f;
    for (int u = 0; u < min(64, seen - t0); ++u) {
      const float pu = __shfl(p, u, 64);
      const int64_t ju = __shfl(j, u, 64);
      for (int c = 0; c < D / 64; ++c) o[c] = fmaf(pu, Elem<T>::to_f32(v[ju * a.v.sn + c * 64 + lane]), o[c]);
    }
  }
  T* out = static_cast<T*>(a.o.ptr) + b * a.o.sb + hq * a.o.sh + i * a.o.sn;
  for (int c = 0; c < D / 64; ++c) out[c * 64 + lane] = Elem<T>::from_f32(o[c] / l);
}

int check_window(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (batch < 1 || n < 1 || n_kv_heads < 1) return D2O_ERR_INVALID_ARG;
  if (dtype != D2O_F32 && dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return D2O_ERR_UNSUPPORTED;
  return D2O_OK;
}

size_t window_bytes(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) { return 256; }

}  // namespace
}  // namespace d2o

using namespace d2o;

extern "C" int d2o_window_workspace_bytes(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                          size_t* bytes) {
  const int rc = check_window(batch, n, n_kv_heads, head_dim, dtype);
  if (rc != D2O_OK) return rc;
  if (!bytes) return D2O_ERR_INVALID_ARG;
  *bytes = window_bytes(batch, n, n_kv_heads, head_dim, dtype);
  return D2O_OK;
}

extern "C" int d2o_window_attend(int32_t batch, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                 int32_t dtype, d2o_view Q, d2o_view K, d2o_view V, const int32_t* lens, int32_t window,
                                 int32_t n_sink, d2o_view O, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_window(batch, n, n_kv_heads, head_dim, dtype);
  if (rc != D2O_OK) return rc;
  const int es = dtype == D2O_BF16 ? 2 : 4;
  if (n_q_heads < 1 || n_q_heads % n_kv_heads || window < 0 || n_sink < 0) return D2O_ERR_INVALID_ARG;
  for (const d2o_view* v : {&Q, &K, &V, &O})
    if (!dense_view_ok(*v, es, true)) return D2O_ERR_INVALID_ARG;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < window_bytes(batch, n, n_kv_heads, head_dim, dtype)) return D2O_ERR_CAPACITY;
  if (int64_t(batch) * n_q_heads > 65535) return D2O_ERR_UNSUPPORTED;
  WindowArgs a{to_view(Q), to_view(K), to_view(V), to_view(O), lens, n, n_q_heads, n_q_heads / n_kv_heads,
               window ? window : INT32_MAX, n_sink};
  const dim3 grid(n, batch * n_q_heads);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == D2O_BF16)
    head_dim == 64 ? window_row<uint16_t, 64><<<grid, 64, 0, s>>>(a) : window_row<uint16_t, 128><<<grid, 64, 0, s>>>(a);
  else
    head_dim == 64 ? window_row<float, 64><<<grid, 64, 0, s>>>(a) : window_row<float, 128><<<grid, 64, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
