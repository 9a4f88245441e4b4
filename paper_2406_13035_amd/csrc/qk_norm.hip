// Norms of queries and keys with the rotation by position (d2o_qk_norm_rope).
#include <algorithm>
#include <cmath>

#include "pages.h"

namespace d2o {
namespace {

constexpr int kMaxPairs = 64;  // head_dim / 2 at most

struct NormArgs {
  View in[2], out[2];       // Q, K
  const void* weight[2];    // [d] or null: ones
  const int32_t* positions;  // [batch][n] or null: pos0 + token
  int32_t batch, n, Hq, heads, per, rot, pos0;  // heads: Hq + Hkv; per: of a workgroup
  float eps;
  double turns[kMaxPairs];  // of pair c, by which a position turns it
};

// A row's 16 elements of a lane, in two pieces of eight.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
  u32x4 x;
  __device__ __forceinline__ void load(const uint16_t* p) { x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? x[i / 2] & 0xFFFF0000u : x[i / 2] << 16); }
  static __device__ __forceinline__ void store(uint16_t* p, const float* f) {
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __bf16(f[i]);
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, y), reinterpret_cast<u32x4*>(p));
  }
};
template <>
struct Eight<float> {
  f32x4 x[2];
  __device__ __forceinline__ void load(const float* p) {
    x[0] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
    x[1] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p) + 1);
  }
  __device__ __forceinline__ float get(int i) const { return x[i / 4][i % 4]; }
  static __device__ __forceinline__ void store(float* p, const float* f) {
    __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(p));
    __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(p) + 1);
  }
};

// y = w x / sqrt(mean(x^2) + eps), then (y_c, y_{c + rot / 2}) turned by position * base^(-2 c / rot) for c < rot / 2.  D / 16 lanes have a row: eight
// elements and the eight that are their partners (of the elements that are not turned, the next eight), so that the rotation exchanges nothing.  A wavefront has
// 1024 / D neighbouring tokens of one head at a time and goes through `per` heads with the same sines and cosines, which are formed once: the angle as a fraction
// of a turn in 64 bits (a position of 2^31 leaves 2^-24 of a turn), sine and cosine of the fraction's 32 bits in 32, then of the rest, sin(x + r) = sin x + r cos x.  U rows are on their way before the first is used.
// Bound by memory: each element is read and written once (32 + 32 heads x 32768 tokens of bf16: 223 us, 4.8 TB/s, where a copy has 5.0).  (The first rows loaded before the
// sines: no shorter for a token, 3 % longer there.)
template <typename T, int D, int U>
__global__ __launch_bounds__(256) void norm_rope(NormArgs a) {
  constexpr int kLanes = D / 16, kTokens = 64 / kLanes;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = lane % kLanes;
  const int64_t at = (int64_t(blockIdx.x) * 4 + w) * kTokens + lane / kLanes;
  const bool is = at < int64_t(a.batch) * a.n;
  const int b = is ? int(at / a.n) : 0, t = is ? int(at % a.n) : 0;
  // the lane's two pieces: elements e0 .. e0 + 7 and e1 .. e1 + 7
  const bool turned = c < a.rot / 16;
  const int e0 = turned ? c * 8 : a.rot + (c - a.rot / 16) * 16, e1 = turned ? c * 8 + a.rot / 2 : e0 + 8;
  float sn[8], cs[8];
  const double pos = a.positions ? double(is ? a.positions[at] : 0) : double(a.pos0) + double(t);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double x = turned ? pos * a.turns[c * 8 + i] : 0.0;
    const double part = x - rint(x);
    const float near = float(part), rest = float((part - double(near)) * 6.283185307179586);
    float s, c;
    sincospif(2.f * near, &s, &c);
    sn[i] = fmaf(rest, c, s);
    cs[i] = fmaf(-rest, s, c);
  }
  float wt[2][16];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      wt[which][i] = a.weight[which] ? Elem<T>::to_f32(static_cast<const T*>(a.weight[which])[(i < 8 ? e0 : e1) + i % 8]) : 1.f;
  const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads);
  for (int h = h0; h < h1; h += U) {
    Eight<T> x[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hh = min(h + u, h1 - 1), which = hh >= a.Hq, head = which ? hh - a.Hq : hh;
      const View& v = a.in[which];
      const T* row = static_cast<const T*>(v.ptr) + b * v.sb + head * v.sh + t * v.sn;
      x[u][0].load(row + e0);
      x[u][1].load(row + e1);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= h1) break;
      const int which = h + u >= a.Hq, head = which ? h + u - a.Hq : h + u;
      float y[16], ss = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        y[i] = x[u][i / 8].get(i % 8);
        ss = fmaf(y[i], y[i], ss);
      }
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) ss += __shfl_xor(ss, o, 64);
      float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
      const bool far = !(ss < 1e37f);
      if (__any(far)) {  // squares that left 32 bits: such rows once more in 64, before the factor as a float loses bits
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) s = fma(double(y[i]), double(y[i]), s);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) s += __shfl_xor(s, o, 64);
        const double rd = 1.0 / sqrt(s * (1.0 / D) + double(a.eps));
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = far ? float(double(y[i]) * rd) : y[i];
        r = far ? 1.f : r;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = y[i] * r * (which ? wt[1][i] : wt[0][i]);
      float o[16];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        o[i] = turned ? y[i] * cs[i] - y[i + 8] * sn[i] : y[i];
        o[i + 8] = turned ? y[i + 8] * cs[i] + y[i] * sn[i] : y[i + 8];
      }
      if (is) {
        const View& v = a.out[which];
        T* row = static_cast<T*>(v.ptr) + b * v.sb + head * v.sh + t * v.sn;
        Eight<T>::store(row + e0, o);
        Eight<T>::store(row + e1, o + 8);
      }
    }
  }
}

template <typename T, int D>
void launch_norm(NormArgs& a, hipStream_t s) {
  constexpr int kTokens = 4 * 1024 / D;  // of a workgroup
  const int64_t blocks = (int64_t(a.batch) * a.n + kTokens - 1) / kTokens;
  // heads of a workgroup: as many as leave four workgroups per CU
  const int64_t want = std::max<int64_t>(1, 1024 / blocks);
  a.per = int(std::max<int64_t>(1, a.heads / want));
  const unsigned parts = unsigned((a.heads + a.per - 1) / a.per);
  constexpr int U = sizeof(T) == 2 ? 4 : 2;
  norm_rope<T, D, U><<<dim3(unsigned(blocks), parts), 256, 0, s>>>(a);
}

}  // namespace
}  // namespace d2o

using namespace d2o;

extern "C" int d2o_qk_norm_rope(int32_t batch, int32_t n, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                d2o_view Q, d2o_view K, const void* q_weight, const void* k_weight, double eps, int32_t rot_dim,
                                const int32_t* positions, int32_t pos0, double rope_base, d2o_view Q_out, d2o_view K_out,
                                void* stream) {
  if (batch < 1 || n < 1 || n_q_heads < 0 || n_kv_heads < 0 || int64_t(n_q_heads) + n_kv_heads < 1) return D2O_ERR_INVALID_ARG;
  if (dtype != D2O_F32 && dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return D2O_ERR_UNSUPPORTED;
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16) return D2O_ERR_INVALID_ARG;
  if (!(eps >= 1e-20) || !(eps <= 1.0) || !(rope_base > 1.0) || !std::isfinite(rope_base)) return D2O_ERR_INVALID_ARG;
  const int es = dtype == D2O_BF16 ? 2 : 4;
  const d2o_view in[2] = {Q, K}, out[2] = {Q_out, K_out};
  const int32_t heads[2] = {n_q_heads, n_kv_heads};
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    if (!dense_view_ok(in[i], es, true) || !dense_view_ok(out[i], es, true)) return D2O_ERR_INVALID_ARG;
    if (!rows_apart(out[i], {batch, heads[i], n}, head_dim)) return D2O_ERR_INVALID_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(q_weight) | reinterpret_cast<uintptr_t>(k_weight)) & (es - 1)) return D2O_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(positions) & 3) return D2O_ERR_INVALID_ARG;
  if (int64_t(n_q_heads) + n_kv_heads > 65535 || int64_t(batch) * n > (int64_t(1) << 28)) return D2O_ERR_UNSUPPORTED;
  NormArgs a;
  for (int i = 0; i < 2; ++i) {
    a.in[i] = to_view(in[i]);
    a.out[i] = to_view(out[i]);
  }
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.positions = positions;
  a.batch = batch;
  a.n = n;
  a.Hq = n_q_heads;
  a.heads = n_q_heads + n_kv_heads;
  a.rot = rot_dim;
  a.pos0 = pos0;
  a.eps = float(eps);
  // base^(-2 c / rot) / (2 pi) as a product, in more bits than the 64-bit result has
  const long double step = rot_dim ? std::pow(static_cast<long double>(rope_base), -2.0L / rot_dim) : 0.0L;
  long double turns = 0.15915494309189533576888376337251436L;
  for (int c = 0; c < kMaxPairs; ++c, turns *= step) a.turns[c] = c < rot_dim / 2 ? double(turns) : 0.0;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == D2O_BF16)
    head_dim == 64 ? launch_norm<uint16_t, 64>(a, s) : launch_norm<uint16_t, 128>(a, s);
  else
    head_dim == 64 ? launch_norm<float, 64>(a, s) : launch_norm<float, 128>(a, s);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
