// Caches in pages: what the kernels of pages_step.hip and pages_evict.hip share.
#pragma once

#include "d2o_internal.h"
#include "device_utils.h"

namespace d2o {

// d2o_pages as the kernels take it; row strides in bytes.
struct PagePool {
  uint8_t* K;
  uint8_t* V;
  int64_t k_page, k_head, k_row, v_page, v_head, v_row;  // bytes
  int8_t* k_exp;
  int8_t* v_exp;
  float* score;
  int32_t* pos;
  const int32_t* table;
  int32_t shift, n_pages, max_pages, Hkv;  // page_size = 1 << shift

  // The page of entry s of sequence b, -1 where the table names none of the pool.
  __device__ __forceinline__ int page_of(int b, int s) const {
    const int p = table[int64_t(b) * max_pages + (s >> shift)];
    return uint32_t(p) < uint32_t(n_pages) ? p : -1;
  }
  __device__ __forceinline__ int row_of(int s) const { return s & ((1 << shift) - 1); }
  __device__ __forceinline__ uint8_t* k_at(int page, int h, int s) const {
    return K + page * k_page + h * k_head + row_of(s) * k_row;
  }
  __device__ __forceinline__ uint8_t* v_at(int page, int h, int s) const {
    return V + page * v_page + h * v_head + row_of(s) * v_row;
  }
  // index into score, pos, k_exp and v_exp
  __device__ __forceinline__ int64_t at(int page, int h, int s) const {
    return ((int64_t(page) * Hkv + h) << shift) + row_of(s);
  }
};

// Checks a description and translates it; D2O_OK or the status to return.
int check_pages(const d2o_pages* p, PagePool* out);
// A view of q, k, v or out tensors of `esize` bytes per element: present, 16-byte aligned, strides in whole 16 bytes, not negative.
bool dense_view_ok(const d2o_view& v, int esize, bool rows);
// The same of a view that is written, of counts[i] batches (pages), heads and rows of d elements: no two of them start at one place or inside each other.
bool rows_apart(const d2o_view& v, const int32_t (&counts)[3], int d);
bool pages_apart(const d2o_pages* p);  // of both pools

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }
size_t pages_step_bytes(const d2o_pages* p, int32_t max_len);   // workspace of d2o_pages_step
size_t pages_evict_bytes(const d2o_pages* p, int32_t max_len);  // of d2o_pages_fill and d2o_pages_evict

// 8-bit rows: x as codes with the row's exponent (fp64 inside, exact), one element; infinities and NaN as NaN, and the exponent is
// that of the others.
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ uint8_t fp8_code(float x, int e) { return is_finite(x) ? fp8_encode(ldexp(double(x), -e)) : uint8_t(0x7F); }
__device__ __forceinline__ float fp8_magnitude(float x) { return is_finite(x) ? fabsf(x) : 0.f; }

}  // namespace d2o
