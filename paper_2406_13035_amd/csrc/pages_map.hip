// Block tables and slot maps from the lengths of requests (d2o_pages_map).
#include <algorithm>

#include "pages.h"

namespace d2o {
namespace {

constexpr int kThreads = 1024;

struct MapArgs {
  int32_t* table;
  const int32_t* lens;
  const int32_t* change;
  int32_t* ring;         // [n_pages] the free pages: `count` of them from `head` on, around the end
  const int32_t* state;  // head, count
  int32_t *lens_out, *state_out, *first, *positions;
  int64_t* slots;
  int32_t* plan;  // [4][batch] as in Plan, then head and count (two launches)
  int32_t batch, shift, n_pages, max_pages, rows;
};

// What the scan over the sequences leaves for the tokens and pages.
struct Plan {
  const int32_t* before;  // [batch] entries before the call
  const int32_t* after;   // and after it
  const int32_t* take;    // first of the pages that it takes, counted from the ring's head
  const int32_t* give;    // first of the places of those it gives back, counted from behind the ring's last page
  const int32_t* first;   // [batch + 1] first row of its new tokens
  int32_t head, count;
};

__device__ __forceinline__ int pages_of(int64_t n, int shift) { return int((n + (int64_t(1) << shift) - 1) >> shift); }

// Inclusive sums over the workgroup of two values, and what all threads together have.
__device__ __forceinline__ void sums(int64_t (&v)[2], int64_t (&all)[2], int64_t (*buf)[kThreads / 64]) {
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t x = __shfl_up((long long)v[0], o, 64), y = __shfl_up((long long)v[1], o, 64);
    if (lane >= o) {
      v[0] += x;
      v[1] += y;
    }
  }
  __syncthreads();
  if (lane == 63) {
    buf[0][w] = v[0];
    buf[1][w] = v[1];
  }
  __syncthreads();
  all[0] = all[1] = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    if (i == w) {
      v[0] += all[0];
      v[1] += all[1];
    }
    all[0] += buf[0][i];
    all[1] += buf[1][i];
  }
}

// The sequences in their order, one per thread and round.  A sequence is served if its wishes and those of all before it, served or not, can be: the
// sums of what is wished for then rise together with the sums of what is taken, and two scans replace a walk from sequence to sequence.
__device__ __forceinline__ void scan(const MapArgs& a, int32_t* before, int32_t* after, int32_t* take, int32_t* give, int32_t* first,
                                     int32_t& head, int32_t& count) {
  __shared__ int64_t buf[2][kThreads / 64];
  __shared__ int taken;
  const int tid = threadIdx.x;
  head = a.state[0];
  if (uint32_t(head) >= uint32_t(a.n_pages)) head = 0;
  count = min(max(a.state[1], 0), a.n_pages);
  if (tid == 0) taken = 0;
  const int64_t most = int64_t(a.max_pages) << a.shift;
  int64_t wished[2] = {0, 0}, done[2] = {0, 0};  // tokens and pages asked for, tokens and pages given
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid;
    const bool is = b < a.batch;
    const int64_t len = is ? min(max(int64_t(a.lens[b]), int64_t(0)), most) : 0, change = is ? a.change[b] : 0;
    int64_t gain = max(change, int64_t(0)), loss = min(max(-change, int64_t(0)), len);
    if (len + gain > most || len + gain > 0x7FFFFFFF) gain = 0;
    const int held = pages_of(len, a.shift), need = pages_of(len + gain, a.shift) - held;
    int64_t v[2] = {gain, need}, all[2];
    sums(v, all, buf);
    const bool served = wished[0] + v[0] <= a.rows && (need == 0 || wished[1] + v[1] <= count);
    const int64_t t0 = wished[1] + v[1] - need;
    wished[0] += all[0];
    wished[1] += all[1];
    if (!served) gain = 0;
    if (served && need) atomicMax(&taken, int(t0) + need);
    const int64_t now = len + gain - loss;
    const int back = loss ? held - pages_of(now, a.shift) : 0;
    int64_t u[2] = {gain, back}, both[2];
    sums(u, both, buf);
    if (is) {
      before[b] = int32_t(len);
      after[b] = int32_t(now);
      take[b] = int32_t(min(t0, int64_t(a.n_pages)));
      give[b] = int32_t(min(done[1] + u[1] - back, int64_t(a.n_pages)));
      first[b] = int32_t(done[0] + u[0] - gain);
      if (first != a.first) a.first[b] = first[b];
      a.lens_out[b] = int32_t(now);
    }
    done[0] += both[0];
    done[1] += both[1];
  }
  __syncthreads();
  if (tid == 0) {
    first[a.batch] = int32_t(done[0]);
    if (first != a.first) a.first[a.batch] = int32_t(done[0]);
    a.state_out[0] = int32_t((int64_t(head) + taken) % a.n_pages);
    a.state_out[1] = int32_t(count - taken + min(done[1], int64_t(a.n_pages - count)));
  }
}

// Row `row` of the packed tokens, of sequence b (-1: of none).  The first token of a new page enters it in the block table.
__device__ __forceinline__ void place(const MapArgs& a, const Plan& p, int row, int b) {
  int64_t slot = -1;
  int at = 0;
  if (b >= 0) {
    const int len = p.before[b];
    at = len + (row - p.first[b]);
    const int index = at >> a.shift, fresh = index - pages_of(len, a.shift), in_page = at & ((1 << a.shift) - 1);
    int32_t* entry = a.table + int64_t(b) * a.max_pages + index;
    int page;
    if (fresh >= 0) {
      page = a.ring[(int64_t(p.head) + p.take[b] + fresh) % a.n_pages];
      if (in_page == 0) *entry = page;
    } else {
      page = *entry;
    }
    if (uint32_t(page) < uint32_t(a.n_pages)) slot = (int64_t(page) << a.shift) + in_page;
  }
  a.slots[row] = slot;
  a.positions[row] = at;
}

// Pages that hold no entry any more, to the ring's end: kGive of a sequence at a time, by one wavefront.
constexpr int kGive = 256;
__device__ __forceinline__ void give_back(const MapArgs& a, const Plan& p, int b, int part) {
  const int now = pages_of(p.after[b], a.shift), held = pages_of(p.before[b], a.shift), lane = threadIdx.x & 63;
  const int i0 = now + part * kGive + lane, end = min(held, now + (part + 1) * kGive);
#pragma unroll
  for (int u = 0; u < kGive / 64; ++u) {
    const int i = i0 + u * 64;
    const int64_t at = int64_t(p.give[b]) + (i - now);
    if (i < end && at < a.n_pages - p.count) a.ring[(int64_t(p.head) + p.count + at) % a.n_pages] = a.table[int64_t(b) * a.max_pages + i];
  }
}

// The last sequence that starts at or before `row`, of `first` [n + 1] from lo on (first[lo] <= row < first[hi]).
__device__ __forceinline__ int owner(const int32_t* first, int row, int lo, int hi) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= row)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Small batches: everything by one workgroup.  Bound by latency: the lengths, two scans, a page's number, the slot (64 sequences: 6.7 us; 256 with 300000 tokens, by two
// launches, 6 and 9).
constexpr int kSmall = 1024, kSmallRows = 4096, kSmallParts = 1024;
__global__ __launch_bounds__(kThreads) void map_small(MapArgs a) {
  __shared__ int32_t before[kSmall], after[kSmall], take[kSmall], give[kSmall], first[kSmall + 1];
  int32_t head, count;
  scan(a, before, after, take, give, first, head, count);
  __syncthreads();
  const Plan p{before, after, take, give, first, head, count};
  const int total = first[a.batch];
  for (int row = threadIdx.x; row < a.rows; row += kThreads) place(a, p, row, row < total ? owner(first, row, 0, a.batch) : -1);
  const int parts = (a.max_pages + kGive - 1) / kGive;
  for (int i = threadIdx.x >> 6; i < a.batch * parts; i += kThreads / 64)
    if (after[i / parts] < before[i / parts]) give_back(a, p, i / parts, i % parts);
}

// Larger ones: the scan ...
__global__ __launch_bounds__(kThreads) void map_scan(MapArgs a) {
  int32_t head, count;
  scan(a, a.plan, a.plan + a.batch, a.plan + 2 * int64_t(a.batch), a.plan + 3 * int64_t(a.batch), a.first, head, count);
  if (threadIdx.x == 0) {
    a.plan[4 * int64_t(a.batch)] = head;
    a.plan[4 * int64_t(a.batch) + 1] = count;
  }
}
// ... then tokens and pages by many workgroups: `blocks` of them the tokens, kPlace each, the others the pages.  A token's sequence is looked up among samples of the
// first rows in LDS, then between two of them.
constexpr int kPlace = 1024, kSamples = 2048;
__global__ __launch_bounds__(256) void map_place(MapArgs a, int blocks) {
  const Plan p{a.plan, a.plan + a.batch, a.plan + 2 * int64_t(a.batch), a.plan + 3 * int64_t(a.batch), a.first, a.plan[4 * int64_t(a.batch)],
               a.plan[4 * int64_t(a.batch) + 1]};
  if (int(blockIdx.x) >= blocks) {
    const int parts = (a.max_pages + kGive - 1) / kGive;
    const int64_t i = int64_t(blockIdx.x - blocks) * 4 + (threadIdx.x >> 6);
    const int b = int(i / parts);
    if (b < a.batch && p.after[b] < p.before[b]) give_back(a, p, b, int(i % parts));
    return;
  }
  __shared__ int32_t sample[kSamples];
  const int step = (a.batch + kSamples - 1) / kSamples, n = (a.batch + step - 1) / step;  // first[0], first[step], ..
  const int total = a.first[a.batch], row0 = blockIdx.x * kPlace;
  if (row0 < total) {
    for (int i = threadIdx.x; i < n; i += 256) sample[i] = a.first[i * step];
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < kPlace / 256; ++u) {
    const int row = row0 + u * 256 + threadIdx.x;
    if (row >= a.rows) break;
    int b = -1;
    if (row < total) {
      const int s = owner(sample, row, 0, n);
      b = step == 1 ? s : owner(a.first, row, s * step, min((s + 1) * step, a.batch));
    }
    place(a, p, row, b);
  }
}

bool is_small(int32_t batch, int32_t max_pages, int32_t rows) {
  return batch <= kSmall && rows <= kSmallRows && int64_t(batch) * ((max_pages + kGive - 1) / kGive) <= kSmallParts;
}

}  // namespace
}  // namespace d2o

using namespace d2o;

extern "C" int d2o_pages_map_workspace_bytes(int32_t batch, int32_t max_pages, int32_t max_tokens, size_t* bytes) {
  if (batch < 1 || max_pages < 1 || max_tokens < 0 || !bytes) return D2O_ERR_INVALID_ARG;
  *bytes = is_small(batch, max_pages, max_tokens) ? 0 : round256((4 * size_t(batch) + 2) * sizeof(int32_t));
  return D2O_OK;
}

extern "C" int d2o_pages_map(int32_t batch, int32_t page_size, int32_t n_pages, int32_t max_pages, int32_t* page_table,
                             const int32_t* lens, const int32_t* change, int32_t* free_pages, const int32_t* free_state,
                             int32_t max_tokens, int32_t* lens_out, int32_t* free_state_out, int32_t* first, int64_t* slots,
                             int32_t* positions, void* workspace, size_t workspace_bytes, void* stream) {
  if (batch < 1 || n_pages < 1 || max_pages < 1 || max_tokens < 0) return D2O_ERR_INVALID_ARG;
  if (page_size < 1 || page_size > 1024 || (page_size & (page_size - 1))) return D2O_ERR_INVALID_ARG;
  if (int64_t(max_pages) * page_size > 0x7FFF0000) return D2O_ERR_INVALID_ARG;
  const void* needed[] = {page_table, lens, change, free_pages, free_state, lens_out, free_state_out, first};
  for (const void* p : needed)
    if (!p || (reinterpret_cast<uintptr_t>(p) & 3)) return D2O_ERR_INVALID_ARG;
  if (max_tokens > 0 && (!slots || !positions)) return D2O_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(slots) & 7) || (reinterpret_cast<uintptr_t>(positions) & 3)) return D2O_ERR_INVALID_ARG;
  size_t need;
  const int rc = d2o_pages_map_workspace_bytes(batch, max_pages, max_tokens, &need);
  if (rc != D2O_OK) return rc;
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < need) return D2O_ERR_CAPACITY;
  const int64_t blocks = (int64_t(max_tokens) + kPlace - 1) / kPlace;
  const int64_t parts = (int64_t(batch) * ((max_pages + kGive - 1) / kGive) + 3) / 4;
  if (blocks + parts > 0xFFFFFF) return D2O_ERR_UNSUPPORTED;  // (a grid holds fewer than 2^32 threads)
  const MapArgs a{page_table, lens, change, free_pages, free_state, lens_out, free_state_out, first, positions, slots,
                  static_cast<int32_t*>(workspace), batch, __builtin_ctz(unsigned(page_size)), n_pages, max_pages, max_tokens};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (need == 0) {
    map_small<<<1, kThreads, 0, s>>>(a);
  } else {
    map_scan<<<1, kThreads, 0, s>>>(a);
    map_place<<<dim3(unsigned(blocks + parts)), 256, 0, s>>>(a, int(blocks));
  }
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
