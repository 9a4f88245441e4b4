// Causal prompt attention over a window of recent tokens and a few first ones (d2o_window_attend).
//
// Query i sees the keys j <= i with j > i - window or j < n_sink.  A workgroup owns a block of query rows and walks the 64-key (bf16)
// or 32-key (fp32) tiles that any of its rows sees: those of the first tokens, then those from its first row's window start to its
// last row.  Both kernels keep S^T = K Q^T in the matrix core's accumulator layout, where a lane owns one query, so that a row's
// maximum and sum are taken in registers, and choose the keys' order such that these registers are the operand of
// O^T = V^T P^T as they are.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace d2o {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kFloor = -3e38f;  // exponent reference before a row has seen a key

struct WindowArgs {
  View q, k, v, o;
  const int32_t* lens;
  int32_t n, Hq, G, window, n_sink;  // window and n_sink: at most n; window: at least 1
  float bias;  // a row sees fewer than 2^bias keys
  // bf16: transposed values and a flag per tile of 64 keys
  uint16_t* vt;  // [B][Hkv][tiles][D][64], infinities and NaN as zero
  float* odd;    // [B][Hkv][tiles] 1 where the tile had any
  int32_t tiles, blocks, reverse, share;  // share: log2 of the query heads of a block
};

// The tiles of BN keys that the rows [r0, r1] see: `sinks` tiles of first tokens, then those from `rest0`.
struct Tiles {
  int sinks, rest0, count;
  __device__ __forceinline__ Tiles(const WindowArgs& a, int r0, int r1, int BN) {
    const int lo = max(0, r0 + 1 - a.window);
    sinks = (min(a.n_sink, r1 + 1) + BN - 1) / BN;
    rest0 = max(lo / BN, sinks);
    const int end = r1 / BN + 1;
    rest0 = min(rest0, end);
    sinks = min(sinks, end);
    count = sinks + end - rest0;
  }
  __device__ __forceinline__ int tile(int t) const { return t < sinks ? t : rest0 + t - sinks; }
};

__device__ __forceinline__ bool sees(const WindowArgs& a, int i, int j) {
  return j <= i && (j > i - a.window || j < a.n_sink);
}
// Whether any of the rows [r0, r1] sees any of the keys [k0, k1], and whether each sees all of them.
__device__ __forceinline__ bool any_seen(const WindowArgs& a, int r0, int r1, int k0, int k1) {
  return k0 <= r1 && (k1 > r0 - a.window || k0 < a.n_sink);
}
__device__ __forceinline__ bool all_seen(const WindowArgs& a, int r0, int r1, int k0, int k1) {
  return k1 <= r0 && (k0 > r1 - a.window || k1 < a.n_sink);
}

// A block's rows are those of BM / 2^share tokens and 2^share query heads of a group, wavefront by wavefront: the heads share K and V, and fewer
// tokens see fewer tiles (8192 tokens, 32 heads on 8, window 1024: 249 -> 226 us).
// Workgroup number -> (block of rows, heads and sequence).  Workgroups go to the chip's eight XCDs, each with an L2 of its own, in
// turn; here each XCD gets a contiguous run of (head, block), so that blocks that share most of their window meet in one L2.
// Without a window (reverse) the work grows with the block's position: the longest blocks of all heads first.
__device__ __forceinline__ void place(const WindowArgs& a, int heads, int& block, int& hz) {
  constexpr int kXcd = 8;
  const int total = a.blocks * heads, lin = blockIdx.x;
  if (a.reverse) {
    block = a.blocks - 1 - lin / heads;
    hz = lin % heads;
    return;
  }
  const int xcd = lin % kXcd, q = total / kXcd, r = total % kXcd, at = xcd * q + min(xcd, r) + lin / kXcd;
  hz = at / a.blocks;
  block = at % a.blocks;
}

__device__ __forceinline__ float max_halves(float v) {  // with the lane 32 away
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return fmaxf(__int_as_float(s[0]), __int_as_float(s[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(s[0]) + __int_as_float(s[1]);
}

// ---- bf16 ----------------------------------------------------------------------------------
// V goes to the matrix core as it is, in bf16, and a probability as the sum of two bf16 terms, p rounded and what that left of it, which hold
// sixteen bits: 2^-17 of p, where one bf16 term would cost 2^-8, as much as the output's own rounding, and one fp16 term 2^-11.  (fp16 also needs
// V brought into its range by powers of two, which no scaling per tile does for values that differ by more than 2^30.)  P V thus takes two
// products per operand read from LDS (32 heads x 32768 tokens, window 4096: 2.28 ms with the first term alone, 2.96 with both).  An infinity or
// NaN of V would reach rows that do not see it (0 x inf): it counts as zero here and is added to the rows that see it at the end.

constexpr int kGroupLd = 512 + 32;  // LDS elements from one group of rows (1 KB, one load instruction) to the next
// A tile's rows of 256 (128) bytes lie four (eight) to a group; chunk k (16 bytes) of a row sits at k ^ x within its four, x from the row:
// the 16 lanes of a 128-bit access phase then meet all banks once.
__device__ __forceinline__ int swz(int chunk, int x) { return ((chunk & ~3) << 3) + (((chunk & 3) ^ x) << 3); }
__device__ __forceinline__ int at256(int row, int chunk) { return (row >> 2) * kGroupLd + (row & 3) * 128 + swz(chunk, row & 3); }
__device__ __forceinline__ int at128(int row, int chunk) { return (row >> 3) * kGroupLd + (row & 7) * 64 + swz(chunk, (row >> 1) & 3); }

constexpr float kLazy = 3.f;       // log2 of the growth the exponent reference tolerates before it moves
constexpr float kFar = 1048576.f;  // exponents whose spacing, 1/8 and more, would blur the reference

// MFMA row -> key offset inside 32 keys, such that accumulator registers 8 kb .. 8 kb + 7 of lane half h hold the keys 16 kb + 8 h .. + 7.
__device__ __forceinline__ int perm_key(int m) { return (m & ~0xC) | ((m & 4) << 1) | ((m & 8) >> 1); }

// V [b][h][n][D] -> vt and odd.  One workgroup per tile.
template <int D>
__global__ __launch_bounds__(256) void window_values(WindowArgs a) {
  __shared__ uint16_t t[64][D + 2];
  __shared__ int odd;
  const int tile = blockIdx.x, Hkv = a.Hq / a.G, bh = blockIdx.y, b = bh / Hkv, hk = bh % Hkv, tid = threadIdx.x;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  if (tile * 64 >= n) return;
  constexpr int kChunks = D / 8, kRows = 256 / kChunks, kRound = 64 / kRows;  // chunks per row, rows per round, rounds
  const uint16_t* src = static_cast<const uint16_t*>(a.v.ptr) + b * a.v.sb + hk * a.v.sh;
  if (tid == 0) odd = 0;
  u32x4 v[kRound];
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kRound; ++u) {
    const int row = u * kRows + tid / kChunks, col = tid % kChunks * 8;
    v[u] = u32x4{0, 0, 0, 0};
    if (tile * 64 + row < n) v[u] = *reinterpret_cast<const u32x4*>(src + int64_t(tile * 64 + row) * a.v.sn + col);
  }
#pragma unroll
  for (int u = 0; u < kRound; ++u) {
    const int row = u * kRows + tid / kChunks, col = tid % kChunks * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if ((v[u][i] & 0x7F800000u) == 0x7F800000u) v[u][i] &= 0x0000FFFFu, bad = true;
      if ((v[u][i] & 0x7F80u) == 0x7F80u) v[u][i] &= 0xFFFF0000u, bad = true;
      *reinterpret_cast<uint32_t*>(&t[row][col + 2 * i]) = v[u][i];
    }
  }
  __syncthreads();
  if (bad) odd = 1;
  uint16_t* dst = a.vt + (int64_t(bh) * a.tiles + tile) * D * 64;
  for (int c = tid; c < D * 8; c += 256) {
    const int dd = c >> 3, kc = (c & 7) * 8;
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = t[kc + 2 * i][dd] | uint32_t(t[kc + 2 * i + 1][dd]) << 16;
    *reinterpret_cast<u32x4*>(dst + dd * 64 + kc) = o;
  }
  __syncthreads();
  if (tid == 0) a.odd[int64_t(bh) * a.tiles + tile] = odd ? 1.f : 0.f;
}

template <int D>
constexpr int tile_elems() { return D / 8 * kGroupLd; }  // a tile of K, and of V^T, in LDS

// NW wavefronts of 32 query rows.  K and V^T tiles are double-buffered in LDS, filled straight from memory; the two halves of the
// wavefronts run half a tile apart, one forming its probabilities on the vector ALU while the other runs P V of its tile and
// Q K^T of the next on the matrix core.
// SPLIT: the two halves own the same rows and take the tiles in turn, each with buffers of its own, and join their softmaxes at the end.
template <int D, int NW, bool SPLIT>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_bf16(WindowArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  constexpr int kElems = tile_elems<D>(), kDC = D / 32, kKS = D / 16, kRW = SPLIT ? NW / 2 : NW, BM = 32 * kRW;  // kRW: wavefronts that share a tile's loads
  const int Hkv = a.Hq / a.G;
  int blk, hz;
  place(a, gridDim.x / a.blocks, blk, hz);
  const int groups = a.Hq >> a.share, b = hz / groups, hq0 = (hz % groups) << a.share, hk = hq0 / a.G;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int tokens = BM >> a.share, r0 = blk * tokens;
  if (r0 >= n) return;
  const int tid = threadIdx.x, w = tid >> 6, half = SPLIT ? w / kRW : 0, ws = __builtin_amdgcn_readfirstlane(w % kRW), lane = tid & 63, m = lane & 31, h = lane >> 5;
  const int hq = hq0 + (w % kRW & ((1 << a.share) - 1));
  const float scale2 = kLog2e / sqrtf(float(D));
  const Tiles tl(a, r0, min(r0 + tokens, n) - 1, 64);
  const int ntile = SPLIT ? (tl.count - half + 1) / 2 : tl.count, rounds = SPLIT ? (tl.count + 1) / 2 : tl.count;  // of this half, of both
  auto tile_of = [&](int t) __attribute__((always_inline)) { return tl.tile(SPLIT ? 2 * t + half : t); };
  uint16_t* Ks = smem + __builtin_amdgcn_readfirstlane(half) * 4 * kElems;  // [2][kElems]
  uint16_t* Vs = Ks + 2 * kElems;                                           // [2][kElems]
  const uint16_t* kbase = static_cast<const uint16_t*>(a.k.ptr) + b * a.k.sb + hk * a.k.sh;
  const int64_t vt0 = (int64_t(b) * Hkv + hk) * a.tiles;
  const uint16_t* vtbase = a.vt + vt0 * D * 64;
  const float* odd = a.odd + vt0;
  // A tile of K is 64 rows of 2 D bytes, one of V^T D rows of 128 bytes; an instruction brings 1 KB.  Through buffer descriptors: rows
  // behind the prompt's end read as zero, a lane's displacement never changes, and the compiler lets the LDS reads of the products
  // return one by one while such loads are on their way (behind global_load_lds, which counts as a flat access, it waits for all).
  constexpr int kRowsK = 512 / D, kLoadsK = 64 / kRowsK / kRW, kLoadsV = D / 8 / kRW;  // rows per instruction, instructions per wavefront
  uint32_t k_off[kLoadsK], v_off[kLoadsV];
#pragma unroll
  for (int i = 0; i < kLoadsK; ++i) {
    const int lr = (ws * kLoadsK + i) * kRowsK + lane / (D / 8), row = (lr & 32) | perm_key(lr & 31);
    k_off[i] = 2 * (uint32_t(row) * uint32_t(a.k.sn) + (D == 128 ? swz(lane & 15, lr & 3) : swz(lane & 7, (lr >> 1) & 3)));
  }
#pragma unroll
  for (int i = 0; i < kLoadsV; ++i) {
    const int row = (ws * kLoadsV + i) * 8 + (lane >> 3);
    v_off[i] = 2 * uint32_t(row * 64 + swz(lane & 7, (row >> 1) & 3));
  }
  auto load_k = [&](int t) __attribute__((always_inline)) {
    const int k0 = __builtin_amdgcn_readfirstlane(tile_of(t)) * 64, last = min(63, n - 1 - k0);
    const auto src = buffer_of(kbase + int64_t(k0) * a.k.sn, 2 * (uint32_t(last) * uint32_t(a.k.sn) + D));
#pragma unroll
    for (int i = 0; i < kLoadsK; ++i) load_lds16(src, k_off[i], Ks + (t & 1) * kElems + (ws * kLoadsK + i) * kGroupLd);
  };
  auto load_v = [&](int t) __attribute__((always_inline)) {
    const auto src = buffer_of(vtbase + int64_t(tile_of(t)) * (D * 64), D * 128);
#pragma unroll
    for (int i = 0; i < kLoadsV; ++i) load_lds16(src, v_off[i], Vs + (t & 1) * kElems + (ws * kLoadsV + i) * kGroupLd);
  };
  const int wr0 = r0 + (w % kRW >> a.share) * 32, q_row = wr0 + m;
  bf16x8 bq[kKS];
  if (!SPLIT || ntile > 0) load_k(0);
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q.ptr) + b * a.q.sb + hq * a.q.sh + int64_t(min(q_row, n - 1)) * a.q.sn;
#pragma unroll
    for (int ks = 0; ks < kKS; ++ks) bq[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16 + h * 8);
  }
  if (!SPLIT || ntile > 0) load_v(0);
  if (ntile > 1) load_k(1);
  float flag = 0.f, flag_next = 0.f;
  if (!SPLIT || ntile > 0) flag_next = odd[tile_of(0)];

  f32x16 o[kDC];
#pragma unroll
  for (int i = 0; i < kDC; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  // mrun: exponent reference of o and lsum, at least `shift` - kLazy = a.bias above the row's maximum: no sum of probabilities is above one, and P V
  // never above the largest value
  const float shift = a.bias + kLazy;
  float mrun = kFloor, lsum = 0.f;
  // A row whose maximum lies beyond kFar has `away`, that maximum or an earlier one, taken from its logits first: what follows sees small numbers.
  // (Looking for such rows takes about 1%: 32768 tokens, window 4096 2.91 -> 2.96 ms.)
  float away = 0.f;  // as an exponent; 0: not such a row
  bool far = false;  // the wavefront has such rows
  f32x16 s[2];
  bf16x8 pb[2][2][2];  // sub-tile, half, term
  auto active = [&](int t) __attribute__((always_inline)) {
    const int k0 = tile_of(t) * 64;
    return any_seen(a, wr0, wr0 + 31, k0, k0 + 63);
  };
  // `moves`: rows whose `away` becomes the tile's maximum; `takes`: rows it is taken from
  auto take_away = [&](auto moves, auto takes) __attribute__((always_inline)) {
#pragma clang fp contract(off)  // (a product that is rounded, so that the maximum less itself is zero)
    float x = -INFINITY;
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int r = 0; r < 16; ++r) x = fmaxf(x, s[st][r]);
    x = max_halves(x) * scale2;
    const float unscale = 1.f / scale2;
    if (moves(x)) {
      mrun -= x - away;
      away = x;
    }
    const bool is = takes();
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[st][r] = is ? (s[st][r] * scale2 - away) * unscale : s[st][r];
  };
  // probabilities of one group of eight registers (sub-tile st, half kb)
  auto form = [&](int st, int kb) __attribute__((always_inline)) {
    float sum = 0.f;
    u32x4 hi, lo;
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(s[st][8 * kb + r], scale2, -mrun)), p1 = __builtin_amdgcn_exp2f(fmaf(s[st][8 * kb + r + 1], scale2, -mrun));
      sum += p0;
      sum += p1;
      uint32_t x = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)p0, (__bf16)p1});
      asm("" : "+v"(x));  // (one conversion of both, of which the compiler would make a third of p0 alone)
      hi[r / 2] = x;
      lo[r / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(p0 - __uint_as_float(x << 16)), (__bf16)(p1 - __uint_as_float(x & 0xFFFF0000u))});
    }
    pb[st][kb][0] = __builtin_bit_cast(bf16x8, hi);
    pb[st][kb][1] = __builtin_bit_cast(bf16x8, lo);
    return sum;
  };
  auto softmax = [&](int t) __attribute__((always_inline)) {
    const int k0 = tile_of(t) * 64;
    if (!all_seen(a, wr0, wr0 + 31, k0, k0 + 63)) {
      // register r of sub-tile st holds key `first` + 32 st + 16 (r / 8) + r % 8
      const int first = k0 + h * 8, last = q_row - first, gone = q_row - a.window - first, sinks = a.n_sink - first;
      const bool ahead = k0 + 63 > wr0, behind = k0 <= wr0 + 31 - a.window;  // keys that follow a row, that its window has left
      if (ahead) {
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (st * 32 + (r >> 3) * 16 + (r & 7) > last) s[st][r] = -INFINITY;
      }
      if (behind) {
        if (k0 >= a.n_sink) {
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (st * 32 + (r >> 3) * 16 + (r & 7) <= gone) s[st][r] = -INFINITY;
        } else {
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int key = st * 32 + (r >> 3) * 16 + (r & 7);
              if (key <= gone && key >= sinks) s[st][r] = -INFINITY;
            }
        }
      }
    }
    if (__builtin_expect(far, false)) take_away([&](float x) { return away != 0.f && x > away + kFar; }, [&] { return away != 0.f; });
    auto reference = [&]() __attribute__((always_inline)) {  // that the tile asks for
      float x = s[0][0];
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int r = 0; r < 16; ++r) x = fmaxf(x, s[st][r]);
      return fmaf(max_halves(x), scale2, shift);
    };
    float cand = reference();
    bool grew = cand > mrun + kLazy;
    if (__any(grew)) {  // wavefront-uniform: no rescale when no row's maximum moved
      const bool leap = grew && away == 0.f && fabsf(cand) > kFar && fabsf(cand) < INFINITY;
      if (__builtin_expect(__any(leap), 0)) {
        far = true;
        take_away([&](float) { return leap; }, [&] { return leap; });
        cand = reference();
        grew = cand > mrun + kLazy;
      }
      const float mnew = grew ? cand : mrun;
      const float f = __builtin_amdgcn_exp2f(mrun - mnew);
      lsum *= f;
      mrun = mnew;
#pragma unroll
      for (int i = 0; i < kDC; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= f;
    }
    float sum = form(0, 0);
    sum += form(0, 1);
    sum += form(1, 0);
    sum += form(1, 1);
    lsum += sum;
  };
  // o += V^T P^T of tile t, then S^T = K Q^T of tile t + 1; LDS operands are fetched two batches of four ahead
  constexpr int kPV = 4 * kDC, kQK = 2 * kKS;
  auto operand = [&](int t, auto i) __attribute__((always_inline)) -> u32x4 {
    constexpr int idx = decltype(i)::value;
    if constexpr (idx < kPV) {
      constexpr int st = idx / (2 * kDC), kb = idx / kDC % 2, dc = idx % kDC;
      return *reinterpret_cast<const u32x4*>(&Vs[(t & 1) * kElems + at128(dc * 32 + m, st * 4 + kb * 2 + h)]);
    }
    const int st = (idx - kPV) & 1, ks = (idx - kPV) >> 1, row = st * 32 + m, chunk = ks * 2 + h;
    return *reinterpret_cast<const u32x4*>(&Ks[((t + 1) & 1) * kElems + (D == 128 ? at256(row, chunk) : at128(row, chunk))]);
  };
  auto issue = [&](auto i, auto term, const u32x4& x) __attribute__((always_inline)) {
    constexpr int idx = decltype(i)::value;
    if constexpr (idx < kPV) {
      constexpr int st = idx / (2 * kDC), kb = idx / kDC % 2, dc = idx % kDC;
      o[dc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pb[st][kb][term], o[dc], 0, 0, 0);
    } else if constexpr (term == 0) {
      constexpr int st = (idx - kPV) & 1, ks = (idx - kPV) >> 1;
      const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      s[st] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), bq[ks], ks == 0 ? zero : s[st], 0, 0, 0);
    }
  };
  auto products = [&](int t, auto first, auto last) __attribute__((always_inline)) {
    constexpr int i0 = decltype(first)::value, NB = (decltype(last)::value - i0) / 4;
    u32x4 A[2][4];
    each<8>([&](auto i) { A[i / 4][i % 4] = operand(t, std::integral_constant<int, i0 + i>{}); });
    each<NB>([&](auto bt) {
      __builtin_amdgcn_sched_barrier(0);
      each<2>([&](auto term) { each<4>([&](auto i) { issue(std::integral_constant<int, i0 + 4 * bt + i>{}, term, A[bt & 1][i]); }); });
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (bt + 2 < NB)
        each<4>([&](auto i) { A[bt & 1][i] = operand(t, std::integral_constant<int, i0 + 4 * (bt + 2) + i>{}); });
    });
  };
  typedef std::integral_constant<int, 0> P0;
  typedef std::integral_constant<int, kPV> P1;
  typedef std::integral_constant<int, kPV + kQK> P2;
  auto matrix = [&](int t, bool pv, bool qk) __attribute__((always_inline)) {  // the wavefront in its matrix phase issues first
    __builtin_amdgcn_s_setprio(1);
    if (pv && qk)
      products(t, P0{}, P2{});
    else if (pv)
      products(t, P0{}, P1{});
    else if (qk)
      products(t, P1{}, P2{});
    __builtin_amdgcn_s_setprio(0);
  };

  const bool late = w >= NW / 2;  // (SPLIT: the second half)
#pragma unroll
  for (int ks = 0; ks < kKS; ++ks) asm volatile("" ::"v"(bq[ks]));  // the queries have arrived
  wait_vm<0>();
  __syncthreads();
  bool now = false;
  for (int t = -1; t < rounds; ++t) {
    const bool more = t + 1 < ntile, next = more && active(t + 1);
    if (t >= 0) {  // K(t) and V(t - 1) were last read before this iteration: their buffers take K(t + 2) and V(t + 1)
      if (t + 2 < ntile) load_k(t + 2);
      if (more) {
        load_v(t + 1);
        flag_next = odd[tile_of(t + 1)];
      }
    }
    if (late && now) softmax(t);
    matrix(t, now, next);
    if (!late && next) softmax(t + 1);
    now = next;
    wait_vm<0>();  // this wavefront's part of the next tiles is in LDS
    flag = fmaxf(flag, flag_next);
    __syncthreads();
  }
  if constexpr (SPLIT) {
    // the second half's rows to LDS (the tiles are done with), the first half adds them to its own
    float* os = reinterpret_cast<float*>(smem) + ws * (kDC * 16 + 4) * 64 + lane;
    if (half) {
      each<kDC>([&](auto dc) { each<16>([&](auto r) { os[(dc * 16 + r) * 64] = o[dc][decltype(r)::value]; }); });
      os[kDC * 16 * 64] = mrun;
      os[(kDC * 16 + 1) * 64] = lsum;
      os[(kDC * 16 + 2) * 64] = flag;
      os[(kDC * 16 + 3) * 64] = away;
    }
    __syncthreads();
    if (half) return;
    const float m1 = os[kDC * 16 * 64] == kFloor ? kFloor : os[kDC * 16 * 64] + (os[(kDC * 16 + 3) * 64] - away), l1 = os[(kDC * 16 + 1) * 64];
    flag = fmaxf(flag, os[(kDC * 16 + 2) * 64]);
    const float M = fmaxf(mrun, m1);
    const float f0 = __builtin_amdgcn_exp2f(mrun - M), f1 = __builtin_amdgcn_exp2f(m1 - M);
    lsum = lsum * f0 + l1 * f1;
    each<kDC>([&](auto dc) {
      each<16>([&](auto r) { o[dc][decltype(r)::value] = o[dc][decltype(r)::value] * f0 + os[(dc * 16 + r) * 64] * f1; });
    });
  }
  if (flag != 0.f) {
    // infinities and NaN of V, which counted as zero above: a row that sees one takes it as it is, whatever its weight
    const uint16_t* vsrc = static_cast<const uint16_t*>(a.v.ptr) + b * a.v.sb + hk * a.v.sh;
    for (int t = 0; t < tl.count; ++t) {
      if (odd[tl.tile(t)] == 0.f) continue;
      const int k0 = tl.tile(t) * 64;
      for (int j = k0; j < min(k0 + 64, n); ++j) {
        if (!sees(a, q_row, j)) continue;
        const uint16_t* row = vsrc + int64_t(j) * a.v.sn;
        each<kDC>([&](auto dc) {
          each<16>([&](auto r) {
            const float x = Elem<uint16_t>::to_f32(row[dc * 32 + (r >> 2) * 8 + h * 4 + (r & 3)]);
            if (!(fabsf(x) < INFINITY)) o[dc][decltype(r)::value] += x;
          });
        });
      }
    }
  }
  const float inv = 1.f / sum_of_halves(lsum);
  if (q_row >= n) return;
  // registers 4 rg .. 4 rg + 3 hold columns 32 dc + 8 rg + 4 h + 0..3: the lanes of a row swap halves of a register pair, so that
  // each stores eight consecutive columns
  uint16_t* out = static_cast<uint16_t*>(a.o.ptr) + b * a.o.sb + hq * a.o.sh + int64_t(q_row) * a.o.sn;
#pragma unroll
  for (int dc = 0; dc < kDC; ++dc)
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = Elem<uint16_t>::from_f32(o[dc][8 * h2 + 2 * i] * inv) | uint32_t(Elem<uint16_t>::from_f32(o[dc][8 * h2 + 2 * i + 1] * inv)) << 16;
      const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
      *reinterpret_cast<u32x4*>(out + dc * 32 + h2 * 16 + h * 8) = u32x4{s0[0], s1[0], s0[1], s1[1]};
    }
}

// ---- fp32 ----------------------------------------------------------------------------------
// Four wavefronts of 16 query rows, tiles of 32 keys, all products on the fp32 matrix instruction (16 x 16 x 4): S^T of 16 keys
// leaves the four keys 4 g + r in register r of lane row g, and register r is the operand of the product whose V rows are
// 4 g + r.  Tiles pass through registers on their way to LDS; an infinity or NaN of V counts as zero there and is added at the end.
// Probabilities are formed as 2^-bias * p: no sum of them is above one, and P V never above the largest value.
template <int D>
__global__ __launch_bounds__(256) void window_f32(WindowArgs a) {
  constexpr int BN = 32, BM = 64, kLd = D + 4, kLoads = BN * D / 4 / 256;
  __shared__ __attribute__((aligned(16))) float Ks[2][BN * kLd], Vs[2][BN * kLd];
  __shared__ int odd;
  int blk, hz;
  place(a, gridDim.x / a.blocks, blk, hz);
  const int groups = a.Hq >> a.share, b = hz / groups, hq0 = (hz % groups) << a.share, hk = hq0 / a.G;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int tokens = BM >> a.share, r0 = blk * tokens;
  if (r0 >= n) return;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4, hq = hq0 + (w & ((1 << a.share) - 1));
  const float scale2 = kLog2e / sqrtf(float(D));
  const Tiles tl(a, r0, min(r0 + tokens, n) - 1, BN);
  const float* kbase = static_cast<const float*>(a.k.ptr) + b * a.k.sb + hk * a.k.sh;
  const float* vbase = static_cast<const float*>(a.v.ptr) + b * a.v.sb + hk * a.v.sh;
  f32x4 kr[kLoads], vr[kLoads];
  auto fetch = [&](int t) __attribute__((always_inline)) {
    const int k0 = tl.tile(t) * BN;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = tid + 256 * i, row = x / (D / 4), col = x % (D / 4) * 4;
      const int64_t j = min(k0 + row, n - 1);
      kr[i] = *reinterpret_cast<const f32x4*>(kbase + j * a.k.sn + col);
      vr[i] = *reinterpret_cast<const f32x4*>(vbase + j * a.v.sn + col);
    }
  };
  auto stage = [&](int buf) __attribute__((always_inline)) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = tid + 256 * i, row = x / (D / 4), col = x % (D / 4) * 4;
      *reinterpret_cast<f32x4*>(&Ks[buf][row * kLd + col]) = kr[i];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!(fabsf(vr[i][j]) < INFINITY)) vr[i][j] = 0.f, bad = true;
      *reinterpret_cast<f32x4*>(&Vs[buf][row * kLd + col]) = vr[i];
    }
    if (bad) odd = 1;
  };
  const int wr0 = r0 + (w >> a.share) * 16, q_row = wr0 + c;
  f32x4 q[D / 16];
  fetch(0);
  const float* qp = static_cast<const float*>(a.q.ptr) + b * a.q.sb + hq * a.q.sh + int64_t(min(q_row, n - 1)) * a.q.sn;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const f32x4*>(qp + i * 16 + g * 4);
  if (tid == 0) odd = 0;
  __syncthreads();
  stage(0);
  __syncthreads();
  float m = kFloor, l = 0.f;
  f32x4 o[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = 0; t < tl.count; ++t) {
    if (t + 1 < tl.count) fetch(t + 1);
    const float *Kt = Ks[t & 1], *Vt = Vs[t & 1];
    const int k0 = tl.tile(t) * BN;
#pragma unroll
    for (int st = 0; st < BN / 16; ++st) {
      const int j0 = k0 + st * 16;
      if (!any_seen(a, wr0, wr0 + 15, j0, j0 + 15)) continue;
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&Kt[(st * 16 + c) * kLd + i * 16 + g * 4]);
#pragma unroll
        for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], q[i][j], s, 0, 0, 0);
      }
      const bool whole = all_seen(a, wr0, wr0 + 15, j0, j0 + 15);
      float mx = m;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[r] *= scale2;
        if (!whole && !sees(a, q_row, j0 + 4 * g + r)) s[r] = -INFINITY;
        mx = fmaxf(mx, s[r]);
      }
      const auto x16 = __builtin_amdgcn_permlane16_swap(__float_as_int(mx), __float_as_int(mx), false, false);
      mx = max_halves(fmaxf(__int_as_float(x16[0]), __int_as_float(x16[1])));
      if (__any(mx > m)) {
        const float f = __builtin_amdgcn_exp2f(m - mx);
        m = mx;
        l *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] *= f;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f((s[r] - m) - a.bias);
        l += p;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(Vt[(st * 16 + 4 * g + r) * kLd + i * 16 + c], p, o[i], 0, 0, 0);
      }
    }
    if (t + 1 < tl.count) stage((t + 1) & 1);
    __syncthreads();
  }
  if (odd)
    for (int t = 0; t < tl.count; ++t)
      for (int j = tl.tile(t) * BN; j < min(tl.tile(t) * BN + BN, n); ++j)
        if (sees(a, q_row, j)) {
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float x = vbase[j * a.v.sn + i * 16 + g * 4 + r];
              if (!(fabsf(x) < INFINITY)) o[i][r] += x;
            }
        }
  const auto x16 = __builtin_amdgcn_permlane16_swap(__float_as_int(l), __float_as_int(l), false, false);
  l = sum_of_halves(__int_as_float(x16[0]) + __int_as_float(x16[1]));
  if (q_row >= n) return;
  const float inv = 1.f / l;
  float* out = static_cast<float*>(a.o.ptr) + b * a.o.sb + hq * a.o.sh + int64_t(q_row) * a.o.sn;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(out + i * 16 + g * 4) = o[i] * inv;
}

// The same for prompts whose blocks of 64 rows leave CUs without work: a workgroup owns 16 rows, its four wavefronts take 16-key tiles
// in turn, straight from memory to registers with the next tile on its way, and join their softmaxes in LDS.  (512 tokens, 4 heads,
// window 64: 13.7 us by the kernel above, 7.1 by this one.)
template <int D>
__global__ __launch_bounds__(256) void window_f32_few(WindowArgs a) {
  constexpr int BN = 16, BM = 16, kI = D / 16, kW = 4;
  __shared__ float so[kW][BM][D + 4], sm[kW][BM], sl[kW][BM];
  __shared__ int odd;
  int blk, hz;
  place(a, gridDim.x / a.blocks, blk, hz);
  const int hq = hz % a.Hq, b = hz / a.Hq, hk = hq / a.G;
  const int n = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int r0 = blk * BM;
  if (r0 >= n) return;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const float scale2 = kLog2e / sqrtf(float(D));
  const Tiles tl(a, r0, min(r0 + BM, n) - 1, BN);
  const float* kbase = static_cast<const float*>(a.k.ptr) + b * a.k.sb + hk * a.k.sh;
  const float* vbase = static_cast<const float*>(a.v.ptr) + b * a.v.sb + hk * a.v.sh;
  if (tid == 0) odd = 0;
  const int q_row = r0 + c;
  f32x4 q[kI], kr[kI], kn[kI];
  float vr[4][kI], vn[4][kI];
  auto fetch = [&](int t, f32x4* kd, float (*vd)[kI]) __attribute__((always_inline)) {
    const int j0 = tl.tile(t) * BN;
    const float* kp = kbase + int64_t(min(j0 + c, n - 1)) * a.k.sn + g * 4;
#pragma unroll
    for (int i = 0; i < kI; ++i) kd[i] = *reinterpret_cast<const f32x4*>(kp + i * 16);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float* vp = vbase + int64_t(min(j0 + 4 * g + r, n - 1)) * a.v.sn + c;
#pragma unroll
      for (int i = 0; i < kI; ++i) vd[r][i] = vp[i * 16];
    }
  };
  if (w < tl.count) fetch(w, kr, vr);
  const float* qp = static_cast<const float*>(a.q.ptr) + b * a.q.sb + hq * a.q.sh + int64_t(min(q_row, n - 1)) * a.q.sn;
#pragma unroll
  for (int i = 0; i < kI; ++i) q[i] = *reinterpret_cast<const f32x4*>(qp + i * 16 + g * 4);
  float m = kFloor, l = 0.f;
  bool bad = false;
  f32x4 o[kI];
#pragma unroll
  for (int i = 0; i < kI; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = w; t < tl.count; t += kW) {
    if (t + kW < tl.count) fetch(t + kW, kn, vn);
    const int j0 = tl.tile(t) * BN;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[i][j], q[i][j], s, 0, 0, 0);
    float mx = m;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[r] *= scale2;
      if (!sees(a, q_row, j0 + 4 * g + r)) s[r] = -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    const auto x16 = __builtin_amdgcn_permlane16_swap(__float_as_int(mx), __float_as_int(mx), false, false);
    mx = max_halves(fmaxf(__int_as_float(x16[0]), __int_as_float(x16[1])));
    const float f = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    l *= f;
#pragma unroll
    for (int i = 0; i < kI; ++i) o[i] *= f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float p = __builtin_amdgcn_exp2f((s[r] - m) - a.bias);
      l += p;
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const bool fine = fabsf(vr[r][i]) < INFINITY;
        bad |= !fine;
        o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(fine ? vr[r][i] : 0.f, p, o[i], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < kI; ++i) kr[i] = kn[i];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < kI; ++i) vr[r][i] = vn[r][i];
  }
  const auto x16 = __builtin_amdgcn_permlane16_swap(__float_as_int(l), __float_as_int(l), false, false);
  l = sum_of_halves(__int_as_float(x16[0]) + __int_as_float(x16[1]));
#pragma unroll
  for (int i = 0; i < kI; ++i) *reinterpret_cast<f32x4*>(&so[w][c][i * 16 + g * 4]) = o[i];
  if (lane < BM) {
    sm[w][lane] = m;
    sl[w][lane] = l;
  }
  __syncthreads();
  if (bad) odd = 1;
  __syncthreads();
  for (int x = tid; x < BM * D; x += 256) {
    const int row = x / D, col = x % D;
    if (r0 + row >= n) break;
    const float M = fmaxf(fmaxf(sm[0][row], sm[1][row]), fmaxf(sm[2][row], sm[3][row]));
    float L = 0.f, y = 0.f;
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      const float f = __builtin_amdgcn_exp2f(sm[i][row] - M);
      L = fmaf(sl[i][row], f, L);
      y = fmaf(so[i][row][col], f, y);
    }
    if (odd)  // infinities and NaN of V: a row that sees one takes it as it is
      for (int t = 0; t < tl.count; ++t)
        for (int j = tl.tile(t) * BN; j < min(tl.tile(t) * BN + BN, n); ++j) {
          const float v = vbase[j * a.v.sn + col];
          if (!(fabsf(v) < INFINITY) && sees(a, r0 + row, j)) y += v;
        }
    (static_cast<float*>(a.o.ptr) + b * a.o.sb + hq * a.o.sh + int64_t(r0 + row) * a.o.sn)[col] = y / L;
  }
}

int check_window(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (batch < 1 || n < 1 || n_kv_heads < 1) return D2O_ERR_INVALID_ARG;
  if (dtype != D2O_F32 && dtype != D2O_BF16) return D2O_ERR_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return D2O_ERR_UNSUPPORTED;
  if (n > 0x7FFF0000 || int64_t(batch) * n_kv_heads > 65535) return D2O_ERR_UNSUPPORTED;
  return D2O_OK;
}

size_t values_bytes(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim) {
  return size_t(batch) * n_kv_heads * ((n + 63) / 64) * head_dim * 64 * sizeof(uint16_t);
}
size_t window_bytes(int32_t batch, int32_t n, int32_t n_kv_heads, int32_t head_dim, int32_t dtype) {
  if (dtype == D2O_F32) return 0;
  return values_bytes(batch, n, n_kv_heads, head_dim) + size_t(batch) * n_kv_heads * ((n + 63) / 64) * sizeof(float);
}

// Query heads that a block of `waves` wavefronts shares, and its blocks of rows.
void share_heads(WindowArgs& a, int waves, int rows) {
  a.share = 0;
  while (a.G % (2 << a.share) == 0 && 2 << a.share <= waves) ++a.share;
  const int tokens = (waves * rows) >> a.share;
  a.blocks = (a.n + tokens - 1) / tokens;
}

template <int D, int NW, bool SPLIT>
hipError_t run_bf16(WindowArgs& a, int batch, hipStream_t s) {
  constexpr int kRW = SPLIT ? NW / 2 : NW, kSmem = (SPLIT ? 8 : 4) * tile_elems<D>() * int(sizeof(uint16_t));
  static_assert(!SPLIT || kSmem >= NW / 2 * (D / 32 * 16 + 4) * 64 * int(sizeof(float)), "the second half's rows");
  share_heads(a, kRW, 32);
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(window_bf16<D, NW, SPLIT>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != hipSuccess) return e;
  window_values<D><<<dim3(a.tiles, batch * (a.Hq / a.G)), 256, 0, s>>>(a);
  window_bf16<D, NW, SPLIT><<<dim3(unsigned(a.blocks) * batch * (a.Hq >> a.share)), 64 * NW, kSmem, s>>>(a);
  return hipGetLastError();
}

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
  if (!rows_apart(O, {batch, n_q_heads, n}, head_dim)) return D2O_ERR_INVALID_ARG;
  const size_t need = window_bytes(batch, n, n_kv_heads, head_dim, dtype);
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < need) return D2O_ERR_CAPACITY;
  if (int64_t(batch) * n_q_heads * ((n + 63) / 64) > 0x7FFFFFFF) return D2O_ERR_UNSUPPORTED;
  if (K.stride_n >= 1 << 24) return D2O_ERR_UNSUPPORTED;  // (displacements inside a tile of 64 keys have 32 bits)
  WindowArgs a{};
  a.q = to_view(Q);
  a.k = to_view(K);
  a.v = to_view(V);
  a.o = to_view(O);
  a.lens = lens;
  a.n = n;
  a.Hq = n_q_heads;
  a.G = n_q_heads / n_kv_heads;
  a.window = window == 0 || window > n ? n : window;
  a.n_sink = std::min(n_sink, n);
  a.bias = float(32 - __builtin_clz(unsigned(std::min<int64_t>(n, int64_t(a.window) + a.n_sink))));
  a.tiles = (n + 63) / 64;
  a.reverse = a.window > n / 2;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == D2O_BF16) {
    a.vt = static_cast<uint16_t*>(workspace);
    a.odd = reinterpret_cast<float*>(static_cast<char*>(workspace) + values_bytes(batch, n, n_kv_heads, head_dim));
    // Wavefronts per workgroup.  Where the chip has a CU for every block of 128 rows, eight, the tiles split over two halves.  Otherwise four,
    // two workgroups (d = 64: three) per CU that hide each other's ends, for heads of 64 and windows below 1024; for larger ones eight, for
    // whose twice as many rows a tile is brought once.  (16384 tokens, 32 heads on 8, d = 128, four and eight: window 128 185 and 198 us, 512 299 and 302,
    // 1024 467 and 462, 4096 1405 and 1354; d = 64, window 2048 499 and 565, 8000 1442 and 1583.  Blocks that all fit at once: four too.)
    const int64_t blocks = int64_t((n + 127) / 128) * n_q_heads * batch;
    const bool four = blocks <= 512 || a.window < 1024;
    hipError_t e;
    if (head_dim == 64)
      e = blocks <= 256 ? run_bf16<64, 8, true>(a, batch, s) : run_bf16<64, 4, false>(a, batch, s);
    else
      e = blocks <= 256 ? run_bf16<128, 8, true>(a, batch, s) : four ? run_bf16<128, 4, false>(a, batch, s) : run_bf16<128, 8, false>(a, batch, s);
    return e == hipSuccess ? D2O_OK : D2O_ERR_HIP;
  }
  const int64_t heads = int64_t(batch) * n_q_heads;
  const bool few = (n + 63) / 64 * heads < 256;  // fewer blocks of 64 rows than CUs
  if (few)
    a.blocks = (n + 15) / 16;
  else
    share_heads(a, 4, 16);
  const dim3 grid(unsigned(a.blocks * (heads >> a.share)));
  const auto kernel = few ? head_dim == 64 ? window_f32_few<64> : window_f32_few<128> : head_dim == 64 ? window_f32<64> : window_f32<128>;
  kernel<<<grid, 256, 0, s>>>(a);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
