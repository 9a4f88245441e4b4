// Attention over a cache in pages whose rows are held in 4 bits: one query token per sequence (d2o_pages_step) and several
// (d2o_pages_attend).
#include "pages_step.h"

namespace d2o {
namespace {

// Query tokens of a batch's sequences stand one behind the other (attend); a sequence's (token, query head of a KV head's group) pairs, in
// this order, are the columns of its products, up to kGroup to a workgroup.
struct AttendArgs : StepArgs {
  const int32_t* first;  // [B + 1] first query token of every sequence
  int32_t n_tokens, batch, groups;  // rows of q; groups of columns, at most
  uint32_t over_g;                  // ceil(2^32 / G): x / G is the upper half of x * over_g for x < 2^28
  __device__ __forceinline__ int token_of(int pair) const { return G == 1 ? pair : int(__umulhi(uint32_t(pair), over_g)); }
};
constexpr int kCols = 16;            // columns of a matrix product
constexpr int kGroup = 32;           // columns of a workgroup at most
constexpr int kLeast4 = kWaves * 2;  // tiles of a workgroup's round: a pair for each wavefront

// Which columns a workgroup has.  Step: the group's query heads of sequence b.
struct Columns {
  int b, base, count;       // sequence, first pair, pairs (0: none)
  int token0, tokens, len;  // (attend) the sequence's first query token, how many it has, its entries
};
// The index-th group of kGroup columns of the batch (of a sequence's, which see more and more, the last one first); all threads of the workgroup.
__device__ __forceinline__ Columns find_columns(const AttendArgs& a, int index) {
  __shared__ int sum[kWaves], found[6];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = (a.batch + 64 * kWaves - 1) / (64 * kWaves), b0 = tid * per, b1 = min(b0 + per, a.batch);
  auto token0 = [&](int b) { return min(max(a.first[b], 0), a.n_tokens); };
  int mine = 0, len = 0, start = 0, end = 0;
  for (int b = b0; b < b1; ++b) {
    start = token0(b);
    end = token0(b + 1);
    len = a.lens[b];  // (of the last one; there is one nearly always)
    mine += (max(end - start, 0) * a.G + kGroup - 1) / kGroup;
  }
  int inc = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(inc, o, 64);
    if (lane >= o) inc += t;
  }
  if (lane == 63) sum[w] = inc;
  if (tid == 0) found[2] = 0;
  __syncthreads();
  for (int i = 0; i < w; ++i) inc += sum[i];
  int at = inc - mine;
  if (index >= at && index < inc)
    for (int b = b0; b < b1; ++b) {
      if (per > 1) {
        start = token0(b);
        end = token0(b + 1);
        len = a.lens[b];
      }
      const int tokens = max(end - start, 0), pairs = tokens * a.G, n = (pairs + kGroup - 1) / kGroup;
      if (index < at + n) {
        const int base = (n - 1 - (index - at)) * kGroup;
        found[0] = b;
        found[1] = base;
        found[2] = min(pairs - base, kGroup);
        found[3] = start;
        found[4] = tokens;
        found[5] = entries_of(len, a.max_len);
        break;
      }
      at += n;
    }
  __syncthreads();
  auto scalar = [&](int i) { return __builtin_amdgcn_readfirstlane(found[i]); };
  return {scalar(0), scalar(1), scalar(2), scalar(3), scalar(4), scalar(5)};
}

// Heads of a step's group that have room in the sixteen columns PARTS times, and the head of column c (kCols: none).
template <int PARTS>
constexpr int kPart = kCols / PARTS;
template <int PARTS>
__device__ __forceinline__ int head_of(int c) {
  return c < PARTS * kPart<PARTS> ? c % kPart<PARTS> : kCols;
}

// What a column sees: entries up to `last`, of these the ones with a position from `lo` on or below n_sink.
struct Sight {
  int last;  // -1: nothing
  int lo;    // (positions are 32-bit numbers: a start below them all is the lowest)
};
__device__ __forceinline__ int window_start(int64_t position, int window) {
  return window == 0 ? INT32_MIN : int(max(position - window + 1, int64_t(INT32_MIN)));
}
__device__ __forceinline__ int row_min(int v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = min(v, __shfl_xor(v, o, 64));
  return v;
}
// The sights of columns c, c + 16, .. (N of them), and the tiles that any of the columns sees; false where there are none.
template <int N>
__device__ __forceinline__ bool sights_of(const AttendArgs& a, const Columns& col, int c, Sight (&mine)[N], TileList& list) {
  int lo = INT32_MAX;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = i * kCols + c, token = a.token_of(col.base + at);
    const bool is = at < col.count;
    mine[i].last = is ? last_seen(col.len, col.tokens, token) : -1;
    mine[i].lo = window_start(a.window != 0 && a.positions && is ? a.positions[col.token0 + token] : mine[i].last, a.window);
    lo = min(lo, is ? mine[i].lo : INT32_MAX);
  }
  list.n = last_seen(col.len, col.tokens, a.token_of(col.base + col.count - 1)) + 1;
  list.last = 0;
  if (list.n == 0) return false;
  list.choose(a, a.window == 0 ? 0 : __builtin_amdgcn_readfirstlane(row_min(lo)), kLeast4);
  return true;
}

// Rows of D 4-bit elements, as the lanes hold them.  K: lane l has row l % 16 of a tile, a quarter of it; V: the 16 lanes of a row of lanes share
// a row, D / 16 elements each.
template <int D>
struct Row4 {
  static constexpr int kSteps = D / 32, kE = D / 16;
  typedef std::conditional_t<D == 128, u32x4, u32x2> KReg;       // also the powers of two of four rows
  typedef std::conditional_t<D == 128, uint32_t, uint16_t> VReg;
};

typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr float kLowest = -3.402823466e38f;  // a maximum before the first logit
constexpr float kFar = 1048576.f;            // exponents whose rounding is no longer small (2^-4)

// a * b as a number of its own, never part of a multiply-add: large logits that are equal have to stay equal when a maximum is taken from them.
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Where a pair of tiles lies, the same for all lanes.
struct Pair {
  int s0[2];      // first entries
  int page[2];    // (pages of whole tiles)
  bool there[2];  // within the share, and on a page
};
// How rows are found.  ROWS: each by its own page number.  TILES, PAIRS: a tile, or a pair of them, lies in one page, whose number and address are the same for
// all lanes and live in scalar registers; a lane adds a displacement of 32 bits that never changes (see the step over wider rows).
enum Finds { ROWS, TILES, PAIRS };

// One share of the tiles that a workgroup's columns see, by its four wavefronts in turn, pairs of tiles at a time; N groups of 16 columns.  As in the
// step over wider rows the logits S^T = K Q^T come from the matrix core, entries by columns, and leave in each lane of row of lanes g one column and the
// entries 4 g .. 4 g + 3 of a tile.  Of two tiles these are eight entries, which is what the lane has to hold of P as the left operand of P V (16 x 16 x 32): P goes from registers to
// the matrix core with no exchange.  The right operand wants eight entries of one element of V: a lane converts the D / 16 elements it has of each of the eight rows
// to bf16 (exact), two elements of one row at a time, and swaps halves between rows: a conversion and a permutation for two values, once for all N groups.
// P goes in as bf16 terms.  The step takes three, which hold all 24 bits: a group of up to five heads stands in the sixteen columns three times, each time for one
// term of the same P, so that one product does for all three and the join adds the parts up (16 x 8192 entries, 8 KV heads of 4: 32 us as with two terms; three products 34);
// one of up to eight twice, for two products (4 KV heads of 8: 23.8 us, with scores 29.8; three products 24.4 and 33.6; two terms 22.9 and 29.0); larger ones take three
// products (2 KV heads of 16: 18.4 us, with scores 29.2; two terms 17.8 and 26.6).  Attention of several tokens, whose columns are all different, takes two, which hold
// 16 bits: a weight is off by 2^-16 of itself at most (three: 1587 -> 1920 us for 2048 tokens on 32768, and bf16 outputs no closer to those of 64 bits in four digits).
// Codes are always finite and powers of two may stand for NaN: where
// columns see different entries, NaN is left out of the product, in which 0 * NaN would reach columns that do not see it, and added to those that do.
template <int D, Finds F, bool STEP, int N, int PARTS>
struct Share {
  typedef Row4<D> R;
  static constexpr int E = R::kE, kExps = D / kBlock4, kSteps = R::kSteps;
  // Attention of several tokens: the next pair's rows are on their way and its keys converted beside the products of the present one (two wavefronts per
  // SIMD).  The step: few registers, so that four wavefronts per SIMD hide the loads (16 x 8192 entries 32 us; in the other manner 38, with three wavefronts 37).
  static constexpr bool kAhead = !STEP;
  const AttendArgs& a;
  const Columns& col;
  const TileList& list;
  const int hk, t0, t1;
  const Sight (&mine)[N];
  const int w, lane, c, g;
  const int all_last, all_lo;
  // rows on their way
  typename R::KReg k[2], vx[2];
  typename R::VReg v[2][4];
  int ke[2];
  uint32_t absent[2];  // (ROWS) bit i: entry i of the tile has no page
  // results: maximum (of the base-2 logits), sum and outputs, register i of om: column 4 g + i, element c * E + index
  float m[N], l[N];
  f32x4 om[N][E];

  __device__ __forceinline__ Pair pair_at(int t) const {
    const auto table = (const __attribute__((address_space(4))) int32_t*)(a.pool.table + int64_t(col.b) * a.pool.max_pages);
    t = min(t, t0 + ((t1 - 1 - t0) & ~1));  // (behind the share: its last pair again)
    Pair p;
    p.s0[0] = list.slot(t);
    p.there[0] = true;
    p.there[1] = t + 1 < t1;
    p.s0[1] = F == PAIRS ? p.s0[0] + kTile : list.slot(min(t + 1, t1 - 1));
#pragma unroll
    for (int i = 0; i < (F == ROWS ? 0 : F == TILES ? 2 : 1); ++i) {
      const int page = table[p.s0[i] >> a.pool.shift];
      const bool is = uint32_t(page) < uint32_t(a.pool.n_pages);
      p.page[i] = is ? page : 0;  // (no page: the pool's first, whose values are not used; rows behind the end lie in the page)
      p.there[i] = p.there[i] && is;
      if (F == PAIRS) {
        p.page[1] = p.page[0];
        p.there[1] = p.there[1] && is;
      }
    }
    return p;
  }
  // Byte `row * stride` of page `page` behind base (strides: launch_*4 sees to it that pages' have 32 bits and rows' 21).
  static __device__ __forceinline__ const uint8_t* at_row(const uint8_t* base, int page, int64_t page_stride, int row, int64_t row_stride) {
    return base + (uint64_t(uint32_t(page)) * uint32_t(page_stride) + uint32_t(row) * uint32_t(row_stride));
  }
  __device__ __forceinline__ const int8_t* exps_at(const int8_t* base, int page, int row) const {
    return base + ((int64_t(page) * a.pool.Hkv + hk) << a.pool.shift) * kExps + row * kExps;
  }
  __device__ __forceinline__ void load_k(const Pair& p) {
    const int rmask = (1 << a.pool.shift) - 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (F != ROWS) {
        const int row = p.s0[i] & rmask;
        const uint8_t* kp = at_row(a.pool.K + hk * a.pool.k_head, p.page[i], a.pool.k_page, row, a.pool.k_row);
        k[i] = *reinterpret_cast<const typename R::KReg*>(kp + (uint32_t(c) * uint32_t(a.pool.k_row) + g * (D / 8)));
        ke[i] = exps_at(a.pool.k_exp, p.page[i], row)[uint32_t(c * kExps + g * kExps / 4)];
      } else {
        // (rows that are not there: the first row of the pool, whose values are not used)
        const int s = p.s0[i] + c, pk = s < list.n ? a.pool.page_of(col.b, s) : -1;
        k[i] = *reinterpret_cast<const typename R::KReg*>((pk >= 0 ? a.pool.k_at(pk, hk, s) : a.pool.K) + g * (D / 8));
        ke[i] = a.pool.k_exp[(pk >= 0 ? a.pool.at(pk, hk, s) : 0) * kExps + g * kExps / 4];
      }
    }
  }
  __device__ __forceinline__ void load_v(const Pair& p) {
    const int rmask = (1 << a.pool.shift) - 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      absent[i] = 0;
      if constexpr (F != ROWS) {
        const int row = p.s0[i] & rmask;
        const uint8_t* vp = at_row(a.pool.V + hk * a.pool.v_head, p.page[i], a.pool.v_page, row, a.pool.v_row);
        const uint32_t voff = uint32_t(4 * g) * uint32_t(a.pool.v_row) + c * (E / 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const auto* at_v = reinterpret_cast<const typename R::VReg*>(vp + uint32_t(r) * uint32_t(a.pool.v_row) + voff);
          v[i][r] = STEP ? __builtin_nontemporal_load(at_v) : *at_v;
        }
        vx[i] = *reinterpret_cast<const typename R::KReg*>(exps_at(a.pool.v_exp, p.page[i], row) + uint32_t(4 * g * kExps));
      } else {
        const int s = p.s0[i] + c, pk = s < list.n ? a.pool.page_of(col.b, s) : -1;
        absent[i] = ~uint32_t(__ballot(pk >= 0)) & 0xFFFFu;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sv = p.s0[i] + 4 * g + r, pv = __shfl(pk, 4 * g + r, 64);
          v[i][r] = *reinterpret_cast<const typename R::VReg*>((pv >= 0 ? a.pool.v_at(pv, hk, sv) : a.pool.V) + c * (E / 2));
          const int8_t* ex = a.pool.v_exp + (pv >= 0 ? a.pool.at(pv, hk, sv) : 0) * kExps;
          if constexpr (D == 128)
            vx[i][r] = *reinterpret_cast<const uint32_t*>(ex);
          else
            vx[i][r / 2] = (r % 2 ? vx[i][r / 2] : 0u) | uint32_t(*reinterpret_cast<const uint16_t*>(ex)) << (16 * (r % 2));
        }
      }
    }
  }
  __device__ __forceinline__ void convert_k(int i, bf16x8 (&to)[kSteps]) const {
    const float scale = fp4_scale(ke[i]);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) to[j] = __builtin_bit_cast(bf16x8, fp4_decode8(k[i][j], scale));
  }
  // elements 2 y and 2 y + 1 of the lane's
  __device__ __forceinline__ void convert_v(int y, bf16x8 (&to)[2], const int (&ve)[2][4]) const {
      u32x4 even, odd;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        auto two = [&](int r) {
          const float scale = fp4_scale(ve[i / 2][r]);
          const uint32_t codes = v[i / 2][r];
          // (which byte has to be a constant)
          const bf16x2 x = y == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)
                           : y == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)
                           : y == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)
                                    : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
          return __builtin_bit_cast(uint32_t, x);
        };
        const uint32_t x0 = two(i % 2 * 2), x1 = two(i % 2 * 2 + 1);
        even[i] = __builtin_amdgcn_perm(x1, x0, 0x05040100);
        odd[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302);
      }
      to[0] = __builtin_bit_cast(bf16x8, even);
      to[1] = __builtin_bit_cast(bf16x8, odd);
  }

  // Probabilities are formed as 2^-bias * p, so that no mean of values of any size overflows.  The step, whose logits and sums make scores, forms
  // (s - maximum) - bias; otherwise one multiply-add is left, from a maximum that is rounded so that it stays exact with bias added, and the sums of P, as it enters
  // the products, come from the matrix core too (P times ones).
  __device__ __forceinline__ void run(const bf16x8 (&q)[N][kSteps], float* lg) {
    const float scale2 = kLog2e / sqrtf(float(D));
    const float bias = list.bias, slack = STEP ? float(kSlack) : kSlack / scale2;
    bool large = false;  // (not STEP) exponents beyond 2^20, where an exact product less a rounded one is no longer small
    const bool by_pos = a.window != 0 && a.pool.pos;
    const int n = list.n;
    f32x4 lm[N];   // (not STEP) sums of P: register i: column 4 g + i
    float ref[N];  // what P is relative to, as an exponent
#pragma unroll
    for (int x = 0; x < N; ++x) {
      ref[x] = m[x] = kLowest;
      l[x] = 0.f;
      lm[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < E; ++e) om[x][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int t = t0 + w * 2;
    bf16x8 kop[2][kSteps];
    Pair now = pair_at(t), next = now;
    if (kAhead && t < t1) {
      load_k(now);
      load_v(now);
      next = pair_at(t + kLeast4);
      convert_k(0, kop[0]);
      convert_k(1, kop[1]);
      load_k(next);
    }
    while (t < t1) {
      if constexpr (!kAhead) {
        now = pair_at(t);
        load_k(now);
        load_v(now);
      }
      bool whole[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        whole[i] = now.there[i] && absent[i] == 0 && now.s0[i] + kTile - 1 <= all_last && !by_pos &&
                   (now.s0[i] >= all_lo || now.s0[i] + kTile <= a.n_sink);
      int ve[2][4];
      uint32_t bad = 0, is = 0xFFu;  // bits 4 i + r: a power of two that stands for NaN; an entry of the sequence, on a page
      const bool all = whole[0] && whole[1];
      auto powers = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if constexpr (D == 128)
              ve[i][r] = __builtin_amdgcn_sbfe(int(vx[i][r]), 8 * (c >> 2), 8);
            else
              ve[i][r] = __builtin_amdgcn_sbfe(int(vx[i][r / 2]), 16 * (r % 2) + 8 * (c >> 3), 8);
          }
        if (!all) {
          is = 0;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              // (no branches: where a lane's vector was changed behind some, one compiler kept the old element)
              const bool in = now.there[i] & (now.s0[i] + 4 * g + r < n) & !(absent[i] >> (4 * g + r) & 1), nan = in & (ve[i][r] == kNan4) & !whole[i];
              bad |= uint32_t(nan) << (4 * i + r);
              is |= uint32_t(in) << (4 * i + r);
              ve[i][r] = whole[i] ? ve[i][r] : in & !nan ? min(ve[i][r], 125) : 0;
            }
        }
      };
      if constexpr (kAhead) powers();  // (else behind the products, which wait for the keys alone)
      const Pair after = kAhead ? pair_at(t + 2 * kLeast4) : now;
      f32x4 s[N][2];
#pragma unroll
      for (int x = 0; x < N; ++x) s[x][0] = s[x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      bf16x8 vop[E / 2][2];
      if constexpr (kAhead) {
#pragma unroll
        for (int y = 0; y < E / 2; ++y) convert_v(y, vop[y], ve);
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int x = 0; x < N; ++x) s[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[i][j], q[x][j], s[x][i], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          convert_k(i, kop[i]);
#pragma unroll
          for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int x = 0; x < N; ++x) s[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kop[i][j], q[x][j], s[x][i], 0, 0, 0);
        }
      }
      if constexpr (kAhead) {
        // one product, then as much of the conversion as runs beside it
#pragma unroll
        for (int i = 0; i < 2 * kSteps * N; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, (9 * E + 8) / (2 * kSteps * N), 0);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) asm volatile("" : "+v"(vop[e / 2][e % 2]));  // (converted here, not later)
        load_v(next);  // (behind the last pair that one again: a branch would have the registers copied, and so waited for)
      }
      if constexpr (!kAhead) powers();
      if constexpr (STEP) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0][i / 4][i % 4] = product(s[0][i / 4][i % 4], scale2);
      }
      uint32_t seen[N];  // bit 4 i + r: column x of the lane's sees entry 4 g + r of tile i
#pragma unroll
      for (int x = 0; x < N; ++x) seen[x] = 0xFFu;
      if (!all) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int e = now.s0[i] + 4 * g + r;
            int at = e;
            if (by_pos) {
              const int p = e < n ? a.pool.page_of(col.b, e) : -1;
              at = p >= 0 ? a.pool.pos[a.pool.at(p, hk, e)] : 0;
            }
#pragma unroll
            for (int x = 0; x < N; ++x) {
              const bool ok = bool(is >> (4 * i + r) & 1) & (e <= mine[x].last) & ((at >= mine[x].lo) | (at < a.n_sink));
              const float logit = s[x][i][r];
              s[x][i][r] = ok ? logit : -INFINITY;
              seen[x] &= ~(uint32_t(!ok) << (4 * i + r));
            }
          }
      }
      if constexpr (STEP) {
        if (lg && c < col.count) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (t + i < t1) *reinterpret_cast<f32x4*>(lg + now.s0[i] + 4 * g) = s[0][i];
        }
      }
      float mx[N];
      bool grown = false;
#pragma unroll
      for (int x = 0; x < N; ++x) {
        mx[x] = m[x];
#pragma unroll
        for (int i = 0; i < 8; ++i) mx[x] = fmaxf(mx[x], s[x][i / 4][i % 4]);
        grown |= mx[x] > m[x] + slack;
      }
      if (__any(grown)) {
#pragma unroll
        for (int x = 0; x < N; ++x) {
          mx[x] = max_rows(mx[x]);
          m[x] = mx[x];
          float to = m[x];
          if constexpr (!STEP) {  // up to 2^20 with as many bits as the sum with bias has; beyond, where each logit is multiplied and rounded first, as those are
            to = product(m[x], scale2);
            to = fabsf(to) > kFar ? to : (to + bias) - bias;
          }
          const float f = __builtin_amdgcn_exp2f(ref[x] - to);
          ref[x] = to;
          l[x] *= f;
          const f32x4 fh = {__shfl(f, 4 * g, 64), __shfl(f, 4 * g + 1, 64), __shfl(f, 4 * g + 2, 64), __shfl(f, 4 * g + 3, 64)};
#pragma unroll
          for (int e = 0; e < E; ++e) om[x][e] *= fh;
          lm[x] *= fh;
        }
        if constexpr (!STEP) {
          bool far = false;
#pragma unroll
          for (int x = 0; x < N; ++x) far |= fabsf(ref[x]) > kFar && m[x] != kLowest;
          large = __any(far);
        }
      }
      float times = scale2, less[N];
#pragma unroll
      for (int x = 0; x < N; ++x) less[x] = -(ref[x] + bias);
      if (large) {
        times = 1.f;
#pragma unroll
        for (int x = 0; x < N; ++x) {
          less[x] = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) s[x][i / 4][i % 4] = (product(s[x][i / 4][i % 4], scale2) - ref[x]) - bias;
        }
      }
#pragma unroll
      for (int x = 0; x < N; ++x) {
        u32x4 hi2, lo2, third2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float p[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float logit = s[x][i / 2][i % 2 * 2 + y];
            p[y] = __builtin_amdgcn_exp2f(STEP ? (logit - ref[x]) - bias : fmaf(logit, times, less[x]));
            if constexpr (STEP) l[x] += p[y];
          }
          // x - h in one instruction each (x itself in the columns that have come to their term).  (Minus zero beside minus one: the pair 0, -1.0 in this
          // order would be written as the constant -1.0, which the instruction reads as a float's bits.)
          auto less_term = [&](const f32x2& x, const bf16x2& h, bool is) __attribute__((always_inline)) {
            const uint32_t one0 = is ? 0x8000BF80u : 0x80008000u, one1 = is ? 0xBF808000u : 0x80008000u;
            return f32x2{__builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, one0), x[0], false),
                         __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, one1), x[1], false)};
          };
          const f32x2 all24 = {p[0], p[1]};
          const bf16x2 h = __builtin_convertvector(all24, bf16x2);
          const f32x2 rest = less_term(all24, h, PARTS == 1 || c >= kPart<PARTS>);
          const bf16x2 l = __builtin_convertvector(rest, bf16x2);
          hi2[i] = __builtin_bit_cast(uint32_t, h);
          lo2[i] = __builtin_bit_cast(uint32_t, l);
          if constexpr (STEP) {
            third2[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(less_term(rest, l, PARTS < 3 || c >= 2 * kPart<PARTS>), bf16x2));
            if (PARTS == 2) third2[i] = c >= kPart<PARTS> ? third2[i] : 0u;
          }
        }
        const bf16x8 hi = __builtin_bit_cast(bf16x8, hi2), lo = __builtin_bit_cast(bf16x8, lo2), third = __builtin_bit_cast(bf16x8, third2);
        if constexpr (kAhead) {
#pragma unroll
          for (int e = 0; e < E; ++e) om[x][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, vop[e / 2][e % 2], om[x][e], 0, 0, 0);
          const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
          lm[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, ones, lm[x], 0, 0, 0);
          lm[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, ones, lm[x], 0, 0, 0);
#pragma unroll
          for (int e = 0; e < E; ++e) om[x][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, vop[e / 2][e % 2], om[x][e], 0, 0, 0);
        } else {
          static_assert(kAhead || N == 1, "V is converted where it is used");
#pragma unroll
          for (int y = 0; y < E / 2; ++y) {
            bf16x8 two[2];
            convert_v(y, two, ve);
            auto add = [&](const bf16x8& term) __attribute__((always_inline)) {
#pragma unroll
              for (int i = 0; i < 2; ++i) om[x][2 * y + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(term, two[i], om[x][2 * y + i], 0, 0, 0);
            };
            add(third);
            if constexpr (PARTS < 3) add(lo);
            if constexpr (PARTS < 2) add(hi);
          }
        }
      }
      if constexpr (kAhead) {
        convert_k(0, kop[0]);
        convert_k(1, kop[1]);
        // the first columns' probabilities; the next ones' beside the products of those before, the next keys' conversion beside the last
        __builtin_amdgcn_sched_group_barrier(0x002, 33, 1);
#pragma unroll
        for (int i = 0; i < N * (2 * E + 2); ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
          __builtin_amdgcn_sched_group_barrier(0x002, 2, 1);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < kSteps; ++j) asm volatile("" : "+v"(kop[i][j]));
        load_k(after);
      }
      if (__any(bad != 0)) {
        // columns that see an entry whose block is NaN: counted by a product of ones
#pragma unroll
        for (int x = 0; x < N; ++x) {
          u32x4 sees, nan;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sees[i] = (seen[x] >> (2 * i) & 1 ? 0x3F80u : 0u) | (seen[x] >> (2 * i + 1) & 1 ? 0x3F800000u : 0u);
            nan[i] = (bad >> (2 * i) & 1 ? 0x3F80u : 0u) | (bad >> (2 * i + 1) & 1 ? 0x3F800000u : 0u);
          }
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          const f32x4 met = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, sees), __builtin_bit_cast(bf16x8, nan), zero, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float poison = met[i] > 0.f ? __uint_as_float(0x7FC00000u) : 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) om[x][e][i] += poison;
          }
        }
      }
      t += kLeast4;
      now = next;
      next = after;
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      m[x] = ref[x];
      l[x] = sum_rows(l[x]);
      if constexpr (!STEP) {  // the lane of column c: register c % 4 of a lane of row c / 4
        const float y = c % 4 == 0 ? lm[x][0] : c % 4 == 1 ? lm[x][1] : c % 4 == 2 ? lm[x][2] : lm[x][3];
        l[x] = __shfl(y, (c >> 2) * 16 + c, 64);
      }
    }
  }
};

template <int D>
struct AttendShared {
  float o[kWaves][kCols][D];
  float ml[kWaves][kCols][2];
  float M[kCols], inv[kCols], sum[kCols];  // of the whole workgroup
  float f[kWaves][kCols];                  // what a wavefront's outputs count for
};

// Four elements of an output.
__device__ __forceinline__ void store_out4(uint16_t* to, const f32x4& o) {
  *reinterpret_cast<u32x2*>(to) = u32x2{uint32_t(Elem<uint16_t>::from_f32(o[0])) | uint32_t(Elem<uint16_t>::from_f32(o[1])) << 16,
                                        uint32_t(Elem<uint16_t>::from_f32(o[2])) | uint32_t(Elem<uint16_t>::from_f32(o[3])) << 16};
}
// Displacement of column `at` in q or out.
__device__ __forceinline__ int64_t column_at(const AttendArgs& a, const View& v, const Columns& col, int hk, int at) {
  const int r = col.base + at, token = a.token_of(r);
  return int64_t(col.token0 + token) * v.sn + int64_t(hk * a.G + r - token * a.G) * v.sh;
}


// A workgroup's share: its columns in N groups of 16.  `part`: which partial result.
template <int D, Finds F, bool STEP, int N, int PARTS>
__device__ __forceinline__ void attend_share(const AttendArgs& a, const Columns& col, const TileList& list, const Sight (&mine)[N], int hk, int share,
                                             int part, AttendShared<D>& sh) {
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4, b = col.b;
  const int t0 = share * list.share, t1 = min(t0 + list.share, list.tiles);
  if (t0 >= t1) return;
  constexpr int E = D / 16, kSteps = D / 32;
  if constexpr (STEP) {
    // the workgroup of the last tile stores the new token, and reads it back as it was encoded
    if (a.kn.ptr && t1 == list.tiles && a.lens[b] <= a.max_len) {
      const int page = a.pool.page_of(b, list.n - 1);
      if (page >= 0) store_new<uint16_t, Code4, D>(a, b, hk, page, list.n - 1, list.last);
      __threadfence_block();
      __syncthreads();
    }
  }
  // where every column sees a tile as a whole: entries up to the first column's last, from the latest window on
  int all_last, all_lo = INT32_MIN;
  if constexpr (STEP) {
    all_last = list.n - 1;
    all_lo = mine[0].lo;
  } else {
    all_last = __builtin_amdgcn_readfirstlane(mine[0].last);
    if (a.window != 0) {
      int latest = INT32_MAX;  // (complement: the minimum of ~lo)
#pragma unroll
      for (int x = 0; x < N; ++x) latest = min(latest, x * kCols + c < col.count ? ~mine[x].lo : INT32_MAX);
      all_lo = __builtin_amdgcn_readfirstlane(~row_min(latest));
    }
  }
  bf16x8 q[N][kSteps];
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const uint16_t* row = nullptr;
    const int head = head_of<PARTS>(c);  // (of the step)
    if (x * kCols + head < col.count) {
      if constexpr (STEP)
        row = static_cast<const uint16_t*>(a.q.ptr) + b * a.q.sb + (hk * a.G + head) * a.q.sh;
      else
        row = static_cast<const uint16_t*>(a.q.ptr) + column_at(a, a.q, col, hk, x * kCols + c);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      q[x][i] = row ? *reinterpret_cast<const bf16x8*>(row + g * (D / 4) + i * 8) : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  }
  float* lg = STEP && a.pool.score ? a.logits + (int64_t(b) * a.Hq + hk * a.G + c) * a.pad : nullptr;
  Share<D, F, STEP, N, PARTS> work{a, col, list, hk, t0, t1, mine, w, lane, c, g, all_last, all_lo};
  work.run(q, lg);
  const bool single = list.shares() == 1;
  // join the wavefronts, 16 columns at a time
#pragma unroll
  for (int x = 0; x < N; ++x) {
    if (x) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<f32x4*>(&sh.o[w][4 * g + i][c * E + e]) = f32x4{work.om[x][e][i], work.om[x][e + 1][i], work.om[x][e + 2][i], work.om[x][e + 3][i]};
    if (lane < kCols) {
      sh.ml[w][lane][0] = work.m[x];
      sh.ml[w][lane][1] = work.l[x];
    }
    __threadfence_block();  // (the logits, which the whole workgroup reads where it is a head's only one)
    __syncthreads();
    const int cols = min(col.count - x * kCols, kCols);
    if (tid < cols) {  // a thread per column: what each wavefront's outputs count for
      float M = sh.ml[0][tid][0], f[kWaves], L = 0.f;
#pragma unroll
      for (int y = 1; y < kWaves; ++y) M = fmaxf(M, sh.ml[y][tid][0]);
#pragma unroll
      for (int y = 0; y < kWaves; ++y) {
        f[y] = __builtin_amdgcn_exp2f(sh.ml[y][tid][0] - M);
        L = fmaf(sh.ml[y][tid][1], f[y], L);
      }
      if (single) {
        sh.M[tid] = M;
        sh.inv[tid] = L == 0.f ? 0.f : ldexpf(1.f / L, -list.bias);
        sh.sum[tid] = L;
      } else {
        const int64_t row = int64_t(part) * (STEP ? a.G : kGroup) + x * kCols + tid;
        a.part_ml[row * 2] = M;
        a.part_ml[row * 2 + 1] = L;
      }
#pragma unroll
      for (int y = 0; y < kWaves; ++y) sh.f[y][tid] = f[y];
    }
    __syncthreads();
    const int at = tid % (D / 4) * 4;
    for (int h = tid / (D / 4); h < cols; h += 64 * kWaves / (D / 4)) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < kWaves; ++y) {
        f32x4 one = *reinterpret_cast<const f32x4*>(&sh.o[y][h][at]);
#pragma unroll
        for (int i = 1; i < PARTS; ++i) one += *reinterpret_cast<const f32x4*>(&sh.o[y][h + i * kPart<PARTS>][at]);
        o += one * sh.f[y][h];
      }
      if (single) {
        const float L = sh.sum[h];
        o = L == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o / L;
        store_out4(STEP ? static_cast<uint16_t*>(a.out.ptr) + b * a.out.sb + (hk * a.G + h) * a.out.sh + at
                        : static_cast<uint16_t*>(a.out.ptr) + column_at(a, a.out, col, hk, x * kCols + h) + at, o);
      } else {
        const int64_t row = int64_t(part) * (STEP ? a.G : kGroup) + x * kCols + h;
        *reinterpret_cast<f32x4*>(a.part_o + row * D + at) = o;
      }
    }
  }
  if constexpr (STEP) {
    if (lg && single) {
      __syncthreads();
      for (int i = tid; i < list.tiles * kTile; i += 64 * kWaves)
        add_scores<1, kCols>(a, list, b, hk, i, 0, list.tiles * kTile, sh.M, sh.inv, [] {});
    }
  }
}

// The step: a workgroup per (share, sequence and KV head), whose columns are the group's query heads.  8 heads x 131072 entries: 33 us, 4.3 TB/s; conversions and
// products take 20 us to issue.
template <int D, Finds F, int PARTS>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(4))) void step_part4(AttendArgs a) {
  __shared__ AttendShared<D> sh;
  const int b = blockIdx.y / a.pool.Hkv, hk = blockIdx.y % a.pool.Hkv;
  const TileList list(a, b, kLeast4);
  if (list.n == 0) {
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i < a.G * D; i += 64 * kWaves) store_out<uint16_t>(a, b, hk * a.G + i / D, i % D, 0.f);
    return;
  }
  const int c = threadIdx.x & 15;
  const Sight mine[1] = {{head_of<PARTS>(c) < a.G ? list.n - 1 : -1, window_start(list.last, a.window)}};
  attend_share<D, F, true, 1, PARTS>(a, Columns{b, 0, a.G, 0, 0, 0}, list, mine, hk, blockIdx.x, blockIdx.y * a.splits + blockIdx.x, sh);
}

// Several tokens per sequence: a workgroup per (group of columns, KV head, share).  2048 tokens on 32768 entries, 32 heads on 8: 1.58 ms, 0.67 PFLOP/s, three executed products
// per two counted; 232 vector instructions and 50 products per pair of tiles and 32 columns, which on this card run beside each other only in part.
template <int D, Finds F>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void attend_part4(AttendArgs a) {
  __shared__ AttendShared<D> sh;
  // neighbouring workgroups are of different KV heads: with eight of them (or a multiple) the groups of a sequence that read one head's rows share an L2
  const int hk = blockIdx.x % a.pool.Hkv, share = blockIdx.x / a.pool.Hkv % a.splits, index = blockIdx.x / a.pool.Hkv / a.splits;
  const int part = (index * a.pool.Hkv + hk) * a.splits + share;
  const Columns col = find_columns(a, index);
  if (col.count <= 0) return;
  auto go = [&](auto groups) __attribute__((always_inline)) {
    constexpr int N = decltype(groups)::value;
    Sight mine[N];
    TileList list;
    if (sights_of<N>(a, col, threadIdx.x & 15, mine, list)) {
      attend_share<D, F, false, N, 1>(a, col, list, mine, hk, share, part, sh);
    } else if (share == 0) {
      for (int i = threadIdx.x; i < col.count * D; i += 64 * kWaves) static_cast<uint16_t*>(a.out.ptr)[column_at(a, a.out, col, hk, i / D) + i % D] = 0;
    }
  };
  if (col.count > kCols)
    go(std::integral_constant<int, kGroup / kCols>{});
  else
    go(std::integral_constant<int, 1>{});
}

// Joins the shares: a workgroup per (16 columns of a group, KV head), 16 lanes per column.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void attend_join4(AttendArgs a) {
  constexpr int kParts = kGroup / kCols, kE = D / 16;
  const int x = blockIdx.x % kParts, hk = blockIdx.x / kParts % a.pool.Hkv, index = blockIdx.x / kParts / a.pool.Hkv;
  const Columns col = find_columns(a, index);
  if (col.count <= x * kCols) return;
  Sight mine[kParts];
  TileList list;
  if (!sights_of<kParts>(a, col, threadIdx.x & 15, mine, list)) return;
  const int ns = list.shares();
  if (ns <= 1) return;
  const int h = x * kCols + int(threadIdx.x >> 4), c = threadIdx.x & 15;
  const bool is = h < col.count;
  const int64_t at0 = (int64_t(index) * a.pool.Hkv + hk) * a.splits * kGroup + (is ? h : x * kCols);  // (share s: + s * kGroup)
  const float* ml = a.part_ml + at0 * 2;
  float M = kLowest, L = 0.f;
  for (int s = c; s < ns; s += 16) M = fmaxf(M, ml[int64_t(s) * kGroup * 2]);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  for (int s = c; s < ns; s += 16) L = fmaf(ml[int64_t(s) * kGroup * 2 + 1], __builtin_amdgcn_exp2f(ml[int64_t(s) * kGroup * 2] - M), L);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) L += __shfl_xor(L, o, 64);
  f32x4 o[kE / 4] = {};
#pragma unroll 4
  for (int s = 0; s < ns; ++s) {
    const float f = __builtin_amdgcn_exp2f(ml[int64_t(s) * kGroup * 2] - M);
#pragma unroll
    for (int y = 0; y < kE / 4; ++y) o[y] += *reinterpret_cast<const f32x4*>(a.part_o + (at0 + int64_t(s) * kGroup) * D + c * kE + y * 4) * f;
  }
  if (!is) return;
  uint16_t* out = static_cast<uint16_t*>(a.out.ptr) + column_at(a, a.out, col, hk, h) + c * kE;
#pragma unroll
  for (int y = 0; y < kE / 4; ++y) store_out4(out + y * 4, L == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[y] / L);
}

// Rows by pairs of tiles where a page holds whole pairs, and displacements, strides and alignment are as at_row and the loads of powers of two take them.
Finds finds_of(const PagePool& p) {
  const bool scalar = p.k_row < (1 << 21) && p.v_row < (1 << 21) && p.k_page < (int64_t(1) << 32) && p.v_page < (int64_t(1) << 32) &&
                      !(reinterpret_cast<uintptr_t>(p.v_exp) & 15);
  return !scalar || p.shift < 4 ? ROWS : p.shift == 4 ? TILES : PAIRS;
}

template <int D, int PARTS>
auto step_kernel(Finds f) {
  return f == PAIRS ? step_part4<D, PAIRS, PARTS> : f == TILES ? step_part4<D, TILES, PARTS> : step_part4<D, ROWS, PARTS>;
}
template <int D>
void launch_step4(AttendArgs& a, int batch, hipStream_t s) {
  const int bh = batch * a.pool.Hkv;
  const Finds f = finds_of(a.pool);
  const auto part = a.G <= kPart<3> ? step_kernel<D, 3>(f) : a.G <= kPart<2> ? step_kernel<D, 2>(f) : step_kernel<D, 1>(f);
  part<<<dim3(a.splits, bh), 64 * kWaves, 0, s>>>(a);
  if (a.splits == 1) return;
  a.joins = batch * a.Hq;
  const int64_t scores = a.pool.score ? int64_t((a.pad + kFinishEntries - 1) / kFinishEntries) * bh : 0;
  const auto finish = a.G == 1 ? step_finish<uint16_t, D, 1> : a.G == 2 ? step_finish<uint16_t, D, 2> : a.G <= 4 ? step_finish<uint16_t, D, 4>
                      : a.G <= 8 ? step_finish<uint16_t, D, 8> : step_finish<uint16_t, D, 16>;
  finish<<<dim3(unsigned(a.joins + scores)), kFinish, 0, s>>>(a, kLeast4);
}

template <int D>
void launch_attend4(const AttendArgs& a, hipStream_t s) {
  const Finds f = finds_of(a.pool);
  const unsigned heads = unsigned(a.groups) * a.pool.Hkv;
  const auto part = f == PAIRS ? attend_part4<D, PAIRS> : f == TILES ? attend_part4<D, TILES> : attend_part4<D, ROWS>;
  part<<<dim3(heads * a.splits), 64 * kWaves, 0, s>>>(a);
  if (a.splits > 1) attend_join4<D><<<dim3(heads * (kGroup / kCols)), 64 * kWaves, 0, s>>>(a);
}

// Groups of columns of n_tokens query tokens, at most: every sequence may leave its last one unfinished.
int64_t column_groups(const d2o_pages* p, int32_t n_tokens) {
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  return std::min(int64_t(n_tokens), int64_t(n_tokens) * G / kGroup + p->batch);
}
// Shares of a group's tiles, for at most `tiles` tiles each: three workgroups per CU, of which two are there at a time, and shares of 32 tiles.  (Sixteen sequences
// of up to 8192 entries, 8 KV heads, 1 to 48 tokens: 91 us with two per CU, 73 with three, 80 with four or eight.)
constexpr int64_t kWanted = 768, kLeastShare = 32;
int attend_splits(int64_t heads, int64_t tiles) { return int(std::max<int64_t>(1, std::min(kWanted / heads, tiles / kLeastShare))); }
// Tiles of a share, so that `splits` of them hold the longest sequence: shorter ones take fewer.
int share_tiles(int64_t tiles, int splits) { return int(((tiles + splits - 1) / splits + kLeast4 - 1) / kLeast4 * kLeast4); }
// Bytes of the partial results of `parts` workgroups.
size_t part_bytes(const d2o_pages* p, int64_t parts) {
  const size_t rows = size_t(parts) * kGroup;
  return round256(rows * p->head_dim * sizeof(float)) + round256(rows * 2 * sizeof(float));
}
// What a call needs, and with how many shares.
size_t attend_bytes(const d2o_pages* p, int32_t max_len, int32_t n_tokens, int* splits) {
  const int64_t heads = column_groups(p, n_tokens) * p->n_kv_heads;
  *splits = attend_splits(heads, most_tiles(p, max_len, 0, 0));
  return *splits > 1 ? part_bytes(p, heads * *splits) : 0;
}
// What every call with as many tokens and entries or fewer needs: large ones have one share and need nothing, smaller ones several.  (heads * splits, where
// splits > 1, is at most kWanted and at most heads times the shares that a group may have, which both do not fall as tokens or entries rise.)
size_t attend_bytes_at_most(const d2o_pages* p, int32_t max_len, int32_t n_tokens) {
  const int64_t heads = column_groups(p, n_tokens) * p->n_kv_heads, shares = most_tiles(p, max_len, 0, 0) / kLeastShare;
  if (shares < 2 || p->n_kv_heads * 2 > kWanted) return 0;
  return part_bytes(p, std::min(kWanted, heads * shares));
}

int check_attend(const d2o_pages* p, PagePool* pool, int32_t n_tokens, int32_t max_len) {
  const int rc = check_pages(p, pool);
  if (rc != D2O_OK) return rc;
  if (!p->cache_fp4) return D2O_ERR_UNSUPPORTED;
  if (n_tokens < 0 || max_len < 1) return D2O_ERR_INVALID_ARG;
  // products of tokens and heads that are formed in 32 bits, and the grid
  if (int64_t(n_tokens) * p->n_q_heads > 0xFFFFFFF || column_groups(p, n_tokens) * p->n_kv_heads > 0xFFFFF) return D2O_ERR_UNSUPPORTED;
  return D2O_OK;
}

}  // namespace

void launch_step4(StepArgs& args, int batch, int D, hipStream_t s) {
  AttendArgs a{args, nullptr, 0, 0, 0, 0};
  if (D == 64)
    launch_step4<64>(a, batch, s);
  else
    launch_step4<128>(a, batch, s);
}

}  // namespace d2o

using namespace d2o;

extern "C" int d2o_pages_attend_workspace_bytes(const d2o_pages* pages, int32_t n_tokens, int32_t max_len, size_t* bytes) {
  const int rc = check_attend(pages, nullptr, n_tokens, max_len);
  if (rc != D2O_OK) return rc;
  if (!bytes) return D2O_ERR_INVALID_ARG;
  *bytes = n_tokens == 0 ? 0 : attend_bytes_at_most(pages, max_len, n_tokens);
  return D2O_OK;
}

extern "C" int d2o_pages_attend(const d2o_pages* pages, d2o_view q, int32_t n_tokens, const int32_t* first, const int32_t* lens,
                                const int32_t* positions, int32_t max_len, int32_t window, int32_t n_sink, d2o_view out,
                                void* workspace, size_t workspace_bytes, void* stream) {
  AttendArgs a{};
  const int rc = check_attend(pages, &a.pool, n_tokens, max_len);
  if (rc != D2O_OK) return rc;
  if (window < 0 || n_sink < 0) return D2O_ERR_INVALID_ARG;
  if (n_tokens == 0) return D2O_OK;
  if (!first || !lens) return D2O_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(first) | reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(positions)) & 3) return D2O_ERR_INVALID_ARG;
  if (!dense_view_ok(q, 2, true) || !dense_view_ok(out, 2, true)) return D2O_ERR_INVALID_ARG;
  if (!rows_apart(out, {1, pages->n_q_heads, n_tokens}, pages->head_dim)) return D2O_ERR_INVALID_ARG;
  if (max_len > int64_t(pages->max_pages) * pages->page_size) return D2O_ERR_CAPACITY;
  const size_t need = attend_bytes(pages, max_len, n_tokens, &a.splits);
  if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return D2O_ERR_INVALID_ARG;
  if (workspace_bytes < need) return D2O_ERR_CAPACITY;
  a.q = to_view(q);
  a.out = to_view(out);
  a.first = first;
  a.lens = lens;
  a.positions = positions;
  a.n_tokens = n_tokens;
  a.batch = pages->batch;
  a.groups = int(column_groups(pages, n_tokens));
  const int64_t heads = int64_t(a.groups) * pages->n_kv_heads;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = need ? a.part_o + round256(size_t(heads) * a.splits * kGroup * pages->head_dim * sizeof(float)) / sizeof(float) : nullptr;
  const int64_t tiles = pages->pos || positions ? most_tiles(pages, max_len, 0, 0) : most_tiles(pages, max_len, window, n_sink, kGroup);
  a.splits = std::min(a.splits, attend_splits(heads, tiles));
  a.share = share_tiles(tiles, a.splits);
  a.Hq = pages->n_q_heads;
  a.G = pages->n_q_heads / pages->n_kv_heads;
  a.over_g = uint32_t(0xFFFFFFFFu / uint32_t(a.G)) + 1;  // (G = 1 is not divided by)
  a.max_len = max_len;
  a.window = window;
  a.n_sink = n_sink;
  a.pairs = 1;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (pages->head_dim == 64)
    launch_attend4<64>(a, s);
  else
    launch_attend4<128>(a, s);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
