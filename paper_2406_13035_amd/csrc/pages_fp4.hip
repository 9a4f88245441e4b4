// Attention over a cache in pages whose rows are held in 4 bits: one query token per sequence (d2o_pages_step) and several
// (d2o_pages_attend).
#include "pages_step.h"

namespace d2o {
namespace {

// Query tokens of a batch's sequences stand one behind the other (attend); a sequence's (token, query head of a KV head's group) pairs, in
// this order, are the columns of its products, sixteen to a workgroup.
struct AttendArgs : StepArgs {
  const int32_t* first;  // [B + 1] first query token of every sequence
  int32_t n_tokens, batch, groups;  // rows of q; groups of columns, at most
  __device__ __forceinline__ int token0(int b) const { return min(max(first[b], 0), n_tokens); }
  __device__ __forceinline__ int tokens(int b) const { return max(token0(b + 1) - token0(b), 0); }
};
constexpr int kCols = 16;
constexpr int kUnits4 = 1;                        // pairs of tiles of a wavefront's round
constexpr int kLeast4 = kWaves * 2 * kUnits4;  // tiles of a workgroup's round

// Which columns a workgroup has.  Step: the group's query heads of sequence b.
struct Columns {
  int b, base, count;  // sequence, first pair, pairs of the sequence from there on (0: none)
};
// The index-th group of kCols columns of the batch; all threads of the workgroup.
__device__ __forceinline__ Columns find_columns(const AttendArgs& a, int index) {
  __shared__ int sum[kWaves], found[3];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int per = (a.batch + 64 * kWaves - 1) / (64 * kWaves), b0 = tid * per, b1 = min(b0 + per, a.batch);
  int mine = 0;
  for (int b = b0; b < b1; ++b) mine += (a.tokens(b) * a.G + kCols - 1) / kCols;
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
      const int pairs = a.tokens(b) * a.G, n = (pairs + kCols - 1) / kCols;
      if (index < at + n) {
        found[0] = b;
        found[1] = (index - at) * kCols;
        found[2] = pairs - found[1];
        break;
      }
      at += n;
    }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1]), __builtin_amdgcn_readfirstlane(found[2])};
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
// Column c's sight, and the tiles that any of the columns sees.  Returns false where there are none.
__device__ __forceinline__ bool sight_of(const AttendArgs& a, const Columns& col, int c, int least, Sight& mine, TileList& list) {
  const int m = a.tokens(col.b), len = min(a.lens[col.b], a.max_len);
  const int token = (col.base + c) / a.G, last_token = (col.base + min(col.count, kCols) - 1) / a.G;
  const bool is = c < col.count;
  mine.last = is ? max(len - m + token, -1) : -1;
  mine.lo = window_start(a.positions && is ? a.positions[a.token0(col.b) + token] : mine.last, a.window);
  list.n = max(len - m + last_token + 1, 0);
  list.last = 0;
  if (list.n == 0) return false;
  const int lo = a.window == 0 ? 0 : __builtin_amdgcn_readfirstlane(row_min(is ? mine.lo : INT32_MAX));
  list.choose(a, lo, least);
  return true;
}

// Rows of D 4-bit elements, as the lanes hold them.  K: lane l has row l % 16 of a tile, a quarter of it; V: the 16 lanes of a row of lanes share
// a row, D / 16 elements each.
template <int D>
struct Row4 {
  static constexpr int kSteps = D / 32, kE = D / 16;
  typedef std::conditional_t<D == 128, u32x4, u32x2> KReg;       // also the powers of two of four rows
  typedef std::conditional_t<D == 128, uint32_t, uint16_t> VReg;
  static __device__ __forceinline__ uint32_t word(const KReg& k, int i) { return k[i]; }
};

// One workgroup per (sequence, KV head, 16 columns, share of the tiles they see).  As in the step over wider rows the logits S^T = K Q^T come from
// the matrix core, entries by columns, and leave in each lane of row of lanes g one column and the entries 4 g .. 4 g + 3 of a tile.  Of two tiles these
// are eight entries, which is what the lane has to hold of P as the left operand of P V (16 x 16 x 32): P goes from registers to the matrix core with no
// exchange.  The right operand wants eight entries of one element of V: a lane converts the D / 16 elements it has of each of the eight rows to
// bf16 (exact), two elements of one row at a time, and swaps halves between rows (a conversion and a permutation for two values).
// P as two bf16 terms, which hold 16 bits: a weight is off by 2^-16 of itself at most.  Codes are always finite and powers of two may stand for NaN: where
// columns see different entries, NaN is left out of the product, in which 0 * NaN would reach columns that do not see it, and added to those that do.
// WIDE: a tile lies in one page (see the step over wider rows).
template <int D, bool WIDE, bool STEP>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void attend_part4(AttendArgs a) {
  typedef Row4<D> R;
  constexpr int E = R::kE, kExps = D / kBlock4, U = kUnits4;
  __shared__ float so[kWaves][kCols][D];
  __shared__ float sml[kWaves][kCols][2];
  __shared__ float sM[kCols], sinv[kCols];
  const int Hkv = a.pool.Hkv;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  Columns col;
  Sight mine;
  TileList list;
  int hk, share, part;  // part: which partial result, in units of shares
  if constexpr (STEP) {
    share = blockIdx.x;
    col.b = blockIdx.y / Hkv;
    hk = blockIdx.y % Hkv;
    col.base = 0;
    col.count = a.G;
    part = blockIdx.y * a.splits + share;
    list = TileList(a, col.b, kLeast4);
    if (list.n == 0) {
      if (share == 0)
        for (int i = tid; i < a.G * D; i += 64 * kWaves) store_out<uint16_t>(a, col.b, hk * a.G + i / D, i % D, 0.f);
      return;
    }
    mine.last = c < a.G ? list.n - 1 : -1;
    mine.lo = window_start(list.last, a.window);
  } else {
    const int index = blockIdx.x / a.splits / Hkv;
    share = blockIdx.x % a.splits;
    hk = blockIdx.x / a.splits % Hkv;
    part = blockIdx.x;
    col = find_columns(a, index);
    if (col.count <= 0) return;
    if (!sight_of(a, col, c, kLeast4, mine, list)) {
      if (share == 0)
        for (int i = tid; i < min(col.count, kCols) * D; i += 64 * kWaves) {
          const int r = col.base + i / D;
          (static_cast<uint16_t*>(a.out.ptr) + int64_t(a.token0(col.b) + r / a.G) * a.out.sn + int64_t(hk * a.G + r % a.G) * a.out.sh)[i % D] = 0;
        }
      return;
    }
  }
  const int b = col.b, cols = min(col.count, kCols);
  const int t0 = share * list.share, t1 = min(t0 + list.share, list.tiles);
  if (t0 >= t1) return;
  const int n = list.n;
  if constexpr (STEP) {
    // the workgroup of the last tile stores the new token, and reads it back as it was encoded
    if (a.kn.ptr && t1 == list.tiles && a.lens[b] <= a.max_len) {
      const int page = a.pool.page_of(b, n - 1);
      if (page >= 0) store_new<uint16_t, Code4, D>(a, b, hk, page, n - 1, list.last);
      __threadfence_block();
      __syncthreads();
    }
  }
  // where every column sees a tile as a whole: entries up to the first column's last, from the last column's window on
  int all_last, all_lo = INT32_MIN;
  if constexpr (!STEP) {
    all_last = __builtin_amdgcn_readfirstlane(__shfl(mine.last, 0, 64));
    if (a.window != 0) {
      all_lo = __builtin_amdgcn_readfirstlane(~row_min(c < cols ? ~mine.lo : INT32_MAX));  // the latest start
    }
  } else {
    all_last = n - 1;
    all_lo = mine.lo;
  }
  const bool by_pos = a.window != 0 && a.pool.pos;
  bf16x8 q[R::kSteps];
  {
    const uint16_t* row = nullptr;
    if (c < cols) {
      const int r = col.base + c;
      if constexpr (STEP)
        row = static_cast<const uint16_t*>(a.q.ptr) + b * a.q.sb + (hk * a.G + r) * a.q.sh;
      else
        row = static_cast<const uint16_t*>(a.q.ptr) + int64_t(a.token0(b) + r / a.G) * a.q.sn + int64_t(hk * a.G + r % a.G) * a.q.sh;
    }
#pragma unroll
    for (int i = 0; i < R::kSteps; ++i)
      q[i] = row ? *reinterpret_cast<const bf16x8*>(row + g * (D / 4) + i * 8) : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  }
  const float scale2 = kLog2e / sqrtf(float(D));
  const float bias = list.bias;  // probabilities are formed as 2^-bias * p, so that no mean of values of any size overflows
  float m = -3.402823466e38f, l = 0.f;
  f32x4 om[E] = {};  // register i: column 4 g + i, element c * E + index
  float* lg = STEP && a.pool.score ? a.logits + (int64_t(b) * a.Hq + hk * a.G + c) * a.pad : nullptr;
  const auto table = (const __attribute__((address_space(4))) int32_t*)(a.pool.table + int64_t(b) * a.pool.max_pages);
  const int rmask = (1 << a.pool.shift) - 1;
  const uint32_t koff = uint32_t(c) * uint32_t(a.pool.k_row) + g * (D / 8), voff = uint32_t(4 * g) * uint32_t(a.pool.v_row) + c * (E / 2);
  for (int t = t0 + w * 2 * U; t < t1; t += kLeast4) {
    typename R::KReg k[2 * U], vx[2 * U];
    typename R::VReg v[2 * U][4];
    int ke[2 * U], s0[2 * U];
    bool there[2 * U], whole[2 * U];
    uint32_t absent[2 * U];  // (not WIDE) bit i: entry i of the tile has no page
#pragma unroll
    for (int u = 0; u < 2 * U; ++u) {
      s0[u] = list.slot(min(t + u, t1 - 1));
      there[u] = t + u < t1;
      absent[u] = 0;
      if constexpr (WIDE) {
        const int page = table[s0[u] >> a.pool.shift];
        there[u] = there[u] && uint32_t(page) < uint32_t(a.pool.n_pages);
        const int p = uint32_t(page) < uint32_t(a.pool.n_pages) ? page : 0;
        const int64_t at = ((int64_t(p) * Hkv + hk) << a.pool.shift) + (s0[u] & rmask);
        const uint8_t* kp = a.pool.K + p * a.pool.k_page + hk * a.pool.k_head + (s0[u] & rmask) * a.pool.k_row;
        const uint8_t* vp = a.pool.V + p * a.pool.v_page + hk * a.pool.v_head + (s0[u] & rmask) * a.pool.v_row;
        k[u] = *reinterpret_cast<const typename R::KReg*>(kp + koff);
        ke[u] = (a.pool.k_exp + at * kExps)[uint32_t(c * kExps + g * kExps / 4)];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[u][r] = __builtin_nontemporal_load(reinterpret_cast<const typename R::VReg*>(vp + r * a.pool.v_row + voff));
        vx[u] = *reinterpret_cast<const typename R::KReg*>(a.pool.v_exp + at * kExps + uint32_t(4 * g * kExps));
      } else {
        // (rows that are not there: the first row of the pool, whose values are not used)
        const int s = s0[u] + c, pk = s < n ? a.pool.page_of(b, s) : -1;
        absent[u] = ~uint32_t(__ballot(pk >= 0)) & 0xFFFFu;
        const uint8_t* kr = pk >= 0 ? a.pool.k_at(pk, hk, s) : a.pool.K;
        k[u] = *reinterpret_cast<const typename R::KReg*>(kr + g * (D / 8));
        ke[u] = a.pool.k_exp[(pk >= 0 ? a.pool.at(pk, hk, s) : 0) * kExps + g * kExps / 4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sv = s0[u] + 4 * g + r, pv = __shfl(pk, 4 * g + r, 64);
          const uint8_t* vr = pv >= 0 ? a.pool.v_at(pv, hk, sv) : a.pool.V;
          v[u][r] = *reinterpret_cast<const typename R::VReg*>(vr + c * (E / 2));
          const int8_t* ex = a.pool.v_exp + (pv >= 0 ? a.pool.at(pv, hk, sv) : 0) * kExps;
          if constexpr (D == 128)
            vx[u][r] = *reinterpret_cast<const uint32_t*>(ex);
          else
            vx[u][r / 2] = (r % 2 ? vx[u][r / 2] : 0u) | uint32_t(*reinterpret_cast<const uint16_t*>(ex)) << (16 * (r % 2));
        }
      }
      whole[u] = there[u] && absent[u] == 0 && s0[u] + kTile - 1 <= all_last && !by_pos &&
                 (s0[u] >= all_lo || s0[u] + kTile <= a.n_sink);
    }
#pragma unroll
    for (int u2 = 0; u2 < U; ++u2) {
      f32x4 s[2];
      int ve[2][4];
      uint32_t bad = 0;      // bit 4 i + r: a power of two that stands for NaN
      uint32_t seen = 0xFFu;  // bit 4 i + r: this lane's column sees entry 4 g + r of tile i
      float mx = m;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = 2 * u2 + i;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        const float scale = fp4_scale(ke[u]);
#pragma unroll
        for (int j = 0; j < R::kSteps; ++j)
          x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fp4_decode8(k[u][j], scale)), q[j], x, 0, 0, 0);
        s[i] = x * scale2;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (D == 128)
            ve[i][r] = __builtin_amdgcn_sbfe(int(vx[u][r]), 8 * (c >> 2), 8);
          else
            ve[i][r] = __builtin_amdgcn_sbfe(int(vx[u][r / 2]), 16 * (r % 2) + 8 * (c >> 3), 8);
        }
        if (!whole[u]) {
          int32_t at[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            at[r] = s0[u] + 4 * g + r;
            if (by_pos) {
              const int p = at[r] < n ? a.pool.page_of(b, at[r]) : -1;
              at[r] = p >= 0 ? a.pool.pos[a.pool.at(p, hk, at[r])] : 0;
            }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            // (no branches: where a lane's vector was changed behind some, one compiler kept the old element)
            const int e = s0[u] + 4 * g + r;
            const bool is = there[u] & (e < n) & !(absent[u] >> (4 * g + r) & 1);
            const bool ok = is & (e <= mine.last) & ((at[r] >= mine.lo) | (at[r] < a.n_sink)), nan = is & (ve[i][r] == kNan4);
            const float logit = s[i][r];
            s[i][r] = ok ? logit : -INFINITY;
            seen &= ~(uint32_t(!ok) << (4 * i + r));
            bad |= uint32_t(nan) << (4 * i + r);
            ve[i][r] = is & !nan ? min(ve[i][r], 125) : 0;
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[i][r]);
        if (lg && c < cols && t + u < t1) *reinterpret_cast<f32x4*>(lg + list.slot(t + u) + 4 * g) = s[i];
      }
      mx = max_rows(mx);
      if (__any(mx > m)) {
        const float f = __builtin_amdgcn_exp2f(m - mx);
        m = mx;
        l *= f;
        const f32x4 fh = {__shfl(f, 4 * g, 64), __shfl(f, 4 * g + 1, 64), __shfl(f, 4 * g + 2, 64), __shfl(f, 4 * g + 3, 64)};
#pragma unroll
        for (int e = 0; e < E; ++e) om[e] *= fh;
      }
      bf16x8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f((s[i / 4][i % 4] - m) - bias);
        l += p;
        hi[i] = __bf16(p);
        lo[i] = __bf16(p - float(hi[i]));
      }
#pragma unroll
      for (int y = 0; y < E / 2; ++y) {  // elements 2 y and 2 y + 1 of the lane's
        u32x4 even, odd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int u = 2 * u2 + i / 2, r = i % 2 * 2;
          auto two = [&](int rr) {
            const float scale = fp4_scale(ve[i / 2][rr]);
            const uint32_t codes = v[u][rr];
            // (which byte has to be a constant)
            const bf16x2 x = y == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)
                             : y == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)
                             : y == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)
                                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
            return __builtin_bit_cast(uint32_t, x);
          };
          const uint32_t x0 = two(r), x1 = two(r + 1);
          even[i] = __builtin_amdgcn_perm(x1, x0, 0x05040100);
          odd[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302);
        }
        om[2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, __builtin_bit_cast(bf16x8, even), om[2 * y], 0, 0, 0);
        om[2 * y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, __builtin_bit_cast(bf16x8, even), om[2 * y], 0, 0, 0);
        om[2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, __builtin_bit_cast(bf16x8, odd), om[2 * y + 1], 0, 0, 0);
        om[2 * y + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, __builtin_bit_cast(bf16x8, odd), om[2 * y + 1], 0, 0, 0);
      }
      if (__any(bad != 0)) {
        // columns that see an entry whose block is NaN: counted by a product of ones
        u32x4 sees, nan;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sees[i] = (seen >> (2 * i) & 1 ? 0x3F80u : 0u) | (seen >> (2 * i + 1) & 1 ? 0x3F800000u : 0u);
          nan[i] = (bad >> (2 * i) & 1 ? 0x3F80u : 0u) | (bad >> (2 * i + 1) & 1 ? 0x3F800000u : 0u);
        }
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const f32x4 met = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, sees), __builtin_bit_cast(bf16x8, nan), zero, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (met[i] > 0.f)
#pragma unroll
            for (int e = 0; e < E; ++e) om[e][i] = __uint_as_float(0x7FC00000u);
      }
    }
  }
  // join the wavefronts
  l = sum_rows(l);
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) so[w][4 * g + i][c * E + e] = om[e][i];
  if (lane < kCols) {
    sml[w][lane][0] = m;
    sml[w][lane][1] = l;
  }
  __threadfence_block();  // (the logits, which the whole workgroup reads where it is a head's only one)
  __syncthreads();
  const bool single = list.shares() == 1;
  for (int i = tid; i < cols * D; i += 64 * kWaves) {
    const int h = i / D, x0 = i % D;
    float M = sml[0][h][0];
#pragma unroll
    for (int x = 1; x < kWaves; ++x) M = fmaxf(M, sml[x][h][0]);
    float L = 0.f, o = 0.f;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const float fx = __builtin_amdgcn_exp2f(sml[x][h][0] - M);
      L = fmaf(sml[x][h][1], fx, L);
      o = fmaf(so[x][h][x0], fx, o);
    }
    const int64_t at = int64_t(part) * (STEP ? a.G : kCols) + h;
    if (single) {
      const float y = L == 0.f ? 0.f : o / L;
      if constexpr (STEP) {
        store_out<uint16_t>(a, b, hk * a.G + h, x0, y);
      } else {
        const int r = col.base + h;
        (static_cast<uint16_t*>(a.out.ptr) + int64_t(a.token0(b) + r / a.G) * a.out.sn + int64_t(hk * a.G + r % a.G) * a.out.sh)[x0] =
            Elem<uint16_t>::from_f32(y);
      }
    } else {
      a.part_o[at * D + x0] = o;
    }
    if (x0 == 0) {
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
      add_scores<1, kCols>(a, list, b, hk, i, 0, list.tiles * kTile, sM, sinv, [] {});
  }
}

// Joins the shares of 16 columns: a workgroup per (group of columns, KV head), a wavefront per column at a time.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void attend_join4(AttendArgs a, int least) {
  const int index = blockIdx.x / a.pool.Hkv, hk = blockIdx.x % a.pool.Hkv;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Columns col = find_columns(a, index);
  if (col.count <= 0) return;
  Sight mine;
  TileList list;
  if (!sight_of(a, col, lane & 15, least, mine, list)) return;
  const int ns = list.shares();
  if (ns <= 1) return;
  for (int h = w; h < min(col.count, kCols); h += kWaves) {
    const int64_t at0 = int64_t(blockIdx.x) * a.splits * kCols + h;  // (share s: + s * kCols)
    const float* ml = a.part_ml + at0 * 2;
    float M = -3.402823466e38f, L = 0.f;
    for (int s = lane; s < ns; s += 64) M = fmaxf(M, ml[int64_t(s) * kCols * 2]);
    M = wave_max(M);
    for (int s = lane; s < ns; s += 64) L = fmaf(ml[int64_t(s) * kCols * 2 + 1], __builtin_amdgcn_exp2f(ml[int64_t(s) * kCols * 2] - M), L);
    L = wave_sum(L);
    float o[D / 64] = {};
#pragma unroll 4
    for (int s = 0; s < ns; ++s) {
      const float f = __builtin_amdgcn_exp2f(ml[int64_t(s) * kCols * 2] - M);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) o[x] = fmaf(a.part_o[(at0 + int64_t(s) * kCols) * D + x * 64 + lane], f, o[x]);
    }
    const int r = col.base + h;
    uint16_t* out = static_cast<uint16_t*>(a.out.ptr) + int64_t(a.token0(col.b) + r / a.G) * a.out.sn + int64_t(hk * a.G + r % a.G) * a.out.sh;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) out[x * 64 + lane] = Elem<uint16_t>::from_f32(L == 0.f ? 0.f : o[x] / L);
  }
}

bool wide_pages(const PagePool& p) {
  // pages that hold whole tiles, displacements that fit, powers of two that can be read sixteen bytes at a time
  return p.shift >= 4 && p.k_row < (1 << 24) && p.v_row < (1 << 24) && !(reinterpret_cast<uintptr_t>(p.v_exp) & 15);
}

template <int D>
void launch_step4(AttendArgs& a, int batch, hipStream_t s) {
  const int bh = batch * a.pool.Hkv;
  const auto part = wide_pages(a.pool) ? attend_part4<D, true, true> : attend_part4<D, false, true>;
  part<<<dim3(a.splits, bh), 64 * kWaves, 0, s>>>(a);
  if (a.splits == 1) return;
  a.joins = batch * a.Hq;
  const int64_t scores = a.pool.score ? int64_t((a.pad + kFinishEntries - 1) / kFinishEntries) * bh : 0;
  step_finish<uint16_t, D, 16><<<dim3(unsigned(a.joins + scores)), kFinish, 0, s>>>(a, kLeast4);
}

template <int D>
void launch_attend4(const AttendArgs& a, hipStream_t s) {
  const auto part = wide_pages(a.pool) ? attend_part4<D, true, false> : attend_part4<D, false, false>;
  const unsigned heads = unsigned(a.groups) * a.pool.Hkv;
  part<<<dim3(heads * a.splits), 64 * kWaves, 0, s>>>(a);
  if (a.splits > 1) attend_join4<D><<<dim3(heads), 64 * kWaves, 0, s>>>(a, kLeast4);
}

// Groups of columns of n_tokens query tokens, at most: every sequence may leave its last one unfinished.
int64_t column_groups(const d2o_pages* p, int32_t n_tokens) {
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  return std::min(int64_t(n_tokens) * ((G + kCols - 1) / kCols), int64_t(n_tokens) * G / kCols + p->batch);
}
size_t attend_bytes(const d2o_pages* p, int32_t max_len, int32_t n_tokens, int* splits) {
  const int64_t heads = column_groups(p, n_tokens) * p->n_kv_heads;
  *splits = step_splits(heads, most_tiles(p, max_len, 0, 0));
  const size_t rows = size_t(heads) * *splits * kCols;
  return *splits > 1 ? round256(rows * p->head_dim * sizeof(float)) + round256(rows * 2 * sizeof(float)) : 0;
}

int check_attend(const d2o_pages* p, PagePool* pool, int32_t n_tokens, int32_t max_len) {
  const int rc = check_pages(p, pool);
  if (rc != D2O_OK) return rc;
  if (!p->cache_fp4) return D2O_ERR_UNSUPPORTED;
  if (n_tokens < 0 || max_len < 1) return D2O_ERR_INVALID_ARG;
  // products of tokens and heads that are formed in 32 bits, and the grid
  if (int64_t(n_tokens) * p->n_q_heads > 0x3FFFFFFF || column_groups(p, n_tokens) * p->n_kv_heads > 0x3FFFFF) return D2O_ERR_UNSUPPORTED;
  return D2O_OK;
}

}  // namespace

void launch_step4(StepArgs& args, int batch, int D, hipStream_t s) {
  AttendArgs a{args, nullptr, 0, 0, 0};
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
  int splits;
  *bytes = n_tokens == 0 ? 0 : attend_bytes(pages, max_len, n_tokens, &splits);
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
  a.part_ml = need ? a.part_o + round256(size_t(heads) * a.splits * kCols * pages->head_dim * sizeof(float)) / sizeof(float) : nullptr;
  a.splits = std::min(a.splits, step_splits(heads, most_tiles(pages, max_len, window, n_sink)));
  a.Hq = pages->n_q_heads;
  a.G = pages->n_q_heads / pages->n_kv_heads;
  a.max_len = max_len;
  a.window = window;
  a.n_sink = n_sink;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (pages->head_dim == 64)
    launch_attend4<64>(a, s);
  else
    launch_attend4<128>(a, s);
  return hipGetLastError() == hipSuccess ? D2O_OK : D2O_ERR_HIP;
}
