// One decode step of a cache that evicts by accumulated attention weight, or whose kept rows are held in 4 bits.
//
// With t = n_seen, e = t - window the position that leaves the ring, x_j the score of row j in units of log2:
//   e goes behind the kept entries, or in the place of the one with the lowest key if its own key is higher (sinks: +inf);
//   the incoming token takes ring slot t % window;
//   out = sum_j p_j v_j over ring and kept entries as they are then, p_j = 2^(x_j - M) / L;
//   by accumulated weight, every entry's key grows by the sum of its p_j over the group's query heads.
//
// Two launches.  The first streams the rows as they lie, cut into shares of a head's ring blocks and kept blocks of 32 rows: a
// workgroup's waves take blocks in turn and keep a running maximum, sum and output, and leave their rows' scores in the workspace.
// Two rows are left out of the stream, because what is at their place differs before and after the step: the ring slot t % window,
// and, when the kept set is full and e may displace an entry, the lowest entry of the share.  The second launch knows the lowest
// entries of all shares: it adds the ones that stay, e if it was taken and the incoming token to the softmax, and with the
// normaliser known adds the weights, each workgroup to its own share's keys; the first workgroup of a head moves the rows.
//
//   S^T[row, head] = K . Q^T       v_mfma_f32_16x16x32_bf16; K rows straight from memory into the A operand
//   O^T[d, head] += V^T . P^T      V in registers, eight rows of a few channels per lane, brought into the A operand's order by
//                                  byte permutes; P from S^T's accumulators without leaving the lane: tile row m = 4 kg + r of
//                                  tile j is row 8 kg + 4 j + r, so a lane's eight probabilities are eight consecutive rows
// P is a bf16 value and the bf16 rounding of what that leaves out: 16 bits, against the 8 of the output.  For up to eight query
// heads the two are columns of one matrix instruction, else two instructions.  fp32 storage: v_mfma_f32_16x16x4_f32 for both
// products, P in 32 bits.
#pragma once
#include "fp4_rows.h"
#include "kept_run.h"

namespace ltea {
namespace {

constexpr int kStreamWaves = 4, kStreamThreads = kStreamWaves * kWave, kFinishThreads = 256;

struct KeptParams {
  int B, Hq, Hkv, window, budget, sink, mass;
  float tau, scale2;             // scale * log2(e)
  const uint8_t* packed;         // null: rows in the storage type
  int32_t* status;
  KeptLayout L;
  float *plan, *shares, *scores;   // workspace
};

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Largest value over the four lanes that hold the same column (lane ^ 16, lane ^ 32).
__device__ __forceinline__ float column_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float column_sum(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// The order in which entries are displaced: lowest key first, of equal keys the latest position (of a caller's equal positions the
// last slot).
struct Entry { uint32_t key; int pos, slot; };       // slot < 0: none
__device__ __forceinline__ bool goes_before(const Entry& a, const Entry& b) {
  if (b.slot < 0) return a.slot >= 0;
  if (a.slot < 0) return false;
  if (a.key != b.key) return a.key < b.key;
  if (a.pos != b.pos) return a.pos > b.pos;
  return a.slot > b.slot;
}
__device__ __forceinline__ Entry first_of_wave(Entry x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const Entry y = {(uint32_t)__shfl_xor((int)x.key, off, kWave), __shfl_xor(x.pos, off, kWave), __shfl_xor(x.slot, off, kWave)};
    if (goes_before(y, x)) x = y;
  }
  return x;
}

// ---- 32 rows of a head in registers ------------------------------------------------------------------------------------------
// Stored rows.  K: piece i of tile j is 16 bytes of row 8 (c / 4) + 4 j + c % 4 of the block.  V: row 8 kg + u, a lane's channels
// are D / 16 consecutive ones of the row.
template <typename T, int D> struct StoredRows {
  static constexpr int kElems = 16 / (int)sizeof(T);        // elements of a piece
  static constexpr int KP = D / (4 * kElems);               // pieces per lane of a K row
  static constexpr int kRow = D * (int)sizeof(T);
  static constexpr int VB = kRow / 16;                      // bytes per lane of a V row: 8, 16 or 32
  u32x4 k[2][KP];
  uint32_t v[8][VB / 4];
  // channel of element x of piece i of lane quarter kg
  static __device__ __forceinline__ int k_channel(int i, int kg, int x) { return 4 * kElems * i + kElems * kg + x; }
  __device__ __forceinline__ void load(const void* ks, const void* vs, int n_rows) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, kg = lane >> 4;
    auto same = [](const void* p) {
      const uint64_t a = reinterpret_cast<uint64_t>(p);
      return reinterpret_cast<void*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 |
                                     (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
    };
    const uint32_t bytes = __builtin_amdgcn_readfirstlane((uint32_t)n_rows * (uint32_t)kRow);
    const auto rk = __builtin_amdgcn_make_buffer_rsrc(same(ks), 0, bytes, 0x00020000);
    const auto rv = __builtin_amdgcn_make_buffer_rsrc(same(vs), 0, bytes, 0x00020000);
    constexpr int kNonTemporal = 2;
    const uint32_t ko = (uint32_t)((8 * (c >> 2) + (c & 3)) * kRow + 16 * kg), vo = (uint32_t)(8 * kg * kRow + VB * c);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < KP; ++i) k[j][i] = __builtin_amdgcn_raw_buffer_load_b128(rk, ko + 4 * j * kRow + 64 * i, 0, kNonTemporal);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if constexpr (VB == 8) {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rv, vo + u * kRow, 0, kNonTemporal);
        v[u][0] = x[0]; v[u][1] = x[1];
      } else {
#pragma unroll
        for (int p = 0; p < VB / 16; ++p) {
          const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rv, vo + u * kRow + 16 * p, 0, kNonTemporal);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[u][4 * p + e] = x[e];
        }
      }
    }
  }
  // rows that do not count hold anything: their values become zeros (their scores are masked)
  __device__ __forceinline__ void clear(uint32_t dead) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (dead >> u & 1u)
#pragma unroll
        for (int e = 0; e < VB / 4; ++e) v[u][e] = 0u;
  }
};

// The same 32 rows in 4 bits: a block as it is stored.
template <int D> struct PackedRows {
  static constexpr int KW = D / 8;         // words per lane: K codes of both tiles, and V codes of eight rows (D = 128: 8, D = 64: 4)
  u32x4 k[D / 64], v[D / 64];
  uint32_t ke;                             // exponent bytes of the lane's row in tiles 0 and 1
  u32x2 ve;                                // of its eight V rows
  static __device__ __forceinline__ int k_channel(int i, int kg, int x) { return (D / 4) * kg + 8 * i + x; }
  __device__ __forceinline__ void load(const uint8_t* block) {
    using P = PackGeo<D>;
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int p = 0; p < D / 64; ++p) {
      k[p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(block) + 64 * p + lane);
      v[p] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(block + P::kV) + 64 * p + lane);
    }
    ke = *reinterpret_cast<const uint16_t*>(block + P::kKe + 2 * (c * P::NG + (D == 128 ? kg : kg >> 1)));
    ve = *reinterpret_cast<const u32x2*>(block + P::kVe + 8 * (kg * P::NG + (D == 128 ? c >> 2 : c >> 3)));
  }
  // codes of K tile j, eight channels i
  __device__ __forceinline__ uint32_t k_codes(int j, int i) const { return D == 128 ? k[j][i] : k[0][2 * j + i]; }
  __device__ __forceinline__ float k_scale(int j) const { return group_scale(ke >> (8 * j) & 255u); }
  // codes of V row u: D = 128 a word, D = 64 the lower half of one
  __device__ __forceinline__ uint32_t v_codes(int u) const { return D == 128 ? v[u >> 2][u & 3] : v[0][u >> 1] >> (16 * (u & 1)); }
  __device__ __forceinline__ float v_scale(int u) const { return group_scale(ve[u >> 2] >> (8 * (u & 3)) & 255u); }
  __device__ __forceinline__ void clear(uint32_t dead) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (dead >> u & 1u) {
        if constexpr (D == 128) v[u >> 2][u & 3] = 0u;
        else v[0][u >> 1] &= u & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        ve[u >> 2] = (ve[u >> 2] & ~(255u << (8 * (u & 3)))) | 127u << (8 * (u & 3));
      }
  }
};

__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float scale, int byte) {
  bf16x2 r;
  switch (byte) {          // an immediate of the instruction
    case 0: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0); break;
    case 1: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1); break;
    case 2: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2); break;
    default: r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3); break;
  }
  return __builtin_bit_cast(uint32_t, r);
}

// ---- scores and outputs of 32 rows --------------------------------------------------------------------------------------------
// Scores x[u] of row 8 kg + u against the lane's column.  qf: the column's query in the channel order of the rows.
template <int D> __device__ __forceinline__ void score_rows(const StoredRows<bf16_t, D>& R, const bf16x8 (&qf)[D / 32], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, R.k[j][i]), qf[i], acc, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * j + r] = acc[r];
  }
}
template <int D> __device__ __forceinline__ void score_rows(const PackedRows<D>& R, const bf16x8 (&qf)[D / 32], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const float sc = R.k_scale(j);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      u32x4 a;
#pragma unroll
      for (int p = 0; p < 4; ++p) a[p] = bf16_pair(R.k_codes(j, i), sc, p);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), qf[i], acc, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * j + r] = acc[r];
  }
}
template <int D> __device__ __forceinline__ void score_rows(const StoredRows<float, D>& R, const float (&qf)[D / 4], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(R.k[j][i][e]), qf[4 * i + e], acc, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * j + r] = acc[r];
  }
}
template <int D> __device__ __forceinline__ void score_rows(const PackedRows<D>& R, const float (&qf)[D / 4], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const float sc = R.k_scale(j);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(code_value(R.k_codes(j, i) >> (4 * e), sc), qf[8 * i + e], acc, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[4 * j + r] = acc[r];
  }
}

// Eight rows of a lane's channels -> operand n (channel n of its channels, rows 0..7), for stored bf16 values two to a word.
template <int N> __device__ __forceinline__ bf16x8 rows_of_channel(const uint32_t (&v)[8][N], int n) {
  u32x4 a;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    a[w] = __builtin_amdgcn_perm(v[2 * w + 1][n / 2], v[2 * w][n / 2], n & 1 ? 0x07060302u : 0x05040100u);
  return __builtin_bit_cast(bf16x8, a);
}

// o[n] += V^T of channel n . P^T.  kTerms: P as one operand (columns hold the terms) or as two.
template <int D, int kTerms> __device__ __forceinline__ void add_values(const StoredRows<bf16_t, D>& R, const bf16x8 (&p)[kTerms], f32x4 (&o)[D / 16]) {
#pragma unroll
  for (int n = 0; n < D / 16; ++n) {
    const bf16x8 a = rows_of_channel(R.v, n);
#pragma unroll
    for (int x = 0; x < kTerms; ++x) o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[x], o[n], 0, 0, 0);
  }
}
template <int D, int kTerms> __device__ __forceinline__ void add_values(const PackedRows<D>& R, const bf16x8 (&p)[kTerms], f32x4 (&o)[D / 16]) {
  uint32_t v[8][D / 32];
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float sc = R.v_scale(u);
#pragma unroll
    for (int w = 0; w < D / 32; ++w) v[u][w] = bf16_pair(R.v_codes(u), sc, w);
  }
#pragma unroll
  for (int n = 0; n < D / 16; ++n) {
    const bf16x8 a = rows_of_channel(v, n);
#pragma unroll
    for (int x = 0; x < kTerms; ++x) o[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p[x], o[n], 0, 0, 0);
  }
}
template <int D> __device__ __forceinline__ void add_values(const StoredRows<float, D>& R, const float (&p)[8], f32x4 (&o)[D / 16]) {
#pragma unroll
  for (int n = 0; n < D / 16; ++n)
#pragma unroll
    for (int u = 0; u < 8; ++u) o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(R.v[u][n]), p[u], o[n], 0, 0, 0);
}
template <int D> __device__ __forceinline__ void add_values(const PackedRows<D>& R, const float (&p)[8], f32x4 (&o)[D / 16]) {
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    const float sc = R.v_scale(u);
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
      o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(code_value(R.v_codes(u) >> (4 * n), sc), p[u], o[n], 0, 0, 0);
  }
}

// ---- a wave's running softmax -------------------------------------------------------------------------------------------------
template <typename T, int D, int GT> struct Running {
  static constexpr bool kTermColumns = sizeof(T) == 2 && GT == 8;
  static constexpr int kTerms = sizeof(T) == 2 && GT == 16 ? 2 : 1;
  float m = -INFINITY, l = 0.f;       // of the lane's column; l: of the lane's rows
  f32x4 o[D / 16];

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // x: scores in log2 units, -inf where the row does not count
  template <typename R> __device__ __forceinline__ void add(const R& rows, const float (&x)[8], bool second_term) {
    float top = x[0];
#pragma unroll
    for (int u = 1; u < 8; ++u) top = fmaxf(top, x[u]);
    const float m_new = fmaxf(m, column_max(top));
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float f = m == -INFINITY ? 0.f : exp2_hw(m - m_new);
      l *= f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[n][r] *= f;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m;      // no row so far
    float p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      p[u] = exp2_hw(x[u] - ref);
      l += p[u];
    }
    if constexpr (sizeof(T) == 4) {
      add_values(rows, p, o);
    } else {
      bf16x8 hi, t[kTerms];
#pragma unroll
      for (int u = 0; u < 8; ++u) hi[u] = (bf16_t)p[u];
      if constexpr (kTermColumns) {
        const float take = second_term ? 1.f : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) t[0][u] = (bf16_t)fmaf(-take, (float)hi[u], p[u]);
      } else {
        t[0] = hi;
#pragma unroll
        for (int u = 0; u < 8; ++u) t[kTerms - 1][u] = (bf16_t)(p[u] - (float)hi[u]);
      }
      add_values<D, kTerms>(rows, t, o);
    }
  }
};

// ---- the leaving token's row as it would be kept --------------------------------------------------------------------------------
// Element of lane `lane` and step s (channel lane + 64 s); PK: what its 4-bit form stands for.
template <typename T, int D, bool PK> __device__ __forceinline__ void load_kept_form(const T* row, float (&x)[D / 64]) {
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int s = 0; s < D / 64; ++s) {
    x[s] = to_f32(row[lane + 64 * s]);
    if constexpr (PK) {
      const uint32_t bits = __float_as_uint(x[s]);
      uint32_t top = bits & 0x7FFFFFFFu;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) {
        const uint32_t y = (uint32_t)__shfl_xor((int)top, off, kWave);
        top = y > top ? y : top;
      }
      const uint32_t ex = group_exponent(top);
      x[s] = code_value(value_code(bits, ex, top), group_scale(ex));
    }
  }
}

// ---- first launch ---------------------------------------------------------------------------------------------------------------
struct Share { int ring0, ring1, kept0, kept1; };      // blocks of 32 rows
__device__ __forceinline__ Share share_of(const KeptParams& P, int split) {
  const int rb = (P.window + 31) / 32, kb = (P.budget + 31) / 32, n = P.L.nsplit;
  return Share{(int)((int64_t)rb * split / n), (int)((int64_t)rb * (split + 1) / n), (int)((int64_t)kb * split / n),
               (int)((int64_t)kb * (split + 1) / n)};
}

template <typename T, int D, bool PK, int GT>
__global__ void __launch_bounds__(kStreamThreads, sizeof(T) == 4 ? 2 : D == 128 ? 2 : 4)
kept_stream_kernel(CacheDev C, KeptParams P, const T* __restrict__ q, const T* __restrict__ k_new) {
  using S = StoredRows<T, D>;
  constexpr int W = kStreamWaves, kRow = D + 4;
  constexpr int kQ = sizeof(T) == 4 ? D / 4 : D / 32;
  using Q = typename std::conditional<sizeof(T) == 4, float, bf16x8>::type;
  __shared__ float red_m[W][16], red_l[W][16];
  __shared__ __align__(16) float red_o[W * 16 * kRow];
  __shared__ Entry red_e[W];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int split = blockIdx.x % P.L.nsplit;
  const int64_t head = blockIdx.x / P.L.nsplit;
  const int b = (int)(head / P.Hkv), h = (int)(head - (int64_t)b * P.Hkv), G = P.L.G;
  const int t = C.n_seen[b], held = P.budget > 0 ? C.ret_count[head] : 0, count = held < P.budget ? held : P.budget;
  const int slot = t % P.window, leaving = t - P.window;
  const float z_e = leaving >= 0 ? C.win_score[head * P.window + slot] : 0.f;
  const bool wants = leaving >= 0 && P.budget > 0 && (leaving < P.sink || z_e > P.tau);
  const bool contest = wants && count >= P.budget;
  const Share sh = share_of(P, split);
  const T* kw = static_cast<const T*>(C.k_win) + head * P.window * D;
  const T* vw = static_cast<const T*>(C.v_win) + head * P.window * D;
  float* plan = P.plan + head * P.L.plan();
  float* rec = P.shares + (head * P.L.nsplit + split) * P.L.share();
  float* scores = P.scores + head * P.L.scores();

  // the share's entry that goes first
  Entry low = {~0u, 0, -1};
  if (contest) {
    const int r1 = 32 * sh.kept1 < count ? 32 * sh.kept1 : count;
    for (int r = 32 * sh.kept0 + tid; r < r1; r += kStreamThreads) {
      const Entry x = {order_key(C.ret_score[head * P.budget + r] + 0.0f), C.ret_pos[head * P.budget + r], r};
      if (goes_before(x, low)) low = x;
    }
    low = first_of_wave(low);
    if (lane == 0) red_e[wave] = low;
    __syncthreads();
    low = red_e[0];
#pragma unroll
    for (int w = 1; w < W; ++w)
      if (goes_before(red_e[w], low)) low = red_e[w];
  }
  low.slot = __builtin_amdgcn_readfirstlane(low.slot);
  if (tid == 0) {
    rec[0] = __uint_as_float(low.key);
    rec[1] = __int_as_float(low.pos);
    rec[2] = __int_as_float(low.slot);
  }
  if (split == 0) {
    if (tid == 0) {
      plan[0] = __int_as_float(t);
      plan[1] = __int_as_float(count);
      plan[2] = z_e;
      plan[3] = __int_as_float(!P.mass && leaving >= 0 && C.n_scored[b] <= leaving);
    }
    // scores of the incoming and of the leaving token
    float kx[2][D / 64];
    load_kept_form<T, D, false>(k_new + head * D, kx[0]);
    load_kept_form<T, D, PK>(kw + (int64_t)slot * D, kx[1]);
    for (int i = wave; i < 2 * G; i += W) {
      const int g = i >> 1, x = i & 1;
      float part = 0.f;
#pragma unroll
      for (int s = 0; s < D / 64; ++s) part = fmaf(to_f32(q[((int64_t)b * P.Hq + h * G + g) * D + lane + 64 * s]), x ? kx[1][s] : kx[0][s], part);
      part = wave_sum(part);
      if (lane == 0) plan[4 + x * G + g] = part * P.scale2;
    }
    if (wave == W - 1) {
      float vx[D / 64];
      load_kept_form<T, D, PK>(vw + (int64_t)slot * D, vx);
#pragma unroll
      for (int s = 0; s < D / 64; ++s) plan[4 + 2 * G + lane + 64 * s] = vx[s];
    }
  }

  const int live_ring = t < P.window ? t : P.window;
  const int col = Running<T, D, GT>::kTermColumns ? c & 7 : c;
  const bool second = Running<T, D, GT>::kTermColumns && c >= 8;
  Running<T, D, GT> run;
  for (int g0 = 0; g0 < G; g0 += GT) {
    run.reset();
    const bool mine = g0 + col < G;
    const T* qr = q + ((int64_t)b * P.Hq + h * G + (mine ? g0 + col : 0)) * D;
    float* my_scores = mine && !second ? scores + (int64_t)(g0 + col) * P.L.slots : nullptr;
    Q qf[kQ];
    // scores of a block -> log2 units, masked; special: a row of it that does not count (or none), n_live rows do
    auto finish_scores = [&](float (&x)[8], int n_live, int special, int64_t at, bool kept) {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int r = 8 * kg + u;
        x[u] *= P.scale2;
        if (kept && r == special && mine && !second) rec[4 + g0 + col] = x[u];
        x[u] = r < n_live && r != special ? x[u] : -INFINITY;
      }
      if (P.mass && my_scores != nullptr) {
        *reinterpret_cast<f32x4*>(my_scores + at + 8 * kg) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4*>(my_scores + at + 8 * kg + 4) = f32x4{x[4], x[5], x[6], x[7]};
      }
    };
    auto dead_rows = [&](int n_live, int special) {
      uint32_t d = 0u;
#pragma unroll
      for (int u = 0; u < 8; ++u) d |= (uint32_t)(8 * kg + u >= n_live || 8 * kg + u == special) << u;
      return d;
    };
    auto stored_blocks = [&](const T* ks, const T* vs, int b0, int b1, int live, int special_row, int64_t at0, bool kept) {
      S R;
      int blk = b0 + wave;
      auto rows_in = [&](int x) { return live - 32 * x < 32 ? live - 32 * x : 32; };
      b1 = b1 < (live + 31) / 32 ? b1 : (live + 31) / 32;
      if (blk < b1) R.load(ks + (int64_t)32 * blk * D, vs + (int64_t)32 * blk * D, rows_in(blk));
      for (; blk < b1; blk += W) {
        const int n_live = rows_in(blk), special = special_row - 32 * blk;
        float x[8];
        score_rows<D>(R, qf, x);
        const bool partial = n_live < 32 || (special >= 0 && special < 32);
        if (partial) R.clear(dead_rows(n_live, special));
        finish_scores(x, n_live, special, at0 + 32 * blk, kept);
        run.add(R, x, second);
        const int next = blk + W;
        if (next < b1) R.load(ks + (int64_t)32 * next * D, vs + (int64_t)32 * next * D, rows_in(next));
      }
    };
    auto load_queries = [&](auto rows) {
      using RT = decltype(rows);
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        if constexpr (sizeof(T) == 4) {
          constexpr int E = std::is_same<RT, S>::value ? 4 : 8;
          qf[i] = mine ? qr[RT::k_channel(i / E, kg, i % E)] : 0.f;
        } else {
          u32x4 x = *reinterpret_cast<const u32x4*>(qr + RT::k_channel(i, kg, 0));
          if (!mine) x = u32x4{0u, 0u, 0u, 0u};
          qf[i] = __builtin_bit_cast(bf16x8, x);
        }
      }
    };
    load_queries(S{});
    stored_blocks(kw, vw, sh.ring0, sh.ring1, live_ring, leaving >= 0 ? slot : -1, 0, false);
    const int64_t at_kept = 32 * (int64_t)((P.window + 31) / 32);
    if constexpr (!PK) {
      stored_blocks(static_cast<const T*>(C.k_ret) + head * P.budget * D, static_cast<const T*>(C.v_ret) + head * P.budget * D,
                    sh.kept0, sh.kept1, count, low.slot, at_kept, true);
    } else {
      load_queries(PackedRows<D>{});
      const uint8_t* blocks = P.packed + head * ((P.budget + 31) / 32) * (int64_t)PackGeo<D>::kBlock;
      PackedRows<D> R;
      const int b1 = sh.kept1 < (count + 31) / 32 ? sh.kept1 : (count + 31) / 32;
      int blk = sh.kept0 + wave;
      if (blk < b1) R.load(blocks + (int64_t)blk * PackGeo<D>::kBlock);
      for (; blk < b1; blk += W) {
        const int n_live = count - 32 * blk < 32 ? count - 32 * blk : 32, special = low.slot - 32 * blk;
        float x[8];
        score_rows<D>(R, qf, x);
        if (n_live < 32 || (special >= 0 && special < 32)) R.clear(dead_rows(n_live, special));
        finish_scores(x, n_live, special, at_kept + 32 * blk, true);
        run.add(R, x, second);
        if (blk + W < b1) R.load(blocks + (int64_t)(blk + W) * PackGeo<D>::kBlock);
      }
    }
    // merge of the waves, then the share's record
    run.l = column_sum(run.l);
    if (kg == 0) { red_m[wave][c] = run.m; red_l[wave][c] = run.l; }
#pragma unroll
    for (int n = 0; n < D / 16; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        red_o[(wave * 16 + c) * kRow + (D / 16) * (4 * kg + r) + n] = run.o[n][r];      // output tile n, row 4 kg + r
      }
    __syncthreads();
    const int heads = G - g0 < GT ? G - g0 : GT;
    for (int i = tid; i < heads * D; i += kStreamThreads) {
      const int g = i / D, d = i - g * D;
      float M = -INFINITY, Ls = 0.f, A = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) M = fmaxf(M, red_m[w][g]);
      const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2_hw(red_m[w][g] - ref);
        float o = red_o[(w * 16 + g) * kRow + d];
        if constexpr (Running<T, D, GT>::kTermColumns) o += red_o[(w * 16 + g + 8) * kRow + d];
        Ls = fmaf(red_l[w][g], f, Ls);
        A = fmaf(o, f, A);
      }
      float* r = rec + 4 + G + (size_t)(g0 + g) * (D + 2);
      if (d == 0) { r[0] = M; r[1] = Ls; }
      r[2 + d] = A;
    }
    __syncthreads();
  }
}

// ---- second launch ----------------------------------------------------------------------------------------------------------------
template <typename T, int D, bool PK>
__global__ void __launch_bounds__(kFinishThreads)
kept_finish_kernel(CacheDev C, KeptParams P, const T* __restrict__ k_new, const T* __restrict__ v_new, T* __restrict__ out) {
  extern __shared__ __align__(16) float lds[];       // [G][nsplit] factors of the shares' outputs, [G] M, [G] 1 / L, [G][nsplit] weights of their lowest entries
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = P.L.nsplit, split = blockIdx.x % n, G = P.L.G;
  const int64_t head = blockIdx.x / n;
  const int b = (int)(head / P.Hkv), h = (int)(head - (int64_t)b * P.Hkv);
  const float* plan = P.plan + head * P.L.plan();
  const float* rec = P.shares + head * n * P.L.share();
  const float* scores = P.scores + head * P.L.scores();
  float* fac = lds;
  float* top = fac + G * n;
  float* inv = top + G;
  float* stay = inv + G;
  const int t = __float_as_int(plan[0]), count = __float_as_int(plan[1]);
  const float z_e = plan[2];
  const bool late = __float_as_int(plan[3]) != 0;
  const int slot = t % P.window, leaving = t - P.window;
  const bool wants = leaving >= 0 && P.budget > 0 && (leaving < P.sink || z_e > P.tau);
  const float e_key = select_key(z_e, leaving, P.sink);

  // what happens to the leaving token: lane s holds the lowest entry of share s
  Entry mine = {~0u, 0, -1};
  if (lane < n) {
    const float* r = rec + lane * P.L.share();
    mine = Entry{__float_as_uint(r[0]), __float_as_int(r[1]), __float_as_int(r[2])};
  }
  const Entry low = first_of_wave(mine);
  int dst = -1;
  if (wants) dst = count < P.budget ? count : low.slot >= 0 && order_key(e_key) > low.key ? low.slot : -1;
  dst = __builtin_amdgcn_readfirstlane(dst);
  const bool stays = mine.slot >= 0 && mine.slot != dst;         // this lane's share's lowest entry is kept

  for (int g = wave; g < G; g += kFinishThreads / kWave) {
    const float* r = rec + (lane < n ? lane : 0) * P.L.share();
    const float m = lane < n ? r[4 + G + (size_t)g * (D + 2)] : -INFINITY, l = lane < n ? r[4 + G + (size_t)g * (D + 2) + 1] : 0.f;
    const float x_s = stays ? r[4 + g] : -INFINITY, x_t = plan[4 + g], x_e = dst >= 0 ? plan[4 + G + g] : -INFINITY;
    const float M = fmaxf(fmaxf(wave_max(fmaxf(m, x_s)), x_t), x_e);
    const float ref = M == -INFINITY ? 0.f : M;
    const float f = exp2_hw(m - ref), w_s = exp2_hw(x_s - ref);
    const float sum = wave_sum(fmaf(l, f, w_s)) + exp2_hw(x_t - ref) + exp2_hw(x_e - ref);
    if (lane < n) { fac[g * n + lane] = f; stay[g * n + lane] = w_s; }
    if (lane == 0) { top[g] = ref; inv[g] = 1.0f / sum; }
  }
  __syncthreads();

  // output: a share of the channels each
  const int items = G * D, i0 = (int)((int64_t)items * split / n), i1 = (int)((int64_t)items * (split + 1) / n);
  for (int i = i0 + tid; i < i1; i += kFinishThreads) {
    const int g = i / D, d = i - g * D;
    float A = exp2_hw(plan[4 + g] - top[g]) * to_f32(v_new[head * D + d]);
    if (dst >= 0) A = fmaf(exp2_hw(plan[4 + G + g] - top[g]), plan[4 + 2 * G + d], A);
    for (int s = 0; s < n; ++s) {
      const float* r = rec + s * P.L.share();
      A = fmaf(r[4 + G + (size_t)g * (D + 2) + 2 + d], fac[g * n + s], A);
      const int low_slot = __float_as_int(r[2]);
      if (low_slot < 0 || low_slot == dst) continue;
      float v;
      if constexpr (PK) {
        const uint8_t* block = P.packed + (head * ((P.budget + 31) / 32) + low_slot / 32) * (int64_t)PackGeo<D>::kBlock;
        v = code_value(block[v_code_at<D>(low_slot % 32, d & ~1)] >> (4 * (d & 1)), group_scale(block[v_exp_at<D>(low_slot % 32, d / 32)]));
      } else {
        v = to_f32(static_cast<const T*>(C.v_ret)[(head * P.budget + low_slot) * D + d]);
      }
      A = fmaf(stay[g * n + s], v, A);
    }
    out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(late ? __builtin_nanf("") : A * inv[g]);
  }

  // weights of this share's entries; a probability that is not a number counts as nothing
  const Share sh = share_of(P, split);
  const int my_low = __float_as_int(rec[split * P.L.share() + 2]);
  auto weight = [&](int64_t at) {
    float w = 0.f;
    for (int g = 0; g < G; ++g) w += fmaxf(exp2_hw(scores[(int64_t)g * P.L.slots + at] - top[g]) * inv[g], 0.f);
    return w;
  };
  auto weight_of = [&](auto score) {
    float w = 0.f;
    for (int g = 0; g < G; ++g) w += fmaxf(exp2_hw(score(g) - top[g]) * inv[g], 0.f);
    return w;
  };
  if (P.mass) {
    const int live = t + 1 < P.window ? t + 1 : P.window;
    const int r1 = 32 * sh.ring1 < live ? 32 * sh.ring1 : live;
    for (int r = 32 * sh.ring0 + tid; r < r1; r += kFinishThreads) {
      float* key = C.win_score + head * P.window + r;
      *key = r == slot ? weight_of([&](int g) { return plan[4 + g]; }) : *key + weight(r);
    }
  }
  const int after = count + (dst == count ? 1 : 0);
  const int k1 = 32 * sh.kept1 < after ? 32 * sh.kept1 : after;
  const int64_t at_kept = 32 * (int64_t)((P.window + 31) / 32);
  for (int r = 32 * sh.kept0 + tid; r < k1; r += kFinishThreads) {
    float* key = C.ret_score + head * P.budget + r;
    if (r == dst) {
      *key = e_key + (P.mass ? weight_of([&](int g) { return plan[4 + G + g]; }) : 0.f);
      C.ret_pos[head * P.budget + r] = leaving;
    } else if (P.mass) {
      *key = *key + (r == my_low ? weight_of([&](int g) { return rec[split * P.L.share() + 4 + g]; }) : weight(at_kept + r));
    }
  }
  if (split != 0) return;

  // the rows that move, and the counters
  T* kw = static_cast<T*>(C.k_win) + (head * P.window + slot) * D;
  T* vw = static_cast<T*>(C.v_win) + (head * P.window + slot) * D;
  if (tid < D) {
    const T ke = kw[tid], ve = vw[tid];
    if (dst >= 0) {
      if constexpr (PK) {
        uint8_t* block = const_cast<uint8_t*>(P.packed) + (head * ((P.budget + 31) / 32) + dst / 32) * (int64_t)PackGeo<D>::kBlock;
        const int r = dst % 32;
        auto put = [&](T x, auto code_at, auto exp_at) {
          const uint32_t bits = __float_as_uint(to_f32(x));
          uint32_t largest = bits & 0x7FFFFFFFu;
#pragma unroll
          for (int off = 16; off > 0; off >>= 1) {
            const uint32_t y = (uint32_t)__shfl_xor((int)largest, off, kWave);
            largest = y > largest ? y : largest;
          }
          const uint32_t ex = group_exponent(largest), code = value_code(bits, ex, largest);
          const uint32_t other = (uint32_t)__shfl_xor((int)code, 1, kWave);
          if ((tid & 1) == 0) block[code_at(r, tid)] = (uint8_t)(code | other << 4);
          if (tid % 32 == 0) block[exp_at(r, tid / 32)] = (uint8_t)ex;
        };
        put(ke, k_code_at<D>, k_exp_at<D>);
        put(ve, v_code_at<D>, v_exp_at<D>);
      } else {
        static_cast<T*>(C.k_ret)[(head * P.budget + dst) * D + tid] = ke;
        static_cast<T*>(C.v_ret)[(head * P.budget + dst) * D + tid] = ve;
      }
    }
    kw[tid] = k_new[head * D + tid];
    vw[tid] = v_new[head * D + tid];
  }
  if (tid == 0) {
    if (after != count) C.ret_count[head] = after;
    if (h == 0) {
      C.n_seen[b] = t + 1;
      if (P.mass) C.n_scored[b] = t + 1;
      if (late && P.status != nullptr) atomicOr(P.status, LTEA_LATE_SCORING);
    }
  }
}

template <typename T, int D>
hipError_t kept_run(const ltea_cfg& cfg, const KeptInputs& in, const ltea_cache& c, int n_seqs, int nsplit, void* workspace,
                    hipStream_t stream) {
  CacheDev C{c.k_win, c.v_win, c.win_score, c.k_ret, c.v_ret, c.ret_score, c.ret_pos, c.ret_count, c.n_seen, c.n_scored};
  KeptParams P;
  P.B = n_seqs; P.Hq = cfg.Hq; P.Hkv = cfg.Hkv; P.window = cfg.window; P.budget = cfg.budget; P.sink = cfg.sink;
  P.mass = in.mass;
  P.tau = cfg.tau_logit;
  P.scale2 = (cfg.softmax_scale > 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
  P.packed = static_cast<const uint8_t*>(in.packed);
  P.status = in.status;
  const int G = cfg.Hq / cfg.Hkv;
  P.L = KeptLayout{G, D, nsplit, 32 * (kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget))};
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv;
  P.plan = static_cast<float*>(workspace);
  P.shares = P.plan + (P.L.plan() * heads + 63) / 64 * 64;
  P.scores = P.shares + (P.L.share() * heads * nsplit + 63) / 64 * 64;
  const dim3 grid((unsigned)(heads * nsplit));
  auto go = [&](auto pk, auto gt) {
    constexpr bool PK = decltype(pk)::value;
    hipLaunchKernelGGL((kept_stream_kernel<T, D, PK, decltype(gt)::value>), grid, dim3(kStreamThreads), 0, stream, C, P,
                       static_cast<const T*>(in.q), static_cast<const T*>(in.k));
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL((kept_finish_kernel<T, D, PK>), grid, dim3(kFinishThreads), (size_t)(2 * G * nsplit + 2 * G) * sizeof(float),
                       stream, C, P, static_cast<const T*>(in.k), static_cast<const T*>(in.v), static_cast<T*>(in.out));
    return hipGetLastError();
  };
  auto by_heads = [&](auto pk) {
    if constexpr (sizeof(T) == 2) {
      if (G <= 8) return go(pk, std::integral_constant<int, 8>{});
    }
    return go(pk, std::integral_constant<int, 16>{});
  };
  return in.packed != nullptr ? by_heads(std::integral_constant<bool, true>{}) : by_heads(std::integral_constant<bool, false>{});
}

}  // namespace
}  // namespace ltea
