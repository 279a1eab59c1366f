// One decode step of a cache that evicts by accumulated attention weight, or whose kept rows are held in 4 bits.
//
// With t = n_seen, e = t - window the position that leaves the ring, x_j the score of row j in units of log2:
//   e goes behind the kept entries, or in the place of the one with the lowest key if its own key is higher (sinks: +inf);
//   the incoming token takes ring slot t % window;
//   out = sum_j p_j v_j over ring and kept entries as they are then, p_j = 2^(x_j - M) / L;
//   by accumulated weight, every entry's key grows by the sum of its p_j over the group's query heads.
//
// A workgroup of four or eight waves streams a head's rows, or one share of them, as they lie: blocks of 32 ring rows and of 32 kept
// rows, its waves taking blocks in turn with a running maximum, sum and output each; by accumulated weight, the scores of all rows are
// kept (in LDS, or in the workspace).
// Two rows are left out of the stream, because what is at their place differs before and after the step: the ring slot t % window,
// and the entry that e displaces.  What replaces them, e as it would be kept and the incoming token, joins the softmax at the end;
// with the normaliser known every key of the head grows by its weight, and the rows move.
// Where heads are few and long, a head is cut into shares and a second launch finishes it.  No share knows the lowest entry of all
// then, so each leaves out its own lowest when e may displace one, and hands its score and value row on beside its maximum, sum and
// output; the second launch adds those that stay, and each of its workgroups the weights of a share's entries.
// A whole head's workgroup counts itself in bits 24..31 of its sequence's first word of ret_count, as ltea_decode_step does, and the
// last one advances the sequence's counters.  Caches whose counts do not fit there take the two launches.
//
//   S^T[row, head] = K . Q^T       v_mfma_f32_16x16x32_bf16; K rows straight from memory into the A operand
//   O^T[d, head] += V^T . P^T      V in registers, eight rows of a few channels per lane, brought into the A operand's order by
//                                  byte permutes; P from S^T's accumulators without leaving the lane: tile row m = 4 kg + r of
//                                  tile j is row 8 kg + 4 j + r, so a lane's eight probabilities are eight consecutive rows
// P is the exact sum of three bf16 terms, so that it keeps its 32 bits beside the 8 of the values.  For up to five query heads the terms
// are columns of one matrix instruction (column 5 * term + head; every lane works out its head's probability and keeps its column's
// term), else three instructions.  fp32 storage: v_mfma_f32_16x16x4_f32 for both products, P in 32 bits.
#pragma once
#include "fp4_rows.h"
#include "kept_run.h"
#include "score_dma.h"

namespace ltea {
namespace {

constexpr int kStepWaves = 4, kStepThreads = kStepWaves * kWave;     // of a workgroup that shares a head, and of the second launch

struct KeptParams {
  int Hq, Hkv, window, budget, sink, mass;
  int scores_in_lds;
  uint32_t count_mask;           // the bits of ret_count that are the count
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

// Entries are displaced lowest key first, of equal keys the latest position first: as one number, the smaller goes first.
struct Entry { unsigned long long order; int slot; };       // slot < 0: none
__device__ __forceinline__ unsigned long long order_of(float key, int pos) {
  return (unsigned long long)order_key(key + 0.0f) << 32 | (0xFFFFFFFFu - (uint32_t)pos);
}
__device__ __forceinline__ Entry first_of_wave(const Entry& x) {
  const unsigned long long m = wave_min_u64(x.order), at = __builtin_amdgcn_ballot_w64(x.order == m);
  return Entry{m, __builtin_amdgcn_readlane(x.slot, (int)__builtin_ctzll(at))};
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
  // n_rows: rows that the memory holds from here on; the others read as zeros (none: nothing is loaded)
  __device__ __forceinline__ void load_k(const void* ks, int n_rows) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, kg = lane >> 4;
    const auto rk = bytes_at(ks, (uint32_t)(n_rows < 0 ? 0 : n_rows < 32 ? n_rows : 32) * (uint32_t)kRow);
    // (known to be small: the constants added below are then part of the instructions, not registers kept over the loop)
    uint32_t ko = (uint32_t)((8 * (c >> 2) + (c & 3)) * kRow + 16 * kg);
    asm volatile("" : "+v"(ko));
    ko &= 16383u;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < KP; ++i) k[j][i] = __builtin_amdgcn_raw_buffer_load_b128(rk, ko + 4 * j * kRow + 64 * i, 0, kNonTemporal);
  }
  __device__ __forceinline__ void load_v(const void* vs, int n_rows) {
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, kg = lane >> 4;
    const auto rv = bytes_at(vs, (uint32_t)(n_rows < 0 ? 0 : n_rows < 32 ? n_rows : 32) * (uint32_t)kRow);
    uint32_t vo = (uint32_t)(8 * kg * kRow + VB * c);
    asm volatile("" : "+v"(vo));
    vo &= 16383u;
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
  // there: whether the block is wanted (nothing is loaded otherwise)
  __device__ __forceinline__ void load(const uint8_t* block, bool there) {
    using P = PackGeo<D>;
    const int lane = threadIdx.x & (kWave - 1), c = lane & 15, kg = lane >> 4;
    const auto r = bytes_at(block, there ? P::kBlock : 0);
    uint32_t at = 16u * lane, at_ke = 2 * (c * P::NG + (D == 128 ? kg : kg >> 1)), at_ve = 8 * (kg * P::NG + (D == 128 ? c >> 2 : c >> 3));
#pragma unroll
    for (int p = 0; p < D / 64; ++p) k[p] = __builtin_amdgcn_raw_buffer_load_b128(r, at + 1024 * p, 0, kNonTemporal);
    ke = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, P::kKe + at_ke, 0, 0);
#pragma unroll
    for (int p = 0; p < D / 64; ++p) v[p] = __builtin_amdgcn_raw_buffer_load_b128(r, P::kV + at + 1024 * p, 0, kNonTemporal);
    ve = __builtin_amdgcn_raw_buffer_load_b64(r, P::kVe + at_ve, 0, 0);
  }
  // codes of K tile j, eight channels i
  __device__ __forceinline__ uint32_t k_codes(int j, int i) const { return D == 128 ? k[j][i] : k[0][2 * j + i]; }
  // 2^E as the conversion takes it: it reads the exponent bits, and gives NaN for 255
  __device__ __forceinline__ float k_scale(int j) const { return __uint_as_float((ke >> (8 * j) & 255u) << 23); }
  // codes of V row u: D = 128 a word, D = 64 the lower half of one
  __device__ __forceinline__ uint32_t v_codes(int u) const { return D == 128 ? v[u >> 2][u & 3] : v[0][u >> 1] >> (16 * (u & 1)); }
  __device__ __forceinline__ float v_scale(int u) const { return __uint_as_float((ve[u >> 2] >> (8 * (u & 3)) & 255u) << 23); }
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

// ---- scores and outputs of 32 rows --------------------------------------------------------------------------------------------
// Scores x[u] of row 8 kg + u against the lane's column.  qf: the column's query in the channel order of the rows; bf16: in LDS, this
// lane's piece i at qf[64 * i] (16 registers less for as many bytes read per block as two rows have).
template <int D> __device__ __forceinline__ void score_rows(const StoredRows<bf16_t, D>& R, const u32x4* qf, float (&x)[8]) {
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const bf16x8 b = __builtin_bit_cast(bf16x8, qf[64 * i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, R.k[j][i]), b, acc[j], 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) x[u] = acc[u >> 2][u & 3];
}
template <int D> __device__ __forceinline__ void score_rows(const PackedRows<D>& R, const u32x4* qf, float (&x)[8]) {
  f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  const float sc[2] = {R.k_scale(0), R.k_scale(1)};
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const bf16x8 b = __builtin_bit_cast(bf16x8, qf[64 * i]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4 a;
#pragma unroll
      for (int p = 0; p < 4; ++p) a[p] = bf16_pair(R.k_codes(j, i), sc[j], p);
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), b, acc[j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int u = 0; u < 8; ++u) x[u] = acc[u >> 2][u & 3];
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
      for (int e = 0; e < 8; e += 2) {
        float a0, a1;
        f32_pair(R.k_codes(j, i), sc, e / 2, a0, a1);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0, qf[8 * i + e], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1, qf[8 * i + e + 1], acc, 0, 0, 0);
      }
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

// o[n] += V^T of channel n . P^T.  kTerms: P as one operand (columns hold the terms) or as three.
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
    for (int n = 0; n < D / 16; n += 2) {
      float a0, a1;
      f32_pair(R.v_codes(u), sc, n / 2, a0, a1);
      o[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a0, p[u], o[n], 0, 0, 0);
      o[n + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a1, p[u], o[n + 1], 0, 0, 0);
    }
  }
}

// ---- a wave's running softmax -------------------------------------------------------------------------------------------------
template <typename T, int D, int GT> struct Running {
  static constexpr bool kTermColumns = sizeof(T) == 2 && GT == 5;
  static constexpr int kTerms = sizeof(T) == 2 && GT == 16 ? 3 : 1;
  float m = -INFINITY, l = 0.f;       // of the lane's column; l: of the lane's rows
  f32x4 o[D / 16];

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // x: q . k, -inf where the row does not count; scale2: softmax scale in log2 units (positive)
  // term: of the lane's column; take: 1, or 0: every term is the leading one (what is finite then is not wanted)
  template <typename R> __device__ __forceinline__ void add(const R& rows, const float (&x)[8], float scale2, int term, float take) {
    float top = x[0];
#pragma unroll
    for (int u = 1; u < 8; ++u) top = fmaxf(top, x[u]);
    const float m_new = fmaxf(m, column_max(top));
    if (__builtin_amdgcn_ballot_w64(m_new > m)) {
      const float f = m == -INFINITY ? 0.f : exp2_hw((m - m_new) * scale2);
      l *= f;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[n][r] *= f;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m * scale2;      // no row so far
    float p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      p[u] = exp2_hw(fmaf(x[u], scale2, -ref));
      l += p[u];
    }
    if constexpr (sizeof(T) == 4) {
      add_values(rows, p, o);
    } else {
      // p = top + middle + rest, exactly, cut to 8 bits each.  Columns: a lane's term is what the ones above it leave, cut in turn.
      auto cut = [](float y) { return __uint_as_float(__float_as_uint(y) & 0xFFFF0000u); };
      const float from_second = kTermColumns ? term > 0 ? 1.f : 0.f : take, from_third = kTermColumns ? term > 1 ? 1.f : 0.f : take;
      u32x4 words[kTerms];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float y[2] = {p[2 * w], p[2 * w + 1]};
        auto pair = [&]() { return __builtin_amdgcn_perm(__float_as_uint(y[1]), __float_as_uint(y[0]), 0x07060302u); };      // upper halves
        if constexpr (!kTermColumns) words[0][w] = pair();
#pragma unroll
        for (int e = 0; e < 2; ++e) y[e] = fmaf(-from_second, cut(y[e]), y[e]);
        if constexpr (!kTermColumns) words[1][w] = pair();
#pragma unroll
        for (int e = 0; e < 2; ++e) y[e] = fmaf(-from_third, cut(y[e]), y[e]);
        words[kTerms - 1][w] = pair();
      }
      bf16x8 t[kTerms];
#pragma unroll
      for (int z = 0; z < kTerms; ++z) t[z] = __builtin_bit_cast(bf16x8, words[z]);
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

// ---- the step -----------------------------------------------------------------------------------------------------------------------
// (Quotients of 32 bits: a head has fewer than 2^24 blocks and at most 64 shares.)
struct Share { int ring0, ring1, kept0, kept1; };      // blocks of 32 rows
__device__ __forceinline__ int part_of(int x, int split, int n) { return (int)((uint32_t)x * (uint32_t)split / (uint32_t)n); }
__device__ __forceinline__ Share share_of(const KeptParams& P, int split) {
  const int rb = (int)(((uint32_t)P.window + 31u) / 32u), kb = (int)(((uint32_t)P.budget + 31u) / 32u), n = P.L.nsplit;
  return Share{part_of(rb, split, n), part_of(rb, split + 1, n), part_of(kb, split, n), part_of(kb, split + 1, n)};
}

// What a step is about, the same in all workgroups of a head.
struct Plan {
  int t, count, slot, leaving;
  float z_e, e_key;
  bool wants, late;        // the leaving token may be kept; it left unscored
};
__device__ __forceinline__ Plan plan_of(const KeptParams& P, int t, int count, float z_e, bool late) {
  Plan p;
  p.t = t; p.count = count; p.slot = t % P.window; p.leaving = t - P.window; p.z_e = z_e;
  p.wants = p.leaving >= 0 && P.budget > 0 && (p.leaving < P.sink || z_e > P.tau);
  p.e_key = select_key(z_e, p.leaving, P.sink);
  p.late = late;
  return p;
}
// Slot that the leaving token goes to, given the entry that goes first of all; -1: none.
__device__ __forceinline__ int target_of(const KeptParams& P, const Plan& p, const Entry& low) {
  const int dst = !p.wants ? -1 : p.count < P.budget ? p.count : low.slot >= 0 && order_key(p.e_key) > (uint32_t)(low.order >> 32) ? low.slot : -1;
  return __builtin_amdgcn_readfirstlane(dst);
}

// The weights of entries join their keys, four rows per thread at a time, and the leaving token's key and position take their slot.
// score4(g, at): scores of slots at .. at + 3 of [ring ++ kept] against query head g; a probability that is not a number counts as
// nothing.  The rows are those of blocks sh.
// What a thread needs first of all, requested ahead: keys of its first rows of either segment and their scores against the first
// four query heads.
struct FirstRows { f32x4 ring, kept, x_ring[4], x_kept[4]; };
__device__ __forceinline__ f32x4 keys_at(const float* keys, int n, int r) {       // of n keys; past them zeros
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(bytes_at(keys, (uint32_t)n * 4u), (uint32_t)r * 4u, 0, 0));
}
__device__ __forceinline__ void request_keys(const CacheDev& C, const KeptParams& P, int64_t head, const Share& sh, FirstRows& F) {
  if (!P.mass) return;
  F.ring = keys_at(C.win_score + head * P.window, P.window, 32 * sh.ring0 + 4 * (int)threadIdx.x);
  F.kept = keys_at(C.ret_score + head * P.budget, P.budget, 32 * sh.kept0 + 4 * (int)threadIdx.x);
}
template <typename F4> __device__ __forceinline__ void request_scores(const KeptParams& P, const Share& sh, FirstRows& F, F4&& score4) {
  if (!P.mass) return;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int gc = g < P.L.G ? g : 0;
    F.x_ring[g] = score4(gc, 32 * sh.ring0 + 4 * (int)threadIdx.x);
    F.x_kept[g] = score4(gc, 32 * ((P.window + 31) / 32) + 32 * sh.kept0 + 4 * (int)threadIdx.x);
  }
}
template <int NT, typename F4>
__device__ __forceinline__ void grow_keys(const CacheDev& C, const KeptParams& P, const Plan& p, int64_t head, const Share& sh, int dst,
                                          const float* xs, const float* top, const float* inv, const FirstRows& first, bool have_scores,
                                          F4&& score4) {
  const int G = P.L.G, tid = threadIdx.x;
  if (!P.mass) {
    if (dst >= 32 * sh.kept0 && dst < 32 * sh.kept1 && tid == 0) {
      C.ret_score[head * P.budget + dst] = p.e_key;
      C.ret_pos[head * P.budget + dst] = p.leaving;
    }
    return;
  }
  auto weight = [&](float x, int g) { return fmaxf(exp2_hw(fmaf(x, P.scale2, -top[g])) * inv[g], 0.f); };
  // keys of rows r0 .. r1 of one segment of n; special: the row of the incoming (or leaving) token, whose key starts at `base`
  auto grow = [&](float* keys, int n, int r0, int r1, int at0, int special, float base, const float* special_x, const f32x4& first_keys,
                  const f32x4 (&first_x)[4]) {
    const auto to = bytes_at(keys, (uint32_t)n * 4u);
    for (int r = r0 + 4 * tid; r < r1; r += 4 * NT) {
      const bool is_first = r == r0 + 4 * tid;
      f32x4 before = first_keys, w = {0.f, 0.f, 0.f, 0.f};
      if (!is_first) before = keys_at(keys, n, r);
      for (int g0 = 0; g0 < G; g0 += 4) {
        f32x4 x[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) x[g] = first_x[g];
        if (!(is_first && have_scores && g0 == 0)) {
#pragma unroll
          for (int g = 0; g < 4; ++g) x[g] = score4(g0 + g < G ? g0 + g : g0, at0 + r);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (g0 + g < G)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] += weight(x[g][i], g0 + g);
      }
      if (special >= r && special < r + 4) {
        float ws = 0.f;
        for (int g = 0; g < G; ++g) ws += weight(special_x[g], g);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (r + i == special) { before[i] = base; w[i] = ws; }
      }
      const f32x4 after = before + w;
      if (r + 4 <= r1) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, after), to, (uint32_t)r * 4u, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (r + i < r1) keys[r + i] = after[i];
      }
    }
  };
  const int live = p.t + 1 < P.window ? p.t + 1 : P.window;
  grow(C.win_score + head * P.window, P.window, 32 * sh.ring0, 32 * sh.ring1 < live ? 32 * sh.ring1 : live, 0, p.slot, 0.f, xs,
       first.ring, first.x_ring);
  const int after = p.count + (dst == p.count ? 1 : 0), k1 = 32 * sh.kept1 < after ? 32 * sh.kept1 : after;
  grow(C.ret_score + head * P.budget, P.budget, 32 * sh.kept0, k1, 32 * ((P.window + 31) / 32), dst, p.e_key, xs + G, first.kept,
       first.x_kept);
  if (dst >= 32 * sh.kept0 && dst < k1 && tid == 0) C.ret_pos[head * P.budget + dst] = p.leaving;
}

// The leaving token's row (ke, ve) to its slot, the incoming token's into the ring.  Threads 0 .. D - 1, a channel each.
template <typename T, int D, bool PK>
__device__ __forceinline__ void move_rows(const CacheDev& C, const KeptParams& P, const Plan& p, int64_t head, int dst, T ke, T ve, T k_in, T v_in) {
  const int d = threadIdx.x;
  T* kw = static_cast<T*>(C.k_win) + (head * P.window + p.slot) * D;
  T* vw = static_cast<T*>(C.v_win) + (head * P.window + p.slot) * D;
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
        if ((d & 1) == 0) block[code_at(r, d)] = (uint8_t)(code | other << 4);
        if (d % 32 == 0) block[exp_at(r, d / 32)] = (uint8_t)ex;
      };
      put(ke, k_code_at<D>, k_exp_at<D>);
      put(ve, v_code_at<D>, v_exp_at<D>);
    } else {
      static_cast<T*>(C.k_ret)[(head * P.budget + dst) * D + d] = ke;
      static_cast<T*>(C.v_ret)[(head * P.budget + dst) * D + d] = ve;
    }
  }
  kw[d] = k_in;
  vw[d] = v_in;
}

__device__ __forceinline__ void advance(const CacheDev& C, const KeptParams& P, int b, const Plan& p) {
  C.n_seen[b] = p.t + 1;
  if (P.mass) C.n_scored[b] = p.t + 1;
}

// What all shares of a head have handed over becomes factors: fac [G][n] of the shares' outputs, stay [G][n] weights of their lowest
// entries that stay (both relative to 2^top), top [G], inv [G] = 1 / sum.  Returns the slot the leaving token goes to.
struct FirstRecord { float order_hi, order_lo, slot, x, m, l, x_in, x_out; };      // of the lane's share and the wave's first query head: requested ahead
template <int D> __device__ __forceinline__ FirstRecord request_record(const KeptParams& P, const float* rec, const float* xs) {
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int n = P.L.nsplit, G = P.L.G, g = wave < G ? wave : 0;
  const float* r = rec + (lane < n ? lane : 0) * P.L.share();
  const float* o = r + 4 + G + D + (size_t)g * (D + 2);
  return FirstRecord{r[0], r[1], r[2], r[4 + g], o[0], o[1], xs[g], xs[G + g]};
}
template <int D>
__device__ __forceinline__ int join_shares(const KeptParams& P, const Plan& p, const float* rec, const float* xs, const FirstRecord& first,
                                           float* fac, float* stay, float* top, float* inv) {
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int n = P.L.nsplit, G = P.L.G;
  const float* r = rec + (lane < n ? lane : 0) * P.L.share();
  Entry mine = {(unsigned long long)__float_as_uint(first.order_hi) << 32 | __float_as_uint(first.order_lo), __float_as_int(first.slot)};
  if (lane >= n) mine = Entry{~0ull, -1};
  const int dst = target_of(P, p, first_of_wave(mine));
  const bool stays = mine.slot >= 0 && mine.slot != dst;
  for (int g = wave; g < G; g += kStepWaves) {
    float x = first.x, m = first.m, l = first.l, x_in = first.x_in, x_out = first.x_out;
    if (g != wave) {
      const float* o = r + 4 + G + D + (size_t)g * (D + 2);
      x = r[4 + g]; m = o[0]; l = o[1]; x_in = xs[g]; x_out = xs[G + g];
    }
    if (lane >= n) { m = -INFINITY; l = 0.f; }
    const float x_s = stays ? x * P.scale2 : -INFINITY, x_t = x_in * P.scale2;
    const float x_e = dst >= 0 ? x_out * P.scale2 : -INFINITY;
    const float M = fmaxf(fmaxf(wave_max(fmaxf(m, x_s)), x_t), x_e);
    const float ref = M == -INFINITY ? 0.f : M;
    const float f = exp2_hw(m - ref), w_s = exp2_hw(x_s - ref);
    const float sum = wave_sum(fmaf(l, f, w_s)) + exp2_hw(x_t - ref) + exp2_hw(x_e - ref);
    if (lane < n) { fac[g * n + lane] = f; stay[g * n + lane] = stays ? w_s : 0.f; }
    if (lane == 0) { top[g] = ref; inv[g] = 1.0f / sum; }
  }
  return dst;
}

// Output element (g, d) of the head from all shares, sixteen of them at a time; of the first sixteen what is handed over is requested
// ahead.
constexpr int kBatch = 16;
struct FirstShares { float o[kBatch], v[kBatch]; };
template <int D>
__device__ __forceinline__ void take_shares(const KeptParams& P, const float* rec, int g, int d, int s0, FirstShares& F) {
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const float* r = rec + (s0 + u < P.L.nsplit ? s0 + u : s0) * P.L.share() + 4 + P.L.G;
    F.v[u] = r[d];
    F.o[u] = r[D + (size_t)g * (D + 2) + 2 + d];
  }
}
template <int D>
__device__ __forceinline__ float joined_output(const KeptParams& P, const float* rec, int g, int d, int dst, const float* xs, float v_in,
                                               float v_e, const float* fac, const float* stay, const float* top, const float* inv,
                                               FirstShares& F) {
  const int n = P.L.nsplit, G = P.L.G;
  float A = exp2_hw(fmaf(xs[g], P.scale2, -top[g])) * v_in;
  if (dst >= 0) A = fmaf(exp2_hw(fmaf(xs[G + g], P.scale2, -top[g])), v_e, A);
  for (int s0 = 0;;) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const bool there = s0 + u < n;
      const int at = g * n + (there ? s0 + u : s0);
      const float w = stay[at];
      if (there) A = fmaf(F.o[u], fac[at], A);
      if (there && w != 0.f) A = fmaf(w, F.v[u], A);        // (a row that does not stay may hold anything)
    }
    s0 += kBatch;
    if (s0 >= n) break;
    take_shares<D>(P, rec, g, d, s0, F);
  }
  return A * inv[g];
}

// WHOLE: the workgroup takes a whole head and finishes it; otherwise a share, and a second launch finishes the head.
// Bound: HBM for long or many heads, else the chain of requests, products and exchanges of one head.  Waves per SIMD: as many as hold
// their registers; D = 128 with three spills (1024 heads of 1024 + 512 rows 148 us, with two 136; 256 heads of 512 + 8192 packed rows
// 78 and 73).
template <typename T, int D, bool PK, int GT, bool WHOLE, int W>
__global__ void __launch_bounds__(W * kWave, sizeof(T) == 4 || D == 128 ? 2 : PK ? 3 : 4)
kept_step_kernel(CacheDev C, KeptParams P, const T* __restrict__ q, const T* __restrict__ k_new, const T* __restrict__ v_new,
                 T* __restrict__ out) {
  using S = StoredRows<T, D>;
  constexpr int NT = W * kWave, kRow = D + 4, kDepth = sizeof(T) == 4 ? 1 : GT == 16 ? 2 : 3;
  // kDepth: blocks of packed rows in flight per wave (GT = 16: three spill, 256 heads of 512 + 4096 rows, eight query heads each, D = 128: 50.8
  // us, two 46.4)
  constexpr int kQ = sizeof(T) == 4 ? D / 4 : D / 32;
  // [W][heads of a pass][kRow] outputs of the waves, [2][G] scores of the incoming and the leaving token, [G] top, [G] inv,
  // [G] scores of the lowest entry, then the scores of all slots [G][slots]
  extern __shared__ __align__(16) float lds[];
  __shared__ float red_m[W][16], red_l[W][16];
  __shared__ Entry red_e[W];
  __shared__ float ve_lds[D];
  __shared__ int pass_again;
  __shared__ __align__(16) u32x4 q_lds[sizeof(T) == 2 ? (PK ? 2 : 1) * kQ * kWave : 1];      // bf16: a pass's queries as B operands, [rows, packed rows][piece][lane]
  __shared__ __align__(16) T rows_lds[4][D];          // keys of the incoming and of the leaving token, the latter's value, the former's
  static_assert(sizeof(red_m) + sizeof(red_l) + sizeof(red_e) + sizeof(ve_lds) + sizeof(pass_again) + sizeof(q_lds) + sizeof(rows_lds) + kKeptLds <= 64 * 1024, "LDS");
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = WHOLE ? 1 : P.L.nsplit, G = P.L.G;
  const uint32_t flat = WHOLE ? blockIdx.x : blockIdx.x / (uint32_t)n;
  const int split = WHOLE ? 0 : (int)(blockIdx.x - flat * (uint32_t)n);
  const int64_t head = flat;
  const int b = (int)(flat / (uint32_t)P.Hkv), h = (int)(flat - (uint32_t)b * (uint32_t)P.Hkv);
  const int heads_at_once = G < GT ? G : GT;
  float* red_o = lds;
  float* xs = red_o + W * heads_at_once * kRow;
  float* top = xs + 2 * G;
  float* inv = top + G;
  float* low_x = inv + G;
  float* rest = xs + (6 * G + 3) / 4 * 4;        // 16-byte aligned
  const Share sh = WHOLE ? Share{0, (int)(((uint32_t)P.window + 31u) / 32u), 0, (int)(((uint32_t)P.budget + 31u) / 32u)} : share_of(P, split);
  const T* kw = static_cast<const T*>(C.k_win) + head * P.window * D;
  const T* vw = static_cast<const T*>(C.v_win) + head * P.window * D;
  const T* kr = static_cast<const T*>(C.k_ret) + head * P.budget * D;
  const T* vr = static_cast<const T*>(C.v_ret) + head * P.budget * D;
  const uint8_t* blocks = P.packed + head * ((P.budget + 31) / 32) * (int64_t)PackGeo<D>::kBlock;
  float* rec = P.shares + (head * n + split) * P.L.share();
  float* scores = P.scores + head * P.L.scores();

  // Requested before anything is known: the scalar words (scalar loads do not wait for rows requested earlier, vector loads return in
  // order), the queries, the first keys of the share, and last the wave's first rows, whatever they hold.
  // this lane's column: a head of the pass and the term of its probabilities (of the last column: none)
  const int col = Running<T, D, GT>::kTermColumns ? c % 5 : c, term = Running<T, D, GT>::kTermColumns ? c / 5 : 0;
  constexpr int kSets = PK ? 2 : 1, kMine = (kSets * kQ + W - 1) / W;      // bf16: pieces of the queries that a wave brings into LDS
  u32x4 q_piece[sizeof(T) == 2 ? kMine : 1];
  auto query_row = [&](int g0) { return q + ((int64_t)b * P.Hq + h * G + (g0 + col < G ? g0 + col : 0)) * D; };
  auto request_queries = [&](int g0) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int piece = wave + i * W, set = piece / kQ, at = piece % kQ;
        const T* row = query_row(g0) + (set == 0 ? S::k_channel(at, kg, 0) : PackedRows<D>::k_channel(at, kg, 0));
        q_piece[i] = *reinterpret_cast<const u32x4*>(row);
      }
    }
  };
  auto put_queries = [&](int g0) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < kMine; ++i)
        if (wave + i * W < kSets * kQ) q_lds[(wave + i * W) * kWave + lane] = term < 3 && g0 + col < G ? q_piece[i] : u32x4{0u, 0u, 0u, 0u};
    }
  };
  request_queries(0);
  int t = load_uniform(C.n_seen + b), held = P.budget > 0 ? load_uniform(C.ret_count + head) : 0, scored = P.mass ? 0 : load_uniform(C.n_scored + b);
  constexpr int kAhead = 2;
  float key_ahead[kAhead];
  int pos_ahead[kAhead];
  const int key0 = 32 * sh.kept0 + tid, key1 = 32 * sh.kept1 < P.budget ? 32 * sh.kept1 : P.budget;
  {
    const uint32_t bytes = (uint32_t)(key1 > 0 ? key1 : 0) * 4u;
    const auto rk = bytes_at(C.ret_score + head * P.budget, bytes), rp = bytes_at(C.ret_pos + head * P.budget, bytes);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {       // (no branches: they would be waited for at its end)
      const uint32_t at = (uint32_t)(key0 + i * NT) * 4u;
      key_ahead[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rk, at, 0, 0));
      pos_ahead[i] = (int)__builtin_amdgcn_raw_buffer_load_b32(rp, at, 0, 0);
    }
  }
  S R;
  const int first_ring = sh.ring0 + wave;
  auto load_ring_k = [&](int blk, bool there) { R.load_k(kw + (int64_t)32 * blk * D, there ? P.window - 32 * blk : 0); };
  auto load_ring_v = [&](int blk, bool there) { R.load_v(vw + (int64_t)32 * blk * D, there ? P.window - 32 * blk : 0); };
  load_ring_k(first_ring, first_ring < sh.ring1);
  load_ring_v(first_ring, first_ring < sh.ring1);
  const int first_kept = sh.kept0 + wave;
  PackedRows<D> K[PK ? kDepth : 1];
  auto request_packed = [&]() {
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      const int blk = first_kept + i * W;
      K[i].load(blocks + (int64_t)blk * PackGeo<D>::kBlock, blk < sh.kept1);
    }
  };
  // (fp32, D = 128: the registers are the ring's.  bf16, D = 128, 256 heads of 1024 + 2400 rows: 56.8 us, requested after the ring 58.6)
  constexpr bool kEarly = PK && (sizeof(T) == 2 || D == 64);
  if constexpr (kEarly) request_packed();
  read_here(t);
  read_here(held);
  read_here(scored);
  held = (int)((uint32_t)held & P.count_mask);
  const int count = held < P.budget ? held : P.budget;
  const bool late = !P.mass && t >= P.window && scored <= t - P.window;
  float z_e = t >= P.window ? load_uniform(C.win_score + head * P.window + t % P.window) : 0.f;
  read_here(z_e);
  const Plan p = plan_of(P, t, count, z_e, late);
  // rows that are needed at the end, straight into LDS
  if (wave < 4 && lane < D * (int)sizeof(T) / 16) {
    const T* row = wave == 0 ? k_new + head * D : wave == 3 ? v_new + head * D : (wave == 1 ? kw : vw) + (int64_t)p.slot * D;
    dma16(make_raw_rsrc(row, (uint32_t)(D * sizeof(T))), (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&rows_lds[wave][0], 16u * (uint32_t)lane);
  }

  // the share's entry that goes first, and whether it is left out of the stream
  Entry low = {~0ull, -1};
  if (p.wants && count >= P.budget) {
    auto look = [&](float key, int pos, int r) {
      const unsigned long long o = order_of(key, pos);
      low.slot = o < low.order ? r : low.slot;
      low.order = o < low.order ? o : low.order;
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (key0 + i * NT < key1) look(key_ahead[i], pos_ahead[i], key0 + i * NT);
    for (int r = key0 + kAhead * NT; r < key1; r += NT) look(C.ret_score[head * P.budget + r], C.ret_pos[head * P.budget + r], r);
    low = first_of_wave(low);
    if (lane == 0) red_e[wave] = low;
    __syncthreads();
    low = red_e[0];
#pragma unroll
    for (int w = 1; w < W; ++w)
      if (red_e[w].order < low.order) low = red_e[w];
  }
  low.slot = __builtin_amdgcn_readfirstlane(low.slot);
  int dst = -1;
  if constexpr (WHOLE) {
    dst = target_of(P, p, low);
    if (dst != low.slot) low.slot = -1;          // it stays: nothing is left out
  }
  const int live_ring = t < P.window ? t : P.window;
  const int ring_end = sh.ring1 < (live_ring + 31) / 32 ? sh.ring1 : (live_ring + 31) / 32;
  const int kept_end = sh.kept1 < (count + 31) / 32 ? sh.kept1 : (count + 31) / 32;
  const int at_kept = 32 * ((P.window + 31) / 32);
  Running<T, D, GT> run;
  T q_ahead[2][D / 64];
  FirstRows first;
  // An infinite value times the lower terms of a probability, zero or of either sign, is not the infinity that the probability itself
  // makes of it: an output that is not finite is what the leading terms give.  Where terms are columns, the leading one is at hand; else
  // a pass with such an output is taken again, all its terms the leading one, for those outputs.
  constexpr bool kTermPasses = Running<T, D, GT>::kTerms > 1;
  float take = 1.f;
  uint32_t not_finite = 0u;        // of this thread's outputs of the pass
  if (kTermPasses && tid == 0) pass_again = 0;
  for (int g0 = 0;;) {
    run.reset();
    const bool mine = g0 + col < G;
    const T* qr = query_row(g0);
    const bool writes = P.mass && mine && term == 0;
    float* my_scores = rest + (int64_t)(g0 + col) * P.L.slots + 8 * kg;                               // in LDS
    const uint32_t my_offset = writes ? (uint32_t)(((g0 + col) * P.L.slots + 8 * kg) * 4) : 1u << 31;      // or in the workspace
    float q_reg[sizeof(T) == 4 ? kQ : 1];      // fp32
    // scores of a block: kept for the weights, then masked; special: a row of it that does not count (or none), n_live rows do
    auto finish_scores = [&](float (&x)[8], int n_live, int special, int at, bool kept, bool partial) {
      const f32x4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
      if (P.scores_in_lds) {
        if (writes) {
          *reinterpret_cast<f32x4*>(my_scores + at) = lo;
          *reinterpret_cast<f32x4*>(my_scores + at + 4) = hi;
        }
      } else if (P.mass) {
        const auto to = bytes_at(scores, (uint32_t)(P.L.scores() * sizeof(float)));
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), to, my_offset + 4u * (uint32_t)at, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), to, my_offset + 4u * (uint32_t)at + 16u, 0, 0);
      }
      if (partial) {
        int r0 = 8 * kg;
        asm volatile("" : "+v"(r0));       // (worked out here)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int r = r0 + u;
          if (kept && r == special && mine && term == 0) low_x[g0 + col] = x[u];
          x[u] = r < n_live && r != special ? x[u] : -INFINITY;
        }
      }
    };
    auto dead_rows = [&](int n_live, int special) {
      int r0 = 8 * kg;
      asm volatile("" : "+v"(r0));
      uint32_t d = 0u;
#pragma unroll
      for (int u = 0; u < 8; ++u) d |= (uint32_t)(r0 + u >= n_live || r0 + u == special) << u;
      return d;
    };
    auto load_queries = [&](auto rows) {       // fp32
      using RT = decltype(rows);
      constexpr int E = std::is_same<RT, S>::value ? 4 : 8;
#pragma unroll
      for (int i = 0; i < kQ; ++i) q_reg[i] = mine ? qr[RT::k_channel(i / E, kg, i % E)] : 0.f;
    };
    auto scores_of = [&](const auto& rows, int set, float (&x)[8]) {
      if constexpr (sizeof(T) == 4) {
        score_rows<D>(rows, q_reg, x);
      } else {
        int at = set * kQ * kWave + lane;
        asm volatile("" : "+v"(at));           // (read again for every block: not held in registers over the loop)
        score_rows<D>(rows, q_lds + at, x);
      }
    };
    // blocks blk, blk + W, .. < end of rows whose first block is requested; next_k / next_v request another one
    auto walk = [&](auto& rows, int blk, int end, int live, int special_row, int at0, bool kept, auto&& next_k, auto&& next_v) {
      for (; blk < end; blk += W) {
        const int n_live = live - 32 * blk < 32 ? live - 32 * blk : 32, special = special_row - 32 * blk;
        const bool partial = n_live < 32 || (special >= 0 && special < 32);
        float x[8];
        scores_of(rows, 0, x);
        next_k(blk + W, blk + W < end);
        if (partial) rows.clear(dead_rows(n_live, special));
        finish_scores(x, n_live, special, at0 + 32 * blk, kept, partial);
        run.add(rows, x, P.scale2, term, take);
        next_v(blk + W, blk + W < end);
      }
    };
    if constexpr (sizeof(T) == 4) load_queries(S{});
    put_queries(g0);
    __syncthreads();
    walk(R, first_ring, ring_end, live_ring, p.leaving >= 0 ? p.slot : -1, 0, false, load_ring_k, load_ring_v);
    if (g0 == 0)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int g = wave + i * W < 2 * G ? (wave + i * W) >> 1 : 0;
#pragma unroll
        for (int s = 0; s < D / 64; ++s) q_ahead[i][s] = q[((int64_t)b * P.Hq + h * G + g) * D + lane + 64 * s];
      }
    if constexpr (!PK) {
      auto load_k = [&](int blk, bool there) { R.load_k(kr + (int64_t)32 * blk * D, there ? P.budget - 32 * blk : 0); };
      auto load_v = [&](int blk, bool there) { R.load_v(vr + (int64_t)32 * blk * D, there ? P.budget - 32 * blk : 0); };
      load_k(first_kept, first_kept < kept_end);
      load_v(first_kept, first_kept < kept_end);
      walk(R, first_kept, kept_end, count, low.slot, at_kept, true, load_k, load_v);
    } else {
      if constexpr (!kEarly) request_packed();
      if constexpr (sizeof(T) == 4) load_queries(PackedRows<D>{});
      for (int blk0 = first_kept; blk0 < kept_end; blk0 += kDepth * W) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
          const int blk = blk0 + i * W;
          if (blk < kept_end) {
            const int n_live = count - 32 * blk < 32 ? count - 32 * blk : 32, special = low.slot - 32 * blk;
            const bool partial = n_live < 32 || (special >= 0 && special < 32);
            float x[8];
            scores_of(K[i], 1, x);
            if (partial) K[i].clear(dead_rows(n_live, special));
            finish_scores(x, n_live, special, at_kept + 32 * blk, true, partial);
            run.add(K[i], x, P.scale2, term, take);
          }
          K[i].load(blocks + (int64_t)(blk + kDepth * W) * PackGeo<D>::kBlock, blk + kDepth * W < kept_end);
        }
      }
    }
    if (g0 == 0) {
      wait_loads();
      __syncthreads();
      if constexpr (WHOLE) request_keys(C, P, head, sh, first);
      // scores of the incoming and of the leaving token; the leaving one's values as they would be kept
      float x_in[D / 64], x_out[D / 64];
      load_kept_form<T, D, false>(rows_lds[0], x_in);
      load_kept_form<T, D, PK>(rows_lds[1], x_out);
      for (int i = wave; i < 2 * G; i += W) {
        const int g = i >> 1, x = i & 1;
        float part = 0.f;
#pragma unroll
        for (int s = 0; s < D / 64; ++s)
          part = fmaf(to_f32(i < 2 * W ? q_ahead[i / W][s] : q[((int64_t)b * P.Hq + h * G + g) * D + lane + 64 * s]), x ? x_out[s] : x_in[s], part);
        part = wave_sum(part);
        if (lane == 0) xs[x * G + g] = part;
      }
      if (wave == W - 1) {
        float v_out[D / 64];
        load_kept_form<T, D, PK>(rows_lds[2], v_out);
#pragma unroll
        for (int s = 0; s < D / 64; ++s) ve_lds[lane + 64 * s] = v_out[s];
      }
    }
    // merge of the waves
    run.l = column_sum(run.l);
    if (kg == 0) { red_m[wave][c] = run.m * P.scale2; red_l[wave][c] = run.l; }
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float o = run.o[x][r];
        if constexpr (Running<T, D, GT>::kTermColumns) {        // the other terms' columns: five and ten lanes on, in the row of 16
          const float middle = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(o), 0x12B, 0xf, 0xf, false));
          const float rest = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(o), 0x126, 0xf, 0xf, false));
          o = fabsf(o) < INFINITY ? o + (middle + rest) : o;
        }
        if (mine && term == 0) red_o[(wave * heads_at_once + col) * kRow + (D / 16) * (4 * kg + r) + x] = o;      // output tile x, row 4 kg + r
      }
    __syncthreads();
    const int heads = G - g0 < GT ? G - g0 : GT;
    uint32_t bit = 1u;               // at most 16 heads * D / NT = 8 outputs
    for (int i = tid; i < heads * D; i += NT, bit <<= 1) {
      if (kTermPasses && take == 0.f && !(not_finite & bit)) continue;
      const int gl = i / D, d = i - gl * D, g = g0 + gl;
      float M = -INFINITY, L = 0.f, A = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) M = fmaxf(M, red_m[w][gl]);
      constexpr bool whole = WHOLE;
      if (whole) {
        M = fmaxf(M, xs[g] * P.scale2);
        if (dst >= 0) M = fmaxf(M, xs[G + g] * P.scale2);
      }
      const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2_hw(red_m[w][gl] - ref);
        L = fmaf(red_l[w][gl], f, L);
        A = fmaf(red_o[(w * heads_at_once + gl) * kRow + d], f, A);
      }
      if (whole) {
        const float w_t = exp2_hw(fmaf(xs[g], P.scale2, -ref)), w_e = dst >= 0 ? exp2_hw(fmaf(xs[G + g], P.scale2, -ref)) : 0.f;
        L += w_t + w_e;
        A = fmaf(w_t, to_f32(rows_lds[3][d]), A);
        if (dst >= 0) A = fmaf(w_e, ve_lds[d], A);
        if (d == 0) { top[g] = ref; inv[g] = 1.0f / L; }
        out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(late ? __builtin_nanf("") : A / L);
      } else {
        float* r = rec + 4 + G + D + (size_t)g * (D + 2);
        if (d == 0) { r[0] = M; r[1] = L; }
        r[2 + d] = A;
      }
      if (kTermPasses && take != 0.f && !(fabsf(A) < INFINITY)) not_finite |= bit;
    }
    if (kTermPasses && take != 0.f && not_finite != 0u) pass_again = 1;
    if (kTermPasses && take == 0.f && tid == 0) pass_again = 0;
    __syncthreads();
    const bool again = kTermPasses && take != 0.f && pass_again != 0;
    take = again ? 0.f : 1.f;
    if (!again) {
      not_finite = 0u;
      g0 += GT;
      if (g0 >= G) break;
    }
    request_queries(g0);
    load_ring_k(first_ring, first_ring < ring_end);          // (here: requested rows are not held through the loops above)
    load_ring_v(first_ring, first_ring < ring_end);
    if constexpr (kEarly) request_packed();
  }

  if constexpr (WHOLE) {
    grow_keys<NT>(C, P, p, head, sh, dst, xs, top, inv, first, false, [&](int g, int at) {
      return *reinterpret_cast<const f32x4*>(P.scores_in_lds ? rest + g * P.L.slots + at : scores + (int64_t)g * P.L.slots + at);
    });
  } else {
    // what the head's other shares, or the second launch, need of this one
    if (tid < D) {
      float v = 0.f;
      if (low.slot >= 0) {
        if constexpr (PK) {
          const uint8_t* block = blocks + (int64_t)(low.slot / 32) * PackGeo<D>::kBlock;
          v = code_value(block[v_code_at<D>(low.slot % 32, tid & ~1)] >> (4 * (tid & 1)), group_scale(block[v_exp_at<D>(low.slot % 32, tid / 32)]));
        } else {
          v = to_f32(vr[(int64_t)low.slot * D + tid]);
        }
      }
      rec[4 + G + tid] = v;
    }
    for (int g = tid; g < G; g += NT) rec[4 + g] = low.slot >= 0 ? low_x[g] : -INFINITY;
    if (tid == 0) {
      rec[0] = __uint_as_float((uint32_t)(low.order >> 32));
      rec[1] = __uint_as_float((uint32_t)low.order);
      rec[2] = __int_as_float(low.slot);
    }
    if (split == 0) {
      float* plan = P.plan + head * P.L.plan();
      for (int g = tid; g < 2 * G; g += NT) plan[4 + g] = xs[g];
      if (tid < D) plan[4 + 2 * G + tid] = ve_lds[tid];
      if (tid == 0) {
        plan[0] = __int_as_float(t);
        plan[1] = __int_as_float(count);
        plan[2] = p.z_e;
        plan[3] = __int_as_float(late);
      }
    }
    return;
  }
  // every row has been read
  if (tid < D) move_rows<T, D, PK>(C, P, p, head, dst, rows_lds[1][tid], rows_lds[2][tid], rows_lds[0][tid], rows_lds[3][tid]);
  if (tid == 0) {
    unsigned* words = reinterpret_cast<unsigned*>(C.ret_count + (int64_t)b * P.Hkv);
    if (dst >= 0 && dst == count) atomicAdd(words + h, 1u);
    const bool last_head = P.Hkv == 1 || (atomicAdd(words, 1u << 24) >> 24) + 1u == (unsigned)P.Hkv;
    if (last_head) {
      if (P.Hkv > 1) atomicSub(words, (unsigned)P.Hkv << 24);
      advance(C, P, b, p);
    }
    if (late && h == 0 && P.status != nullptr) atomicOr(P.status, LTEA_LATE_SCORING);
  }
}

// ---- second launch: a head's shares are joined by as many workgroups, each for its own share's keys and a part of the output --------------
template <typename T, int D, bool PK>
__global__ void __launch_bounds__(kStepThreads)
kept_finish_kernel(CacheDev C, KeptParams P, const T* __restrict__ k_new, const T* __restrict__ v_new, T* __restrict__ out) {
  extern __shared__ __align__(16) float lds[];
  const int tid = threadIdx.x;
  const int n = P.L.nsplit, G = P.L.G;
  const uint32_t flat = blockIdx.x / (uint32_t)n;
  const int split = (int)(blockIdx.x - flat * (uint32_t)n);
  const int64_t head = flat;
  const int b = (int)(flat / (uint32_t)P.Hkv), h = (int)(flat - (uint32_t)b * (uint32_t)P.Hkv);
  const float* plan = P.plan + head * P.L.plan();
  const float* rec = P.shares + head * n * P.L.share();
  const float* scores = P.scores + head * P.L.scores();
  float* fac = lds;
  float* stay = fac + G * n;
  float* top = stay + G * n;
  float* inv = top + G;
  const float* xs = plan + 4;
  const Share sh = share_of(P, split);
  const auto from = bytes_at(scores, (uint32_t)(P.L.scores() * sizeof(float)));
  auto score4 = [&](int g, int at) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (uint32_t)(g * P.L.slots + at) * 4u, 0, 0));
  };
  const int items = G * D, i0 = part_of(items, split, n) + tid, i1 = part_of(items, split + 1, n);
  // everything whose place is known is requested before anything is waited for
  const FirstRecord record = request_record<D>(P, rec, xs);
  FirstShares F;
  FirstRows first;
  request_keys(C, P, head, sh, first);
  request_scores(P, sh, first, score4);
  const float plan_t = plan[0], plan_count = plan[1], plan_z = plan[2], plan_late = plan[3];
  take_shares<D>(P, rec, i0 < items ? i0 / D : 0, i0 % D, 0, F);
  const Plan p = plan_of(P, __float_as_int(plan_t), __float_as_int(plan_count), plan_z, __float_as_int(plan_late) != 0);
  T ke = T(0), ve = T(0), k_in = T(0), v_in = T(0);
  if (split == 0 && tid < D) {
    ke = static_cast<const T*>(C.k_win)[(head * P.window + p.slot) * D + tid];
    ve = static_cast<const T*>(C.v_win)[(head * P.window + p.slot) * D + tid];
    k_in = k_new[head * D + tid];
    v_in = v_new[head * D + tid];
  }
  const int dst = join_shares<D>(P, p, rec, xs, record, fac, stay, top, inv);
  __syncthreads();
  for (int i = i0; i < i1; i += kStepThreads) {
    const int g = i / D, d = i - g * D;
    if (i != i0) take_shares<D>(P, rec, g, d, 0, F);
    const float y = joined_output<D>(P, rec, g, d, dst, xs, to_f32(v_new[head * D + d]), plan[4 + 2 * G + d], fac, stay, top, inv, F);
    out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(p.late ? __builtin_nanf("") : y);
  }
  grow_keys<kStepThreads>(C, P, p, head, sh, dst, xs, top, inv, first, true, score4);
  if (split != 0) return;
  if (tid < D) move_rows<T, D, PK>(C, P, p, head, dst, ke, ve, k_in, v_in);
  if (tid == 0) {
    if (dst >= 0 && dst == p.count) C.ret_count[head] = p.count + 1;
    if (h == 0) {
      advance(C, P, b, p);
      if (p.late && P.status != nullptr) atomicOr(P.status, LTEA_LATE_SCORING);
    }
  }
}

template <typename T, int D>
hipError_t kept_run(const ltea_cfg& cfg, const KeptInputs& in, const ltea_cache& c, int n_seqs, KeptSplit split, void* workspace,
                    hipStream_t stream) {
  CacheDev C{c.k_win, c.v_win, c.win_score, c.k_ret, c.v_ret, c.ret_score, c.ret_pos, c.ret_count, c.n_seen, c.n_scored};
  KeptParams P;
  P.Hq = cfg.Hq; P.Hkv = cfg.Hkv; P.window = cfg.window; P.budget = cfg.budget; P.sink = cfg.sink;
  P.mass = in.mass;
  P.tau = cfg.tau_logit;
  P.scale2 = (cfg.softmax_scale > 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
  P.packed = static_cast<const uint8_t*>(in.packed);
  P.status = in.status;
  const int G = cfg.Hq / cfg.Hkv, nsplit = split.shares;
  const KeptForm form = kept_form(cfg, split, in.mass);
  P.L = KeptLayout{G, D, nsplit, 32 * (kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget))};
  P.count_mask = form.whole ? 0xFFFFu : 0xFFFFFFFFu;
  P.scores_in_lds = form.scores_in_lds;
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv;
  P.plan = static_cast<float*>(workspace);
  P.shares = P.plan + (P.L.plan() * heads + 63) / 64 * 64;
  P.scores = P.shares + (P.L.share() * heads * nsplit + 63) / 64 * 64;      // (there by weight only, where they are not in LDS)
  const dim3 grid((unsigned)(heads * nsplit));
  auto launch = [&](auto pk, auto gt, auto finishes, auto waves) {
    constexpr bool PK = decltype(pk)::value, WHOLE = decltype(finishes)::value;
    constexpr int GT = decltype(gt)::value, W = decltype(waves)::value;
    hipLaunchKernelGGL((kept_step_kernel<T, D, PK, GT, WHOLE, W>), grid, dim3(W * kWave), form.lds, stream, C, P,
                       static_cast<const T*>(in.q), static_cast<const T*>(in.k), static_cast<const T*>(in.v), static_cast<T*>(in.out));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || WHOLE) return e;
    hipLaunchKernelGGL((kept_finish_kernel<T, D, PK>), grid, dim3(kStepThreads), (size_t)(2 * G * nsplit + 2 * G) * sizeof(float),
                       stream, C, P, static_cast<const T*>(in.k), static_cast<const T*>(in.v), static_cast<T*>(in.out));
    return hipGetLastError();
  };
  using std::integral_constant;
  using std::true_type;
  auto go = [&](auto pk, auto gt) {
    const integral_constant<int, kStepWaves> four;
    if (!form.whole) return launch(pk, gt, std::false_type{}, four);
    if (form.waves == 8) return launch(pk, gt, true_type{}, integral_constant<int, 8>{});
    return launch(pk, gt, true_type{}, four);
  };
  auto by_heads = [&](auto pk) {
    if constexpr (sizeof(T) == 2) {
      if (G <= 5) return go(pk, integral_constant<int, 5>{});
    }
    return go(pk, integral_constant<int, 16>{});
  };
  return in.packed != nullptr ? by_heads(true_type{}) : by_heads(std::false_type{});
}

}  // namespace
}  // namespace ltea
