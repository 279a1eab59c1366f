// One decode step of a cache that evicts by accumulated attention weight, or whose kept rows are held in 4 bits.
//
// With t = n_seen, e = t - window the position that leaves the ring, x_j the score of row j in units of log2:
//   e goes behind the kept entries, or in the place of the one with the lowest key if its own key is higher (sinks: +inf);
//   the incoming token takes ring slot t % window;
//   out = sum_j p_j v_j over ring and kept entries as they are then, p_j = 2^(x_j - M) / L;
//   by accumulated weight, every entry's key grows by the sum of its p_j over the group's query heads.
//
// A workgroup of four waves streams one share of a head's rows as they lie, blocks of 32 ring rows and of 32 kept rows, its waves
// taking blocks in turn with a running maximum, sum and output each; the scores of all rows are kept (in LDS, or in the workspace).
// Two rows are left out of the stream, because what is at their place differs before and after the step: the ring slot t % window,
// and the entry that e displaces.  What replaces them, e as it would be kept and the incoming token, joins the softmax at the end;
// with the normaliser known every key of the head grows by its weight, and the rows move.
// Where heads are few, a head is cut into shares.  No share knows the lowest entry of all then, so each leaves out its own lowest
// when e may displace one, and hands its score and value row on beside its maximum, sum and output: whoever finishes the head adds
// those that stay.  That is the share that arrives last, or a second launch whose workgroups add the weights to a share each
// (launches of very long heads, and caches whose counts do not fit, see below).
// Arrivals are counted in the upper bits of ret_count as ltea_decode_step does it (bits 16..23 of a head's word its shares, bits
// 24..31 of a sequence's first word its heads), handed-over words go past the XCD's own L2 (agent scope), and nobody waits for
// anybody.
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

constexpr int kStepWaves = 4, kStepThreads = kStepWaves * kWave;

struct KeptParams {
  int B, Hq, Hkv, window, budget, sink, mass;
  int fused;                     // the head is finished in the first launch
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

// `bytes` bytes at p, the same in all lanes; what lies past them reads as zeros and is not written.
__device__ __forceinline__ auto bytes_at(const void* p, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(p);        // (the compiler does not see that this is the same in all lanes)
  void* same = reinterpret_cast<void*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32 |
                                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a));
  return __builtin_amdgcn_make_buffer_rsrc(same, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
constexpr int kNonTemporal = 2, kPastL2 = 16;              // of buffer instructions

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

// ---- the step -----------------------------------------------------------------------------------------------------------------------
struct Share { int ring0, ring1, kept0, kept1; };      // blocks of 32 rows
__device__ __forceinline__ Share share_of(const KeptParams& P, int split) {
  const int rb = (P.window + 31) / 32, kb = (P.budget + 31) / 32, n = P.L.nsplit;
  return Share{(int)((int64_t)rb * split / n), (int)((int64_t)rb * (split + 1) / n), (int)((int64_t)kb * split / n),
               (int)((int64_t)kb * (split + 1) / n)};
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

// A word that another workgroup of this launch wrote, or one of an earlier launch.
template <bool SHARED> __device__ __forceinline__ float take(const float* p) {
  if constexpr (SHARED) return __hip_atomic_load(const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else return *p;
}
__device__ __forceinline__ void give(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The weights of entries join their keys, four rows per thread at a time, and the leaving token's key and position take their slot.
// score4(g, at): scores of slots at .. at + 3 of [ring ++ kept] against query head g; a probability that is not a number counts as
// nothing.  The rows are those of blocks sh.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <typename F>
__device__ __forceinline__ void grow_keys(const CacheDev& C, const KeptParams& P, const Plan& p, int64_t head, const Share& sh, int dst,
                                          const float* xs, const float* top, const float* inv, F&& score4) {
  const int G = P.L.G, tid = threadIdx.x;
  if (!P.mass) {
    if (dst >= 32 * sh.kept0 && dst < 32 * sh.kept1 && tid == 0) {
      C.ret_score[head * P.budget + dst] = p.e_key;
      C.ret_pos[head * P.budget + dst] = p.leaving;
    }
    return;
  }
  auto weight = [&](float x, int g) { return fmaxf(exp2_hw(x - top[g]) * inv[g], 0.f); };
  // keys of rows r0 .. r1 of one segment; special: the row of the incoming (or leaving) token, whose key starts at `base`
  auto grow = [&](float* keys, int r0, int r1, int at0, int special, float base, const float* special_x) {
    for (int r = r0 + 4 * tid; r < r1; r += 4 * kStepThreads) {
      float before[4], w[4] = {0.f, 0.f, 0.f, 0.f};
      const bool all = r + 4 <= r1;
      if (all) {
        const f32x4_any x = *reinterpret_cast<const f32x4_any*>(keys + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] = x[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) before[i] = keys[r + i < r1 ? r + i : r1 - 1];
      }
      for (int g0 = 0; g0 < G; g0 += 4) {
        f32x4 x[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) x[g] = score4(g0 + g < G ? g0 + g : g0, at0 + r);
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] += g0 + g < G ? weight(x[g][i], g0 + g) : 0.f;
      }
      if (special >= r && special < r + 4) {
        float ws = 0.f;
        for (int g = 0; g < G; ++g) ws += weight(special_x[g], g);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (r + i == special) { before[i] = base; w[i] = ws; }
      }
      if (all) {
        *reinterpret_cast<f32x4_any*>(keys + r) = f32x4_any{before[0] + w[0], before[1] + w[1], before[2] + w[2], before[3] + w[3]};
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (r + i < r1) keys[r + i] = before[i] + w[i];
      }
    }
  };
  const int live = p.t + 1 < P.window ? p.t + 1 : P.window;
  grow(C.win_score + head * P.window, 32 * sh.ring0, 32 * sh.ring1 < live ? 32 * sh.ring1 : live, 0, p.slot, 0.f, xs);
  const int after = p.count + (dst == p.count ? 1 : 0), k1 = 32 * sh.kept1 < after ? 32 * sh.kept1 : after;
  grow(C.ret_score + head * P.budget, 32 * sh.kept0, k1, 32 * ((P.window + 31) / 32), dst, p.e_key, xs + G);
  if (dst >= 32 * sh.kept0 && dst < k1 && tid == 0) C.ret_pos[head * P.budget + dst] = p.leaving;
}

// The leaving token's row to its slot, the incoming token's into the ring.  Threads 0 .. D - 1.
template <typename T, int D, bool PK>
__device__ __forceinline__ void move_rows(const CacheDev& C, const KeptParams& P, const Plan& p, int64_t head, int dst, T k_in, T v_in) {
  const int d = threadIdx.x;
  T* kw = static_cast<T*>(C.k_win) + (head * P.window + p.slot) * D;
  T* vw = static_cast<T*>(C.v_win) + (head * P.window + p.slot) * D;
  if (dst >= 0) {
    const T ke = kw[d], ve = vw[d];
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
template <bool SHARED, int D>
__device__ __forceinline__ int join_shares(const KeptParams& P, const Plan& p, const float* rec, const float* xs, float* fac, float* stay,
                                           float* top, float* inv) {
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
  const int n = P.L.nsplit, G = P.L.G;
  const float* r = rec + (lane < n ? lane : 0) * P.L.share();
  Entry mine = {(unsigned long long)__float_as_uint(take<SHARED>(r)) << 32 | __float_as_uint(take<SHARED>(r + 1)), __float_as_int(take<SHARED>(r + 2))};
  if (lane >= n) mine = Entry{~0ull, -1};
  const int dst = target_of(P, p, first_of_wave(mine));
  const bool stays = mine.slot >= 0 && mine.slot != dst;
  for (int g = wave; g < G; g += kStepWaves) {
    const float* o = r + 4 + G + D + (size_t)g * (D + 2);
    const float m = lane < n ? take<SHARED>(o) : -INFINITY, l = lane < n ? take<SHARED>(o + 1) : 0.f;
    const float x_s = stays ? take<SHARED>(r + 4 + g) : -INFINITY, x_t = xs[g], x_e = dst >= 0 ? xs[G + g] : -INFINITY;
    const float M = fmaxf(fmaxf(wave_max(fmaxf(m, x_s)), x_t), x_e);
    const float ref = M == -INFINITY ? 0.f : M;
    const float f = exp2_hw(m - ref), w_s = exp2_hw(x_s - ref);
    const float sum = wave_sum(fmaf(l, f, w_s)) + exp2_hw(x_t - ref) + exp2_hw(x_e - ref);
    if (lane < n) { fac[g * n + lane] = f; stay[g * n + lane] = stays ? w_s : 0.f; }
    if (lane == 0) { top[g] = ref; inv[g] = 1.0f / sum; }
  }
  return dst;
}

// Output element (g, d) of the head from all shares.
template <bool SHARED, typename T, int D>
__device__ __forceinline__ float joined_output(const KeptParams& P, const float* rec, int g, int d, int dst, const float* xs, float v_in,
                                               float v_e, const float* fac, const float* stay, const float* top, const float* inv) {
  const int n = P.L.nsplit, G = P.L.G;
  float A = exp2_hw(xs[g] - top[g]) * v_in;
  if (dst >= 0) A = fmaf(exp2_hw(xs[G + g] - top[g]), v_e, A);
  constexpr int kBatch = 16;
  for (int s0 = 0; s0 < n; s0 += kBatch) {
    float o[kBatch], v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float* r = rec + (s0 + u < n ? s0 + u : s0) * P.L.share() + 4 + G;
      v[u] = take<SHARED>(r + d);
      o[u] = take<SHARED>(r + D + (size_t)g * (D + 2) + 2 + d);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + u >= n) break;
      A = fmaf(o[u], fac[g * n + s0 + u], A);
      const float w = stay[g * n + s0 + u];
      if (w != 0.f) A = fmaf(w, v[u], A);        // (a row that does not stay may hold anything)
    }
  }
  return A * inv[g];
}

// How a head is finished: by its one workgroup, by the last of its shares, or by the second launch.
enum { kWhole, kLastShare, kSecondLaunch };

template <typename T, int D, bool PK, int GT, int MODE>
__global__ void __launch_bounds__(kStepThreads, sizeof(T) == 4 ? 2 : D == 128 ? (PK ? 2 : 3) : PK ? 3 : 4)
kept_step_kernel(CacheDev C, KeptParams P, const T* __restrict__ q, const T* __restrict__ k_new, const T* __restrict__ v_new,
                 T* __restrict__ out) {
  using S = StoredRows<T, D>;
  constexpr int W = kStepWaves, kRow = D + 4, kDepth = sizeof(T) == 4 ? 1 : 3;      // kDepth: blocks of packed rows in flight per wave
  constexpr int kQ = sizeof(T) == 4 ? D / 4 : D / 32;
  using Q = typename std::conditional<sizeof(T) == 4, float, bf16x8>::type;
  // [W][heads of a pass][kRow] outputs of the waves, [2][G] scores of the incoming and the leaving token, [G] top, [G] inv,
  // [G] scores of the lowest entry, then the scores of all slots [G][slots], or the shares' factors [2][G][nsplit]
  extern __shared__ __align__(16) float lds[];
  __shared__ float red_m[W][16], red_l[W][16];
  __shared__ Entry red_e[W];
  __shared__ float ve_lds[D];
  __shared__ int last_lds;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = MODE == kWhole ? 1 : P.L.nsplit, split = MODE == kWhole ? 0 : blockIdx.x % n, G = P.L.G;
  const int64_t head = MODE == kWhole ? blockIdx.x : blockIdx.x / n;
  const int b = (int)(head / P.Hkv), h = (int)(head - (int64_t)b * P.Hkv);
  const int heads_at_once = G < GT ? G : GT;
  float* red_o = lds;
  float* xs = red_o + W * heads_at_once * kRow;
  float* top = xs + 2 * G;
  float* inv = top + G;
  float* low_x = inv + G;
  float* rest = xs + (6 * G + 3) / 4 * 4;        // 16-byte aligned
  const Share sh = share_of(P, split);
  const T* kw = static_cast<const T*>(C.k_win) + head * P.window * D;
  const T* vw = static_cast<const T*>(C.v_win) + head * P.window * D;
  const T* kr = static_cast<const T*>(C.k_ret) + head * P.budget * D;
  const T* vr = static_cast<const T*>(C.v_ret) + head * P.budget * D;
  const uint8_t* blocks = P.packed + head * ((P.budget + 31) / 32) * (int64_t)PackGeo<D>::kBlock;
  float* rec = P.shares + (head * n + split) * P.L.share();
  float* scores = P.scores + head * P.L.scores();

  // Requested before anything is known: the wave's first ring block, whatever it holds, and the first keys of the share.
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
  if constexpr (PK) request_packed();
  constexpr int kAhead = 2;
  float key_ahead[kAhead];
  int pos_ahead[kAhead];
  const int key0 = 32 * sh.kept0 + tid, key1 = 32 * sh.kept1 < P.budget ? 32 * sh.kept1 : P.budget;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int r = key0 + i * kStepThreads;
    const bool there = r < key1;
    key_ahead[i] = there ? C.ret_score[head * P.budget + r] : 0.f;
    pos_ahead[i] = there ? C.ret_pos[head * P.budget + r] : 0;
  }
  float x_in[D / 64], x_out[D / 64], v_out[D / 64];
  load_kept_form<T, D, false>(k_new + head * D, x_in);
  const int t = C.n_seen[b];
  const int held = P.budget > 0 ? (int)((uint32_t)C.ret_count[head] & P.count_mask) : 0, count = held < P.budget ? held : P.budget;
  const bool late = !P.mass && t >= P.window && C.n_scored[b] <= t - P.window;
  const Plan p = plan_of(P, t, count, t >= P.window ? C.win_score[head * P.window + t % P.window] : 0.f, late);
  load_kept_form<T, D, PK>(kw + (int64_t)p.slot * D, x_out);
  load_kept_form<T, D, PK>(vw + (int64_t)p.slot * D, v_out);

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
      if (key0 + i * kStepThreads < key1) look(key_ahead[i], pos_ahead[i], key0 + i * kStepThreads);
    for (int r = key0 + kAhead * kStepThreads; r < key1; r += kStepThreads) look(C.ret_score[head * P.budget + r], C.ret_pos[head * P.budget + r], r);
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
  if constexpr (MODE == kWhole) {
    dst = target_of(P, p, low);
    if (dst != low.slot) low.slot = -1;          // it stays: nothing is left out
  }
  // scores of the incoming and of the leaving token; the leaving one's values as they would be kept
  for (int i = wave; i < 2 * G; i += W) {
    const int g = i >> 1, x = i & 1;
    float part = 0.f;
#pragma unroll
    for (int s = 0; s < D / 64; ++s) part = fmaf(to_f32(q[((int64_t)b * P.Hq + h * G + g) * D + lane + 64 * s]), x ? x_out[s] : x_in[s], part);
    part = wave_sum(part);
    if (lane == 0) xs[x * G + g] = part * P.scale2;
  }
  if (wave == W - 1)
#pragma unroll
    for (int s = 0; s < D / 64; ++s) ve_lds[lane + 64 * s] = v_out[s];

  const int live_ring = t < P.window ? t : P.window;
  const int ring_end = sh.ring1 < (live_ring + 31) / 32 ? sh.ring1 : (live_ring + 31) / 32;
  const int kept_end = sh.kept1 < (count + 31) / 32 ? sh.kept1 : (count + 31) / 32;
  const int at_kept = 32 * ((P.window + 31) / 32);
  const int col = Running<T, D, GT>::kTermColumns ? c & 7 : c;
  const bool second = Running<T, D, GT>::kTermColumns && c >= 8;
  Running<T, D, GT> run;
  for (int g0 = 0; g0 < G; g0 += GT) {
    run.reset();
    const bool mine = g0 + col < G;
    const T* qr = q + ((int64_t)b * P.Hq + h * G + (mine ? g0 + col : 0)) * D;
    const bool writes = P.mass && mine && !second;
    float* my_scores = rest + (int64_t)(g0 + col) * P.L.slots + 8 * kg;                               // in LDS
    const uint32_t my_offset = writes ? (uint32_t)(((g0 + col) * P.L.slots + 8 * kg) * 4) : 1u << 31;      // or in the workspace
    Q qf[kQ];
    // scores of a block -> log2 units, kept for the weights, then masked; special: a row of it that does not count (or none), n_live rows do
    auto finish_scores = [&](float (&x)[8], int n_live, int special, int at, bool kept, bool partial) {
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] *= P.scale2;
      const f32x4 lo = {x[0], x[1], x[2], x[3]}, hi = {x[4], x[5], x[6], x[7]};
      if (P.scores_in_lds) {
        if (writes) {
          *reinterpret_cast<f32x4*>(my_scores + at) = lo;
          *reinterpret_cast<f32x4*>(my_scores + at + 4) = hi;
        }
      } else if (P.mass) {
        constexpr int kFlags = MODE == kLastShare ? kPastL2 : 0;     // another workgroup of this launch may read them
        const auto to = bytes_at(scores, (uint32_t)(P.L.scores() * sizeof(float)));
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), to, my_offset + 4u * (uint32_t)at, 0, kFlags);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), to, my_offset + 4u * (uint32_t)at + 16u, 0, kFlags);
      }
      if (partial) {
        int r0 = 8 * kg;
        asm volatile("" : "+v"(r0));       // (worked out here)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int r = r0 + u;
          if (kept && r == special && mine && !second) low_x[g0 + col] = x[u];
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
    // blocks blk, blk + W, .. < end of rows whose first block is requested; next_k / next_v request another one
    auto walk = [&](auto& rows, int blk, int end, int live, int special_row, int at0, bool kept, auto&& next_k, auto&& next_v) {
      for (; blk < end; blk += W) {
        const int n_live = live - 32 * blk < 32 ? live - 32 * blk : 32, special = special_row - 32 * blk;
        const bool partial = n_live < 32 || (special >= 0 && special < 32);
        float x[8];
        score_rows<D>(rows, qf, x);
        next_k(blk + W, blk + W < end);
        if (partial) rows.clear(dead_rows(n_live, special));
        finish_scores(x, n_live, special, at0 + 32 * blk, kept, partial);
        run.add(rows, x, second);
        next_v(blk + W, blk + W < end);
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
    if (g0 > 0) {
      load_ring_k(first_ring, first_ring < ring_end);
      load_ring_v(first_ring, first_ring < ring_end);
    }
    walk(R, first_ring, ring_end, live_ring, p.leaving >= 0 ? p.slot : -1, 0, false, load_ring_k, load_ring_v);
    if constexpr (!PK) {
      auto load_k = [&](int blk, bool there) { R.load_k(kr + (int64_t)32 * blk * D, there ? P.budget - 32 * blk : 0); };
      auto load_v = [&](int blk, bool there) { R.load_v(vr + (int64_t)32 * blk * D, there ? P.budget - 32 * blk : 0); };
      load_k(first_kept, first_kept < kept_end);
      load_v(first_kept, first_kept < kept_end);
      walk(R, first_kept, kept_end, count, low.slot, at_kept, true, load_k, load_v);
    } else {
      if (g0 > 0) request_packed();
      load_queries(PackedRows<D>{});
      for (int blk0 = first_kept; blk0 < kept_end; blk0 += kDepth * W) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) {
          const int blk = blk0 + i * W;
          if (blk < kept_end) {
            const int n_live = count - 32 * blk < 32 ? count - 32 * blk : 32, special = low.slot - 32 * blk;
            const bool partial = n_live < 32 || (special >= 0 && special < 32);
            float x[8];
            score_rows<D>(K[i], qf, x);
            if (partial) K[i].clear(dead_rows(n_live, special));
            finish_scores(x, n_live, special, at_kept + 32 * blk, true, partial);
            run.add(K[i], x, second);
          }
          K[i].load(blocks + (int64_t)(blk + kDepth * W) * PackGeo<D>::kBlock, blk + kDepth * W < kept_end);
        }
      }
    }
    // merge of the waves
    run.l = column_sum(run.l);
    if (kg == 0) { red_m[wave][c] = run.m; red_l[wave][c] = run.l; }
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float o = run.o[x][r];
        if constexpr (Running<T, D, GT>::kTermColumns) o += __shfl_xor(o, 8, kWave);
        if (mine && !second) red_o[(wave * heads_at_once + col) * kRow + (D / 16) * (4 * kg + r) + x] = o;      // output tile x, row 4 kg + r
      }
    __syncthreads();
    const int heads = G - g0 < GT ? G - g0 : GT;
    for (int i = tid; i < heads * D; i += kStepThreads) {
      const int gl = i / D, d = i - gl * D, g = g0 + gl;
      float M = -INFINITY, L = 0.f, A = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) M = fmaxf(M, red_m[w][gl]);
      constexpr bool whole = MODE == kWhole;
      if (whole) {
        M = fmaxf(M, xs[g]);
        if (dst >= 0) M = fmaxf(M, xs[G + g]);
      }
      const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2_hw(red_m[w][gl] - ref);
        L = fmaf(red_l[w][gl], f, L);
        A = fmaf(red_o[(w * heads_at_once + gl) * kRow + d], f, A);
      }
      if (whole) {
        const float w_t = exp2_hw(xs[g] - ref), w_e = dst >= 0 ? exp2_hw(xs[G + g] - ref) : 0.f;
        L += w_t + w_e;
        A = fmaf(w_t, to_f32(v_new[head * D + d]), A);
        if (dst >= 0) A = fmaf(w_e, ve_lds[d], A);
        if (d == 0) { top[g] = ref; inv[g] = 1.0f / L; }
        out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(late ? __builtin_nanf("") : A / L);
      } else {
        float* r = rec + 4 + G + D + (size_t)g * (D + 2);
        if (d == 0) { give(r, M); give(r + 1, L); }
        give(r + 2 + d, A);
      }
    }
    __syncthreads();
  }

  if constexpr (MODE == kWhole) {
    grow_keys(C, P, p, head, sh, dst, xs, top, inv, [&](int g, int at) {
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
      give(rec + 4 + G + tid, v);
    }
    for (int g = tid; g < G; g += kStepThreads) give(rec + 4 + g, low.slot >= 0 ? low_x[g] : -INFINITY);
    if (tid == 0) {
      give(rec, __uint_as_float((uint32_t)(low.order >> 32)));
      give(rec + 1, __uint_as_float((uint32_t)low.order));
      give(rec + 2, __int_as_float(low.slot));
    }
    if constexpr (MODE == kSecondLaunch) {
      if (split != 0) return;
      float* plan = P.plan + head * P.L.plan();
      for (int g = tid; g < 2 * G; g += kStepThreads) plan[4 + g] = xs[g];
      if (tid < D) plan[4 + 2 * G + tid] = ve_lds[tid];
      if (tid == 0) {
        plan[0] = __int_as_float(t);
        plan[1] = __int_as_float(count);
        plan[2] = p.z_e;
        plan[3] = __int_as_float(late);
      }
      return;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what this thread gave is there
    __syncthreads();
    if (tid == 0) last_lds = (atomicAdd(reinterpret_cast<unsigned*>(C.ret_count + head), 1u << 16) >> 16 & 255u) + 1u == (unsigned)n;
    __syncthreads();
    if (!last_lds) return;
    const float* all = P.shares + head * n * P.L.share();
    float* fac = rest;
    float* stay = fac + G * n;
    dst = join_shares<true, D>(P, p, all, xs, fac, stay, top, inv);
    __syncthreads();
    for (int i = tid; i < G * D; i += kStepThreads) {
      const int g = i / D, d = i - g * D;
      const float y = joined_output<true, T, D>(P, all, g, d, dst, xs, to_f32(v_new[head * D + d]), ve_lds[d], fac, stay, top, inv);
      out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(late ? __builtin_nanf("") : y);
    }
    const auto from = bytes_at(scores, (uint32_t)(P.L.scores() * sizeof(float)));
    grow_keys(C, P, p, head, Share{0, (P.window + 31) / 32, 0, (P.budget + 31) / 32}, dst, xs, top, inv, [&](int g, int at) {
      return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (uint32_t)(g * P.L.slots + at) * 4u, 0, kPastL2));
    });
  }
  // every row has been read
  if (tid < D) move_rows<T, D, PK>(C, P, p, head, dst, k_new[head * D + tid], v_new[head * D + tid]);
  if (tid == 0) {
    const unsigned delta = (dst >= 0 && dst == count ? 1u : 0u) - (n > 1 ? (unsigned)n << 16 : 0u);
    unsigned* words = reinterpret_cast<unsigned*>(C.ret_count + (int64_t)b * P.Hkv);
    if (delta != 0u) atomicAdd(words + h, delta);
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
  const int n = P.L.nsplit, split = blockIdx.x % n, G = P.L.G;
  const int64_t head = blockIdx.x / n;
  const int b = (int)(head / P.Hkv), h = (int)(head - (int64_t)b * P.Hkv);
  const float* plan = P.plan + head * P.L.plan();
  const float* rec = P.shares + head * n * P.L.share();
  const float* scores = P.scores + head * P.L.scores();
  float* fac = lds;
  float* stay = fac + G * n;
  float* top = stay + G * n;
  float* inv = top + G;
  const Plan p = plan_of(P, __float_as_int(plan[0]), __float_as_int(plan[1]), plan[2], __float_as_int(plan[3]) != 0);
  const float* xs = plan + 4;
  const int dst = join_shares<false, D>(P, p, rec, xs, fac, stay, top, inv);
  __syncthreads();
  const int items = G * D, i0 = (int)((int64_t)items * split / n), i1 = (int)((int64_t)items * (split + 1) / n);
  for (int i = i0 + tid; i < i1; i += kStepThreads) {
    const int g = i / D, d = i - g * D;
    const float y = joined_output<false, T, D>(P, rec, g, d, dst, xs, to_f32(v_new[head * D + d]), plan[4 + 2 * G + d], fac, stay, top, inv);
    out[((int64_t)b * P.Hq + h * G + g) * D + d] = from_f32<T>(p.late ? __builtin_nanf("") : y);
  }
  grow_keys(C, P, p, head, share_of(P, split), dst, xs, top, inv,
            [&](int g, int at) { return *reinterpret_cast<const f32x4*>(scores + (int64_t)g * P.L.slots + at); });
  if (split != 0) return;
  if (tid < D) move_rows<T, D, PK>(C, P, p, head, dst, k_new[head * D + tid], v_new[head * D + tid]);
  if (tid == 0) {
    if (dst >= 0 && dst == p.count) C.ret_count[head] = p.count + 1;
    if (h == 0) {
      advance(C, P, b, p);
      if (p.late && P.status != nullptr) atomicOr(P.status, LTEA_LATE_SCORING);
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
  // counts fit ret_count's upper bits, and what is left to the last share to arrive is not more than a second launch costs
  P.fused = cfg.budget > 0 && cfg.budget < (1 << 16) && cfg.Hkv <= 255 && (nsplit == 1 || !in.mass || P.L.scores() <= kKeptLastShare);
  P.count_mask = P.fused ? 0xFFFFu : 0xFFFFFFFFu;
  P.scores_in_lds = P.fused && nsplit == 1 && P.L.scores() * sizeof(float) <= kKeptScoresLds;
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv;
  P.plan = static_cast<float*>(workspace);
  P.shares = P.plan + (P.L.plan() * heads + 63) / 64 * 64;
  P.scores = P.shares + (P.L.share() * heads * nsplit + 63) / 64 * 64;
  const dim3 grid((unsigned)(heads * nsplit));
  auto go_mode = [&](auto pk, auto gt, auto mode) {
    constexpr bool PK = decltype(pk)::value;
    constexpr int GT = decltype(gt)::value;
    const size_t rest = P.scores_in_lds ? (in.mass ? P.L.scores() : 0) : P.fused && nsplit > 1 ? 2 * (size_t)G * nsplit : 0;
    const size_t bytes = ((size_t)kStepWaves * (G < GT ? G : GT) * (D + 4) + 6 * (size_t)G + 4 + rest) * sizeof(float);
    hipLaunchKernelGGL((kept_step_kernel<T, D, PK, GT, decltype(mode)::value>), grid, dim3(kStepThreads), bytes, stream, C, P, static_cast<const T*>(in.q),
                       static_cast<const T*>(in.k), static_cast<const T*>(in.v), static_cast<T*>(in.out));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || P.fused) return e;
    hipLaunchKernelGGL((kept_finish_kernel<T, D, PK>), grid, dim3(kStepThreads), (size_t)(2 * G * nsplit + 2 * G) * sizeof(float),
                       stream, C, P, static_cast<const T*>(in.k), static_cast<const T*>(in.v), static_cast<T*>(in.out));
    return hipGetLastError();
  };
  auto go = [&](auto pk, auto gt) {
    if (!P.fused) return go_mode(pk, gt, std::integral_constant<int, kSecondLaunch>{});
    return nsplit == 1 ? go_mode(pk, gt, std::integral_constant<int, kWhole>{}) : go_mode(pk, gt, std::integral_constant<int, kLastShare>{});
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
