// Launchers of the step over kept entries (kept_step.h), and the conversion of kept rows to 4 bits and back.
#include <initializer_list>
#include "fp4_rows.h"
#include "kept_run.h"

namespace ltea {
namespace {

// ---- rows <-> 4 bits ------------------------------------------------------------------------------------------------------------
// One workgroup per block of 32 rows of a head; a thread takes eight channels of a row at a time, four neighbouring threads a group.
// Bound: HBM (D = 128, bf16: 512 bytes of row against 136), with everything a workgroup reads requested at once and the chip's
// conversions (16 sequences x 8 heads x 8192 rows: 108 us there and 95 back; rounding by comparisons 193 there).
constexpr int kPackThreads = 256;

// Eight channels as the workgroup's memory holds them.
template <typename T> struct Eight {
  uint32_t w[2 * sizeof(T)];
  template <typename R> __device__ __forceinline__ void load(const R& rsrc, uint32_t at) {
#pragma unroll
    for (int p = 0; p < (int)sizeof(T) / 2; ++p) {
      const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + 16 * p, 0, kNonTemporal);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[4 * p + e] = x[e];
    }
  }
  template <typename R> __device__ __forceinline__ void store(const R& rsrc, uint32_t at) const {
#pragma unroll
    for (int p = 0; p < (int)sizeof(T) / 2; ++p)
      __builtin_amdgcn_raw_buffer_store_b128(u32x4{w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]}, rsrc, at + 16 * p, 0, kNonTemporal);
  }
  // bits of the largest magnitude as fp32
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0u;
#pragma unroll
    for (int e = 0; e < (int)(2 * sizeof(T)); ++e) {
      if constexpr (sizeof(T) == 4) {
        const uint32_t a = w[e] & 0x7FFFFFFFu;
        m = a > m ? a : m;
      } else {
        const uint32_t a = w[e] << 16 & 0x7FFFFFFFu, b = w[e] & 0x7FFF0000u;
        m = a > m ? a : m;
        m = b > m ? b : m;
      }
    }
    return m;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) c = pair_codes(c, __uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]), scale, i);
      else c = pair_codes(c, w[i], scale, i);
    }
    return c;
  }
  __device__ __forceinline__ uint32_t signs() const {       // codes of zeros with the values' signs
    uint32_t c = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) c |= (sizeof(T) == 4 ? w[i % (2 * sizeof(T))] >> 31 : w[i / 2] >> (16 * (i & 1) + 15) & 1u) << (4 * i + 3);
    return c;
  }
  __device__ __forceinline__ void set(uint32_t c, float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        float a, b;
        f32_pair(c, scale, i, a, b);
        w[2 * i] = __float_as_uint(a);
        w[2 * i + 1] = __float_as_uint(b);
      } else {
        w[i] = bf16_pair(c, scale, i);
      }
    }
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads)
kept_pack_kernel(const T* __restrict__ k_ret, const T* __restrict__ v_ret, const int32_t* __restrict__ ret_count, int budget,
                 int n_blocks, uint32_t first, uint8_t* __restrict__ packed) {
  const int64_t head = (first + blockIdx.x) / (uint32_t)n_blocks;
  const int blk = (int)(first + blockIdx.x - (uint32_t)head * (uint32_t)n_blocks);
  const int count = ret_count[head], left = (count < budget ? count : budget) - 32 * blk;
  if (left <= 0) return;
  uint8_t* out = packed + (head * n_blocks + blk) * (int64_t)PackGeo<D>::kBlock;
  constexpr int kEach = 32 * D / 8 / kPackThreads;          // items of K, and of V, per thread
  static_assert(kEach * kPackThreads * 8 == 32 * D, "whole rounds");
  const int64_t row0 = (head * budget + 32 * blk) * D;
  const uint32_t bytes = (uint32_t)((left < 32 ? left : 32) * D * (int)sizeof(T));      // rows past them read as zeros
  const auto rk = bytes_at(k_ret + row0, bytes), rv = bytes_at(v_ret + row0, bytes);
  Eight<T> x[2][kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) x[0][i].load(rk, (uint32_t)(threadIdx.x + i * kPackThreads) * 8u * (uint32_t)sizeof(T));
#pragma unroll
  for (int i = 0; i < kEach; ++i) x[1][i].load(rv, (uint32_t)(threadIdx.x + i * kPackThreads) * 8u * (uint32_t)sizeof(T));
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int item = threadIdx.x + i * kPackThreads, d = 8 * (item % (D / 8)), r = item / (D / 8);
      uint32_t top = x[is_v][i].top();
      uint32_t other = __builtin_amdgcn_update_dpp(0, top, 0xB1, 0xf, 0xf, false);      // lane ^ 1
      top = other > top ? other : top;
      other = __builtin_amdgcn_update_dpp(0, top, 0x4E, 0xf, 0xf, false);               // lane ^ 2
      top = other > top ? other : top;
      const uint32_t ex = group_exponent(top);
      uint32_t codes = x[is_v][i].codes(group_scale(ex));
      if (top < 0x03800000u) codes = x[is_v][i].signs();
      if (ex == 255u) codes = 0x77777777u;
      if (r >= left) continue;
      if (!is_v) {
        *reinterpret_cast<uint32_t*>(out + k_code_at<D>(r, d)) = codes;
      } else if constexpr (D == 128) {
        *reinterpret_cast<uint32_t*>(out + v_code_at<D>(r, d)) = codes;
      } else {
        *reinterpret_cast<uint16_t*>(out + v_code_at<D>(r, d)) = (uint16_t)codes;
        *reinterpret_cast<uint16_t*>(out + v_code_at<D>(r, d + 4)) = (uint16_t)(codes >> 16);
      }
      if (d % 32 == 0) out[is_v ? v_exp_at<D>(r, d / 32) : k_exp_at<D>(r, d / 32)] = (uint8_t)ex;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads)
kept_unpack_kernel(const uint8_t* __restrict__ packed, const int32_t* __restrict__ ret_count, int budget, int n_blocks, uint32_t first,
                   T* __restrict__ k_ret, T* __restrict__ v_ret) {
  const int64_t head = (first + blockIdx.x) / (uint32_t)n_blocks;
  const int blk = (int)(first + blockIdx.x - (uint32_t)head * (uint32_t)n_blocks);
  const int count = ret_count[head], left = (count < budget ? count : budget) - 32 * blk;
  if (left <= 0) return;
  const uint8_t* in = packed + (head * n_blocks + blk) * (int64_t)PackGeo<D>::kBlock;
  constexpr int kEach = 32 * D / 8 / kPackThreads;
  const int64_t row0 = (head * budget + 32 * blk) * D;
  const uint32_t bytes = (uint32_t)((left < 32 ? left : 32) * D * (int)sizeof(T));      // rows past them are not written
  const auto rk = bytes_at(k_ret + row0, bytes), rv = bytes_at(v_ret + row0, bytes);
  uint32_t codes[2][kEach], ex[2][kEach];
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int item = threadIdx.x + i * kPackThreads, d = 8 * (item % (D / 8)), r = item / (D / 8);
      if (!is_v || D == 128) codes[is_v][i] = *reinterpret_cast<const uint32_t*>(in + (is_v ? v_code_at<D>(r, d) : k_code_at<D>(r, d)));
      else codes[is_v][i] = *reinterpret_cast<const uint16_t*>(in + v_code_at<D>(r, d)) | (uint32_t)*reinterpret_cast<const uint16_t*>(in + v_code_at<D>(r, d + 4)) << 16;
      ex[is_v][i] = in[is_v ? v_exp_at<D>(r, d / 32) : k_exp_at<D>(r, d / 32)];
    }
#pragma unroll
  for (int is_v = 0; is_v < 2; ++is_v)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      Eight<T> x;
      x.set(codes[is_v][i], __uint_as_float(ex[is_v][i] << 23));
      x.store(is_v ? rv : rk, (uint32_t)(threadIdx.x + i * kPackThreads) * 8u * (uint32_t)sizeof(T));
    }
}

// Workgroups (shares) of a head and their waves.  A launch takes 256 CUs.
// More heads than CUs: a head's workgroup of four waves, several of them on a CU (1024 heads of 1024 + 512 rows, D = 128: 136 us,
// with eight waves 156; 257, 300 and 384 heads of them 54, 56 and 59 us, with eight 64, 66 and 68; 257, 384 and 512 heads of 1024 +
// 2400 packed rows 68, 74 and 84, with eight 79, 88 and 100; of 768 + 512 rows with four query heads, D = 64, 27.7, 30.4 and 32.5,
// with eight 28.1, 30.9 and 32.8).  Fewer: eight waves (256 heads of 512 + 8192 packed rows, D = 128: 73 us, with four 85), but
// four for few short heads (8 heads of 768 + 512 rows 15.4 us, with eight 16.3; 64 heads 17.5 and 17.8). Few heads of 48 blocks of
// rows or more are cut, in 8 shares or a power of two that leaves each 16 blocks: 8 heads of 768 + 1024 rows 16.1 us in 8 (whole
// 18.2, in 5 17.0), 32 of 768 + 2001 packed 15.7 in 8 (whole 20.6, in 6 and 10 16.5 and 17.4), 8 of 768 + 16384 packed 21.3 in 16
// and 21.0 in 32 (whole 73.9, in 8 26.5), 8 of 768 + 32768 packed 23.4 in 32 (in 16 and 64 27.2 and 30.4: reading the shares grows
// with them); wide rows in more, a share for each 128 KB (2 heads of 768 + 4000 fp32 rows, D = 128: 22.7 us in 32, 25.9 in 16, 25.0
// in 64; 4 of 768 + 16384: 33.4 in 64, 37.7 in 32).  Shorter heads do not gain (40 blocks: 15.4 us whole and in 8).  Where a head
// gets fewer than four CUs packed rows do not gain either (128 heads of 1024 + 8192: 45 us whole, 47 in 2), stored ones do (128 of
// 1024 + 2048: 55 whole, 43 in 2).
constexpr int64_t kCus = 256;
KeptSplit split_of(const ltea_cfg& cfg, int n_seqs, bool packed) {
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv, G = cfg.Hq / cfg.Hkv, fill = kCus / heads;
  const int64_t blocks = (int64_t)kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget);
  if (fill < 1) return KeptSplit{1, 4};
  if (blocks < 48 || fill < (packed ? 4 : 2)) return KeptSplit{1, blocks < 64 && fill > 2 ? 4 : 8};
  const int64_t row = 2 * cfg.D * (cfg.dtype == LTEA_F32 ? 4 : 2), kept = packed ? 2 * (cfg.D / 2 + cfg.D / 32) : row;
  const int64_t by_bytes = (cfg.window * row + cfg.budget * kept) / (128 * 1024), by_blocks = blocks / 16 < 32 ? blocks / 16 : 32;
  int64_t n = 8;
  while (2 * n <= (by_bytes > by_blocks ? by_bytes : by_blocks)) n *= 2;
  for (const int64_t limit : {fill, kKeptMaxFactors / G, (int64_t)kKeptMaxShares}) n = n < limit ? n : limit;
  return KeptSplit{(int)n, 4};
}

// scored: heads whose scores are kept here.  (What shares hand over has its place also where heads are finished whole: a few KB a head.)
size_t kept_floats(const ltea_cfg& cfg, int64_t heads, int64_t shares, int64_t scored) {
  const KeptLayout L{cfg.Hq / cfg.Hkv, cfg.D, 1, 32 * (kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget))};
  auto up = [](size_t x) { return (x + 63) / 64 * 64; };
  return up(L.plan() * heads) + up(L.share() * shares) + L.scores() * scored;
}

}  // namespace

size_t kept_packed_bytes(const ltea_cfg& cfg, int n_seqs) {
  return (size_t)n_seqs * cfg.Hkv * kept_blocks_of(cfg.budget) * 34 * cfg.D;
}

size_t kept_workspace(const ltea_cfg& cfg, int n_seqs, bool packed, bool mass) {
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv;
  if (heads == 0) return 0;
  const KeptSplit s = split_of(cfg, n_seqs, packed);
  return kept_floats(cfg, heads, heads * s.shares, mass && !kept_form(cfg, s, mass).scores_in_lds ? heads : 0) * sizeof(float);
}
// With and without packed rows, and not less for more sequences.  Scores: of all heads, or of no more than are ever cut or take eight waves.
size_t kept_workspace_most(const ltea_cfg& cfg, int n_seqs, bool mass) {
  const int64_t heads = (int64_t)n_seqs * cfg.Hkv;
  if (heads == 0) return 0;
  const int64_t scored = heads > kCus && kept_form(cfg, KeptSplit{1, 4}, mass).scores_in_lds ? kCus : heads;
  return kept_floats(cfg, heads, heads > kCus ? heads : kCus, mass ? scored : 0) * sizeof(float);
}

bool kept_step_supported(const ltea_cfg& cfg, int n_seqs) {
  if (cfg.Hq / cfg.Hkv > kKeptMaxGroup) return false;
  // a head's scores are addressed by 32-bit offsets
  if (((int64_t)kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget)) * 128 * (cfg.Hq / cfg.Hkv) >= (int64_t)1 << 31) return false;
  return (int64_t)n_seqs * cfg.Hkv <= kMaxThreads / 256;      // (more heads than CUs: a workgroup of four waves each)
}

hipError_t launch_kept_step(const ltea_cfg& cfg, const void* q, const void* k, const void* v, void* out, const ltea_cache& c,
                            const void* packed, bool mass, int n_seqs, int32_t* status, void* workspace, hipStream_t stream) {
  const KeptInputs in{q, k, v, out, packed, status, mass};
  const KeptSplit n = split_of(cfg, n_seqs, packed != nullptr);
  if (cfg.dtype == LTEA_F32)
    return cfg.D == 64 ? kept_run_f32_64(cfg, in, c, n_seqs, n, workspace, stream)
                       : kept_run_f32_128(cfg, in, c, n_seqs, n, workspace, stream);
  return cfg.D == 64 ? kept_run_bf16_64(cfg, in, c, n_seqs, n, workspace, stream)
                     : kept_run_bf16_128(cfg, in, c, n_seqs, n, workspace, stream);
}

hipError_t launch_kept_convert(const ltea_cfg& cfg, const ltea_cache& c, void* packed, bool to_packed, int n_seqs, hipStream_t stream) {
  const int n_blocks = kept_blocks_of(cfg.budget);
  const int64_t grid = (int64_t)n_seqs * cfg.Hkv * n_blocks;
  if (grid == 0) return hipSuccess;
  auto go = [&](auto tag, auto dim) {
    using T = decltype(tag);
    constexpr int D = decltype(dim)::value;
    constexpr int64_t kMost = kMaxThreads / kPackThreads;
    for (int64_t first = 0; first < grid; first += kMost) {
      const dim3 blocks((unsigned)(grid - first < kMost ? grid - first : kMost));
      if (to_packed)
        hipLaunchKernelGGL((kept_pack_kernel<T, D>), blocks, dim3(kPackThreads), 0, stream, static_cast<const T*>(c.k_ret),
                           static_cast<const T*>(c.v_ret), c.ret_count, cfg.budget, n_blocks, (uint32_t)first, static_cast<uint8_t*>(packed));
      else
        hipLaunchKernelGGL((kept_unpack_kernel<T, D>), blocks, dim3(kPackThreads), 0, stream, static_cast<const uint8_t*>(packed),
                           c.ret_count, cfg.budget, n_blocks, (uint32_t)first, static_cast<T*>(c.k_ret), static_cast<T*>(c.v_ret));
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  if (cfg.dtype == LTEA_F32)
    return cfg.D == 64 ? go(float{}, std::integral_constant<int, 64>{}) : go(float{}, std::integral_constant<int, 128>{});
  return cfg.D == 64 ? go(bf16_t{}, std::integral_constant<int, 64>{}) : go(bf16_t{}, std::integral_constant<int, 128>{});
}

}  // namespace ltea
