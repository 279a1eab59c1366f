// Attention weight that every token of a prompt has received: mass[h][j] = sum over the query heads of KV head h and the queries i
// that see j of exp(scale q_i . k_j - lse_i).
//
//   S[key, query] = K . Q^T    v_mfma_f32_32x32x16_bf16 (fp32: v_mfma_f32_32x32x2_f32), K held in registers for the life of a wave,
//                              Q tiles of 64 rows through LDS
//   mass[key] += 2^(S c - lse_i log2(e))
// A lane owns one query column, so lse is one register, and keeps sums of its 16 keys per block that meet over the lanes once, at
// the end.  Products of bf16 values are exact in fp32 and nothing is rounded to fewer bits.
//
// A workgroup takes 4 waves x KB blocks of 32 keys of one (sequence, KV head) and a part of the queries that can see them, all
// query heads of the group.  Parts meet in a second launch, in their order: same bits every time, and sums of at most 2048 queries
// per head in one register chain.
#include "ltea_common.h"
#include "ltea_kernels.h"
#include "mfma_tiles.h"

namespace ltea {
namespace {

constexpr int kThreads = 256, kTileRows = 64;
template <typename T> constexpr int kKeyBlocks = sizeof(T) == 4 ? 1 : 2;      // of 32 keys per wave
template <typename T> constexpr int kTileKeys = 4 * 32 * kKeyBlocks<T>;

struct MassParams {
  int n_seqs, tiles_upper, Hq, Hkv, window, last, parts, part_rows;
  int64_t total;
  float scale2;
};

// Queries of a sequence of n tokens that can see a key of [lo, hi) and count.
__device__ __forceinline__ void queries_of(const MassParams& P, int n, int lo, int hi, int& q0, int& q1) {
  const int first = P.last > 0 && n > P.last ? n - P.last : 0;
  q0 = lo > first ? lo : first;
  const int64_t reach = (int64_t)hi - 1 + P.window;
  q1 = reach < n ? (int)reach : n;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2)
attention_mass_kernel(const T* __restrict__ q, int64_t q_st, int64_t q_sh, const T* __restrict__ k, int64_t k_st, int64_t k_sh,
                      const int32_t* __restrict__ cu, const float* __restrict__ lse, MassParams P, float* __restrict__ sums) {
  constexpr int KB = kKeyBlocks<T>, kKeys = kTileKeys<T>;
  constexpr int kRow = D * (int)sizeof(T), PPR = kRow / 16, KP = PPR / 2;       // 16-byte pieces of a row, and per lane
  constexpr int kLoads = kTileRows * PPR / kThreads;
  __shared__ __align__(1024) uint8_t tile[2][kTileRows * kRow];
  __shared__ float tile_lse[2][kTileRows];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 31, hb = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int part = blockIdx.x % P.parts, h = blockIdx.x / P.parts % P.Hkv, flat = blockIdx.x / P.parts / P.Hkv;
  int seq, tile_i, lo, n;
  if (!locate_tile(cu, P.n_seqs, kKeys, flat, seq, tile_i, lo, n)) return;
  const int key0 = tile_i * kKeys, key1 = key0 + kKeys < n ? key0 + kKeys : n;
  int q0, q1;
  queries_of(P, n, key0, key1, q0, q1);
  q0 += part * P.part_rows;
  q1 = q1 < q0 + P.part_rows ? q1 : q0 + P.part_rows;
  const int G = P.Hq / P.Hkv;

  // this wave's keys
  const int my0 = key0 + wave * 32 * KB;
  u32x4 kf[KB][KP];
#pragma unroll
  for (int x = 0; x < KB; ++x) {
    const int j = my0 + 32 * x + c;
    const u32x4* row = reinterpret_cast<const u32x4*>(k + (int64_t)(lo + (j < n ? j : n - 1)) * k_st + h * k_sh);
#pragma unroll
    for (int i = 0; i < KP; ++i) kf[x][i] = row[2 * i + hb];
  }
  float sum[KB][16];
#pragma unroll
  for (int x = 0; x < KB; ++x)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[x][r] = 0.f;

  const int per_head = q1 > q0 ? (q1 - q0 + kTileRows - 1) / kTileRows : 0, tiles = per_head * G;
  // piece p of row r lies at p ^ swizzle(r): sixteen consecutive rows at one piece then cover all banks
  auto swizzle = [](int r) { return PPR == 8 ? (r >> 1) & 7 : r & 15; };
  u32x4 held[kLoads];
  float held_lse = 0.f;
  auto request = [&](int i) {
    const int g = i / per_head, r0 = q0 + (i - g * per_head) * kTileRows;
    const T* base = q + (int64_t)lo * q_st + (int64_t)(h * G + g) * q_sh;
#pragma unroll
    for (int x = 0; x < kLoads; ++x) {
      const int piece = tid + kThreads * x, r = piece / PPR;
      const int row = r0 + r < n ? r0 + r : n - 1;
      held[x] = reinterpret_cast<const u32x4*>(base + (int64_t)row * q_st)[piece % PPR];
    }
    if (tid < kTileRows) {
      const float y = r0 + tid < q1 ? lse[(int64_t)(h * G + g) * P.total + lo + r0 + tid] : INFINITY;
      held_lse = fabsf(y) < INFINITY ? y * 1.4426950408889634f : INFINITY;       // no query, or one whose lse is not finite: counts nothing
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int x = 0; x < kLoads; ++x) {
      const int piece = tid + kThreads * x, r = piece / PPR;
      *reinterpret_cast<u32x4*>(&tile[buf][r * kRow + 16 * ((piece % PPR) ^ swizzle(r))]) = held[x];
    }
    if (tid < kTileRows) tile_lse[buf][tid] = held_lse;
  };
  if (tiles > 0) { request(0); put(0); }
  __syncthreads();
  for (int i = 0; i < tiles; ++i) {
    const int buf = i & 1;
    if (i + 1 < tiles) request(i + 1);
    const int r0 = q0 + (i % per_head) * kTileRows;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int i0 = r0 + 32 * half, r = 32 * half + c;
      // no query, no key, all queries before the wave's keys, or all keys out of their windows
      if (i0 >= q1 || my0 >= n || i0 + 31 < my0 || i0 - (my0 + 32 * KB - 1) >= P.window) continue;
      const float l2 = tile_lse[buf][r];
      const bool dead = !(l2 < INFINITY);
      u32x4 qf[KP];
#pragma unroll
      for (int p = 0; p < KP; ++p) qf[p] = *reinterpret_cast<const u32x4*>(&tile[buf][r * kRow + 16 * ((2 * p + hb) ^ swizzle(r))]);
      if (__builtin_amdgcn_ballot_w64(dead)) {
        if (dead)
#pragma unroll
          for (int p = 0; p < KP; ++p) qf[p] = u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int x = 0; x < KB; ++x) {
        const int j0 = my0 + 32 * x;
        f32x16 s;
#pragma unroll
        for (int y = 0; y < 16; ++y) s[y] = 0.f;
#pragma unroll
        for (int p = 0; p < KP; ++p) {
          if constexpr (sizeof(T) == 2) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[x][p]), __builtin_bit_cast(bf16x8, qf[p]), s, 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[x][p][e]), __uint_as_float(qf[p][e]), s, 0, 0, 0);
          }
        }
        const bool whole = i0 >= j0 + 31 && i0 + 31 - j0 < P.window;        // every query of the block sees every key
        if (whole) {
#pragma unroll
          for (int y = 0; y < 16; ++y) sum[x][y] += __builtin_amdgcn_exp2f(fmaf(s[y], P.scale2, -l2));
        } else {
          const int i_q = i0 + c;
#pragma unroll
          for (int y = 0; y < 16; ++y) {
            const int ago = i_q - (j0 + 8 * (y / 4) + 4 * hb + y % 4);
            const float e = __builtin_amdgcn_exp2f(fmaf(s[y], P.scale2, -l2));
            sum[x][y] += ago >= 0 && ago < P.window ? e : 0.f;
          }
        }
      }
    }
    if (i + 1 < tiles) put(buf ^ 1);
    __syncthreads();
  }
  float* to = sums + ((int64_t)part * P.Hkv + h) * P.total + lo;
#pragma unroll
  for (int x = 0; x < KB; ++x)
#pragma unroll
    for (int y = 0; y < 16; ++y) {
      float v = sum[x][y];
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
      const int j = my0 + 32 * x + 8 * (y / 4) + 4 * hb + y % 4;
      if (c == 0 && j < n) to[j] = v;
    }
}

__global__ void __launch_bounds__(kThreads)
mass_parts_kernel(const float* __restrict__ sums, int parts, int64_t n, float* __restrict__ mass) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  float v = 0.f;
  for (int p = 0; p < parts; ++p) v += sums[p * n + i];
  mass[i] = v;
}

struct Split { int parts, rows; };
// Parts of the queries: as many as fill the chip a few times over, at most 2048 queries each.
Split split_of(const ltea_cfg& cfg, const SeqView& sv, int last) {
  const int64_t keys = cfg.dtype == LTEA_F32 ? kTileKeys<float> : kTileKeys<bf16_t>;
  const int64_t groups = (sv.total_tokens / keys + 1) * cfg.Hkv;
  int64_t reach = cfg.window + keys - 1 < sv.max_seqlen ? cfg.window + keys - 1 : sv.max_seqlen;
  if (last > 0 && last < reach) reach = last;
  int64_t parts = (1024 + groups - 1) / groups;
  if (parts < (reach + 2047) / 2048) parts = (reach + 2047) / 2048;
  int64_t rows = ((reach + parts - 1) / parts + kTileRows - 1) / kTileRows * kTileRows;
  return Split{(int)((reach + rows - 1) / rows), (int)rows};
}

}  // namespace

size_t mass_workspace(const ltea_cfg& cfg, const SeqView& sv, int last) {
  const Split s = split_of(cfg, sv, last);
  return s.parts > 1 ? (size_t)s.parts * cfg.Hkv * sv.total_tokens * sizeof(float) : 0;
}
// Of any call of up to so many tokens: a part for every 2048 queries of the longest sequence and one more, or as many as fill the chip.
size_t mass_workspace_most(const ltea_cfg& cfg, int64_t total, int32_t max_seqlen) {
  const size_t keys = cfg.dtype == LTEA_F32 ? kTileKeys<float> : kTileKeys<bf16_t>;
  return (1024 * keys + (size_t)cfg.Hkv * total * (2 + (size_t)max_seqlen / 2048)) * sizeof(float);
}

// The grid is a 32-bit number.
bool mass_supported(const ltea_cfg& cfg, const SeqView& sv, int last) {
  const int64_t keys = cfg.dtype == LTEA_F32 ? kTileKeys<float> : kTileKeys<bf16_t>;
  return sv.total_tokens == 0 || (sv.total_tokens / keys + sv.n_seqs) * cfg.Hkv * split_of(cfg, sv, last).parts <= INT32_MAX;
}

hipError_t launch_attention_mass(const ltea_cfg& cfg, const void* q, int64_t q_st, int64_t q_sh, const void* k, int64_t k_st, int64_t k_sh,
                                 const SeqView& sv, const float* lse, int last, float* mass, void* workspace, hipStream_t stream) {
  if (sv.total_tokens == 0) return hipSuccess;
  const Split s = split_of(cfg, sv, last);
  MassParams P;
  P.n_seqs = sv.n_seqs; P.Hq = cfg.Hq; P.Hkv = cfg.Hkv; P.window = cfg.window; P.last = last;
  P.parts = s.parts; P.part_rows = s.rows; P.total = sv.total_tokens;
  P.scale2 = (cfg.softmax_scale > 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)cfg.D)) * 1.4426950408889634f;
  float* sums = s.parts > 1 ? static_cast<float*>(workspace) : mass;
  auto go = [&](auto tag, auto dim) {
    using T = decltype(tag);
    constexpr int D = decltype(dim)::value;
    P.tiles_upper = (int)(sv.total_tokens / kTileKeys<T> + sv.n_seqs);
    hipLaunchKernelGGL((attention_mass_kernel<T, D>), dim3((unsigned)((int64_t)P.tiles_upper * cfg.Hkv * s.parts)), dim3(kThreads), 0,
                       stream, static_cast<const T*>(q), q_st, q_sh, static_cast<const T*>(k), k_st, k_sh, sv.cu_seqlens, lse, P, sums);
    return hipGetLastError();
  };
  const hipError_t e = cfg.dtype == LTEA_F32
                           ? (cfg.D == 64 ? go(float{}, std::integral_constant<int, 64>{}) : go(float{}, std::integral_constant<int, 128>{}))
                           : (cfg.D == 64 ? go(bf16_t{}, std::integral_constant<int, 64>{}) : go(bf16_t{}, std::integral_constant<int, 128>{}));
  if (e != hipSuccess || s.parts == 1) return e;
  const int64_t n = sv.total_tokens * cfg.Hkv;
  hipLaunchKernelGGL(mass_parts_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, sums, s.parts, n, mass);
  return hipGetLastError();
}

}  // namespace ltea
