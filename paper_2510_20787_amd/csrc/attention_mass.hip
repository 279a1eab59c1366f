// Attention weight that every token of a prompt has received: mass[h][j] = sum over the query heads of KV head h and the queries i
// that see j of exp(scale q_i . k_j - lse_i).
//
//   S[key, query] = K . Q^T    v_mfma_f32_32x32x16_bf16 (fp32: v_mfma_f32_32x32x2_f32), K held in registers for the life of a wave,
//                              Q tiles of 128 rows (fp32: 64) through LDS
//   mass[key] += 2^(S c - lse_i log2(e))
// A lane owns one query column, so lse is one register, and keeps sums of its 16 keys per block that meet over the lanes once, at
// the end.  Products of bf16 values are exact in fp32 and nothing is rounded to fewer bits.
//
// Bound: a wave's issue.  32 x 32 scores take 128 cycles of exponentials and 128 of scale and sum beside 64 (D = 64) or 128 (D =
// 128) of matrix instructions, which overlap little: 4 x 4096 tokens, 32/8 heads, D = 64: 223 us (615 TFLOP/s of products; vector
// instructions issue in 77 % of the clocks in which a CU has work, matrix instructions in 31 %, and it has some in 79 %: 2176
// workgroups in 768 places), 32768 tokens, 32 heads, D = 128: 4270 us (1.03 PFLOP/s; 4190 to 4460 over several boxes; 67 %, 51 %
// and 96 %).  Two blocks of 32 keys per wave: at D = 64 three take 271 us and four 342 (fewer waves); 16 x 16 instructions 8515 us
// for the long prompt where these took 4560 at the time (registers).
//
// A workgroup takes 4 waves x KB blocks of 32 keys of one (sequence, KV head) and a part of the queries that can see them, all
// query heads of the group.  Parts meet in a second launch, in their order: same bits every time, and sums of at most 2048 queries
// per head in one register chain.  Only parts that reach a key write sums for it; where a window keeps the others away, parts are counted
// from the first that does.  Prompts of more parts than a launch takes (16, or as many as fill the chip) take several pairs of launches,
// so that the sums need no more room than that.
#include "ltea_common.h"
#include "ltea_kernels.h"
#include "mfma_tiles.h"

namespace ltea {
namespace {

constexpr int kThreads = 256, kStepRows = 64;
// Rows of a tile of queries: steps of 64, one barrier.  bf16: two steps (4 x 4096 tokens, 32/8 heads, D = 64: 227 us, with one 267;
// 32768 tokens, 32 heads, D = 128: 4316 and 4363); fp32 fills the LDS with one.
template <typename T, int D> constexpr int kRows = sizeof(T) == 2 ? 128 : 64;
// Blocks of 32 keys per wave, keys per workgroup
template <typename T, int D> constexpr int kKeyBlocks = sizeof(T) == 4 ? 1 : 2;
template <typename T, int D> constexpr int kTileKeys = 4 * 32 * kKeyBlocks<T, D>;
int64_t tile_keys(const ltea_cfg& cfg) {
  if (cfg.dtype == LTEA_F32) return kTileKeys<float, 64>;
  return cfg.D == 64 ? kTileKeys<bf16_t, 64> : kTileKeys<bf16_t, 128>;
}

struct MassParams {
  int n_seqs, tiles_upper, Hq, Hkv, window, last, part_rows, head_parts, part_heads, units;
  int slot0, slots;              // of this launch
  bool relative, whole;          // slots count from a key's first part; sums are the weights: one part in all
  int64_t total;
  float scale2;
};

// Of a sequence of n tokens, the counting queries [first, n) lie in parts of part_rows.  Slot 0 begins at query `from` for the keys
// [lo, hi), which queries before `end` see.
struct Slots {
  uint32_t from, end;
  __device__ __forceinline__ Slots(const MassParams& P, int n, int lo, int hi) {
    const int first = P.last > 0 && n > P.last ? n - P.last : 0;
    const uint32_t reach = (uint32_t)hi - 1u + (uint32_t)P.window, rows = (uint32_t)P.part_rows;
    from = (uint32_t)first + (P.relative && lo > first ? (uint32_t)(lo - first) / rows * rows : 0u);
    end = reach < (uint32_t)n ? reach : (uint32_t)n;
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 2)
attention_mass_kernel(const T* __restrict__ q, int64_t q_st, int64_t q_sh, const T* __restrict__ k, int64_t k_st, int64_t k_sh,
                      const int32_t* __restrict__ cu, const float* __restrict__ lse, MassParams P, float* __restrict__ sums) {
  constexpr int KB = kKeyBlocks<T, D>, kKeys = kTileKeys<T, D>;
  constexpr int kTileRows = kRows<T, D>, kSteps = kTileRows / kStepRows;
  constexpr int kRow = D * (int)sizeof(T), PPR = kRow / 16, KP = PPR / 2;       // 16-byte pieces of a row, and per lane
  constexpr int kLoads = kTileRows * PPR / kThreads;
  __shared__ __align__(1024) uint8_t tile[2][kTileRows * kRow];
  __shared__ float tile_lse[2][kTileRows];
  __shared__ int tile_whole[2][kSteps];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), c = lane & 31, hb = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // An XCD takes whole (part, KV head) units: the key tiles that read the same queries run side by side on its L2.  Late parts, which
  // the most keys see, first.
  const int unit = (int)(blockIdx.x % 8 + blockIdx.x / 8 / P.tiles_upper * 8), flat = (int)(blockIdx.x / 8 % P.tiles_upper);
  if (unit >= P.units) return;
  const int of_launch = P.slots * P.head_parts - 1 - unit / P.Hkv, h = unit % P.Hkv;
  int seq, tile_i, lo, n;
  if (!locate_tile(cu, P.n_seqs, kKeys, flat, seq, tile_i, lo, n)) return;
  const int key0 = tile_i * kKeys, key1 = key0 + kKeys < n ? key0 + kKeys : n;
  float* to = sums + ((int64_t)of_launch * P.Hkv + h) * P.total + lo;
  const Slots slots(P, n, key0, key1);
  const uint32_t from_q = slots.from + (uint32_t)(P.slot0 + of_launch / P.head_parts) * (uint32_t)P.part_rows, to_q = from_q + (uint32_t)P.part_rows;
  const int q0 = from_q > (uint32_t)key0 ? (int)from_q : key0, q1 = to_q < slots.end ? (int)to_q : (int)slots.end;
  if (from_q >= slots.end || q1 <= q0) {
    if (P.whole)
      for (int j = key0 + tid; j < key1; j += kThreads) to[j] = 0.f;
    return;
  }
  const int G = P.Hq / P.Hkv, g0 = of_launch % P.head_parts * P.part_heads, g1 = g0 + P.part_heads < G ? g0 + P.part_heads : G;

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

  // piece p of row r lies at p ^ swizzle(r): sixteen consecutive rows at one piece then cover all banks
  auto swizzle = [](int r) { return PPR == 8 ? (r >> 1) & 7 : r & 15; };
  const uint32_t row_bytes = (uint32_t)(q_st * (int64_t)sizeof(T));
  uint32_t from[kLoads], into[kLoads];                     // of this thread's pieces: in memory from the tile's first row, in the LDS tile
#pragma unroll
  for (int x = 0; x < kLoads; ++x) {
    const int piece = tid + kThreads * x, r = piece / PPR, p = piece % PPR;
    from[x] = (uint32_t)r * row_bytes + 16u * p;
    into[x] = (uint32_t)(r * kRow + 16 * (p ^ swizzle(r)));
  }
  u32x4 held[kLoads];
  float held_lse = 0.f;
  // the tile of query head h * G + g from row r0 on: rows past the sequence's end read as zeros
  auto request = [&](int g, int r0) {
    const T* base = q + (int64_t)(lo + r0) * q_st + (int64_t)(h * G + g) * q_sh;
    const int rows = n - r0 < kTileRows ? n - r0 : kTileRows;
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, (uint32_t)(rows - 1) * row_bytes + (uint32_t)kRow, 0x00020000);
#pragma unroll
    for (int x = 0; x < kLoads; ++x) held[x] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, from[x], 0, 0);
    if (wave < kSteps) held_lse = lse[(int64_t)(h * G + g) * P.total + lo + (r0 + tid < n ? r0 + tid : n - 1)];
  };
  auto put = [&](int buf, int r0) {
#pragma unroll
    for (int x = 0; x < kLoads; ++x) *reinterpret_cast<u32x4*>(&tile[buf][into[x]]) = held[x];
    if (wave < kSteps) {
      const bool counts = r0 + tid < q1 && fabsf(held_lse) < INFINITY;     // a query whose lse is not finite counts nothing
      tile_lse[buf][tid] = counts ? held_lse * 1.4426950408889634f : INFINITY;
      const bool all = __builtin_amdgcn_ballot_w64(counts) == ~0ull;
      if (lane == 0) tile_whole[buf][wave] = all;
    }
  };
  // The block whose scores are there but whose exponentials are not taken yet: they go between the next block's matrix instructions.
  f32x16 s[2];
  float pending = 0.f;
#pragma unroll
  for (int y = 0; y < 16; ++y) s[1][y] = -INFINITY;
  auto mma = [](const u32x4& a, const u32x4& b, const f32x16& acc) {
    if constexpr (sizeof(T) == 2) {
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
      f32x16 r = acc;
#pragma unroll
      for (int e = 0; e < 4; ++e) r = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), r, 0, 0, 0);
      return r;
    }
  };
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto load_q = [&](int buf, int half, u32x4 (&qf)[KP], float& l2) {
    const int r = 32 * half + c;
    l2 = tile_lse[buf][r];
#pragma unroll
    for (int p = 0; p < KP; ++p) qf[p] = *reinterpret_cast<const u32x4*>(&tile[buf][r * kRow + 16 * ((2 * p + hb) ^ swizzle(r))]);
  };
  request(g0, q0);
  put(0, q0);
  __syncthreads();
  int g = g0, r0 = q0;
  for (int buf = 0; g < g1; buf ^= 1) {
    const bool wraps = r0 + kTileRows >= q1;
    const int g_next = wraps ? g + 1 : g, r_next = wraps ? q0 : r0 + kTileRows;
    if (g_next < g1) request(g_next, r_next);
#pragma unroll 1
    for (int step = 0; step < kSteps; ++step) {
      // every query of the step counts and sees every key of the wave
      const int r1 = r0 + kStepRows * step;
      const bool plain = tile_whole[buf][step] && r1 >= my0 + 32 * KB - 1 && r1 + kStepRows - 1 - my0 < P.window && my0 < n;
      if (plain) {
        u32x4 qf[KP];
        float l2 = 0.f, l_old = pending;
#pragma unroll
        for (int st = 0; st < 2 * KB; ++st) {
          const int half = st / KB, x = st % KB, now = st & 1, old = now ^ 1, xo = (st + KB * 2 - 1) % KB;
          if (x == 0) load_q(buf, 2 * step + half, qf, l2);
          s[now] = zero;
          // the first matrix instruction goes before the exponentials that wait for the last one of the block before
#pragma unroll
          for (int p = 0; p < KP; ++p) {
            s[now] = mma(kf[x][p], qf[p], s[now]);
            if (p > 0)
#pragma unroll
              for (int y = 16 * (p - 1) / (KP - 1); y < 16 * p / (KP - 1); ++y)
                sum[xo][y] += __builtin_amdgcn_exp2f(fmaf(s[old][y], P.scale2, -l_old));
            if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
          }
          l_old = l2;
        }
        pending = l2;
      }
      if (!plain && my0 < n) {
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          sum[KB - 1][y] += __builtin_amdgcn_exp2f(fmaf(s[1][y], P.scale2, -pending));
          s[1][y] = -INFINITY;
        }
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const int i0 = r1 + 32 * half;
          // no query, all queries before the wave's keys, or all keys out of their windows
          if (i0 >= q1 || i0 + 31 < my0 || i0 - (my0 + 32 * KB - 1) >= P.window) continue;
          u32x4 qf[KP];
          float l2;
          load_q(buf, 2 * step + half, qf, l2);
          const int i_q = l2 < INFINITY ? i0 + c : -1;      // a query that does not count sees nothing, whatever its row and the keys hold
#pragma unroll
          for (int x = 0; x < KB; ++x) {
            const int j0 = my0 + 32 * x;
            f32x16 z = zero;
#pragma unroll
            for (int p = 0; p < KP; ++p) z = mma(kf[x][p], qf[p], z);
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const int ago = i_q - (j0 + 8 * (y / 4) + 4 * hb + y % 4);
              const float e = __builtin_amdgcn_exp2f(fmaf(z[y], P.scale2, -l2));
              sum[x][y] += ago >= 0 && ago < P.window ? e : 0.f;
            }
          }
        }
        pending = 0.f;
      }
    }
    if (g_next < g1) put(buf ^ 1, r_next);
    __syncthreads();
    g = g_next;
    r0 = r_next;
  }
#pragma unroll
  for (int y = 0; y < 16; ++y) sum[KB - 1][y] += __builtin_amdgcn_exp2f(fmaf(s[1][y], P.scale2, -pending));
  // Sums over the 32 query columns, halving the sums that a lane holds at every step: lane c ends with the one of y = c / 2.
#pragma unroll
  for (int x = 0; x < KB; ++x) {
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum[x][y]), __float_as_uint(sum[x][y + 8]), false, false);
      sum[x][y] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#pragma unroll
    for (int w = 4; w > 0; w >>= 1)
#pragma unroll
      for (int y = 0; y < w; ++y) {
        const bool upper = c & 2 * w;
        const float keep = upper ? sum[x][y + w] : sum[x][y], give = upper ? sum[x][y] : sum[x][y + w];
        sum[x][y] = keep + __shfl_xor(give, 2 * w, kWave);
      }
    const float v = sum[x][0] + __shfl_xor(sum[x][0], 1, kWave);
    const int y = c >> 1, j = my0 + 32 * x + 8 * (y / 4) + 4 * hb + y % 4;
    if ((c & 1) == 0 && j < n) to[j] = v;
  }
}

// The sums of a launch's parts, in their order, join those of the launches before.  A workgroup per key tile of the first kernel.
template <int kKeys>
__global__ void __launch_bounds__(kKeys)
mass_parts_kernel(const float* __restrict__ sums, const int32_t* __restrict__ cu, MassParams P, float* __restrict__ mass) {
  const int h = blockIdx.x / P.tiles_upper, flat = blockIdx.x - h * P.tiles_upper;
  int seq, tile_i, lo, n;
  if (!locate_tile(cu, P.n_seqs, kKeys, flat, seq, tile_i, lo, n)) return;
  const int key0 = tile_i * kKeys, key1 = key0 + kKeys < n ? key0 + kKeys : n, j = key0 + threadIdx.x;
  if (j >= key1) return;
  float* to = mass + h * P.total + lo + j;
  const float* from = sums + h * P.total + lo + j;
  float v = P.slot0 == 0 ? 0.f : *to;
  const Slots slots(P, n, key0, key1);
  const uint32_t rows = (uint32_t)P.part_rows;
  uint32_t q = slots.from + (uint32_t)P.slot0 * rows;
#pragma unroll 4
  for (int u = 0, hp = 0; u < P.slots * P.head_parts; ++u) {
    const float x = from[(int64_t)u * P.Hkv * P.total];      // (of a part that does not reach: anything)
    if (q < slots.end && q + rows > (uint32_t)key0) v += x;
    if (++hp == P.head_parts) { hp = 0; q += rows; }
  }
  *to = v;
}

struct Split { int slots, each, rows, head_parts, heads; bool relative; };      // parts that reach a key, and of one launch; rows and query heads of one
constexpr int64_t kFill = 2048, kOnce = 512, kEach = 16;
// Parts of the queries: as many as fill the chip a few times over (4 x 4096 tokens, 32/8 heads: 226 us; half as many workgroups 258, twice
// 231), at most 2048 queries each and 64 at least (300 fp32 tokens, 2 heads: 10.6 us, with 128 14.6).  Where those are not even two
// workgroups a CU, the query heads of a group are shared out too (300 tokens, 32/8 heads: 17.1 -> 11.6 us; filling the chip as often as
// above by heads, 1000 tokens take 27.4 us instead of 21.8).
// A launch takes 16 parts, or as many as fill the chip, and no more than a grid holds: sums of 64 bytes a token and KV head, whatever the length (131072 tokens, 8 heads,
// D = 128: 17.95 ms in four pairs of launches, 17.87 in one with four times the room).  With a window only the parts that reach a key have a
// slot (the same with a window of 2048: 0.82 ms, with a slot for every part 1.19).
Split split_of(const ltea_cfg& cfg, const SeqView& sv, int last) {
  const int64_t keys = tile_keys(cfg), G = cfg.Hq / cfg.Hkv;
  const int64_t groups = (sv.total_tokens / keys + 1) * cfg.Hkv;
  const int64_t reach = last > 0 && last < sv.max_seqlen ? last : sv.max_seqlen;
  const int64_t fill = (kFill + groups - 1) / groups;
  int64_t parts = fill;
  if (parts < (reach + 2047) / 2048) parts = (reach + 2047) / 2048;
  const int64_t rows = ((reach + parts - 1) / parts + kStepRows - 1) / kStepRows * kStepRows;
  parts = (reach + rows - 1) / rows;
  const int64_t most = kOnce / (groups * parts), heads = most < 2 ? G : most < G ? (G + most - 1) / most : 1;
  const int64_t head_parts = (G + heads - 1) / heads;
  // a key tile and its window: so many queries, which begin anywhere in a part
  const int64_t seen = (cfg.window + keys - 1 + rows - 2) / rows + 1, slots = seen < parts ? seen : parts;
  // (units of eight key heads and parts, see the kernel)
  const int64_t room = (kMaxThreads / kThreads / (sv.total_tokens / keys + sv.n_seqs) - 7) / (cfg.Hkv * head_parts);
  int64_t each = fill > kEach ? fill : kEach;
  if (each > room) each = room > 1 ? room : 1;
  return Split{(int)slots, (int)(slots < each ? slots : each), (int)rows, (int)head_parts, (int)heads, seen < parts};
}

}  // namespace

size_t mass_workspace(const ltea_cfg& cfg, const SeqView& sv, int last) {
  const Split s = split_of(cfg, sv, last);
  const int64_t sums = (int64_t)s.each * s.head_parts;
  return s.slots * s.head_parts > 1 ? (size_t)sums * cfg.Hkv * sv.total_tokens * sizeof(float) : 0;
}
// Of any call of up to so many tokens: sums for every 2048 queries of the longest sequence and one more, but not more than a launch takes,
// or as many as fill the chip.
size_t mass_workspace_most(const ltea_cfg& cfg, int64_t total, int32_t max_seqlen) {
  const size_t keys = tile_keys(cfg), sums = 2 + (size_t)max_seqlen / 2048;
  return (kFill * keys + (size_t)cfg.Hkv * total * (sums < kEach ? sums : kEach)) * sizeof(float);
}

// The threads of a launch and the offsets inside a tile of queries are 32-bit numbers.
bool mass_supported(const ltea_cfg& cfg, const SeqView& sv, int64_t q_st, int last) {
  if (q_st * (cfg.dtype == LTEA_F32 ? 4 : 2) * 128 >= (int64_t)1 << 31) return false;
  if (sv.total_tokens == 0) return true;
  const Split s = split_of(cfg, sv, last);
  return (sv.total_tokens / tile_keys(cfg) + sv.n_seqs) * ((int64_t)cfg.Hkv * s.each * s.head_parts + 7) <= kMaxThreads / kThreads;
}

hipError_t launch_attention_mass(const ltea_cfg& cfg, const void* q, int64_t q_st, int64_t q_sh, const void* k, int64_t k_st, int64_t k_sh,
                                 const SeqView& sv, const float* lse, int last, float* mass, void* workspace, hipStream_t stream) {
  if (sv.total_tokens == 0) return hipSuccess;
  const Split s = split_of(cfg, sv, last);
  MassParams P;
  P.n_seqs = sv.n_seqs; P.Hq = cfg.Hq; P.Hkv = cfg.Hkv; P.window = cfg.window; P.last = last;
  P.part_rows = s.rows; P.head_parts = s.head_parts; P.part_heads = s.heads; P.total = sv.total_tokens;
  P.relative = s.relative; P.whole = s.slots * s.head_parts == 1;
  P.scale2 = (cfg.softmax_scale > 0.f ? cfg.softmax_scale : 1.0f / sqrtf((float)cfg.D)) * 1.4426950408889634f;
  P.tiles_upper = (int)(sv.total_tokens / tile_keys(cfg) + sv.n_seqs);
  float* sums = P.whole ? mass : static_cast<float*>(workspace);
  auto go = [&](auto tag, auto dim) {
    using T = decltype(tag);
    constexpr int D = decltype(dim)::value, kKeys = kTileKeys<T, D>;
    for (P.slot0 = 0; P.slot0 < s.slots; P.slot0 += s.each) {
      P.slots = s.slots - P.slot0 < s.each ? s.slots - P.slot0 : s.each;
      P.units = cfg.Hkv * P.slots * s.head_parts;
      hipLaunchKernelGGL((attention_mass_kernel<T, D>), dim3((unsigned)((int64_t)P.tiles_upper * ((P.units + 7) / 8 * 8))), dim3(kThreads), 0,
                         stream, static_cast<const T*>(q), q_st, q_sh, static_cast<const T*>(k), k_st, k_sh, sv.cu_seqlens, lse, P, sums);
      hipError_t e = hipGetLastError();
      if (e != hipSuccess || P.whole) return e;
      hipLaunchKernelGGL(mass_parts_kernel<kKeys>, dim3((unsigned)(P.tiles_upper * cfg.Hkv)), dim3(kKeys), 0, stream, sums, sv.cu_seqlens, P, mass);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
  };
  if (cfg.dtype == LTEA_F32) return cfg.D == 64 ? go(float{}, std::integral_constant<int, 64>{}) : go(float{}, std::integral_constant<int, 128>{});
  return cfg.D == 64 ? go(bf16_t{}, std::integral_constant<int, 64>{}) : go(bf16_t{}, std::integral_constant<int, 128>{});
}

}  // namespace ltea
