// What the launchers (kept.hip) and the kernels (kept_step.h, instantiated per storage type and head size in kept_step_*.hip) of
// the decode step over a cache that evicts by accumulated attention weight, or whose kept rows are in 4 bits, share.
#pragma once
#include "decode_run.h"

namespace ltea {

struct KeptInputs { const void *q, *k, *v; void* out; const void* packed; int32_t* status; bool mass; };

constexpr int kKeptMaxShares = 64;       // lanes of a wave
constexpr int kKeptMaxGroup = 128;       // query heads per KV head

constexpr int kKeptMaxFactors = 6144;    // query heads times shares: two numbers each in the second launch's LDS
constexpr size_t kKeptScoresLds = 40 * 1024;    // bytes of a head's scores that stay in LDS
constexpr size_t kKeptLds = 52 * 1024;          // bytes of LDS that a workgroup asks for beside its fixed arrays

struct KeptSplit { int shares, waves; };        // of a head; waves of a workgroup that takes a whole one, if their outputs fit

// What the workgroups of a head hand to the finishing launch, in floats of the workspace.
struct KeptLayout {
  int G, D, nsplit, slots;
  // per head: t, count, bits of the leaving token's key, late; scores of the incoming and of the leaving token [2][G]; V row of the
  // leaving token as it would be kept [D]
  __host__ __device__ size_t plan() const { return 4 + 2 * (size_t)G + D; }
  // per share: its lowest entry (its place in the order, two words, slot, pad), that entry's scores [G] and V row [D], maximum, sum and output [G][D + 2]
  __host__ __device__ size_t share() const { return 4 + (size_t)G + D + (size_t)G * (D + 2); }
  // per head: the scores of all slots [G][slots]
  __host__ __device__ size_t scores() const { return (size_t)G * slots; }
};

inline int kept_blocks_of(int rows) { return (int)(((int64_t)rows + 31) / 32); }

// What a step launches.
struct KeptForm {
  bool whole;                    // one launch: a head's workgroup finishes it, where its count fits ret_count's upper bits
  int waves;
  bool scores_in_lds;            // by weight: else the scores of all slots are kept in the workspace
  size_t lds;                    // bytes that a workgroup asks for
};
inline KeptForm kept_form(const ltea_cfg& cfg, KeptSplit split, bool mass) {
  const int G = cfg.Hq / cfg.Hkv, pass = G < 16 ? G : 16;          // query heads of a pass
  KeptForm f;
  f.whole = split.shares == 1 && cfg.budget > 0 && cfg.budget < (1 << 16) && cfg.Hkv <= 255;
  f.waves = f.whole && split.waves == 8 && pass * cfg.D <= 1024 ? 8 : 4;          // (the outputs of eight waves: 34 KB)
  f.lds = ((size_t)f.waves * pass * (cfg.D + 4) + 6 * (size_t)G + 4) * sizeof(float);
  const size_t scores = (size_t)G * 32 * ((size_t)kept_blocks_of(cfg.window) + kept_blocks_of(cfg.budget)) * sizeof(float);
  f.scores_in_lds = mass && f.whole && scores <= kKeptScoresLds && f.lds + scores <= kKeptLds;
  if (f.scores_in_lds) f.lds += scores;
  return f;
}

#define LTEA_KEPT_RUN(name)                                                                                       \
  hipError_t name(const ltea_cfg& cfg, const KeptInputs& in, const ltea_cache& c, int n_seqs, KeptSplit split, void* workspace, \
                  hipStream_t stream)
LTEA_KEPT_RUN(kept_run_f32_64);
LTEA_KEPT_RUN(kept_run_f32_128);
LTEA_KEPT_RUN(kept_run_bf16_64);
LTEA_KEPT_RUN(kept_run_bf16_128);

}  // namespace ltea
