// Instances of the step over kept entries: see kept_step.h.
#include "kept_step.h"

namespace ltea {

LTEA_KEPT_RUN(kept_run_f32_64) { return kept_run<float, 64>(cfg, in, c, n_seqs, split, workspace, stream); }
LTEA_KEPT_RUN(kept_run_f32_128) { return kept_run<float, 128>(cfg, in, c, n_seqs, split, workspace, stream); }

}  // namespace ltea
