// Instances of the step over kept entries: see kept_step.h.
#include "kept_step.h"

namespace ltea {

LTEA_KEPT_RUN(kept_run_bf16_128) { return kept_run<bf16_t, 128>(cfg, in, c, n_seqs, split, workspace, stream); }

}  // namespace ltea
