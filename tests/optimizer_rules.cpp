// The sizes of the norm's launches, for tests that evaluate them without a GPU.
#include "wash_internal.h"

extern "C" {
void rule_norm(int layout, int n_models, unsigned units, int elem_bytes, int sm_count, unsigned *out)
{
    const wash::NormPlan plan = wash::norm_plan(layout, n_models, units, elem_bytes, sm_count);
    const int together = plan.bytes / (8 * elem_bytes);
    const wash::NormGrid grid = wash::norm_grid(layout, n_models, units, plan.threads, together, plan.blocks);
    out[0] = static_cast<unsigned>(plan.threads);
    out[1] = static_cast<unsigned>(together);
    out[2] = grid.n_chunks;
    out[3] = grid.per_model;
}
unsigned long long rule_norm_partials(int layout, int n_models, int sm_count) { return wash::norm_partials(layout, n_models, sm_count); }
unsigned rule_chunk_units(int layout, int n_models) { return wash::chunk_units(layout, n_models); }
}
