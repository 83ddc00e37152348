// Causal attention of sequences' new tokens over the paged key-value cache: the kernels are in
// prefill_tile.h.
#include "prefill_tile.h"

// Enough for every call: 2 groups of a head's slots (see plan_of: groups + tiles of a prefill, which has no more tiles than groups
// where it splits any; 4/3 groups of a tree's call).
size_t prefill_work_bytes(int kvh, int dim)
{
    const size_t groups = (size_t)std::max(groups_of(dim) / kvh, 1) * 2;
    return groups * sizeof(Split) + groups * kvh * WAVES * part_floats(dim) * sizeof(float);
}

// Whether the call's tiles fit one launch.
bool prefill_fits(const KvDev &c, int heads) { return tiles_of(c, heads) * c.kvh < (1ll << 23); }

hipError_t launch_prefill(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s)
{
    if (type == SAE_KV_BF16) return launch_dim<SAE_KV_BF16, false>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_dim<SAE_KV_F16, false>(c, a, dim, s);
    return launch_dim<SAE_KV_FP8, false>(c, a, dim, s);
}
