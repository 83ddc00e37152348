// Attention of drafted tokens that form trees over the paged key-value cache: the kernels of
// prefill_tile.h, whose rows see the cached prefix, their ancestors and themselves.
//
// A tree comes as its tokens' parents.  Which tokens a row sees is a row of bits in LDS, made from the
// parents in log2(tokens) rounds by the workgroups whose keys reach into the tree (or that a window's
// depths matter to); a step of 64 keys takes from it two words a row, shifted to the step's
// first key.  Steps before the tree cost what they cost in a prompt.
#include "prefill_tile.h"

hipError_t launch_tree(const KvDev &c, const AttnArgs &a, int type, int dim, hipStream_t s)
{
    if (type == SAE_KV_BF16) return launch_dim<SAE_KV_BF16, true>(c, a, dim, s);
    if (type == SAE_KV_F16) return launch_dim<SAE_KV_F16, true>(c, a, dim, s);
    return launch_dim<SAE_KV_FP8, true>(c, a, dim, s);
}
