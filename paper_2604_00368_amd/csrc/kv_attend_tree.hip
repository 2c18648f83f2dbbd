// tent_kv_attend_tree: attention of a tree of drafted tokens.  The kernels are those of kv_attend.h, in which what a row sees of its
// sequence's rows is the bits of its mask.
#include "kv_attend.h"

using namespace tent;

namespace {

int check_tree(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args)
{
    const int rc = check(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (args->flags & TENT_KV_ATTEND_ALL) return TENT_ERR_INVALID;
    return batch->n_seqs && batch->n_rows && args->window && args->window < batch->max_rows ? TENT_ERR_RANGE : TENT_OK;
}

}  // namespace

extern "C" int tent_kv_attend_tree_workspace(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args, uint64_t* bytes)
{
    const int rc = check_tree(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (!bytes) return TENT_ERR_INVALID;
    *bytes = batch->n_seqs == 0 || batch->n_rows == 0 ? 0 : shape_of(*cache, *batch, *args, true).workspace;
    return TENT_OK;
}

extern "C" int tent_kv_attend_tree(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args, const tent_kv_tree* tree,
                                   void* stream)
{
    const int rc = check_tree(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (!tree || tree->reserved) return TENT_ERR_INVALID;
    if (batch->n_seqs == 0 || batch->n_rows == 0) return TENT_OK;
    if (!tree->masks || ((uintptr_t)tree->masks & 7u)) return TENT_ERR_INVALID;
    if ((uint64_t)tree->mask_stride * 64 < batch->max_rows) return TENT_ERR_RANGE;
    return attend<true>(cache, batch, args, tree, stream);
}
