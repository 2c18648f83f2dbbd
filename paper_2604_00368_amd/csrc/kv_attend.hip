// tent_kv_attend: what it enqueues is in kv_attend.h.
#include "kv_attend.h"

using namespace tent;

extern "C" int tent_kv_attend_workspace(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args,
                                        uint64_t* bytes)
{
    const int rc = check(cache, batch, args);
    if (rc != TENT_OK) return rc;
    if (!bytes) return TENT_ERR_INVALID;
    *bytes = batch->n_seqs == 0 || batch->n_rows == 0 ? 0 : shape_of(*cache, *batch, *args, false).workspace;
    return TENT_OK;
}

extern "C" int tent_kv_attend(const tent_kv_cache* cache, const tent_kv_batch* batch, const tent_kv_attend_args* args, void* stream)
{
    const int rc = check(cache, batch, args);
    return rc != TENT_OK ? rc : attend<false>(cache, batch, args, nullptr, stream);
}
