// Launches of the cache's page operations (arguments checked by the C entries).
#pragma once
#include "common.cuh"

namespace gdn {

int pool_launches(const gdn_cache_desc* d);          // launches that a call with these pools needs to move pages
int fork_launches(const gdn_cache_desc* d);
cudaError_t launch_cache_copy(const gdn_cache_desc* d, const int32_t* src, const int32_t* dst, int32_t count);
cudaError_t launch_cache_fork(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* parents, const int32_t* children,
                              const int32_t* tokens, int32_t count);
cudaError_t launch_cache_free(const gdn_cache_desc* d, int32_t* refcounts, int32_t* tables, const int32_t* rows, int32_t count);
cudaError_t launch_cache_compact(const gdn_cache_desc* d, const int32_t* refcounts, const int32_t* tables, int32_t* out_refcounts, int32_t* out_tables,
                                 int32_t* page_map, int32_t* live);

}  // namespace gdn
