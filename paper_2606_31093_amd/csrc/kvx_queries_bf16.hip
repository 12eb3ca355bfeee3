// kvx_queries_bf16.hip -- the kernels of kvx_queries.h for bfloat16 rows over a bfloat16 cache.

#include "kvx_queries.h"

namespace kvx {

int launch_queries_bf16(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream) {
    return launch_type<false, false>(p, first, n, stream);
}

}  // namespace kvx
