// kvx_queries_bf16_e4m3.hip -- the kernels of kvx_queries.h for bfloat16 rows over an e4m3 cache.

#include "kvx_queries.h"

namespace kvx {

int launch_queries_bf16_e4m3(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream) {
    return launch_type<false, true>(p, first, n, stream);
}

}  // namespace kvx
