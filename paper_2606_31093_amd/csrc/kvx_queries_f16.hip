// kvx_queries_f16.hip -- the kernels of kvx_queries.h for half rows over a half cache.

#include "kvx_queries.h"

namespace kvx {

int launch_queries_f16(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream) {
    return launch_type<true, false>(p, first, n, stream);
}

}  // namespace kvx
