// Few rows over the cache, bf16 queries.
#include "attend_rows.hpp"

namespace mcf {
int attend::launch_rows_bf16(const Params &p, int size, int row_blocks, int waves, unsigned blocks, void *stream) {
    return launch_rows<__bf16>(p, size, row_blocks, waves, blocks, stream);
}
} // namespace mcf
