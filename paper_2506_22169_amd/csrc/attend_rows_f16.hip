// Few rows over the cache, f16 queries.
#include "attend_rows.hpp"

namespace mcf {
int attend::launch_rows_f16(const Params &p, int size, int row_blocks, int waves, unsigned blocks, void *stream) {
    return launch_rows<_Float16>(p, size, row_blocks, waves, blocks, stream);
}
} // namespace mcf
