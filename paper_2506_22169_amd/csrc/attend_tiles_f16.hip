// Many rows over the cache, f16 queries.
#include "attend_tiles.hpp"

namespace mcf {
int attend::launch_tiles_f16(const Params &p, int size, int waves, unsigned blocks, void *stream) {
    return launch_tiles<_Float16>(p, size, waves, blocks, stream);
}
} // namespace mcf
