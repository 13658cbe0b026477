// Many rows over the cache, bf16 queries.
#include "attend_tiles.hpp"

namespace mcf {
int attend::launch_tiles_bf16(const Params &p, int size, int waves, unsigned blocks, void *stream) {
    return launch_tiles<__bf16>(p, size, waves, blocks, stream);
}
} // namespace mcf
