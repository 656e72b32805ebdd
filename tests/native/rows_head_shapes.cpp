// Prints the side of a product's tiles (csrc/launch_sizes.hpp), and 1 where they keep more steps on their way, for
// the numbers on stdin: rows, columns, most parts, bytes of an element.
#include <inttypes.h>
#include <stdio.h>

#include "launch_sizes.hpp"

int main()
{
    int64_t m, n, most, elem;
    while (scanf("%" SCNd64 " %" SCNd64 " %" SCNd64 " %" SCNd64, &m, &n, &most, &elem) == 4) {
        const ul::TileShape s = ul::tile_shape(m, n, most, elem);
        printf("%" PRId64 " %d\n", ul::tile_side(s), s == ul::TileShape::tiny_deep);
    }
    return 0;
}
