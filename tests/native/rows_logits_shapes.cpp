// Prints the side of the logits' tiles (csrc/launch_sizes.hpp), and 1 where they keep more steps on their way, for the
// numbers on stdin: the table's rows, h's, bytes of an element.
#include <inttypes.h>
#include <stdio.h>

#include "launch_sizes.hpp"

int main()
{
    int64_t rows, n, elem;
    while (scanf("%" SCNd64 " %" SCNd64 " %" SCNd64, &rows, &n, &elem) == 3) {
        const ul::TileShape s = ul::logits_shape(rows, n, elem);
        printf("%" PRId64 " %d\n", ul::tile_side(s), s == ul::TileShape::tiny_deep);
    }
    return 0;
}
