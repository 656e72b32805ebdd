// Prints the norm's workgroups of csrc/launch_sizes.hpp for the numbers on stdin, one line per line read.
#include <inttypes.h>
#include <stdio.h>

#include "launch_sizes.hpp"

int main()
{
    int64_t work, threads;
    while (scanf("%" SCNd64 " %" SCNd64, &work, &threads) == 2) printf("%" PRId64 "\n", ul::norm_grid(work, threads));
    return 0;
}
