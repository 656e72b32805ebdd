// Prints the norm's workgroups of csrc/launch_sizes.hpp for the numbers on stdin, one line per line read.
#include <inttypes.h>
#include <stdio.h>

#include "launch_sizes.hpp"

int main()
{
    int64_t work, threads;
    int32_t cols;
    while (scanf("%" SCNd64 " %" SCNd32 " %" SCNd64, &work, &cols, &threads) == 3)
        printf("%" PRId64 "\n", ul::norm_grid(work, cols, threads));
    return 0;
}
