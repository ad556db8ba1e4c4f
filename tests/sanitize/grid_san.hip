// Built for the host with AddressSanitizer and UndefinedBehaviorSanitizer: launch grids for any number of workgroups keep to the limits of a launch.
#include <stdio.h>

#include "../../paper_2402_02320_amd/csrc/generation.hpp"

using namespace spin;

int main()
{
    // up to the words of one tensor, 64 elements a workgroup
    for (size_t blocks = 1; blocks <= (size_t)1 << 34; blocks = blocks + blocks / 3 + 1)
        for (size_t near : {blocks - 1, blocks, blocks + 1}) {
            if (near == 0) continue;
            const dim3 g = grid_of(near);
            const size_t all = (size_t)g.x * g.y;
            if ((size_t)g.x * 256 > 0xffffffffu || g.y > kMaxGrid || g.z != 1 || all < near || all - near >= g.x) {
                printf("%zu workgroups: %u x %u x %u\n", near, g.x, g.y, g.z);
                return 1;
            }
        }
    printf("grid run ok\n");
    return 0;
}
