// Grids of many workgroups (launch_grid() of csrc/experts.h): every workgroup has its place, fewer places stand empty than the grid has rows, and no axis has 2^32 threads, with
// 1024 threads a workgroup, the most that a launch may have.  Prints "grids ok".
#include <stdio.h>

#include "../paper_2505_19115_amd/csrc/experts.h"

using namespace nvfp4;

int main()
{
    const int64_t most = INT32_MAX;
    for (int64_t at = 1; at <= most; at = at < most / 2 ? 2 * at : at == most ? most + 1 : most)
        for (int64_t n = at > 3 ? at - 3 : 1; n <= at + 3 && n <= most; ++n) {
            const dim3 g = launch_grid(n);
            const int64_t places = (int64_t)g.x * g.y;
            if (places < n || places - n >= g.y || places > UINT32_MAX || g.z != 1 || (int64_t)g.x * 1024 > UINT32_MAX || g.y > 65535) {
                fprintf(stderr, "%lld workgroups: %u x %u\n", (long long)n, g.x, g.y);
                return 1;
            }
        }
    printf("grids ok\n");
    return 0;
}
