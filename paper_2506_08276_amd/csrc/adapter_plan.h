// Which kernel a projection with adapters goes through.  Host code without HIP types.
#pragma once
#include <stdint.h>

enum ProjectTile { PROJECT_32 = 0, PROJECT_64, PROJECT_256 };

// rows x N x K: project_kernel with tiles of 32 x 32 or 64 x 64 (four wavefronts share K), or project_large_kernel (256 x 256, from K of 256 on).
// 32 x 32 while its blocks fit the chip at once; beyond, what the busiest CU's tiles take.  Microseconds of the kernel, rank 16, bf16:
//   rows x N x K          32      64      256 |                          64     256
//    48 x  768 x  768    4.6     6.5       - |  2000 x 2304 x  768      27      27
//   300 x  384 x 1536    6.5    10.6       - |  4000 x  768 x  768      17      26
//   300 x  768 x  768    5.4     7.5       - |  4000 x 2304 x  768      47      28
//   500 x  768 x  768    8.1     7.6       - |  8000 x  384 x 1536      28      37
//   800 x  384 x  384    5.9     6.4      20 |  8000 x  768 x  768      30      27
//   800 x  768 x  768   10.8     8.0      26 |  8000 x 2304 x  768      85      51
//   800 x 2304 x  768   24.6    15.0      26 | 16000 x  384 x  384      22      21
//  1300 x  384 x 1536   11.3    11.2      37 | 32000 x  384 x 1536     100      47
inline ProjectTile choose_project(int cus, int64_t rows, int N, int K)
{
    auto tiles = [&](int size) { return ((rows + size - 1) / size) * ((N + size - 1) / size); };
    auto rounds = [&](int size) { return (double)((tiles(size) + cus - 1) / cus); };
    if (tiles(32) <= cus) return PROJECT_32;
    const double us64 = 4.0 + rounds(64) * (1.2 + 0.0044 * K), us256 = rounds(256) * (13.5 + 0.0155 * K);
    return K >= 256 && us256 < us64 ? PROJECT_256 : PROJECT_64;
}
