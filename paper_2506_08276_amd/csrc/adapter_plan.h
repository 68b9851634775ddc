// Which kernel a projection with adapters goes through, sums of row numbers that stay below 2^31, which matrices share bytes.  Code without HIP types.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define PLAN_FN __host__ __device__ inline
#else
#define PLAN_FN inline
#endif

constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;  // of 256 threads in a launch, which takes fewer than 2^32 threads

// Whether low_kernel's blocks share K, one per tile of 16 rows: up to four of them per CU; beyond, wavefronts of their own for 32 rows each read less.
inline bool low_shares_k(int cus, int tiles) { return tiles < 4 * cus; }

// Whether a tile of `height` rows has any of `rows`: tile * height may pass 2^31 behind the last one.
PLAN_FN bool tile_has_rows(int tile, int height, int rows) { return tile <= (rows - 1) / height; }
// Slot `base` of a chunk of n, or the one behind the chunk: what a wavefront asks for ahead may lie some hundred behind it.
PLAN_FN int chunk_slot(int first, int n, int base) { return first + (base < n ? base : n); }

enum ProjectTile { PROJECT_32 = 0, PROJECT_64, PROJECT_256, PROJECT_96 };

// rows x N x K: project_kernel with tiles of 32 x 32, 64 x 64 or 64 x 96 (four wavefronts share K), or project_large_kernel (256 x 256, from K of 256 on).
// 32 x 32 while its blocks fit the chip at once; 64 x 96 (one block per CU) where its blocks do and those of 64 x 64 do not; beyond, what the busiest CU's tiles take.
// Microseconds of the kernel, rank 16, bf16:
//   rows x N x K          32      64      96     256 |                          64      96     256
//    48 x  768 x  768    4.6     6.4       -       - |  4000 x  384 x  384     9.0     7.9      19
//   300 x  384 x 1536    6.2    10.2       -       - |  4000 x  768 x  768      17       -      25
//   300 x  768 x  768    5.2     6.9       -       - |  4000 x 2304 x  768      43       -      29
//   500 x  768 x  768    7.7     7.0       -      27 |  8000 x  384 x 1536      28       -      38
//   500 x 2304 x  768   15.7    11.9     8.8      27 |  8000 x  768 x  768      29       -      27
//   800 x  384 x  384    5.4     6.0       -      20 |  8000 x 2304 x  768      81       -      50
//   800 x  768 x  768   10.2     7.4       -      25 | 16000 x  384 x  384      23       -      20
//   800 x 2304 x  768   22.5    13.2       -      26 | 32000 x  384 x 1536     101       -      48
//  1300 x  384 x 1536   10.7    10.6       -      36 |  2000 x 2304 x  768      25       -      27
//  2000 x  768 x  768   18.5    11.0     9.0      25 |  3391 x  384 x 1536      19    13.4      38
// Those are with one or two adapters per tile.  In project_large_kernel every adapter of a tile is a pair of slabs for each 32 of its ranks (16, in fp16), 1.7 us however few
// rows it has; in project_kernel up to 32 of a group's are on their way together, 0.08 us of a tile's for 16 ranks of one.  Single tokens, the whole call, K of 768, the
// chosen one marked; worst of 270 cases with K of 384 to 2304: 7 % behind the better of the two, without these terms 4 times.
//   rows x N, adapters x rank, type   pairs of a tile      64      256 |  rows x N, adapters x rank, type   pairs of a tile      64      256
//   4000 x  768   1024 x 16  bf16          70            *36.4   155.7 |   8000 x 2304     64 x 64  fp16          16            130.4  *138.8
//   8000 x  768   1024 x 16  bf16          39            *48.0   103.0 |   8000 x 2304     64 x 64  bf16           8            123.1   *98.6
//   8000 x  768   4000 x 16  bf16         122            *99.1   284.4 |  32000 x 2304   1024 x 64  bf16          22            721.6  *530.1
//   8000 x 2304   4000 x 16  bf16         122           *301.6   638.7 |  64000 x 2304   4000 x 16  bf16          20            922.5  *691.2
inline int segment_pairs(int rank, int pieces) { return ((rank + 15) / 16 * pieces + 1) / 2; }  // pieces: bf16 numbers that hold one of `up`'s

// What the adapters of a batch are to the tiles: pairs of slabs in tiles of 256 rows, and sixteens of ranks of every adapter in every group of 32 rows.
struct AdapterLoad {
    int most_pairs = 0;  // of one tile
    int64_t pairs = 0, sixteens = 0;
};

inline ProjectTile choose_project(int cus, int64_t rows, int N, int K, AdapterLoad load = AdapterLoad())
{
    auto tiles_of = [&](int height, int width) { return ((rows + height - 1) / height) * ((N + width - 1) / width); };
    auto tiles = [&](int size) { return tiles_of(size, size); };
    auto rounds = [&](int size) { return (double)((tiles(size) + cus - 1) / cus); };
    if (tiles(32) <= cus) return PROJECT_32;
    if (tiles(64) > cus && tiles_of(64, 96) <= cus) return PROJECT_96;
    auto beyond_two = [](double v) { return v > 2 ? v - 2 : 0; };
    const double us64 = 4.0 + rounds(64) * (1.2 + 0.0044 * K + 0.08 * beyond_two((double)load.sixteens / ((rows + 63) / 64)));
    const double mean = rounds(256) * beyond_two((double)load.pairs / ((rows + 255) / 256)), most = beyond_two(load.most_pairs);
    const double us256 = rounds(256) * (13.5 + 0.0155 * K) + 1.7 * (mean > most ? mean : most);
    return K >= 256 && us256 < us64 ? PROJECT_256 : PROJECT_64;
}

// Whether any of `rows` rows of a_cols elements at `a`, lda elements apart, shares a byte with any of b's; lda >= a_cols, ldb >= b_cols.  Rows of one may lie between those of
// the other.
inline bool rows_overlap(uint64_t a, int64_t lda, int64_t a_cols, uint64_t b, int64_t ldb, int64_t b_cols, int64_t rows, int size)
{
    typedef __int128 Wide;
    const Wide a_step = (Wide)lda * size, b_step = (Wide)ldb * size, a_bytes = (Wide)a_cols * size, b_bytes = (Wide)b_cols * size, d = (Wide)b - a;
    if (rows < 1 || d >= (rows - 1) * a_step + a_bytes || -d >= (rows - 1) * b_step + b_bytes) return false;
    auto meets = [&](int64_t j) {  // b's row j against the last of a's rows that begin before its end: those before that one end earlier
        const Wide start = d + j * b_step, last = start + b_bytes - 1;
        if (last < 0) return false;
        const Wide i = last / a_step < rows - 1 ? last / a_step : rows - 1;
        return i * a_step + a_bytes > start;
    };
    if (lda == ldb || rows == 1) return meets(0) || meets(rows - 1);  // all rows lie alike; the first or the last one has a's rows on both sides
    for (int64_t j = 0; j < rows; ++j)
        if (meets(j)) return true;
    return false;
}
