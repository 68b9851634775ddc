// Projections with low-rank adapters beside a shared weight, and their gradients (gfx950).
#include <math.h>
#include <string.h>

#include <algorithm>
#include <exception>
#include <initializer_list>
#include <new>
#include <type_traits>
#include <vector>

#include "adapter_gemm.h"

namespace {

// ------------------------------------------------------------------ layouts
// W[N][K] (or, transposed, W[K][N] read by columns) in the MFMA's operand order: [N / 32][K / 16][lane][8], lane l holding column l & 31 and the K
// of 8 (l >> 5) on.  Zeros beyond N and K, up to a multiple of 32 and of 128.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const T *w, int N, int K, int transposed, T *out)
{
    const int ksteps = project_ksteps(K);
    const size_t pieces = (size_t)((N + 31) >> 5) * ksteps * 64;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (size_t)gridDim.x * 256) {
        const int lane = (int)(i & 63), step = (int)((i >> 6) % ksteps), ct = (int)((i >> 6) / ksteps);
        const int n = ct * 32 + (lane & 31), k = step * 16 + (lane >> 5) * 8;
        Raw8<T> v;
        for (int j = 0; j < 8; ++j)
            v.v[j] = n < N && k + j < K ? (transposed ? w[(size_t)(k + j) * N + n] : w[(size_t)n * K + k + j]) : (T)0.f;
        v.store(out + i * 8, 8);
    }
}

// up[n][r] (IS_UP) or down[r][n] of the used adapters in the order that the products read, see adapter.h: one piece of 8 ranks of a column per thread and step.
// In the low-rank activations' launch, beside them.
template <class T, bool IS_UP>
__device__ inline void lay_out(const T *from, const int32_t *used, const int4 *adapters, int n_used, int R, int N, bf16_t *to, int block, int blocks)
{
    constexpr int UP = Frag<T>::PIECES;
    const int R16 = rank_groups(R), column_tiles = (N + 31) >> 5;
    const size_t items = (size_t)n_used * column_tiles * R16 * 64;
    for (size_t i = (size_t)block * 256 + threadIdx.x; i < items; i += (size_t)blocks * 256) {
        const int lane = (int)(i & 63), k = (int)((i >> 6) % R16), a = used[(i >> 6) / R16 / column_tiles];
        const int n = (int)((i >> 6) / R16 % column_tiles) * 32 + (lane & 31), r = k * 16 + (lane >> 5) * 8, left = adapters[a].z - r;
        Raw8<T> v;
        v.v = typename Vec8<T>::type{};
        if (n < N && left > 0) {
            if constexpr (IS_UP) {
                v.load(from + ((size_t)a * N + n) * R + r, min(left, 8));
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) v.v[j] = from[((size_t)a * R + r + j) * N + n];
            }
        }
        f32x8 f = v.wide();
#pragma unroll
        for (int e = 0; e < UP; ++e) *reinterpret_cast<bf16x8 *>(to + ((i >> 6) * UP * 64 + e * 64 + lane) * 8) = take_piece(f);
    }
}

// Before the gradients: `up` of the used adapters transposed (up[n][r] -> up_t[r][n], blocks of 32 x 32, so that the low-rank activations' kernel reads rows of it as it
// reads `down`), and `down` laid out for the product.  A few hundred KB: a launch, 5 to 6 us.
template <class T>
__global__ __launch_bounds__(256) void lay_out_kernel(const T *down, const T *up, const int32_t *used, const int4 *adapters, int n_used, int R, int K,
                                                      int N, T *up_t, bf16_t *down_packed, int transposing)
{
    if ((int)blockIdx.x >= transposing) {
        lay_out<T, false>(down, used, adapters, n_used, R, K, down_packed, blockIdx.x - transposing, gridDim.x - transposing);
        return;
    }
    __shared__ T tile[32][34];
    const int tiles_n = (N + 31) / 32, tiles_r = (R + 31) / 32;
    const int n0 = blockIdx.x % tiles_n * 32, r0 = blockIdx.x / tiles_n % tiles_r * 32, number = blockIdx.x / tiles_n / tiles_r;
    const T *from = up + (size_t)used[number] * N * R;
    T *to = up_t + (size_t)number * N * R;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    for (int j = ty; j < 32; j += 8)
        if (n0 + j < N && r0 + tx < R) tile[j][tx] = from[(size_t)(n0 + j) * R + r0 + tx];
    __syncthreads();
    for (int j = ty; j < 32; j += 8)
        if (r0 + j < R && n0 + tx < N) to[(size_t)(r0 + j) * N + n0 + tx] = tile[tx][j];
}

// ------------------------------------------------------------------ low-rank activations
// low[row][r] = sum over k of x[row][k] down[a][r][k] for 16 RT slots of one adapter, in MFMA 16x16x32: a lane ends with four ranks of a row.
// They go out as they are, by row (`low`, if wanted), and times the adapter's scale in the pieces that the product reads, by slot.
// SPLIT: a block per tile, whose four wavefronts share K; else a wavefront per tile, of 32 rows, as reading `down` again for every 16 of them would
// cost as much as reading x.  Blocks from `low_blocks` on lay out `up`.  Bound by memory and the way there: 83 229 rows of 768, rank 16, take 29 us (4.8 TB/s with what
// it writes), with 16 rows per wavefront 31.5; rank 32 38 and 46, K of 2304 82 and 106.  48 rows of 768: 4.2 us, a launch and two dependent reads.
template <class T, int NT, int RT, bool SPLIT>
__global__ __launch_bounds__(256) void low_kernel(const T *x, int64_t ldx, const T *down, int R, int K, const int32_t *row_of, const int4 *tiles,
                                                  int n_tiles, int low_blocks, int compact, float *low, bf16_t *pieces, const int4 *adapters, const T *up,
                                                  int N, const int32_t *used, int n_used, bf16_t *up_packed)
{
    if ((int)blockIdx.x >= low_blocks) {
        lay_out<T, true>(up, used, adapters, n_used, R, N, up_packed, blockIdx.x - low_blocks, gridDim.x - low_blocks);
        return;
    }
    typedef typename Frag<T>::type F;
    static_assert(!SPLIT || RT == 1, "");
    __shared__ f32x4 part[SPLIT ? 4 : 1][SPLIT ? NT : 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, q = lane >> 4;
    const int index = SPLIT ? blockIdx.x : blockIdx.x * 4 + wave;
    if (index >= n_tiles) return;
    const int4 tile = tiles[index];
    const int n = tile.z & 0xffff, rank = tile.z >> 16, groups = (rank + 15) >> 4;
    const float scale = rank ? __int_as_float(adapters[tile.x].w) : 0.f;
    int64_t row[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) row[t] = row_of[tile.y + min(t * 16 + j, n - 1)];
    f32x4 acc[RT][NT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int g = 0; g < NT; ++g) acc[t][g] = f32x4{};
    if (rank) {
        const T *xp[RT], *ap[NT];
#pragma unroll
        for (int t = 0; t < RT; ++t) xp[t] = x + row[t] * ldx + q * 8;
#pragma unroll
        for (int g = 0; g < NT; ++g) ap[g] = down + ((size_t)(compact ? tile.w : tile.x) * R + min(g * 16 + j, rank - 1)) * K + q * 8;
        const int steps = (K + 31) >> 5, per = SPLIT ? (steps + 3) >> 2 : steps;
        const int from = SPLIT ? wave * per : 0, to = min(steps, from + per);
        constexpr int U = RT > 1 || NT > 2 ? 2 : 4;  // steps whose operands are on their way together
        for (int s = from; s < to; s += U) {
            F xf[U][RT], af[U][NT];
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const bool in = s + i < to && (s + i) * 32 + q * 8 < K;  // K is a multiple of 8
                    xf[i][t] = *(in ? reinterpret_cast<const F *>(xp[t] + (s + i) * 32) : reinterpret_cast<const F *>(&zero_piece));
                }
#pragma unroll
            for (int g = 0; g < NT; ++g)
                if (g < groups)
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        const bool in = s + i < to && (s + i) * 32 + q * 8 < K;
                        af[i][g] = *(in ? reinterpret_cast<const F *>(ap[g] + (s + i) * 32) : reinterpret_cast<const F *>(&zero_piece));
                    }
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int g = 0; g < NT; ++g)
                    if (g < groups)
#pragma unroll
                        for (int t = 0; t < RT; ++t) acc[t][g] = mfma16(af[i][g], xf[i][t], acc[t][g]);
        }
        if constexpr (SPLIT) {
#pragma unroll
            for (int g = 0; g < NT; ++g) part[wave][g][lane] = acc[0][g];
            __syncthreads();
#pragma unroll
            for (int g = 0; g < NT; ++g) acc[0][g] = (part[0][g][lane] + part[1][g][lane]) + (part[2][g][lane] + part[3][g][lane]);
        }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t * 16 + j >= n) continue;
        bf16_t *to = pieces + (int64_t)(tile.y + t * 16 + j) * rank_groups(R) * 32;
#pragma unroll
        for (int g = 0; g < NT; ++g) {
            const int r = g * 16 + q * 4;
            if (SPLIT && (g & 3) != wave) continue;
            f32x4 v = acc[t][g];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = r + i < rank ? v[i] : 0.f;
            if (low && r < R) *reinterpret_cast<f32x4 *>(low + row[t] * R + r) = v;
            if (g < groups) {
                v *= scale;
                f32x4 first, second;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    first[i] = first_piece(v[i]);
                    second[i] = behind_first(v[i]);  // rounded, as nothing comes behind it
                }
                *reinterpret_cast<bf16x4 *>(to + g * 32 + q * 4) = __builtin_convertvector(first, bf16x4);
                *reinterpret_cast<bf16x4 *>(to + g * 32 + 16 + q * 4) = __builtin_convertvector(second, bf16x4);
            }
        }
    }
}

// ------------------------------------------------------------------ the projection
// out[row][n] = sum over k of x[row][k] W[n][k] + bias[n] + the adapter's part, tiles of 32 TM x 32 TN slots and columns.  Four wavefronts share K, every fourth step of 16
// each, so that together they read whole lines of x (2000 x 384 x 1536, the whole call: 14.2 us, with a quarter of K in a row each 16.6); operands from memory
// to registers, U steps ahead; their sums meet in LDS.  The adapters come first, while the first operands are on their way.  For few rows, where the time
// of one tile is what counts: 48 x 768 x 768 4.4 to 5.8 us by the number of runs, bound by the reads that wait for each other (row number, x; runs, pieces,
// `up`); 3391 x 384 x 1536 in tiles of 64 x 96 13.4 us, in 64 x 64 (two on some units) 18.8.  Beyond that the larger tile reads less.
template <class T, int TM, int TN, int U>
__global__ __launch_bounds__(256, 2) void project_kernel(const T *x, int64_t ldx, const T *w, const float *bias, int N, int K, const int32_t *row_of,
                                                      int rows, const int32_t *run_ptr, const int2 *runs, const bf16_t *pieces, int R16,
                                                      const bf16_t *up, T *out, int64_t ldo)
{
    typedef typename Frag<T>::type F;
    constexpr int BM = 32 * TM, BN = 32 * TN, PITCH = BN + 4;
    __shared__ float sums[4][BM][PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    // Blocks go round-robin to the 8 XCDs: those of one take a run of tiles, all columns of a few rows (3391 x 384 x 1536 in 64 x 64: 18 us, with
    // columns apart 24).
    const int tiles_n = (N + BN - 1) / BN, tile = (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3));
    const int tile_n = tile % tiles_n, tile_m = tile / tiles_n;
    if (!tile_has_rows(tile_m, BM, rows)) return;
    const int ksteps = project_ksteps(K), used = (K + 15) >> 4;
    const T *xp[TM], *wp[TN];
    int2 my_run[TM];
    int count[TM];
#pragma unroll
    for (int mi = 0; mi < TM; ++mi) xp[mi] = x + (int64_t)row_of[tile_m * BM + mi * 32 + l32] * ldx + half * 8;
#pragma unroll
    for (int mi = 0; mi < TM; ++mi) {
        const int group = tile_m * TM + mi, begin = group * 32 < rows ? run_ptr[group] : 0;
        count[mi] = group * 32 < rows ? run_ptr[group + 1] - begin : 0;
        my_run[mi] = int2{};
        if (lane < count[mi]) my_run[mi] = runs[begin + lane];
    }
    const int last_ct = (N - 1) >> 5;
#pragma unroll
    for (int ni = 0; ni < TN; ++ni) wp[ni] = w + ((size_t)min(tile_n * TN + ni, last_ct) * ksteps * 64 + lane) * 8;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
        for (int ni = 0; ni < TN; ++ni) acc[mi][ni] = f32x16{};
    F xf[U][TM], wf[U][TN];
    auto fetch = [&](int i, int s) {  // zeros of x beyond K; behind the last step that one again, for nothing
        s = min(s, used - 1);
        const bool in = s * 16 + half * 8 < K;
#pragma unroll
        for (int ni = 0; ni < TN; ++ni) wf[i][ni] = *reinterpret_cast<const F *>(wp[ni] + (size_t)s * 512);
#pragma unroll
        for (int mi = 0; mi < TM; ++mi) xf[i][mi] = *(in ? reinterpret_cast<const F *>(xp[mi] + s * 16) : reinterpret_cast<const F *>(&zero_piece));
    };
#pragma unroll
    for (int i = 0; i < U; ++i) fetch(i, wave + 4 * i);
#pragma unroll
    for (int mi = 0; mi < TM; ++mi)
        add_adapters<TN, Frag<T>::PIECES>(acc[mi], my_run[mi], count[mi], tile_m * TM + mi, wave, 4,
                                          pieces + (int64_t)min(tile_m * BM + mi * 32 + l32, rows - 1) * R16 * 32, up, R16, last_ct + 1, tile_n * TN);
    auto multiply = [&](int i) {
#pragma unroll
        for (int mi = 0; mi < TM; ++mi)
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) acc[mi][ni] = mfma32(wf[i][ni], xf[i][mi], acc[mi][ni]);
    };
    int s = wave;
    for (; s + 4 * U < used; s += 4 * U) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            multiply(i);
            fetch(i, s + 4 * (U + i));
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i)  // a step beyond the last is not multiplied: W may hold infinities
        if (s + 4 * i < used) multiply(i);
#pragma unroll
    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
        for (int ni = 0; ni < TN; ++ni)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = {acc[mi][ni][4 * g], acc[mi][ni][4 * g + 1], acc[mi][ni][4 * g + 2], acc[mi][ni][4 * g + 3]};
                *reinterpret_cast<f32x4 *>(&sums[wave][mi * 32 + l32][ni * 32 + 8 * g + 4 * half]) = v;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < BM * BN / 8; i += 256) {
        const int m = i / (BN / 8), c = i % (BN / 8) * 8, col = tile_n * BN + c, slot = tile_m * BM + m;
        if (col >= N || slot >= rows) continue;  // N is a multiple of 8
        f32x8 v = {};
        if (bias) __builtin_memcpy(&v, bias + col, sizeof(v));
#pragma unroll
        for (int p = 0; p < 4; ++p) v += *reinterpret_cast<const f32x8 *>(&sums[p][m][c]);
        Raw8<T> o;
        o.round(v);
        *reinterpret_cast<typename Vec8<T>::type *>(out + (int64_t)row_of[slot] * ldo + col) = o.v;
    }
}

// ------------------------------------------------------------------ the adapters' gradients
// Eight rows of eight 16-bit elements, transposed: out[f] holds element f of the rows in order.
__device__ inline void transpose8(const u32x4 (&in)[8], u32x4 (&out)[8])
{
#pragma unroll
    for (int f = 0; f < 8; ++f)
#pragma unroll
        for (int p = 0; p < 4; ++p)  // rows 2p and 2p + 1
            out[f][p] = __builtin_amdgcn_perm(in[2 * p + 1][f >> 1], in[2 * p][f >> 1], f & 1 ? 0x07060302 : 0x05040100);
}

// 32 rows' share of sum over rows of h[row][r] p[row][c], to 24 bits of h: three pieces of it; fp16 elements are two bf16 pieces exactly.
__device__ inline f32x4 outer_step(const bf16x8 (&h)[3], const bf16x8 &p, f32x4 c)
{
    c = mfma16(h[2], p, c);
    c = mfma16(h[1], p, c);
    return mfma16(h[0], p, c);
}
__device__ inline f32x4 outer_step(const bf16x8 (&h)[3], const f16x8 &p, f32x4 c)
{
    f32x8 v = __builtin_convertvector(p, f32x8);
    const bf16x8 p1 = take_piece(v), p2 = take_piece(v);
    c = mfma16(h[2], p2, c);
    c = mfma16(h[2], p1, c);
    c = mfma16(h[1], p2, c);
    c = mfma16(h[1], p1, c);
    c = mfma16(h[0], p2, c);
    return mfma16(h[0], p1, c);
}

// partial[chunk][r][c] = sum over the chunk's rows of low[row][r] p[row][c]: c < K from x and the low-rank gradients (down's), then N from dout and the
// low-rank activations (up's).  A block takes 128 columns and 16 NR ranks, its wavefronts 32 rows each in turn; a lane reads 16 bytes of a row and turns
// eight rows of them, in registers, into the MFMA operands of its eight columns; low goes through LDS, 16 bytes of a row per lane on the way in.  The next
// rows are on their way while these are multiplied, and the numbers of those after them.  Bound by the bytes in flight (204 registers, two wavefronts per SIMD):
// 82 953 rows, 768 + 768 columns, rank up to 32: 75 us, 3.4 TB/s (72 with pieces rounded to nearest, which makes NaN of infinities).
template <class T, int NR>
__global__ __launch_bounds__(256) void outer_kernel(const T *x, int64_t ldx, const T *dout, int64_t ldd, const float *grad_low, const float *low, int R,
                                                    int K, int N, const int32_t *row_of, const int2 *chunks, float *partial)
{
    constexpr int PITCH = 36;  // rows of a rank's 32, in steps of 16 bytes, and all banks by ranks
    __shared__ __attribute__((aligned(16))) float sums[16 * NR][128];
    __shared__ __attribute__((aligned(16))) float turned[4][16 * NR][PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, j = lane & 15;
    const int strips_k = (K + 127) / 128, strips = strips_k + (N + 127) / 128, strip = blockIdx.x % strips;
    const int2 chunk = chunks[blockIdx.x / strips];
    const int n = chunk.y & 0xffff, rank = chunk.y >> 16, r0 = blockIdx.y * 16 * NR;
    if (r0 >= rank) return;
    const bool of_x = strip < strips_k;
    const T *p = of_x ? x : dout;
    const int64_t ld = of_x ? ldx : ldd;
    const float *h = (of_x ? grad_low : low) + r0 + (lane & 3) * 4;
    const int C = of_x ? K : N, c0 = (of_x ? strip : strip - strips_k) * 128, col = c0 + j * 8;
    const bool has_col = col < C;
    f32x4 acc[NR][8];
#pragma unroll
    for (int g = 0; g < NR; ++g)
#pragma unroll
        for (int f = 0; f < 8; ++f) acc[g][f] = f32x4{};
    int row[8], h_row[2];
    u32x4 d[8];
    f32x4 hv[NR][2];
    auto number = [&](int base) {  // the table goes on behind the last slot: what is read there is not used
        __builtin_memcpy(row, row_of + chunk_slot(chunk.x, n, base + q * 8), sizeof(row));
#pragma unroll
        for (int i = 0; i < 2; ++i) h_row[i] = row_of[chunk_slot(chunk.x, n, base + i * 16 + (lane >> 2))];
    };
    auto request = [&](int base) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            d[i] = base + q * 8 + i < n && has_col ? *reinterpret_cast<const u32x4 *>(p + row[i] * ld + col) : u32x4{};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int g = 0; g < NR; ++g)
                hv[g][i] = base + i * 16 + (lane >> 2) < n && r0 + g * 16 + (lane & 3) * 4 < R
                               ? *reinterpret_cast<const f32x4 *>(h + (int64_t)h_row[i] * R + g * 16) : f32x4{};
    };
    number(wave * 32);
    request(wave * 32);
    number(wave * 32 + 128);
    for (int base = wave * 32; base < n; base += 128) {
        u32x4 t[8];
        bf16x8 piece[NR][3];
        __builtin_amdgcn_wave_barrier();  // LDS serves a wavefront's accesses in order
#pragma unroll
        for (int g = 0; g < NR; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) turned[wave][g * 16 + (lane & 3) * 4 + e][i * 16 + (lane >> 2)] = hv[g][i][e];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int g = 0; g < NR; ++g) {
            f32x8 v;
            __builtin_memcpy(&v, __builtin_assume_aligned(&turned[wave][g * 16 + j][q * 8], 16), sizeof(v));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_canonicalizef(v[i]);  // a NaN whose upper half is an infinity's
#pragma unroll
            for (int i = 0; i < 3; ++i) piece[g][i] = take_piece(v);
        }
        transpose8(d, t);
        request(base + 128);
        number(base + 256);
#pragma unroll
        for (int f = 0; f < 8; ++f)
#pragma unroll
            for (int g = 0; g < NR; ++g) acc[g][f] = outer_step(piece[g], __builtin_bit_cast(typename Frag<T>::type, t[f]), acc[g][f]);
    }
    for (int w = 0; w < 4; ++w) {  // the wavefronts' sums, in order
        if (wave == w)
#pragma unroll
            for (int g = 0; g < NR; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x8 v;
#pragma unroll
                    for (int f = 0; f < 8; ++f) v[f] = acc[g][f][e];
                    f32x8 *to = reinterpret_cast<f32x8 *>(&sums[g * 16 + q * 4 + e][j * 8]);
                    *to = w ? *to + v : v;
                }
        __syncthreads();
    }
    float *to = partial + (size_t)(blockIdx.x / strips) * R * (K + N) + (of_x ? 0 : K) + c0;
    for (int i = threadIdx.x; i < 16 * NR * 32; i += 256) {
        const int r = i >> 5, c = (i & 31) * 4;
        if (r0 + r < rank && c0 + c < C) *reinterpret_cast<f32x4 *>(to + (size_t)(r0 + r) * (K + N) + c) = *reinterpret_cast<const f32x4 *>(&sums[r][c]);
    }
}

// ddown[a][r][k] and dup[a][n][r] from the chunks' sums, in their order; 0 where an adapter has no rows, and beyond its rank.  13.5 MB of sums: 4.9 us.
__global__ __launch_bounds__(1024) void outer_sum_kernel(const float *partial, const int4 *adapters, int R, int K, int N, float *ddown, float *dup)
{
    __shared__ float tile[32][33];
    const int4 a = adapters[blockIdx.z];
    const int c0 = blockIdx.x * 32, r0 = blockIdx.y * 32, tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = c0 + tx, r = r0 + ty;
    float s = 0.f;
    if (r < a.z && c < K + N) {
        const float *from = partial + ((size_t)a.x * R + r) * (K + N) + c;
        const size_t step = (size_t)R * (K + N);
        for (int i = 0; i < a.y; i += 8) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + j < a.y ? from[(i + j) * step] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
    }
    s *= __int_as_float(a.w);
    if (r < R && c < K) ddown[((size_t)blockIdx.z * R + r) * K + c] = s;
    if (c0 + 32 <= K) return;
    tile[ty][tx] = s;
    __syncthreads();
    const int n = c0 + ty - K;
    if (n >= 0 && n < N && r0 + tx < R) dup[((size_t)blockIdx.z * N + n) * R + r0 + tx] = tile[tx][ty];
}

template <class K>
int allow_lds(K kernel, int bytes)
{
    LEANN_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return LEANN_OK;
}

template <class F>
int with_half_type(int dtype, F f)
{
    if (dtype == LEANN_BF16) return f((bf16_t *)nullptr);
    return f((f16_t *)nullptr);
}

int launched(const char *call)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LEANN_OK;
    leann_set_error("%s: launch failed: %s", call, hipGetErrorString(e));
    return LEANN_EDEVICE;
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

int check_half_rows(const char *call, const char *what, const void *p, int64_t ld, int64_t cols)
{
    if (!p || !aligned16(p)) {
        leann_set_error("%s: %s is null or not aligned to 16 bytes", call, what);
        return LEANN_EINVAL;
    }
    if (ld < cols || ld % 8) {
        leann_set_error("%s: rows of %s are %lld elements apart, need at least %lld and a multiple of 8", call, what, (long long)ld, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

// The launch of the low-rank activations: blocks for them, for rows without adapter, too, if those are to be zeros, and for `up` of N columns in the product's order.
struct LowLaunch {
    bool split;  // four wavefronts share K
    int tiles;
    int64_t low_blocks, blocks;
};
LowLaunch plan_low(const leann_ctx *ctx, const leann_adapter_rows *rows, bool with_zeros, int N)
{
    LowLaunch l;
    l.split = low_shares_k(ctx->num_cus, rows->n_tiles);
    l.tiles = l.split ? (with_zeros ? rows->n_tiles : rows->n_adapted_tiles) : with_zeros ? rows->n_wide_tiles : rows->n_adapted_wide_tiles;
    l.low_blocks = l.split ? l.tiles : (l.tiles + 3) / 4;
    const int64_t laying = ((int64_t)rows->n_used * ((N + 31) / 32) * rank_groups(rows->max_rank) * 64 + 255) / 256;
    l.blocks = l.low_blocks ? l.low_blocks + std::min<int64_t>(laying, ctx->num_cus * 4) : 0;
    return l;
}

// What a product's adapters need: the low-rank activations in pieces (and as they are, if wanted; with_zeros: zeros for rows without adapter, too), `up` laid
// out (up: from here, in the same launch; null: it is there already).
template <class T>
void enqueue_low(leann_ctx *ctx, const leann_adapter_rows *rows, const T *x, int64_t ldx, int K, const T *down, int compact, float *low, bool with_zeros,
                 bf16_t *pieces, const T *up, int N, bf16_t *up_packed)
{
    const int R = rows->max_rank;
    const LowLaunch l = plan_low(ctx, rows, with_zeros, up ? N : 0);
    if (!l.blocks) return;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks), dim3(256), 0, ctx->stream, x, ldx, down, R, K, rows->row_of, l.split ? rows->tiles : rows->wide_tiles,
                           l.tiles, (int)l.low_blocks, compact, low, pieces, rows->adapters, up, N, rows->used, rows->n_used, up_packed);
    };
    static_assert(WIDE_ROWS == 32, "two tiles of 16");
    if (R <= 16) l.split ? go(low_kernel<T, 1, 1, true>) : go(low_kernel<T, 1, 2, false>);
    else if (R <= 32) l.split ? go(low_kernel<T, 2, 1, true>) : go(low_kernel<T, 2, 2, false>);
    else if (R <= 64) l.split ? go(low_kernel<T, 4, 1, true>) : go(low_kernel<T, 4, 2, false>);
    else l.split ? go(low_kernel<T, 8, 1, true>) : go(low_kernel<T, 8, 2, false>);
}

struct ProjectLaunch {
    ProjectTile tile;
    int64_t blocks;
};
ProjectLaunch plan_project(const leann_ctx *ctx, const leann_adapter_rows *rows, int dtype, int64_t ldx, int N, int K)
{
    ProjectLaunch l;
    l.tile = choose_project(ctx->num_cus, rows->T, N, K, rows->load[(dtype == LEANN_F16 ? Frag<f16_t>::PIECES : Frag<bf16_t>::PIECES) - 1]);
    if (l.tile == PROJECT_256 && rows->T * ldx / 8 >= 0xffffff00ll) l.tile = PROJECT_64;  // beyond the large tiles' offsets
    const int height = l.tile == PROJECT_32 ? 32 : l.tile == PROJECT_256 ? 256 : 64, width = l.tile == PROJECT_96 ? 96 : height;
    l.blocks = ((rows->T + height - 1) / height * ((N + width - 1) / width) + 7) / 8 * 8;
    if (l.tile == PROJECT_256) l.blocks = std::min<int64_t>(l.blocks, ctx->num_cus);
    return l;
}

// out = x w^T + bias + the adapters' part
template <class T>
void enqueue_project(leann_ctx *ctx, const leann_adapter_rows *rows, const T *x, int64_t ldx, const T *w, const float *bias, int N, int K,
                     const bf16_t *pieces, const bf16_t *up, T *out, int64_t ldo)
{
    const int R16 = rank_groups(rows->max_rank);
    const ProjectLaunch l = plan_project(ctx, rows, std::is_same_v<T, f16_t> ? LEANN_F16 : LEANN_BF16, ldx, N, K);
    if (l.tile == PROJECT_256) {
        typedef ProjectCfg<2, 4, 2> Cfg;
        static_assert(Cfg::BM == 256 && Cfg::BN == 256, "");
        const int tiles_n = (N + Cfg::BN - 1) / Cfg::BN;
        hipLaunchKernelGGL((project_large_kernel<T, 2, 4, 2>), dim3((unsigned)l.blocks), dim3(512), Cfg::SMEM, ctx->stream, x, ldx, w, bias, N, K, rows->row_of,
                           (int)rows->T, rows->seg_ptr, rows->segs, pieces, R16, up, out, ldo, tiles_n);
        return;
    }
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.blocks), dim3(256), 0, ctx->stream, x, ldx, w, bias, N, K, rows->row_of, (int)rows->T, rows->run_ptr,
                           rows->runs, pieces, R16, up, out, ldo);
    };
    if (l.tile == PROJECT_32) go(project_kernel<T, 1, 1, 8>);
    else if (l.tile == PROJECT_64) go(project_kernel<T, 2, 2, 4>);
    else go(project_kernel<T, 2, 3, 4>);
}

// Before the first launch of a call: all of its launches.
int check_launches(const char *call, std::initializer_list<int64_t> blocks)
{
    for (int64_t b : blocks)
        if (b > MAX_BLOCKS) {
            leann_set_error("%s: rows, columns and adapters of this number are not covered (%lld workgroups in a launch, at most %lld)", call, (long long)b,
                            (long long)MAX_BLOCKS);
            return LEANN_ESHAPE;
        }
    return LEANN_OK;
}

size_t pieces_bytes(const leann_adapter_rows *rows) { return up256((size_t)rows->T * rank_groups(rows->max_rank) * 64 + 64); }  // 64: read past the last one's, see request_pieces
size_t packed_bytes(const leann_adapter_rows *rows, int N)  // room for fp16's two pieces
{
    return up256((size_t)rows->n_used * ((N + 31) / 32) * rank_groups(rows->max_rank) * 2048);
}

template <class T>
void enqueue_outer(leann_ctx *ctx, const leann_adapter_rows *rows, const T *x, int64_t ldx, const T *dout, int64_t ldd, const float *grad_low,
                   const float *low, int K, int N, float *partial)
{
    const int R = rows->max_rank, strips = (K + 127) / 128 + (N + 127) / 128;
    auto go = [&](auto kernel, int ranks) {
        hipLaunchKernelGGL(kernel, dim3(strips * rows->n_chunks, (R + ranks - 1) / ranks), dim3(256), 0, ctx->stream, x, ldx, dout, ldd, grad_low, low, R,
                           K, N, rows->row_of, rows->chunks, partial);
    };
    if (R <= 16) go(outer_kernel<T, 1>, 16);
    else go(outer_kernel<T, 2>, 32);
}

int check_apart(const char *call, const char *a, const void *a_dev, int64_t lda, int64_t a_cols, const char *b, const void *b_dev, int64_t ldb, int64_t b_cols,
                int64_t rows)
{
    if (!rows_overlap((uint64_t)a_dev, lda, a_cols, (uint64_t)b_dev, ldb, b_cols, rows, 2)) return LEANN_OK;
    leann_set_error("%s: %s overlaps %s", call, a, b);
    return LEANN_EINVAL;
}

int check_pair(const char *call, const leann_ctx *ctx, const leann_projection *proj, const leann_adapter_rows *rows)
{
    if (!ctx || !proj || !rows) {
        leann_set_error("%s: null context, projection or rows", call);
        return LEANN_EINVAL;
    }
    if (proj->device != ctx->device || rows->device != ctx->device) {
        leann_set_error("%s: the projection or the rows belong to another device", call);
        return LEANN_EINVAL;
    }
    return LEANN_OK;
}

// The tables of a batch: 27 us for 48 rows of 48 requests, 42 for 6560 of 96, 98 for 83 229 of 512, with the allocation and the copy.
int make_rows(leann_ctx *ctx, const int32_t *rows_of_request, const int32_t *adapter_of_request, int32_t n_requests, const int32_t *rank,
              const float *scale, int32_t n_adapters, int32_t max_rank, leann_adapter_rows *out)
{
    int64_t T = 0;
    std::vector<int64_t> start((size_t)n_requests + 1, 0);
    for (int i = 0; i < n_requests; ++i) start[i + 1] = T += rows_of_request[i];
    auto of = [&](int i) { return adapter_of_request[i] >= 0 && rank[adapter_of_request[i]] > 0 ? adapter_of_request[i] : n_adapters; };
    // requests by adapter (those without one, or with one of rank 0, last), in their order
    std::vector<int32_t> first(n_adapters + 2, 0), order(n_requests);
    for (int i = 0; i < n_requests; ++i) ++first[of(i) + 1];
    for (int a = 0; a <= n_adapters; ++a) first[a + 1] += first[a];
    {
        std::vector<int32_t> next(first.begin(), first.end() - 1);
        for (int i = 0; i < n_requests; ++i) order[next[of(i)]++] = i;
    }
    std::vector<int32_t> row_of;
    row_of.reserve(T + 256 + 8);
    std::vector<int64_t> slot_of(n_adapters + 2, 0);  // an adapter's first slot
    for (int a = 0; a <= n_adapters; ++a) {
        for (int j = first[a]; j < first[a + 1]; ++j)
            for (int64_t r = start[order[j]]; r < start[order[j] + 1]; ++r) row_of.push_back((int32_t)r);
        slot_of[a + 1] = (int64_t)row_of.size();
    }
    while (row_of.size() % 256) row_of.push_back(row_of[T - 1]);
    row_of.insert(row_of.end(), 8, 0);  // outer_kernel reads eight at a time

    const int64_t adapted = slot_of[n_adapters];
    // Rows of a chunk of outer_kernel: as many as leave one chunk for every third CU (times the blocks of 128 columns, twelve at 768 + 768), 64 at least, 2048 at most.
    // 82 953 rows 768 -> 768, ranks up to 32: 229 us for the whole gradient, with chunks half as long 239 (their sums are written and read again).
    const int chunk_rows = (int)std::min<int64_t>(2048, std::max<int64_t>(64, (adapted / std::max(1, ctx->num_cus / 3) + 63) / 64 * 64));
    std::vector<int4> tiles, wide, segs, adapters(n_adapters);
    std::vector<int2> runs, chunks;
    std::vector<int32_t> used, run_ptr((T + 31) / 32 + 1, 0), seg_ptr((T + 255) / 256 + 1, 0);
    auto bits = [](float f) {
        int32_t i;
        memcpy(&i, &f, sizeof(i));
        return i;
    };
    for (int a = 0; a <= n_adapters; ++a) {
        const int64_t from = slot_of[a], to = slot_of[a + 1];
        const int r = a < n_adapters ? rank[a] : 0, number = (int)used.size();
        if (a == n_adapters) {
            out->n_adapted_tiles = (int)tiles.size();
            out->n_adapted_wide_tiles = (int)wide.size();
        }
        for (int64_t s = from; s < to; s += WIDE_ROWS)
            wide.push_back(int4{a < n_adapters ? a : -1, (int)s, (int)std::min<int64_t>(WIDE_ROWS, to - s) | r << 16, number});
        for (int64_t s = from; s < to; s += 16) tiles.push_back(int4{a < n_adapters ? a : -1, (int)s, (int)std::min<int64_t>(16, to - s) | r << 16, number});
        if (a == n_adapters) break;
        adapters[a] = int4{(int)chunks.size(), 0, r, bits(scale[a])};
        for (int64_t s = from; s < to; s += chunk_rows) chunks.push_back(int2{(int)s, (int)std::min<int64_t>(chunk_rows, to - s) | r << 16});
        adapters[a].y = (int)chunks.size() - adapters[a].x;
        for (int64_t s = from; s < to;) {
            const int64_t group = s / 32, end = std::min<int64_t>(to, (group + 1) * 32);
            runs.push_back(int2{(int)s, (int)(end - s) | r << 8 | (int)((uint32_t)number << 16)});
            ++run_ptr[group + 1];
            s = end;
        }
        for (int64_t s = from; s < to;) {
            const int64_t tile = s / 256, end = std::min<int64_t>(to, (tile + 1) * 256);
            segs.push_back(int4{(int)s, (int)end, r, number});
            ++seg_ptr[tile + 1];
            s = end;
        }
        if (to > from) used.push_back(a);
    }
    for (size_t g = 1; g < seg_ptr.size(); ++g) {
        seg_ptr[g] += seg_ptr[g - 1];
        for (int pieces = 1; pieces <= 2; ++pieces) {
            int n = 0;
            for (int i = seg_ptr[g - 1]; i < seg_ptr[g]; ++i) n += segment_pairs(segs[i].z, pieces);
            AdapterLoad &l = out->load[pieces - 1];
            l.most_pairs = std::max(l.most_pairs, n);
            l.pairs += n;
        }
    }
    for (AdapterLoad &l : out->load)
        for (const int2 &run : runs) l.sixteens += rank_groups(run.y >> 8 & 255);
    for (size_t g = 1; g < run_ptr.size(); ++g) run_ptr[g] += run_ptr[g - 1];

    out->device = ctx->device;
    out->T = T;
    out->n_adapters = n_adapters;
    out->max_rank = max_rank;
    out->n_used = (int)used.size();
    out->n_tiles = (int)tiles.size();
    out->n_wide_tiles = (int)wide.size();
    out->n_chunks = (int)chunks.size();
    std::vector<char> image;
    auto put = [&](const auto &v) {
        const size_t at = up256(image.size()), bytes = v.size() * sizeof(v[0]);
        image.resize(at + bytes);
        if (bytes) memcpy(image.data() + at, v.data(), bytes);
        return at;
    };
    const size_t at[10] = {put(row_of), put(run_ptr), put(runs), put(tiles), put(chunks), put(adapters), put(used), put(seg_ptr), put(segs), put(wide)};
    LEANN_TRY(ctx->reserve(out->mem, std::max<size_t>(image.size(), 1)));
    LEANN_HIP(hipMemcpyAsync(out->mem.p, image.data(), image.size(), hipMemcpyHostToDevice, ctx->stream));
    LEANN_HIP(hipStreamSynchronize(ctx->stream));
    const char *base = (const char *)out->mem.p;
    out->row_of = (const int32_t *)(base + at[0]);
    out->run_ptr = (const int32_t *)(base + at[1]);
    out->runs = (const int2 *)(base + at[2]);
    out->tiles = (const int4 *)(base + at[3]);
    out->chunks = (const int2 *)(base + at[4]);
    out->adapters = (const int4 *)(base + at[5]);
    out->used = (const int32_t *)(base + at[6]);
    out->seg_ptr = (const int32_t *)(base + at[7]);
    out->segs = (const int4 *)(base + at[8]);
    out->wide_tiles = (const int4 *)(base + at[9]);
    return LEANN_OK;
}

}  // namespace

int adapter_init_device()
{
    LEANN_TRY(allow_lds(project_large_kernel<bf16_t, 2, 4, 2>, ProjectCfg<2, 4, 2>::SMEM));
    return allow_lds(project_large_kernel<f16_t, 2, 4, 2>, ProjectCfg<2, 4, 2>::SMEM);
}

extern "C" {

void leann_projection_free(leann_projection *p)
{
    if (!p) return;
    (void)hipSetDevice(p->device);
    for (DevBuf *b : {&p->w, &p->wt, &p->bias}) b->release();
    delete p;
}

void leann_adapter_rows_free(leann_adapter_rows *p)
{
    if (!p) return;
    (void)hipSetDevice(p->device);
    p->mem.release();
    delete p;
}

int leann_projection_create(leann_ctx *ctx, const void *w_dev, const float *bias_dev, int32_t n_out, int32_t n_in, int dtype, int with_gradient,
                            leann_projection **out)
{
    static const char *call = "leann_projection_create";
    if (!ctx || !w_dev || !out || n_out < 1 || n_in < 1 || (dtype != LEANN_BF16 && dtype != LEANN_F16)) {
        leann_set_error("%s: null argument, no rows or columns, or a type other than bf16 and f16", call);
        return LEANN_EINVAL;
    }
    if (n_out % 8 || n_in % 8 || n_out > 65536 || n_in > 65536) {
        leann_set_error("%s: %d x %d is not covered (multiples of 8, at most 65536)", call, n_out, n_in);
        return LEANN_ESHAPE;
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    leann_projection *p = new (std::nothrow) leann_projection();
    if (!p) {
        leann_set_error("%s: no host memory", call);
        return LEANN_ENOMEM;
    }
    p->device = ctx->device;
    p->dtype = dtype;
    p->n_out = n_out;
    p->n_in = n_in;
    auto packed = [&](int N, int K) { return (size_t)((N + 31) / 32) * project_ksteps(K) * 1024; };
    int rc = ctx->reserve(p->w, packed(n_out, n_in));
    if (rc == LEANN_OK && with_gradient) rc = ctx->reserve(p->wt, packed(n_in, n_out));
    if (rc == LEANN_OK && bias_dev) rc = ctx->reserve(p->bias, n_out * sizeof(float));
    if (rc == LEANN_OK)
        rc = with_half_type(dtype, [&](auto *type) {
            typedef std::remove_pointer_t<decltype(type)> T;
            hipLaunchKernelGGL(pack_kernel<T>, dim3(1024), dim3(256), 0, ctx->stream, (const T *)w_dev, n_out, n_in, 0, (T *)p->w.p);
            if (with_gradient) hipLaunchKernelGGL(pack_kernel<T>, dim3(1024), dim3(256), 0, ctx->stream, (const T *)w_dev, n_in, n_out, 1, (T *)p->wt.p);
            return launched(call);
        });
    if (rc == LEANN_OK && bias_dev) {
        const hipError_t e = hipMemcpyAsync(p->bias.p, bias_dev, n_out * sizeof(float), hipMemcpyDeviceToDevice, ctx->stream);
        if (e != hipSuccess) {
            leann_set_error("%s: copying the bias failed: %s", call, hipGetErrorString(e));
            rc = LEANN_EDEVICE;
        }
    }
    if (rc == LEANN_OK) {
        const hipError_t e = hipStreamSynchronize(ctx->stream);  // the caller may free the weight
        if (e != hipSuccess) {
            leann_set_error("%s: %s", call, hipGetErrorString(e));
            rc = LEANN_EDEVICE;
        }
    }
    if (rc != LEANN_OK) {
        leann_projection_free(p);
        return rc;
    }
    *out = p;
    return LEANN_OK;
}

int leann_adapter_rows_create(leann_ctx *ctx, const int32_t *rows_of_request_host, const int32_t *adapter_of_request_host, int32_t n_requests,
                              const int32_t *rank_host, const float *scale_host, int32_t n_adapters, int32_t max_rank, leann_adapter_rows **out)
{
    static const char *call = "leann_adapter_rows_create";
    if (!ctx || !out || n_requests < 0 || n_adapters < 1 || !rank_host || !scale_host ||
        (n_requests > 0 && (!rows_of_request_host || !adapter_of_request_host))) {
        leann_set_error("%s: null argument, negative request count or no adapters", call);
        return LEANN_EINVAL;
    }
    if (max_rank < 8 || max_rank > 128 || max_rank % 8) {
        leann_set_error("%s: room for %d ranks is not covered (a multiple of 8, at most 128)", call, max_rank);
        return LEANN_ESHAPE;
    }
    int64_t T = 0;
    for (int i = 0; i < n_requests; ++i) {
        if (rows_of_request_host[i] < 0 || adapter_of_request_host[i] < -1 || adapter_of_request_host[i] >= n_adapters) {
            leann_set_error("%s: request %d has a negative row count or an adapter outside [-1, %d)", call, i, n_adapters);
            return LEANN_EINVAL;
        }
        T += rows_of_request_host[i];
    }
    for (int a = 0; a < n_adapters; ++a)
        if (rank_host[a] < 0 || rank_host[a] > max_rank || !std::isfinite(scale_host[a])) {
            leann_set_error("%s: adapter %d has a rank outside [0, %d] or a scale that is not finite", call, a, max_rank);
            return LEANN_EINVAL;
        }
    if (T > 0x7fffffffll - 256) {
        leann_set_error("%s: %lld rows are not covered (below 2^31 - 256)", call, (long long)T);
        return LEANN_ESHAPE;
    }
    if (n_adapters > 65535) {
        leann_set_error("%s: %d adapters are not covered (at most 65535)", call, n_adapters);
        return LEANN_ESHAPE;
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    leann_adapter_rows *p = nullptr;
    int rc;
    try {
        p = new leann_adapter_rows();
        rc = make_rows(ctx, rows_of_request_host, adapter_of_request_host, n_requests, rank_host, scale_host, n_adapters, max_rank, p);
    } catch (const std::exception &) {
        leann_set_error("%s: no host memory", call);
        rc = LEANN_ENOMEM;
    }
    if (rc != LEANN_OK) {
        leann_adapter_rows_free(p);
        return rc;
    }
    *out = p;
    return LEANN_OK;
}

int leann_adapter_project(leann_ctx *ctx, const leann_projection *proj, const leann_adapter_rows *rows, const void *x_dev, int64_t ldx,
                          const void *down_dev, const void *up_dev, void *out_dev, int64_t ldo, float *low_dev)
{
    static const char *call = "leann_adapter_project";
    LEANN_TRY(check_pair(call, ctx, proj, rows));
    if (rows->T == 0) return LEANN_OK;
    LEANN_TRY(check_half_rows(call, "x", x_dev, ldx, proj->n_in));
    LEANN_TRY(check_half_rows(call, "out", out_dev, ldo, proj->n_out));
    if (!down_dev || !up_dev || !aligned16(down_dev) || !aligned16(up_dev) || !aligned16(low_dev)) {
        leann_set_error("%s: the adapters' matrices are null, or they or low are not aligned to 16 bytes", call);
        return LEANN_EINVAL;
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    const int N = proj->n_out, K = proj->n_in;
    LEANN_TRY(check_launches(call, {plan_low(ctx, rows, low_dev != nullptr, N).blocks, plan_project(ctx, rows, proj->dtype, ldx, N, K).blocks}));
    LEANN_TRY(check_apart(call, "out", out_dev, ldo, N, "x", x_dev, ldx, K, rows->T));
    std::lock_guard<std::mutex> turn(ctx->op_work_mutex);
    LEANN_TRY(ctx->reserve(ctx->op_work, pieces_bytes(rows) + packed_bytes(rows, N)));
    bf16_t *pieces = (bf16_t *)ctx->op_work.p, *packed = (bf16_t *)((char *)ctx->op_work.p + pieces_bytes(rows));
    return with_half_type(proj->dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        enqueue_low<T>(ctx, rows, (const T *)x_dev, ldx, K, (const T *)down_dev, 0, low_dev, low_dev != nullptr, pieces, (const T *)up_dev, N, packed);
        enqueue_project<T>(ctx, rows, (const T *)x_dev, ldx, (const T *)proj->w.p, (const float *)proj->bias.p, N, K, pieces, packed, (T *)out_dev, ldo);
        return launched(call);
    });
}

int leann_adapter_project_backward(leann_ctx *ctx, const leann_projection *proj, const leann_adapter_rows *rows, const void *dout_dev, int64_t ldd,
                                   const void *x_dev, int64_t ldx, const float *low_dev, const void *down_dev, const void *up_dev, void *dx_dev,
                                   int64_t lddx, float *ddown_dev, float *dup_dev)
{
    static const char *call = "leann_adapter_project_backward";
    LEANN_TRY(check_pair(call, ctx, proj, rows));
    if ((rows->T > 0 && !dx_dev && !ddown_dev) || !ddown_dev != !dup_dev) {
        leann_set_error("%s: no output, or only one of ddown and dup", call);
        return LEANN_EINVAL;
    }
    if (dx_dev && !proj->wt.p) {
        leann_set_error("%s: the projection was created without gradient", call);
        return LEANN_EINVAL;
    }
    const int N = proj->n_out, K = proj->n_in, R = rows->max_rank;
    if (rows->T > 0) {
        LEANN_TRY(check_half_rows(call, "dout", dout_dev, ldd, N));
        if (dx_dev) LEANN_TRY(check_half_rows(call, "dx", dx_dev, lddx, K));
        if (ddown_dev) LEANN_TRY(check_half_rows(call, "x", x_dev, ldx, K));
        if (!down_dev || !up_dev || (ddown_dev && !low_dev) || !aligned16(down_dev) || !aligned16(up_dev) || !aligned16(low_dev)) {
            leann_set_error("%s: the adapters' matrices or low are null or not aligned to 16 bytes", call);
            return LEANN_EINVAL;
        }
    }
    const int64_t transposing = (int64_t)rows->n_used * ((N + 31) / 32) * ((R + 31) / 32);
    const int64_t laying = dx_dev ? ((int64_t)rows->n_used * ((K + 31) / 32) * rank_groups(R) * 64 + 255) / 256 : 0;
    const int64_t lay_out_blocks = transposing + std::min<int64_t>(laying, ctx->num_cus * 4);
    const int64_t outer_blocks = ddown_dev ? (int64_t)rows->n_chunks * ((K + 127) / 128 + (N + 127) / 128) : 0;
    LEANN_TRY(check_launches(call, {lay_out_blocks, plan_low(ctx, rows, false, 0).blocks, dx_dev && rows->T ? plan_project(ctx, rows, proj->dtype, ldd, K, N).blocks : 0,
                                    outer_blocks}));
    if (dx_dev) LEANN_TRY(check_apart(call, "dx", dx_dev, lddx, K, "dout", dout_dev, ldd, N, rows->T));
    if (dx_dev && ddown_dev) LEANN_TRY(check_apart(call, "dx", dx_dev, lddx, K, "x", x_dev, ldx, K, rows->T));
    LEANN_HIP(hipSetDevice(ctx->device));
    const size_t low_bytes = up256((size_t)rows->T * R * sizeof(float)), up_bytes = up256((size_t)rows->n_used * R * N * 2),
                 partial_bytes = ddown_dev ? (size_t)rows->n_chunks * R * (K + N) * sizeof(float) : 0;
    std::lock_guard<std::mutex> turn(ctx->op_work_mutex);
    LEANN_TRY(ctx->reserve(ctx->op_work,
                           std::max<size_t>(1, pieces_bytes(rows) + packed_bytes(rows, K) + low_bytes + up_bytes + partial_bytes)));
    char *work = (char *)ctx->op_work.p;
    auto take = [&](size_t bytes) {
        char *p = work;
        work += bytes;
        return p;
    };
    bf16_t *pieces = (bf16_t *)take(pieces_bytes(rows)), *packed = (bf16_t *)take(packed_bytes(rows, K));
    float *grad_low = (float *)take(low_bytes);
    char *up_at = take(up_bytes);
    float *partial = (float *)take(partial_bytes);
    return with_half_type(proj->dtype, [&](auto *type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        T *up_t = (T *)up_at;
        if (rows->n_used) {
            hipLaunchKernelGGL(lay_out_kernel<T>, dim3((unsigned)lay_out_blocks), dim3(256), 0, ctx->stream, (const T *)down_dev, (const T *)up_dev, rows->used,
                               rows->adapters, rows->n_used, R, K, N, up_t, packed, (int)transposing);
            enqueue_low<T>(ctx, rows, (const T *)dout_dev, ldd, N, up_t, 1, ddown_dev ? grad_low : nullptr, false, pieces, (const T *)nullptr, 0,
                           (bf16_t *)nullptr);
        }
        if (dx_dev && rows->T)
            enqueue_project<T>(ctx, rows, (const T *)dout_dev, ldd, (const T *)proj->wt.p, nullptr, K, N, pieces, packed, (T *)dx_dev, lddx);
        if (ddown_dev) {
            if (rows->n_chunks)
                enqueue_outer<T>(ctx, rows, (const T *)x_dev, ldx, (const T *)dout_dev, ldd, grad_low, low_dev, K, N, partial);
            hipLaunchKernelGGL(outer_sum_kernel, dim3((K + N + 31) / 32, (R + 31) / 32, rows->n_adapters), dim3(1024), 0, ctx->stream, partial,
                               rows->adapters, R, K, N, ddown_dev, dup_dev);
        }
        return launched(call);
    });
}

}  // extern "C"
