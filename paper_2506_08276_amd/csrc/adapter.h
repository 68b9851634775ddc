// What the kernels of projections with low-rank adapters share: handles, tables, MFMA operands (gfx950).
#pragma once
#include "adapter_plan.h"
#include "rows.h"

// The shared projection, as the kernels read it: W and, for gradients, its transpose in the MFMA's operand order.
struct leann_projection {
    int device = 0, dtype = 0;
    int32_t n_out = 0, n_in = 0;
    DevBuf w, wt, bias;
};

constexpr int WIDE_ROWS = 32;

// Which rows of a batch go through which adapter.  Rows are put in an order, their slots, in which an adapter's rows are adjacent (those without one
// last), so that a tile of rows meets few adapters.  All tables lie in one allocation.
struct leann_adapter_rows {
    int device = 0;
    int64_t T = 0;
    int32_t n_adapters = 0, max_rank = 0, n_used = 0;
    int32_t n_tiles = 0, n_adapted_tiles = 0;  // of 16 slots of one adapter; tiles of rows without one come last
    int32_t n_wide_tiles = 0, n_adapted_wide_tiles = 0;  // likewise, of 32
    int32_t n_chunks = 0;                      // of up to chunk_rows slots of one adapter
    AdapterLoad load[2];                       // by the pieces of an element of `up`, less one
    DevBuf mem;
    const int32_t *row_of = nullptr;     // [T, up to a multiple of 256: the last row again, 8 more]
    const int32_t *run_ptr = nullptr;    // [32-slot groups + 1]
    const int2 *runs = nullptr;          // first slot, slots | rank << 8 | number among the used adapters << 16
    const int32_t *seg_ptr = nullptr;    // [256-slot tiles + 1]
    const int4 *segs = nullptr;          // a tile's adapters: first slot, slot behind the last, rank, number among the used adapters
    const int4 *tiles = nullptr;         // adapter, first slot, slots | rank << 16, number among the used adapters
    const int4 *wide_tiles = nullptr;    // likewise
    const int2 *chunks = nullptr;        // by adapter: first slot, slots | rank << 16
    const int4 *adapters = nullptr;      // [n_adapters] first chunk, chunks, rank, scale
    const int32_t *used = nullptr;       // [n_used] adapters that have rows
};

namespace {

// Steps of 16 of K in a packed weight: whole numbers of four slabs of 32, zeros beyond K.
__host__ __device__ inline int project_ksteps(int K) { return (K + 127) / 128 * 8; }

__device__ u32x4 zero_piece;  // zeros, read instead of what rows hold beyond K (not a constant: the compiler would make a branch of the choice, and a wait)

template <class T>
struct Frag;
template <>
struct Frag<bf16_t> {
    typedef bf16x8 type;
    typedef bf16x4 four;
    static constexpr int PIECES = 1;  // bf16 numbers that hold one exactly
};
template <>
struct Frag<f16_t> {
    typedef f16x8 type;
    typedef f16x4 four;
    static constexpr int PIECES = 2;
};

__device__ inline f32x16 mfma32(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma32(const f16x8 &a, const f16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(const f16x8 &a, const f16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// A number as a sum of bf16 pieces of 8 bits each, cut off, not rounded: all have the number's sign and none is zero unless the number is (where nothing is left, 2^-126 stands
// for it), so that an infinity on either side of a product is the definition's infinity, where a piece of zero or of the other sign would make NaN of it.  An infinity is
// its first piece, NaN stays NaN.  Two pieces hold 16 bits of a value (11 of fp16's), three all 24.  (Numbers below 2^-126 may be lost.)
constexpr float LEAST_PIECE = 0x1p-126f;
__device__ inline float first_piece(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ inline float behind_first(float v)  // max takes the number where the difference of infinities is none
{
    return __builtin_copysignf(__builtin_fmaxf(__builtin_fabsf(v - first_piece(v)), __builtin_fminf(__builtin_fabsf(v), LEAST_PIECE)), v);
}

// The first pieces of eight values; v becomes what is behind them.
__device__ inline bf16x8 take_piece(f32x8 &v)
{
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = behind_first(v[i]);
    return __builtin_bit_cast(bf16x8, p);
}

// Low-rank activations go into the matrix instructions as two pieces of 8 bits, 16 ranks of a row as 32 numbers, first pieces first: [slot][ranks / 16][32],
// times the adapter's scale.  On bf16 MFMAs for both types: they are sums in fp32 and may leave fp16's range.  What is left out is 2^-16 of each term, where the
// output's own rounding is 2^-9 or 2^-12.  `up` is laid out anew in each call, as its values change from step to step in training: in operand order
// [used adapter][columns / 32][ranks / 16][piece][lane][8], zeros beyond rank and columns; fp16 numbers are two pieces exactly.
__host__ __device__ inline int rank_groups(int R) { return (R + 15) >> 4; }

// The adapters' part of one 32-slot group's tiles: acc[ni] += up[columns of tile ni] pieces[slots]^T for every run of the group that is number `first`,
// `first + step`, ...  A lane holds one slot of the output, so a run that is not the whole group changes only the lanes that are its own: another request's
// infinities stay with it.  Lane l holds run l of the group's `count`; with an adapter per row, what bounds it is the runs' latency, so B of them have
// their first 16 ranks on the way together.
template <int TN, int UP>
__device__ inline void add_adapters(f32x16 (&acc)[TN], const int2 &my_run, int count, int group, int first, int step, const bf16_t *pieces,
                                    const bf16_t *up, int R16, int column_tiles, int column_tile)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    constexpr int B = TN * UP == 1 ? 4 : 2;
    if (first >= count) return;
    auto piece = [&](int k, int which) { return *reinterpret_cast<const bf16x8 *>(pieces + k * 32 + which * 16 + half * 8); };
    const bf16x8 h1 = piece(0, 0), h2 = piece(0, 1);
    size_t at[TN];  // of the lane's piece of a column tile; behind the last one: the last one's, for nothing
#pragma unroll
    for (int ni = 0; ni < TN; ++ni) at[ni] = (size_t)min(column_tile + ni, column_tiles - 1) * R16 * UP * 512 + lane * 8;
    for (int i = first; i < count; i += B * step) {
        bf16x8 f[B][TN][UP];
        int z[B], slot[B];
#pragma unroll
        for (int r = 0; r < B; ++r) {
            const int from = min(i + r * step, count - 1);
            slot[r] = __builtin_amdgcn_readlane(my_run.x, from) - group * 32;
            z[r] = __builtin_amdgcn_readlane(my_run.y, from);
            const bf16_t *u = up + (size_t)((uint32_t)z[r] >> 16) * column_tiles * R16 * UP * 512;
#pragma unroll
            for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                for (int e = 0; e < UP; ++e) f[r][ni][e] = *reinterpret_cast<const bf16x8 *>(u + at[ni] + e * 512);
        }
#pragma unroll
        for (int r = 0; r < B; ++r) {
            if (i + r * step >= count) break;
            const int steps = rank_groups(z[r] >> 8 & 255);
            const bool own = l32 >= slot[r] && l32 < slot[r] + (z[r] & 255);
            const bf16_t *u = up + (size_t)((uint32_t)z[r] >> 16) * column_tiles * R16 * UP * 512;
            f32x16 sum[TN];
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) {
                sum[ni] = acc[ni];
#pragma unroll
                for (int e = 0; e < UP; ++e) {
                    sum[ni] = mfma32(f[r][ni][e], h2, sum[ni]);
                    sum[ni] = mfma32(f[r][ni][e], h1, sum[ni]);
                }
            }
            for (int k = 1; k < steps; ++k) {
                const bf16x8 k1 = piece(k, 0), k2 = piece(k, 1);
#pragma unroll
                for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                    for (int e = 0; e < UP; ++e) {
                        const bf16x8 g = *reinterpret_cast<const bf16x8 *>(u + at[ni] + (k * UP + e) * 512);
                        sum[ni] = mfma32(g, k2, sum[ni]);
                        sum[ni] = mfma32(g, k1, sum[ni]);
                    }
            }
#pragma unroll
            for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[ni][j] = own ? sum[ni][j] : acc[ni][j];
        }
    }
}

}  // namespace
