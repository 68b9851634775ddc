// What the kernels of projections with low-rank adapters share: handles, tables, MFMA operands (gfx950).
#pragma once
#include "rows.h"

// The shared projection, as the kernels read it: W and, for gradients, its transpose in the MFMA's operand order.
struct leann_projection {
    int device = 0, dtype = 0;
    int32_t n_out = 0, n_in = 0;
    DevBuf w, wt, bias;
};

// Which rows of a batch go through which adapter.  Rows are put in an order, their slots, in which an adapter's rows are adjacent (those without one
// last), so that a tile of rows meets few adapters.  All tables lie in one allocation.
struct leann_adapter_rows {
    int device = 0;
    int64_t T = 0;
    int32_t n_adapters = 0, max_rank = 0, n_used = 0;
    int32_t n_tiles = 0, n_adapted_tiles = 0;  // of 16 slots of one adapter; tiles of rows without one come last
    int32_t n_chunks = 0;                      // of up to chunk_rows slots of one adapter
    DevBuf mem;
    const int32_t *row_of = nullptr;     // [T, up to a multiple of 256: the last row again]
    const int32_t *run_ptr = nullptr;    // [32-slot groups + 1]
    const int4 *runs = nullptr;          // adapter, first slot, slots | rank << 8 | number among the used adapters << 16, scale
    const int4 *tiles = nullptr;         // adapter, first slot, slots | rank << 16, number among the used adapters
    const int4 *chunks = nullptr;        // likewise, by adapter
    const int4 *adapters = nullptr;      // [n_adapters] first chunk, chunks, rank, scale
    const int32_t *used = nullptr;       // [n_used] adapters that have rows
};

namespace {

// Steps of 16 of K in a packed weight: whole numbers of four slabs of 32, zeros beyond K.
__host__ __device__ inline int project_ksteps(int K) { return (K + 127) / 128 * 8; }

template <class T>
struct Frag;
template <>
struct Frag<bf16_t> {
    typedef bf16x8 type;
    typedef bf16x4 four;
};
template <>
struct Frag<f16_t> {
    typedef f16x8 type;
    typedef f16x4 four;
};

__device__ inline f32x16 mfma32(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma32(const f16x8 &a, const f16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(const f16x8 &a, const f16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The next 8 bits of eight values: what is left of v is exact.  Two pieces hold 16 bits of a value, three all 24.
__device__ inline bf16x8 take_piece(f32x8 &v)
{
    const bf16x8 p = __builtin_convertvector(v, bf16x8);
    v -= __builtin_convertvector(p, f32x8);
    return p;
}

// One step of 16 ranks of an adapter's part, acc += up low^T, on bf16 MFMAs for both types: the low-rank activations are fp32 and may leave
// fp16's range.  They go in as two pieces of 8 bits (2^-17 of each term, where the output's own rounding is 2^-8 or 2^-11); fp16 weights are
// two pieces exactly, of whose four products the smallest is left out.
__device__ inline f32x16 adapter_step(const bf16x8 &up, const bf16x8 &h1, const bf16x8 &h2, f32x16 c)
{
    c = mfma32(up, h2, c);
    return mfma32(up, h1, c);
}
__device__ inline f32x16 adapter_step(const f16x8 &up, const bf16x8 &h1, const bf16x8 &h2, f32x16 c)
{
    f32x8 u = __builtin_convertvector(up, f32x8);
    const bf16x8 u1 = take_piece(u), u2 = take_piece(u);
    c = mfma32(u1, h2, c);
    c = mfma32(u2, h1, c);
    return mfma32(u1, h1, c);
}

// The adapters' part of one 32-slot group's tiles: acc[ni] += scale * up[columns of tile ni] low[slots]^T for every run of the group that is
// number `first`, `first + step`, ...  A lane holds one slot of the output, so a run that is not the whole group changes only the lanes that are its own:
// another request's infinities stay with it.
template <class T, int TN>
__device__ inline void add_adapters(f32x16 (&acc)[TN], const int32_t *run_ptr, const int4 *runs, int group, int first, int step, const float *low_row,
                                    const T *up, int R, int N, int col, bool compact)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, l32 = lane & 31;
    const int begin = run_ptr[group], count = run_ptr[group + 1] - begin;
    for (int i = first; i < count; i += step) {
        const int4 run = runs[begin + i];
        const int rank = run.z >> 8 & 255, from = run.y - group * 32, to = from + (run.z & 255);
        const float scale = __int_as_float(run.w);
        const bool own = l32 >= from && l32 < to;
        const T *u = up + (size_t)(compact ? (uint32_t)run.z >> 16 : (uint32_t)run.x) * N * R;
        f32x16 sum[TN];
#pragma unroll
        for (int ni = 0; ni < TN; ++ni) sum[ni] = acc[ni];
        for (int k = 0; k < rank; k += 16) {
            const int at = k + half * 8, n = rank - at;  // n: of this lane's eight ranks those that exist
            f32x8 h = {};
            if (n > 0) __builtin_memcpy(&h, low_row + at, sizeof(h));  // zeros beyond the rank
            h *= scale;
            const bf16x8 h1 = take_piece(h), h2 = take_piece(h);
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) {
                typename Frag<T>::type f = {};
                if (n > 0) {
                    f = *reinterpret_cast<const typename Frag<T>::type *>(u + (size_t)min(col + ni * 32 + l32, N - 1) * R + at);
#pragma unroll
                    for (int j = 1; j < 8; ++j) f[j] = j < n ? f[j] : (T)0.f;  // what lies beyond the rank may be anything
                }
                sum[ni] = adapter_step(f, h1, h2, sum[ni]);
            }
        }
#pragma unroll
        for (int ni = 0; ni < TN; ++ni)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[ni][j] = own ? sum[ni][j] : acc[ni][j];
    }
}

}  // namespace
