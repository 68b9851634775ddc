// What the kernels of attention and of its gradient share: the plan, tiles in LDS, MFMA operands, masks and the bias (gfx950).
#pragma once
#include "attention_plan.h"
#include "rows.h"

constexpr int ATT_MOST_DISTANCE = 1024;
constexpr float ATT_LEAST_SCALE = 0x1p-20f, ATT_MOST_SCALE = 0x1p20f;
constexpr int64_t ATT_MOST_LD = (int64_t)1 << 22;  // 256 rows are within a buffer's 2^31 bytes
constexpr int ATT_LDS = 160 * 1024;                  // of a compute unit
constexpr int ATT_WHOLE = 256;                      // keys and queries that one block's gradient kernel takes
constexpr int ATT_EXT = 104;  // a wavefront's 32 rows and 64 of the other side have relative positions in a range of 95; sums of theirs touch nine places more

// What the two gradient kernels go through.
struct AttentionSides {
    int32_t n_tiles = 0, n_query_items = 0, n_key_items = 0, n_joins = 0, n_slots = 0;  // tiles: of queries
    int32_t key_waves = 4;  // wavefronts of 32 keys of their own in a block for keys: 4 or 2
    const AttentionTile *query_tiles = nullptr, *key_tiles = nullptr;
    const AttentionItem *query_items = nullptr, *key_items = nullptr;
    const AttentionJoin *joins = nullptr;
};
// Sequences that one block takes whole, as tiles of all their keys.
struct AttentionWhole {
    int32_t n_tiles = 0, n_items = 0;
    const AttentionTile *tiles = nullptr;
    const AttentionItem *items = nullptr;
};

// One batch's sequences: tables on the device, in one allocation.
struct leann_attention_plan {
    int device = 0;
    int32_t heads = 0, kv_heads = 0, dim = 0;
    int64_t Tq = 0, Tk = 0;
    int32_t left = -1, right = -1, sinks = 0;  // as the kernels take them: no limit is a bound behind every position
    int32_t distance = 0, buckets = 0;         // distance: of the table below, no longer than the sequences make it
    int32_t query_waves = 0;                   // wavefronts of a forward block, 32 queries each
    int32_t n_items = 0, n_joins = 0, n_slots = 0;
    int32_t join_rows = 0;                     // of a join, the most
    DevBuf mem;
    const AttentionTile *tiles = nullptr;
    const AttentionItem *items = nullptr;
    const AttentionJoin *joins = nullptr;
    AttentionSides all, others;  // every sequence, and those that are not in:
    AttentionWhole whole[2];     // up to 128 keys and queries, up to 256
    const int32_t *bucket_of = nullptr;  // [2 distance + 1]
};

// A matrix of a call, for its checks.
struct AttentionMatrix {
    const char *name;
    const void *p;
    int64_t ld, cols, rows;
};

int att_launched(const char *call);
int att_check_call(const char *call, const leann_ctx *ctx, const leann_attention_plan *plan, int dtype, float scale, const float *bias_dev);
int att_check_rows(const char *call, const char *what, const void *p, int64_t ld, int64_t cols);
int att_check_apart(const char *call, const AttentionMatrix &a, const AttentionMatrix &b);

// What a kernel needs of a plan besides tables.
struct AttentionShape {
    int32_t heads, share;  // heads, and how many of them share a key head
    int32_t dim;
    int32_t left, right, sinks, distance;
    float scale;
};
AttentionShape att_shape(const leann_attention_plan *p, float scale);

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

template <class T>
struct Half8;
template <>
struct Half8<bf16_t> {
    typedef bf16x8 type;
    static constexpr uint32_t EXPONENT = 0x7f80;
};
template <>
struct Half8<f16_t> {
    typedef f16x8 type;
    static constexpr uint32_t EXPONENT = 0x7c00;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

__device__ inline f32x16 att_mfma(const bf16x8 &a, const bf16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 att_mfma(const f16x8 &a, const f16x8 &b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ inline f32x4 att_mfma16(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Tiles of 64 rows of DP elements (the head's size, zeros up to 32, 64 or 128) lie in LDS as rows of 16-byte chunks, chunk c of row r at c ^ att_swizzle(r): 16 rows' reads
// of one chunk, and the reads of four adjacent rows' 64 bytes that transpose, reach all banks.
template <int DP>
__device__ inline int att_swizzle(int row)
{
    if constexpr (DP == 32) return (row >> 2) & 3;
    else if constexpr (DP == 64) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
    else return (row & 3) << 2 | ((row >> 2) & 3);
}

typedef __attribute__((address_space(3))) void lds_t;
__device__ inline void lds_request(__amdgpu_buffer_rsrc_t b, uint32_t offset, void *to)  // 16 bytes per lane, to `to` and on in the lanes' order
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lds_t *)to, 16, (int)offset, 0, 0, 0);
}

// Requests for a tile, from memory to LDS without registers: 1 KB each, one of NW wavefronts' share of them.  A lane fetches the chunk that belongs at its place.  Rows behind the
// sequence's last and columns behind the head's are out of the buffer's bounds and come as zeros.
template <class T, int DP, int NW>
struct TileRequests {
    static constexpr int CPR = DP / 8, RPI = 64 / CPR, N = ATT_STEP / RPI / NW;
    uint32_t at[N];  // byte offsets in the tile

    __device__ inline void init(int64_t ld, int dim, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = (i * NW + wave) * RPI + lane / CPR, ch = (lane % CPR) ^ att_swizzle<DP>(row);
            at[i] = ch * 8 < dim ? (uint32_t)(row * ld + ch * 8) * 2 : 0x80000000u;
        }
    }
    // 64 rows from `base` on, of which `rows` are the sequence's; all arguments are the same in every lane
    __device__ inline void request(const T *base, int64_t ld, int rows, int dim, T *lds, int wave) const
    {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(base), 0, (int)(((min(rows, ATT_STEP) - 1) * ld + dim) * 2), 0x00020000);
#pragma unroll
        for (int i = 0; i < N; ++i) lds_request(rsrc, at[i], lds + (i * NW + wave) * 512);
    }
};

// Waits until no more than VM of the wavefront's memory requests are on their way, and for its LDS accesses; then for the other wavefronts.  Nothing is moved across.
template <int VM>
__device__ inline void wait_for_requests()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | 0x70);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ inline void block_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Infinities and NaN of an operand.  Where a tile is partly hidden they have to be taken out: a row of the other side that does not see them would get NaN from a product with
// zero.
template <class T>
struct Finite {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
    __device__ inline void look(const typename Half8<T>::type &f)
    {
        const u32x4 v = __builtin_bit_cast(u32x4, f);
#pragma unroll
        for (int w = 0; w < 4; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[w] & 0x7fff7fffu));
    }
    __device__ inline bool all() const { return !__ballot((most[0] >= Half8<T>::EXPONENT) | (most[1] >= Half8<T>::EXPONENT)); }  // in every lane
    __device__ static inline void keep(typename Half8<T>::type &f)
    {
        u32x4 v = __builtin_bit_cast(u32x4, f);
        constexpr uint32_t E = Half8<T>::EXPONENT;
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] &= ((v[w] & E) == E ? 0u : 0xffffu) | ((v[w] & E << 16) == E << 16 ? 0u : 0xffff0000u);
        f = __builtin_bit_cast(typename Half8<T>::type, v);
    }
};

// Operand A (or B) of a 32x32x16 product: rows row0 + lane % 32 of a tile, elements 16 step + 8 (lane / 32) and on.
template <class T, int DP>
__device__ inline typename Half8<T>::type row_operand(const T *lds, int row0, int step, int lane)
{
    const int row = row0 + (lane & 31), ch = step * 2 + (lane >> 5);
    return *reinterpret_cast<const typename Half8<T>::type *>(lds + row * DP + ((ch ^ att_swizzle<DP>(row)) << 3));
}

// Operand A of the transposed tile: lane l holds column col0 + l % 32 and, in slots 0..3 and 4..7, the rows row0 + 4 (l / 32) + {0..3} and 8 more: exactly the rows that
// accumulator registers 8u .. 8u + 7 of a 32x32 product hold (row0 = 16 u), so that those are the other operand as they are.  16 lanes read four rows of 16 elements and
// get a column of four each.
// The reads are written out, each group with its wait behind it: before the builtin's, the compiler waits for every request from memory to LDS that is on its way, the tiles ahead
// among them (LDS arrays and requests look alike to it).
template <int FROM>
__device__ inline void transposed4(const uint32_t (&a)[4], s16x4 (&o)[4])
{
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%8\n\t"
                 "ds_read_b64_tr_b16 %2, %6 offset:%8\n\tds_read_b64_tr_b16 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(FROM));
}
template <int FROM>
__device__ inline void transposed8(const uint32_t (&a)[8], s16x4 (&o)[8])
{
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%16\n\tds_read_b64_tr_b16 %1, %9 offset:%16\n\tds_read_b64_tr_b16 %2, %10 offset:%16\n\t"
                 "ds_read_b64_tr_b16 %3, %11 offset:%16\n\tds_read_b64_tr_b16 %4, %12 offset:%16\n\tds_read_b64_tr_b16 %5, %13 offset:%16\n\t"
                 "ds_read_b64_tr_b16 %6, %14 offset:%16\n\tds_read_b64_tr_b16 %7, %15 offset:%16\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "n"(FROM));
}
template <int FROM, int NEXT>
__device__ inline void transposed4_twice(const uint32_t (&a)[4], s16x4 (&o)[8])
{
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %9 offset:%12\n\tds_read_b64_tr_b16 %2, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %3, %11 offset:%12\n\tds_read_b64_tr_b16 %4, %8 offset:%13\n\tds_read_b64_tr_b16 %5, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %10 offset:%13\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(FROM), "n"(NEXT));
}

template <class T, int DP>
struct Columns {
    typedef typename Half8<T>::type V8;
    static constexpr int ND = DP / 32, GROUP = 16 * DP * 2;  // bytes of 16 rows
    uint32_t at[2 * ND];                                     // of rows 0 and 8 of each 32 columns

    __device__ inline void init(int lane)
    {
#pragma unroll
        for (int i = 0; i < 2 * ND; ++i) {
            const int row = 4 * (lane >> 5) + ((lane & 15) >> 2) + 8 * (i & 1), col = (i >> 1) * 32 + (lane & 16) + 4 * (lane & 3);
            at[i] = (row * DP + (((col >> 3) ^ att_swizzle<DP>(row)) << 3) + (col & 7)) * 2;
        }
    }
    __device__ static inline V8 join(const s16x4 &a, const s16x4 &b) { return __builtin_bit_cast(V8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)); }
    __device__ static inline uint32_t place(const T *lds) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const T *)lds; }

    // two groups, rows ROW .. ROW + 15 and the next 16
    template <int ROW>
    __device__ inline void two(const T *tile, V8 (&f)[2][ND]) const
    {
        constexpr int FROM = ROW / 16 * GROUP;
        const uint32_t base = place(tile);
        if constexpr (ND == 1) {
            const uint32_t a[4] = {base + at[0], base + at[1], base + at[0] + GROUP, base + at[1] + GROUP};
            s16x4 o[4];
            transposed4<FROM>(a, o);
            f[0][0] = join(o[0], o[1]);
            f[1][0] = join(o[2], o[3]);
        } else if constexpr (ND == 2) {
            const uint32_t a[4] = {base + at[0], base + at[1], base + at[2], base + at[3]};
            s16x4 o[8];
            transposed4_twice<FROM, FROM + GROUP>(a, o);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i >> 1][i & 1] = join(o[2 * i], o[2 * i + 1]);
        } else {
            uint32_t a[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = base + at[i];
            s16x4 o[8];
            transposed8<FROM>(a, o);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[0][i] = join(o[2 * i], o[2 * i + 1]);
            transposed8<FROM + GROUP>(a, o);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[1][i] = join(o[2 * i], o[2 * i + 1]);
        }
    }
    // one group of two tiles, rows ROW .. ROW + 15
    template <int ROW>
    __device__ inline void both(const T *one, const T *other, V8 (&f)[ND], V8 (&g)[ND]) const
    {
        constexpr int FROM = ROW / 16 * GROUP;
        const uint32_t b = place(one), c = place(other);
        if constexpr (ND == 1) {
            const uint32_t a[4] = {b + at[0], b + at[1], c + at[0], c + at[1]};
            s16x4 o[4];
            transposed4<FROM>(a, o);
            f[0] = join(o[0], o[1]);
            g[0] = join(o[2], o[3]);
        } else {
#pragma unroll
            for (int d = 0; d < ND; d += 2) {
                const uint32_t a[8] = {b + at[2 * d], b + at[2 * d + 1], b + at[2 * d + 2], b + at[2 * d + 3],
                                       c + at[2 * d], c + at[2 * d + 1], c + at[2 * d + 2], c + at[2 * d + 3]};
                s16x4 o[8];
                transposed8<FROM>(a, o);
                f[d] = join(o[0], o[1]);
                f[d + 1] = join(o[2], o[3]);
                g[d] = join(o[4], o[5]);
                g[d + 1] = join(o[6], o[7]);
            }
        }
    }
};

// A lane's operand row from memory: row lane % 32 from `base` on, zeros behind the `rows` that there are.
template <class T, int DP>
__device__ inline void load_rows(const T *base, int64_t ld, int rows, int dim, int lane, typename Half8<T>::type (&f)[DP / 16])
{
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(base), 0, rows > 0 ? (int)(((min(rows, 32) - 1) * ld + dim) * 2) : 0, 0x00020000);
    const uint32_t from = (uint32_t)((lane & 31) * ld + (lane >> 5) * 8) * 2;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const uint32_t at = s * 16 + (lane >> 5) * 8 < dim ? from + s * 32 : 0x80000000u;
        f[s] = __builtin_bit_cast(typename Half8<T>::type, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
    }
}

// Waits here until operands from memory are there.  Left to the compiler, the wait is where they are first used, in the loop over tiles, and there it is one for all of the
// tiles that are on their way, in every turn.
template <class V8, int NS>
__device__ inline void arrived(V8 (&f)[NS])
{
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        u32x4 v = __builtin_bit_cast(u32x4, f[s]);
        asm volatile("" : "+v"(v));
        f[s] = __builtin_bit_cast(V8, v);
    }
}

// Number of accumulator register r's row, less 4 (lane / 32).
constexpr __device__ int acc_row(int r) { return 8 * (r >> 2) + (r & 3); }

// Eight registers of an accumulator, rounded to nearest: an operand.
template <class T>
__device__ inline typename Half8<T>::type rounded(const f32x16 &a, int u)
{
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a[8 * u + i];
    return __builtin_convertvector(v, typename Half8<T>::type);
}

// Sum, or maximum, over the two lanes that hold one column.
__device__ inline float both_halves_sum(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ inline float both_halves_max(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Stores a transposed result: lane l holds column (row of the output) l % 32 of ND tiles of 32 elements.  Two groups of four rows are swapped between the halves
// so that a lane has eight adjacent elements.
template <class T, int ND>
__device__ inline void store_columns(const f32x16 (&o)[ND], float factor, T *row, bool valid, int dim, int lane)
{
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            f32x8 f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = o[dt][8 * g + i] * factor;
            u32x4 w = __builtin_bit_cast(u32x4, __builtin_convertvector(f, typename Half8<T>::type));
            const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const int at = dt * 32 + 16 * g + 8 * (lane >> 5);
            if (valid && at < dim) *reinterpret_cast<u32x4 *>(row + at) = u32x4{a[0], b[0], a[1], b[1]};
        }
}

// Goes through `rows` rows of memory from row j0 on and calls f(row number, row) for those that have an infinity or NaN; all lanes together.
template <class T, class F>
__device__ inline void for_nonfinite_rows(const T *base, int64_t ld, int j0, int rows, int dim, int lane, F f)
{
    for (int i = 0; i < rows; ++i) {
        const T *row = base + (int64_t)(j0 + i) * ld;
        bool any = false;
        for (int d = lane; d < dim; d += 64) any |= !(__builtin_fabsf((float)row[d]) < INFINITY);
        if (__ballot(any)) f(j0 + i, row);
    }
}

// Adds to a transposed result (see store_columns) what was taken out of those rows, where the lane's column sees the row.
template <class T, int ND, class Seen>
__device__ inline void add_nonfinite(f32x16 (&o)[ND], const T *base, int64_t ld, int j0, int rows, int dim, int lane, Seen seen)
{
    for_nonfinite_rows<T>(base, ld, j0, min(rows, ATT_STEP), dim, lane, [&](int j, const T *row) {
        const bool mine = seen(j);
        int from = 4 * (lane >> 5);
        asm volatile("" : "+v"(from));  // else the tests below leave the loop, and take scalar registers from the common path
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int d = dt * 32 + 8 * c + from;
                if (d >= dim) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = (float)row[d + e];
                    if (mine && !(__builtin_fabsf(x) < INFINITY)) o[dt][4 * c + e] += x;
                }
            }
    });
}

__host__ __device__ inline int bias_entries(int distance) { return 2 * distance + 1 + 2 * ATT_EXT; }

// LDS of a block that takes a sequence whole (whole_grad_kernel): NW wavefronts, rows of DP.
template <int DP, int NW>
struct WholeCfg {
    static constexpr int KEYS = 32 * NW, STAGE = 32 * DP;  // elements of a stage's Q, or dO
    static constexpr int K_BYTES = KEYS * DP * 2, STAGES_BYTES = 2 * 2 * STAGE * 2, DS_BYTES = 32 * KEYS * 2, NUMBERS_BYTES = KEYS * 2 * (int)sizeof(float);
    static constexpr int FIXED = K_BYTES + STAGES_BYTES + DS_BYTES + NUMBERS_BYTES;
    // With a bias one table, with its gradient two more per wavefront.
    static int bytes(int distance, bool bias, bool dbias) { return FIXED + (bias ? ((bias_entries(distance) + 3) & ~3) * 4 * (dbias ? 1 + 2 * NW : 1) : 0); }
};

// The bias of one head by relative position, in units of the scores before they are scaled, so that the products of queries and keys add to it:
// [2 distance + 1 + 2 ATT_EXT], the ends repeated, which stand for all beyond; 0 where no position is from `least` to `most`.  A finite bias beyond 2^100 counts as 2^100, which scores of any size are
// lost against: a row of them is even, as it would be in numbers without end, and no difference is one of infinities.
__device__ inline void make_bias(float *table, const float *bias, const int32_t *bucket_of, const AttentionShape &a, int head, int least = INT32_MIN, int most = INT32_MAX)
{
    const float inverse = 1.f / __builtin_fabsf(a.scale);
    least = min(max(least, -a.distance), a.distance), most = min(max(most, -a.distance), a.distance);
    for (int i = threadIdx.x; i < bias_entries(a.distance); i += blockDim.x) {
        const int d = min(max(i - ATT_EXT, 0), 2 * a.distance);
        float b = bias[(int64_t)bucket_of[d] * a.heads + head];
        if (d - a.distance < least || d - a.distance > most) b = 0.f;
        table[i] = (__builtin_fabsf(b) < INFINITY ? __builtin_fmaxf(__builtin_fminf(b, 0x1p100f), -0x1p100f) : b) * inverse;
    }
}

// An index into LDS that is one register: the compiler would otherwise put the array's own place into each of the offsets that follow, which a read of two numbers has no
// room for.
__device__ inline int one_register(int i)
{
    asm volatile("" : "+v"(i));
    return i;
}

// The scale's sign goes into the queries.
template <class V8, int NS>
__device__ inline void take_sign(V8 (&f)[NS], float scale)
{
    if (scale >= 0.f) return;
#pragma unroll
    for (int s = 0; s < NS; ++s) f[s] = __builtin_bit_cast(V8, __builtin_bit_cast(u32x4, f[s]) ^ 0x80008000u);
}

// Which of 64 keys hide from some of the wavefront's queries: those behind a query's last one, those before its first one, or neither.
struct Edges {
    bool behind, before;
};
__device__ inline Edges edges(const AttentionShape &a, int p, int queries, int j, int keys)
{
    return {j + keys - 1 > p + a.right || keys < ATT_STEP, j < p + queries - 1 - a.left && j + keys > a.sinks};
}

// What `queries` queries at positions from p on see of `keys` keys from key j on: nothing, or all of them.
struct Sight {
    bool none, all;
};
__device__ inline Sight sight(const AttentionShape &a, int p, int queries, int j, int keys)
{
    // the first query sees the fewest keys ahead, the last one the fewest behind
    const int last = p + queries - 1, end = j + keys - 1;
    const bool none = queries <= 0 || keys <= 0 || j > last + a.right || (end < p - a.left && j >= a.sinks);
    const bool all = end <= p + a.right && (j >= last - a.left || end < a.sinks);
    return {none, all};
}

}  // namespace
